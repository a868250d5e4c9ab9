// Generation with a sliding window and sinks: one token per sequence over caches of any capacity.
//
// Position t lies in row t while t < capacity, else in row sinks + (t - sinks) mod (capacity - sinks).  The keys of a step are the sinks,
// then the window in order of position, the new token last (read from k_new and v_new: its cache row is written by the same launch).
//
// Memory bounds a step: every visible row of K and V is read once for all query heads of its KV head.  A wavefront takes 32 keys at a
// time and needs no other: S^T = K Q^T with the keys as A operand straight from memory (a lane reads its key's pieces) and up to 32 query
// heads as B; the values pass through a part of LDS of the wavefront's own, where they are turned (focus_window.h); O^T += V^T P^T.
// The next 32 keys' loads are on their way meanwhile.  Work-groups of four wavefronts share a walk, several share the walk of a
// head where there are few sequences; their partial softmaxes are joined in LDS, then by a second launch, each in a fixed order.
#include "focus_window.h"

#include <algorithm>

namespace focus {

using namespace window;

namespace {

constexpr int COLS = 32;                    // query heads of a work-group
template <typename T, int D> constexpr int dec_waves() { return D * (int)sizeof(T) > 256 ? 1 : 2; }

// What a sequence's step reads.
struct Step {
    int pos, sinks, start, count;           // position; visible sinks; first position of the window behind them; keys
    int slot0, ring;                        // cache row of `start`; rows that go round
    bool live;
};
__device__ inline int cache_row(int pos, int n, int sinks) { return pos < n ? pos : sinks + (pos - sinks) % (n - sinks); }
__device__ inline Step step_of(const WindowArgs& A, int pos)
{
    Step s;
    s.pos = pos;
    s.ring = A.n - A.sinks;
    s.live = pos >= 0 && (pos < A.n || s.ring >= A.window);
    if (!s.live) { s.sinks = s.start = s.count = s.slot0 = 0; return s; }
    s.sinks = min(A.sinks, pos + 1);
    s.start = max(s.sinks, pos - A.window + 1);
    s.count = s.sinks + max(0, pos - s.start + 1);
    s.slot0 = s.start <= pos ? cache_row(s.start, A.n, A.sinks) : 0;
    return s;
}

// work-groups that share the keys of a (batch, KV head, 32 query heads): two for each compute unit in all, of four rounds of 32 keys at
// least, so that each wavefront has one
int decode_parts(const WindowArgs& A)
{
    const int G = A.Hq / A.Hkv;
    const long long rows = (long long)A.B * A.Hkv * ((G + COLS - 1) / COLS);
    const long long keys = std::min((long long)A.window + A.sinks, (long long)A.n);
    const long long most = (keys + 127) / 128;
    return (int)std::max(1ll, std::min(most, (512 + rows - 1) / rows));
}

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(WTHR, (dec_waves<T, D>())) void window_step_kernel(WindowArgs A, int parts, const int* __restrict__ pos_dev,
                                                                              const T* __restrict__ q, const T* __restrict__ kn,
                                                                              const T* __restrict__ vn, T* kc, T* vc, float* __restrict__ part,
                                                                              T* __restrict__ out, float* __restrict__ lse)
{
    typedef Tile<T, D, 32> TL;
    typedef Piece<T> P;
    constexpr bool AHEAD = D * (int)sizeof(T) <= 256;         // loads of the next keys during the products of these (registers)
    constexpr int VBX = TL::BYTES / 1024;                     // loads of a round of V
    constexpr int JOIN = COLS * (D + 4) * 4;
    constexpr int SMEM = 4 * TL::BYTES > JOIN ? 4 * TL::BYTES : JOIN;
    __shared__ __attribute__((aligned(256))) char smem[SMEM];
    __shared__ float s_m[4][COLS], s_l[4][COLS];
    const int lane = threadIdx.x & 63, hh = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = A.Hq / A.Hkv, shares = (G + COLS - 1) / COLS;
    const int p0 = blockIdx.x % parts, share = blockIdx.x / parts % shares, hk = blockIdx.x / parts / shares % A.Hkv;
    const int b = blockIdx.x / parts / shares / A.Hkv;
    const Step S = step_of(A, pos_dev[b]);
    if (!S.live) return;
    const size_t kv = (size_t)b * A.Hkv + hk;
    T *kcb = kc + kv * A.n * D, *vcb = vc + kv * A.n * D;
    const T *knb = kn + kv * D, *vnb = vn + kv * D;
    if (p0 == 0 && share == 0) {                              // the new rows
        const size_t row = (size_t)cache_row(S.pos, A.n, A.sinks) * D;
        for (int i = threadIdx.x; i < 2 * TL::PIECES; i += WTHR) {
            const bool val = i >= TL::PIECES;
            const int piece = val ? i - TL::PIECES : i;
            *(u32x4*)((char*)((val ? vcb : kcb) + row) + 16 * piece) = load_piece(val ? vnb : knb, piece);
        }
    }
    const int heads = min(COLS, G - share * COLS), h0 = hk * G + share * COLS;
    const T* qrow = q + ((size_t)b * A.Hq + h0 + min(col, heads - 1)) * D;
    u32x4 qf[AHEAD ? TL::KS : 1];
    if constexpr (AHEAD) {
#pragma unroll
        for (int s = 0; s < TL::KS; ++s) qf[s] = load_piece(qrow, 2 * s + hh);
    }
    f32x16 o[TL::DB];
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) o[i] = 0.f;
    constexpr float LOWER = P::EXP == 0x7c007c00u ? 6.f : 0.f;          // as in the forward pass
    float m = -1e30f, l = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;
    // element offset of key u's row in the caches; the new token (the last key) lies elsewhere
    auto row_of = [&](int u, const T* cache, const T* fresh) -> const T* {
        if (u >= S.count - 1) return fresh;
        int row = u;
        if (u >= S.sinks) {
            row = S.slot0 + (u - S.sinks);
            if (row >= A.n) row -= S.ring;
        }
        return cache + (size_t)row * D;
    };
    u32x4 kf[AHEAD ? TL::KS : 1], vr[AHEAD ? VBX : 1];
    auto load_k = [&](int u0) {
        const T* r = row_of(min(u0 + col, S.count - 1), kcb, knb);
#pragma unroll
        for (int s = 0; s < (AHEAD ? TL::KS : 0); ++s) kf[s] = load_piece(r, 2 * s + hh);
    };
    const int cplace = TL::comps_place(lane);
    char* mine = smem + wave * TL::BYTES;
    // V: row r of the round to its place, 16 bytes a lane
    auto load_v = [&](int u0, int i, u32x4* x) {
        const int id = 64 * i + lane, r = id / (TL::RPITCH / 16), piece = (id % (TL::RPITCH / 16)) ^ TL::turn_of_row(r);
        u32x4 y = {0u, 0u, 0u, 0u};
        if (u0 + r < S.count && piece < TL::PIECES) y = load_piece(row_of(u0 + r, vcb, vnb), piece);
        *x = y;
    };
    auto store_v = [&](int i, const u32x4* x) { *(u32x4*)(mine + 16 * (64 * i + lane)) = *x; };

    // rounds of 32 keys: this work-group's share of them, its wavefronts in turn
    const int rounds = (S.count + 31) / 32;
    const int r0 = (int)((long long)rounds * p0 / parts), r1 = (int)((long long)rounds * (p0 + 1) / parts);
    if (AHEAD && r0 + wave < r1) {
        load_k(32 * (r0 + wave));
#pragma unroll
        for (int i = 0; i < (AHEAD ? VBX : 0); ++i) load_v(32 * (r0 + wave), i, &vr[AHEAD ? i : 0]);
    }
    for (int r = r0 + wave; r < r1; r += 4) {
        const int u0 = 32 * r;
        f32x16 x = 0.f;
        if constexpr (AHEAD) {
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) x = P::mma(kf[s], qf[s], x);
#pragma unroll
            for (int i = 0; i < VBX; ++i) store_v(i, &vr[i]);
            if (r + 4 < r1) {
                load_k(u0 + 128);
#pragma unroll
                for (int i = 0; i < VBX; ++i) load_v(u0 + 128, i, &vr[i]);
            }
        } else {
            const T* kr = row_of(min(u0 + col, S.count - 1), kcb, knb);
#pragma unroll 4
            for (int s = 0; s < TL::KS; ++s) x = P::mma(load_piece(kr, 2 * s + hh), load_piece(qrow, 2 * s + hh), x);
#pragma unroll 2
            for (int i = 0; i < VBX; ++i) {
                u32x4 y;
                load_v(u0, i, &y);
                store_v(i, &y);
            }
        }
        own_fence();
        if (CAP) tanh_scores<T>(x, ci);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = u0 + 8 * (i / 4) + 4 * hh + i % 4 < S.count ? x[i] : -INFINITY;
            top = fmaxf(top, x[i]);
        }
        top = halves_max(top) * c;
        const bool over = top > m + LOWER + 8.f;
        if (__any(over)) {
            const float to = over ? top - LOWER : m, f = exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int i = 0; i < TL::DB; ++i) o[i] *= f;
        }
        float p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -m));
            l += p[i];
        }
#pragma unroll
        for (int s = 0; s < TL::US; ++s) {
            const u32x4 pf = P::pack(p + s * P::E);
#pragma unroll
            for (int db = 0; db < TL::DB; ++db) o[db] = P::mma(TL::comps_piece(mine, cplace, db, s), pf, o[db]);
        }
        own_fence();
    }
    // the four wavefronts' softmaxes become one: a common reference, then the sums one after the other
    l = halves_sum(l);
    if (hh == 0) { s_m[wave][col] = m; s_l[wave][col] = l; }
    __syncthreads();                                          // (and LDS changes its use)
    float M = s_m[0][col];
#pragma unroll
    for (int i = 1; i < 4; ++i) M = fmaxf(M, s_m[i][col]);
    const float f = exp2f(m - M);
    float* sum = (float*)smem;                                // [COLS][D + 4]
    for (int turn = 0; turn < 4; ++turn) {
        if (wave == turn) {
#pragma unroll
            for (int db = 0; db < TL::DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int comp = 32 * db + 8 * (i / 4) + 4 * hh + i % 4;
                    if (comp >= D) continue;
                    float* at = sum + col * (D + 4) + comp;
                    *at = turn ? *at + o[db][i] * f : o[db][i] * f;
                }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < heads * D; i += WTHR) {
        const int head = i / D, comp = i % D;
        float mm = s_m[0][head], ll = 0.f;
#pragma unroll
        for (int w = 1; w < 4; ++w) mm = fmaxf(mm, s_m[w][head]);
#pragma unroll
        for (int w = 0; w < 4; ++w) ll += s_l[w][head] * exp2f(s_m[w][head] - mm);
        const float val = sum[head * (D + 4) + comp];
        const size_t bh = (size_t)b * A.Hq + h0 + head;
        if (parts == 1) {
            const float y = val / ll;
            const float ys[8] = {y, y, y, y, y, y, y, y};
            const u32x4 pk = P::pack(ys);
            __builtin_memcpy(out + bh * D + comp, &pk, sizeof(T));
            if (lse && comp == 0) lse[bh] = (mm + log2f(ll)) * LN2;
        } else {
            float* slot = part + (bh * parts + p0) * (D + 2);
            slot[comp] = val;
            if (comp == 0) { slot[D] = mm; slot[D + 1] = ll; }
        }
    }
}

// out and lse of a head from its work-groups' partial softmaxes (all of a thread's loads are on their way before the first is needed)
template <typename T>
__global__ __launch_bounds__(256) void window_step_join_kernel(WindowArgs A, int parts, const int* __restrict__ pos_dev,
                                                             const float* __restrict__ part, T* __restrict__ out, float* __restrict__ lse)
{
    constexpr int AT_ONCE = 16;
    const size_t bh = blockIdx.x;
    const int d = A.d, comp = threadIdx.x;
    const float* slots = part + bh * parts * (d + 2);
    const int pos = pos_dev[bh / A.Hq];
    float M = -1e30f, l = 0.f, sum = 0.f;
    for (int i0 = 0; i0 < parts; i0 += AT_ONCE) {
        float m[AT_ONCE], ls[AT_ONCE], o[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const bool there = i0 + i < parts;
            const float* s = slots + (size_t)(there ? i0 + i : 0) * (d + 2);
            m[i] = there ? s[d] : -1e30f;
            ls[i] = there ? s[d + 1] : 0.f;
            o[i] = there && comp < d ? s[comp] : 0.f;
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) top = fmaxf(top, m[i]);
        const float f = exp2f(M - top);
        l *= f;
        sum *= f;
        M = top;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const float g = i0 + i < parts ? exp2f(m[i] - M) : 0.f;
            l += ls[i] * g;
            sum += o[i] * g;
        }
    }
    if (!step_of(A, pos).live || comp >= d) return;           // (what a skipped sequence's slots hold is not used)
    const float y = sum / l;
    const float ys[8] = {y, y, y, y, y, y, y, y};
    const u32x4 pk = Piece<T>::pack(ys);
    __builtin_memcpy(out + bh * d + comp, &pk, sizeof(T));
    if (lse && comp == 0) lse[bh] = (M + log2f(l)) * LN2;
}

// The rows that a prompt leaves in the caches: row r holds the last position below the sequence's length that lies there.
__global__ __launch_bounds__(WTHR) void window_fill_kernel(WindowArgs A, int capacity, int pieces, const char* __restrict__ k,
                                                          const char* __restrict__ v, char* __restrict__ kc, char* __restrict__ vc, int es)
{
    const int b = blockIdx.y / A.Hkv, hk = blockIdx.y % A.Hkv;
    const Sequence sq = sequence_of(A, b);
    const long long id = (long long)blockIdx.x * WTHR + threadIdx.x;
    const int row = (int)(id / pieces), piece = (int)(id % pieces);
    if (row >= capacity || row >= sq.len) return;
    int pos = row;
    if (sq.len > capacity && row >= A.sinks) {
        const int ring = capacity - A.sinks;                  // (>= window: checked by the caller)
        pos = row + (sq.len - 1 - row) / ring * ring;
    }
    const long long from = ((long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)(sq.first + pos) * A.ks[2]) * es + 16 * piece;
    const long long to = (((long long)b * A.Hkv + hk) * capacity + row) * (long long)pieces * 16 + 16 * piece;
    *(u32x4*)(kc + to) = *(const u32x4*)(k + from);
    *(u32x4*)(vc + to) = *(const u32x4*)(v + from);
}

template <typename T, int D, bool CAP>
hipError_t launch_cap(const WindowArgs& A, const int* pos, const void* q, const void* kn, const void* vn, void* kc, void* vc, char* ws,
                      void* out, float* lse, hipStream_t st)
{
    const int parts = decode_parts(A), G = A.Hq / A.Hkv;
    const long long groups = (long long)A.B * A.Hkv * ((G + COLS - 1) / COLS) * parts;
    if (groups > 0x7fffffffll) return hipErrorInvalidConfiguration;
    window_step_kernel<T, D, CAP><<<(unsigned)groups, WTHR, 0, st>>>(A, parts, pos, (const T*)q, (const T*)kn, (const T*)vn, (T*)kc, (T*)vc,
                                                                    (float*)ws, (T*)out, lse);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    window_step_join_kernel<T><<<A.B * A.Hq, D <= 64 ? 64 : D <= 128 ? 128 : 256, 0, st>>>(A, parts, pos, (const float*)ws, (T*)out, lse);
    return hipGetLastError();
}
template <typename T, int D, typename... X>
hipError_t launch_d(const WindowArgs& A, X... x)
{
    return A.softcap > 0.f ? launch_cap<T, D, true>(A, x...) : launch_cap<T, D, false>(A, x...);
}
template <typename T, typename... X>
hipError_t launch_t(const WindowArgs& A, X... x)
{
    switch (A.d) {
        case 64: return launch_d<T, 64>(A, x...);
        case 80: return launch_d<T, 80>(A, x...);
        case 96: return launch_d<T, 96>(A, x...);
        case 128: return launch_d<T, 128>(A, x...);
        default: return launch_d<T, 256>(A, x...);
    }
}

}  // namespace

size_t window_decode_workspace(const WindowArgs& A)
{
    const int parts = decode_parts(A);
    return parts == 1 ? 0 : (size_t)A.B * A.Hq * parts * (A.d + 2) * sizeof(float);
}

hipError_t launch_window_decode(const WindowArgs& A, const int* pos, const void* q, const void* kn, const void* vn, void* kc, void* vc,
                                char* ws, void* out, float* lse, hipStream_t st)
{
    if (A.dtype == 0) return launch_t<float>(A, pos, q, kn, vn, kc, vc, ws, out, lse, st);
    if (A.dtype == 1) return launch_t<uint16_t>(A, pos, q, kn, vn, kc, vc, ws, out, lse, st);
    return launch_t<f16_bits>(A, pos, q, kn, vn, kc, vc, ws, out, lse, st);
}

hipError_t launch_window_fill(const WindowArgs& A, int capacity, const void* k, const void* v, void* kc, void* vc, hipStream_t st)
{
    const int es = A.dtype == 0 ? 4 : 2, pieces = A.d * es / 16;
    const long long work = (long long)std::min(capacity, A.span_max) * pieces;
    window_fill_kernel<<<dim3((unsigned)((work + WTHR - 1) / WTHR), A.B * A.Hkv), WTHR, 0, st>>>(A, capacity, pieces, (const char*)k,
                                                                                              (const char*)v, (char*)kc, (char*)vc, es);
    return hipGetLastError();
}

}  // namespace focus
