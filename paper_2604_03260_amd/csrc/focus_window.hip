// Attention of a sliding window with sinks, forward: row i sees key j iff j <= i and (i - j < window or j < sinks).
//
// One pass over the keys a tile of rows can see, with a running reference and sum of the softmax:
//   S^T = K Q^T  (A = keys by rows, B = the wavefront's 32 queries, held in registers)
//   P^T = exp2(scale' S^T - m), one row of the softmax per lane (and half-wave), so its maximum and sum are sums in a lane
//   O^T += V^T P^T (A = values by components; P^T is the B operand as the first product left it, focus_window.h)
// A work-group is four wavefronts that share the staged keys; each owns 32 rows of one query head.  The heads of a KV head come first, then
// the next rows: with four heads all four walk in step, and the walk is as short as the window allows.  Keys and values go straight to
// LDS; the values' rows are turned by the LDS reads, so no copy of them in another order is needed and the call is one launch without
// workspace.  (Turned in registers on their way, 16 v_perm and 8 stores per 4 x 8 components, they took a fifth of the time.)
// Two buffers, one barrier per tile of 32 keys.
// The reference m of a row moves only when its maximum has risen by more than 8 (log2 units): O is rarely rescaled, and the
// probabilities stay below 2^8.  IEEE halves lose bits below 2^-14: there the reference lies 6 lower, so what is dropped is below 2^-31 of the
// largest, 2^-11 of the sum over 2^20 keys.
#include "focus_window.h"

#include <algorithm>

namespace focus {

using namespace window;

namespace {

constexpr int KEY_TILE = 32;
// Wavefronts per SIMD: as many as the queries and the output leave registers for.  They are what hides the waits of a step whose parts depend on each
// other (128 components of 16 bits, tiles of 32 keys: two 775 us, three 650 to 710 us by box; tiles of 64 keys, whose two buffers leave room for two
// work-groups only, 785 us; 32768 tokens of 32/8 heads, window 1024).  Scores a block ahead of the softmax and operands a step ahead
// of the products, with two wavefronts, were 769 us.
template <typename T, int D> constexpr int fwd_waves() { return D * (int)sizeof(T) > 384 ? 1 : D * (int)sizeof(T) > 256 ? 2 : 3; }

constexpr float START = -1e30f;              // the reference of a row before its first key

// One tile of keys for a wavefront's rows: scores, the rows' references and sums, and the output.  edge: some pair is hidden.
template <typename T, int D, bool CAP>
WINDOW_INLINE __device__ inline void attend(const WindowArgs& A, const char* kt, const char* vt, int rplace, int cplace, const u32x4 (&qf)[Tile<T, D, 32>::KS],
                                            int row, int tkey, int hh, bool edge, float c, float ci, float& m, float& l, f32x16 (&o)[Tile<T, D, 32>::DB])
{
    typedef Tile<T, D, 32> TL;
    typedef Piece<T> P;
    constexpr float LOWER = P::EXP == 0x7c007c00u ? 6.f : 0.f;          // IEEE halves, see above
    const int rp = opaque(rplace), cp = opaque(cplace);
    f32x16 x = 0.f;
#pragma unroll
    for (int s = 0; s < TL::KS; ++s) x = P::mma(TL::rows_piece(kt, rp, s), qf[s], x);
    settle<T>();
    if (CAP) tanh_scores<T>(x, ci);
    if (edge) {
        const int key = opaque(tkey + 4 * hh);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = visible(row, key + 8 * (i / 4) + i % 4, A.window, A.sinks) ? x[i] : -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, x[j]);
    top = halves_max(top) * c;
    const bool over = top > m + (LOWER + 8.f);
    if (__any(over)) {                                // (a row's bits do not depend on its neighbours)
        const float to = over ? top - LOWER : m, f = __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= f;
#pragma unroll
        for (int j = 0; j < TL::DB; ++j) o[j] *= f;
    }
    u32x4 pf[TL::US];
#pragma unroll
    for (int s = 0; s < TL::US; ++s) {
        float p[8];
#pragma unroll
        for (int j = 0; j < P::E; ++j) {
            p[j] = __builtin_amdgcn_exp2f(fmaf(x[s * P::E + j], c, -m));
            l += p[j];
        }
        pf[s] = P::pack(p);
    }
#pragma unroll
    for (int s = 0; s < TL::US; ++s)
#pragma unroll
        for (int db = 0; db < TL::DB; ++db) o[db] = P::mma(TL::comps_piece(vt, cp, db, s), pf[s], o[db]);
    settle<T>();
}

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(WTHR, (fwd_waves<T, D>())) void window_fwd_kernel(WindowArgs A, int blocks, const T* __restrict__ q,
                                                                             const T* __restrict__ k, const T* __restrict__ v,
                                                                             T* __restrict__ out, float* __restrict__ lse)
{
    constexpr int R = KEY_TILE;
    typedef Tile<T, D, R> TL;
    __shared__ __attribute__((aligned(256))) char s_k[2][TL::BYTES], s_v[2][TL::BYTES];
    __shared__ unsigned s_bad[2];
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // (b, KV head, four of the (rows, query head) of it, the head fastest)
    const int G = A.Hq / A.Hkv, fours = (blocks * G + 3) / 4;
    const long long w = work_of((long long)A.B * A.Hkv * fours);
    if (w < 0) return;
    const int four = (int)(w % fours), hk = (int)(w / fours % A.Hkv), b = (int)(w / fours / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    const int tile0 = four * 4 / G * 32;                      // first row of the work-group
    if (tile0 >= sq.len) return;
    const int row0 = (four * 4 + wave) / G * 32;              // of the wavefront
    const int h = hk * G + (four * 4 + wave) % G;
    const bool idle = row0 >= sq.len;                         // no rows: the wavefront only helps to stage
    const int row = row0 + (lane & 31);
    const bool real = row < sq.len;
    const T* qrow = q + (long long)sq.tb * A.qs[0] + (long long)h * A.qs[1] + (long long)(sq.first + (real ? row : sq.len - 1)) * A.qs[2];
    const T* kb = k + (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)sq.first * A.ks[2];
    const T* vb = v + (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)sq.first * A.ks[2];

    u32x4 qf[TL::KS];
#pragma unroll
    for (int s = 0; s < TL::KS; ++s) qf[s] = load_piece(qrow, 2 * s + hh);
    f32x16 o[TL::DB];
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) o[i] = 0.f;
    float m = START, l = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;

    const Walk W(A, tile0, min((four * 4 + 3) / G * 32 + 32, sq.len) - 1);
    const int pitch = (int)(A.ks[2] * (long long)sizeof(T));
    Dma<T, D, R, 4> dma;
    dma.init(wave, lane, pitch);
    auto fetch = [&](int t) WINDOW_INLINE {
        const int key = W.key_at(t);
        dma.load(kb + (long long)key * A.ks[2], pitch, sq.len - key, s_k[t & 1], wave, lane);
        dma.load(vb + (long long)key * A.ks[2], pitch, sq.len - key, s_v[t & 1], wave, lane);
    };
    if (threadIdx.x < 2) s_bad[threadIdx.x] = 0u;
    fetch(0);
    landed(qf);
    const int rplace = TL::rows_place(lane), cplace = TL::comps_place(lane);
#pragma unroll 1
    for (int t = 0; t < W.tiles; ++t) {
        const int buf = t & 1, tkey = W.key_at(t);
        dma_wait();
        __syncthreads();
        const bool edge = W.edge(tkey, A);
        if (edge) {
            scrub<T, D, R>(s_v[buf], &s_bad[buf], threadIdx.x, WTHR);
            __syncthreads();
        }
        if (t + 1 < W.tiles) fetch(t + 1);
        const Block kind = idle ? HIDDEN : block_kind(row0, tkey, A.window, A.sinks);
        if (kind != HIDDEN) {
            attend<T, D, CAP>(A, s_k[buf], s_v[buf], rplace, cplace, qf, row, tkey, hh, kind == EDGE, c, ci, m, l, o);
            if (edge) {
                const unsigned marks = s_bad[buf];
                if (marks != 0u && spoiled_by<true>(marks, row, tkey, hh, A.window, A.sinks)) l = __builtin_nanf("");
            }
        }
        if (edge) {                                           // (the marks have been seen by all before they go)
            __syncthreads();
            if (threadIdx.x == 0) s_bad[buf] = 0u;
        }
    }
    if (idle) return;
    l = halves_sum(l);
    T* orow = real ? out + (long long)sq.tb * A.os[0] + (long long)h * A.os[1] + (long long)(sq.first + row) * A.os[2] : nullptr;
    store_row<T, D>(orow, o, 1.f / l, lane);
    if (lse && real && hh == 0) lse[((long long)sq.tb * A.Hq + h) * A.n + sq.first + row] = (m + log2f(l)) * LN2;
}

// The same for few rows: a work-group has 32 rows of one head, its wavefronts take the tiles of their walk in turn, each through LDS of its own and
// without a barrier, and their outputs are joined in LDS, in order.
template <typename T, int D> constexpr int few_lds() { return std::max(8 * Tile<T, D, 32>::BYTES, 4 * 32 * (D + 4) * 4) + 2048; }
template <typename T, int D, bool CAP>
__global__ __launch_bounds__(WTHR, 1) void window_fwd_few_kernel(WindowArgs A, int blocks, const T* __restrict__ q, const T* __restrict__ k,
                                                                 const T* __restrict__ v, T* __restrict__ out, float* __restrict__ lse)
{
    typedef Tile<T, D, 32> TL;
    constexpr int PITCH = D + 4;                              // floats of a row in the join
    __shared__ __attribute__((aligned(256))) char smem[few_lds<T, D>() - 2048];
    __shared__ float s_m[4][32], s_l[4][32];
    __shared__ unsigned s_bad[4];
    const int lane = threadIdx.x & 63, hh = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long w = work_of((long long)A.B * A.Hq * blocks);
    if (w < 0) return;
    const int row0 = (int)(w % blocks) * 32, h = (int)(w / blocks % A.Hq), b = (int)(w / blocks / A.Hq), hk = h / (A.Hq / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    if (row0 >= sq.len) return;
    const int row = row0 + col;
    const T* qrow = q + (long long)sq.tb * A.qs[0] + (long long)h * A.qs[1] + (long long)(sq.first + min(row, sq.len - 1)) * A.qs[2];
    const T* kb = k + (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)sq.first * A.ks[2];
    const T* vb = v + (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)sq.first * A.ks[2];
    u32x4 qf[TL::KS];
#pragma unroll
    for (int s = 0; s < TL::KS; ++s) qf[s] = load_piece(qrow, 2 * s + hh);
    f32x16 o[TL::DB];
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) o[i] = 0.f;
    float m = START, l = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;
    const Walk W(A, row0, min(row0 + 31, sq.len - 1));
    const int pitch = (int)(A.ks[2] * (long long)sizeof(T));
    char *kt = smem + 2 * wave * TL::BYTES, *vt = kt + TL::BYTES;
    const int rplace = TL::rows_place(lane), cplace = TL::comps_place(lane);
    if (lane == 0) s_bad[wave] = 0u;
#pragma unroll 1
    for (int t = wave; t < W.tiles; t += 4) {
        const int tkey = W.key_at(t);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the tile before has been read
        Dma<T, D, 32, 1> dma;
        dma.init(0, opaque(lane), pitch);
        dma.load(kb + (long long)tkey * A.ks[2], pitch, sq.len - tkey, kt, 0, lane);
        dma.load(vb + (long long)tkey * A.ks[2], pitch, sq.len - tkey, vt, 0, lane);
        dma_wait();
        own_fence();
        const bool edge = block_kind(row0, tkey, A.window, A.sinks) == EDGE;
        if (edge) {
            scrub<T, D, 32>(vt, &s_bad[wave], lane, 64);
            own_fence();
        }
        attend<T, D, CAP>(A, kt, vt, rplace, cplace, qf, row, tkey, hh, edge, c, ci, m, l, o);
        if (edge) {
            const unsigned marks = s_bad[wave];
            if (marks != 0u && spoiled_by<true>(marks, row, tkey, hh, A.window, A.sinks)) l = __builtin_nanf("");
            own_fence();
            if (lane == 0) s_bad[wave] = 0u;
        }
    }
    l = halves_sum(l);
    if (hh == 0) { s_m[wave][col] = m; s_l[wave][col] = l; }
    __syncthreads();                                          // (behind the last tiles too)
    float top = s_m[0][col], sum = 0.f;
#pragma unroll
    for (int i = 1; i < 4; ++i) top = fmaxf(top, s_m[i][col]);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += s_l[i][col] * __builtin_amdgcn_exp2f(s_m[i][col] - top);
    const float f = __builtin_amdgcn_exp2f(m - top) / sum;
    float* joined = (float*)smem;                             // [wave][row][PITCH]
#pragma unroll
    for (int db = 0; db < TL::DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (32 * db + 8 * j >= D) continue;
            const float4 x = {o[db][4 * j] * f, o[db][4 * j + 1] * f, o[db][4 * j + 2] * f, o[db][4 * j + 3] * f};
            *(float4*)(joined + (size_t)(32 * wave + col) * PITCH + 32 * db + 8 * j + 4 * hh) = x;
        }
    __syncthreads();
    const int real = min(32, sq.len - row0);
    T* ob = out + (long long)sq.tb * A.os[0] + (long long)h * A.os[1] + (long long)(sq.first + row0) * A.os[2];
    for (int id = threadIdx.x; id < real * (D / 4); id += WTHR) {
        const int r = id / (D / 4), at = id % (D / 4) * 4;
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float y = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) y += joined[(32 * i + r) * PITCH + at + e];
            x[e] = x[4 + e] = y;
        }
        const u32x4 y = Piece<T>::pack(x);
        T* to = ob + (long long)r * A.os[2] + at;
        if constexpr (sizeof(T) == 4) *(u32x4*)to = y;
        else { uint2 z; z.x = y[0]; z.y = y[1]; *(uint2*)to = z; }
    }
    if (lse && wave == 0 && hh == 0 && row < sq.len) lse[((long long)sq.tb * A.Hq + h) * A.n + sq.first + row] = (top + log2f(sum)) * LN2;
}

// Few rows: all work-groups of the kernel for them fit the machine at once.  Then four wavefronts on one walk end sooner than one walk each (us, window 128 and
// 1024 with 4 sinks: bf16, 12 heads of 64, 1024 tokens: 17.1 -> 8.8 and 33.9 -> 15.8; fp32, the same: 35.1 -> 17.0 and 94.7 -> 46.6; bf16, 32/8 heads
// of 128, 512 tokens: 13.7 -> 12.5 and 22.5 -> 15.2).  Beyond, they copy every tile four times as often (12 heads of 64, 4096 tokens: 19.6 against 22.7; 32/8
// heads of 128, 1024 tokens: 15.6 against 23.4, though 39.7 against 36.5 with the long window).
template <typename T, int D, bool CAP>
hipError_t launch_cap(const WindowArgs& A, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st)
{
    const int G = A.Hq / A.Hkv, blocks = (A.span_max + 31) / 32;
    const long long groups = work_groups((long long)A.B * A.Hkv * ((blocks * G + 3) / 4));
    if constexpr (D * (int)sizeof(T) <= 512) {                // (what fits LDS)
        if (4 * groups <= 256 * (163840 / few_lds<T, D>())) {
            window_fwd_few_kernel<T, D, CAP><<<(unsigned)work_groups((long long)A.B * A.Hq * blocks), WTHR, 0, st>>>(
                A, blocks, (const T*)q, (const T*)k, (const T*)v, (T*)out, lse);
            return hipGetLastError();
        }
    }
    if (groups > 0x7fffffffll) return hipErrorInvalidConfiguration;
    window_fwd_kernel<T, D, CAP><<<(unsigned)groups, WTHR, 0, st>>>(A, blocks, (const T*)q, (const T*)k, (const T*)v, (T*)out, lse);
    return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_d(const WindowArgs& A, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st)
{
    return A.softcap > 0.f ? launch_cap<T, D, true>(A, q, k, v, out, lse, st) : launch_cap<T, D, false>(A, q, k, v, out, lse, st);
}
template <typename T>
hipError_t launch_t(const WindowArgs& A, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st)
{
    switch (A.d) {
        case 64: return launch_d<T, 64>(A, q, k, v, out, lse, st);
        case 80: return launch_d<T, 80>(A, q, k, v, out, lse, st);
        case 96: return launch_d<T, 96>(A, q, k, v, out, lse, st);
        case 128: return launch_d<T, 128>(A, q, k, v, out, lse, st);
        default: return launch_d<T, 256>(A, q, k, v, out, lse, st);
    }
}

}  // namespace

hipError_t launch_window_fwd(const WindowArgs& A, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st)
{
    if (A.dtype == 0) return launch_t<float>(A, q, k, v, out, lse, st);
    if (A.dtype == 1) return launch_t<uint16_t>(A, q, k, v, out, lse, st);
    return launch_t<f16_bits>(A, q, k, v, out, lse, st);
}

}  // namespace focus
