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
// A wavefront's walk is a sequence of blocks of 32 keys, one step each, in which the vector units and the matrix cores have independent work:
//   step i:  softmax of block i  beside  S of block i + 1 and O += V P of block i - 1
// so K is a block ahead of the softmax and V a block behind it, both in two buffers, with one barrier per tile.
// The reference m of a row moves only when its maximum has risen by more than 8 (log2 units): O is rarely rescaled, and the
// probabilities stay below 2^8.  IEEE halves lose bits below 2^-14: there the reference lies 6 lower, so what is dropped is below 2^-31 of the
// largest, 2^-11 of the sum over 2^20 keys.
#include "focus_window.h"

#include <type_traits>

namespace focus {

using namespace window;

namespace {

template <typename T, int D> constexpr int key_tile() { return sizeof(T) == 4 || D > 128 ? 32 : 64; }
// wavefronts per SIMD: the queries and the output of 256 components (fp32: above 96) alone fill half of the registers
template <typename T, int D> constexpr int fwd_waves() { return D * (int)sizeof(T) > 384 ? 1 : 2; }

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(WTHR, (fwd_waves<T, D>())) void window_fwd_kernel(WindowArgs A, int blocks, const T* __restrict__ q,
                                                                             const T* __restrict__ k, const T* __restrict__ v,
                                                                             T* __restrict__ out, float* __restrict__ lse)
{
    constexpr int R = key_tile<T, D>(), U = R / 32;           // keys and steps of a tile
    // Operands of the products are read a step ahead where the registers hold them.  K is fetched KFETCH tiles ahead of the softmax, V VFETCH
    constexpr bool AHEAD = D * (int)sizeof(T) <= 256;
    static_assert(AHEAD || U == 1, "without operands ahead a tile is one block");
    constexpr int KFETCH = AHEAD && U == 1 ? 3 : 2, VFETCH = AHEAD ? 1 : 0;
    typedef Tile<T, D, R> TL;
    typedef Piece<T> P;
    __shared__ __attribute__((aligned(256))) char s_k[2][TL::BYTES], s_v[2][TL::BYTES];
    __shared__ unsigned s_bad[4][2];
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
    constexpr float LOWER = P::EXP == 0x7c007c00u ? 6.f : 0.f;          // IEEE halves, see above
    float m = -1e30f, l = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;

    const Walk W(A, sq, tile0, min((four * 4 + 3) / G * 32 + 32, sq.len) - 1, U);
    auto key_at = [&](int t) WINDOW_INLINE { return W.key_at(t, R); };
    const int pitch = (int)(A.ks[2] * (long long)sizeof(T));
    Dma<T, D, R, 4> dma;
    dma.init(wave, lane, pitch);
    // (behind the last tile: its rows again, in bounds and never used)
    auto fetch = [&](const T* base, char* bufs, int t) WINDOW_INLINE {
        const int key = key_at(min(t, W.tiles - 1));
        dma.load(base + (long long)key * A.ks[2], pitch, sq.len - key, bufs + (t & 1) * TL::BYTES, wave, lane);
    };
    // V of tile t has landed and is about to be read
    auto check = [&](int t) WINDOW_INLINE {
        if (threadIdx.x < 2) s_bad[(t + 1) & 3][threadIdx.x] = 0u;
        if (t >= 0 && W.edge(key_at(t), R, A)) {
            scrub<T, D, R>(s_v[t & 1], s_bad[t & 3]);
            __syncthreads();
        }
    };
    if (threadIdx.x < 8) s_bad[threadIdx.x >> 1][threadIdx.x & 1] = 0u;
    fetch(kb, s_k[0], 0);
    fetch(kb, s_k[0], 1);
    if constexpr (AHEAD) fetch(vb, s_v[0], 0);
    else
        for (int i = threadIdx.x; i < TL::BYTES / 16; i += WTHR) *(u32x4*)(s_v[1] + 16 * i) = u32x4{0u, 0u, 0u, 0u};   // (met by weights of zero)
    dma_wait();
    __syncthreads();

    const int rplace = TL::rows_place(lane), cplace = TL::comps_place(lane);
    f32x16 x = 0.f;                                           // scores of the step's block, then of the next one
    u32x4 pf[TL::US];                                         // probabilities of the block before
    u32x4 ka[AHEAD ? TL::KS : 1], va[AHEAD ? TL::US * TL::DB : 1];
#pragma unroll
    for (int s = 0; s < TL::US; ++s) pf[s] = 0u;
#pragma unroll
    for (int s = 0; s < (AHEAD ? TL::US * TL::DB : 1); ++s) va[s] = 0u;
    // hides what a row does not see, once the scores are there (blocks from key open0 to open1 hide nothing)
    const int open0 = row0 + 32 - A.window, open1 = row0 - 31;
    auto finish = [&](int key0) WINDOW_INLINE {
        if (CAP) tanh_scores<T>(x, ci);
        if (key0 >= open0 && key0 <= open1) return;
        if (block_kind(row0, key0, A.window, A.sinks) == OPEN) return;
        const int key = opaque(key0 + 4 * hh);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = visible(row, key + 8 * (i / 4) + i % 4, A.window, A.sinks) ? x[i] : -INFINITY;
    };
    // the values of a block, in tile t, place u, have been met: were there marked ones among them?
    auto look = [&](int t, int u) WINDOW_INLINE {
        const int key = key_at(t);
        if (!W.edge(key, R, A)) return;
        const unsigned marks = s_bad[t & 3][u];
        if (marks != 0u && spoiled_by<true>(marks, row, key + 32 * u, hh, A.window, A.sinks)) l = __builtin_nanf("");
    };
    // softmax of the scores x, then the next block's scores and the last block's values.  With operands ahead, those of the next step are read
    // between the products, each into the registers that a product has just read: knext, vnext say where.  Else they are read where they are needed.
    auto products = [&](const char* kbuf, const char* vbuf) WINDOW_INLINE {
        const int rp = opaque(rplace), cp = opaque(cplace);
        __builtin_amdgcn_sched_barrier(0);
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) top = fmaxf(top, x[j]);
        top = halves_max(top) * c;
        const bool over = top > m + (LOWER + 8.f), rescale = __any(over);
        const float to = over ? top - LOWER : m, f = __builtin_amdgcn_exp2f(m - to);      // (a row's bits do not depend on its neighbours)
        m = to;
        l *= f;
        u32x4 pn[TL::US];
#pragma unroll
        for (int s = 0; s < TL::US; ++s) {
            float p[8];
#pragma unroll
            for (int j = 0; j < P::E; ++j) {
                p[j] = __builtin_amdgcn_exp2f(fmaf(x[s * P::E + j], c, -m));
                l += p[j];
            }
            pn[s] = P::pack(p);
            asm volatile("" : "+v"(pn[s]));                   // (found here, not behind the products)
        }
        __builtin_amdgcn_sched_barrier(0);
        x = 0.f;
        if constexpr (AHEAD) {
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) {
                x = P::mma(ka[s], qf[s], x);
                ka[s] = TL::rows_piece(kbuf, rp, s);
            }
#pragma unroll
            for (int s = 0; s < TL::US; ++s)
#pragma unroll
                for (int db = 0; db < TL::DB; ++db) {
                    o[db] = P::mma(va[s * TL::DB + db], pf[s], o[db]);
                    va[s * TL::DB + db] = TL::comps_piece(vbuf, cp, db, s);
                }
            constexpr int READS = sizeof(T) == 4 ? 4 : 2;
#pragma unroll
            for (int j = 0; j < TL::KS; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, sizeof(T) == 4 ? 4 : 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
#pragma unroll
            for (int j = 0; j < TL::US * TL::DB; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, sizeof(T) == 4 ? 4 : 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
            }
        } else {
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) x = P::mma(TL::rows_piece(kbuf, rp, s), qf[s], x);
#pragma unroll
            for (int s = 0; s < TL::US; ++s)
#pragma unroll
                for (int db = 0; db < TL::DB; ++db) o[db] = P::mma(TL::comps_piece(vbuf, cp, db, s), pf[s], o[db]);
        }
#pragma unroll
        for (int s = 0; s < TL::US; ++s) pf[s] = pn[s];
        __builtin_amdgcn_sched_barrier(0);
        if (rescale) {
#pragma unroll
            for (int j = 0; j < TL::DB; ++j) o[j] *= f;
        }
    };
    At before = {AHEAD ? 0 : 1, 0}, here = {0, 0}, next = after<U>(here, W);
    auto kat = [&](At a) WINDOW_INLINE { return s_k[0] + (a.t & 1) * TL::BYTES + TL::BLOCK * a.u; };
    auto vat = [&](At a) WINDOW_INLINE { return s_v[0] + (a.t & 1) * TL::BYTES + TL::BLOCK * a.u; };
#pragma unroll
    for (int s = 0; s < TL::KS; ++s) x = P::mma(TL::rows_piece(s_k[0], rplace, s), qf[s], x);
    finish(key_at(0));
    if constexpr (AHEAD) {
#pragma unroll
        for (int s = 0; s < TL::KS; ++s) ka[s] = TL::rows_piece(kat(next), rplace, s);
        if constexpr (U == 1) {
            __syncthreads();                                  // (K of tile 2 goes where that of tile 0 was)
            fetch(kb, s_k[0], 2);
        }
    }
#pragma unroll 1
    for (int i = 0; i < W.blocks; ++i) {
        if (here.u == 0) {                                    // the first step of a tile
            dma_wait();
            __syncthreads();
            check(AHEAD ? here.t : here.t - 1);
            fetch(kb, s_k[0], here.t + KFETCH);
            fetch(vb, s_v[0], here.t + VFETCH);
        }
        const At third = after<U>(next, W);
        if constexpr (AHEAD) products(kat(third), vat(here));
        else products(kat(next), vat(before));
        finish(key_at(next.t) + 32 * next.u);
        if (i > 0) look(before.t, before.u);
        before = here;
        here = next;
        next = third;
    }
    dma_wait();                                               // (nothing may land in LDS after the work-group's end)
    if constexpr (!AHEAD) {
        __syncthreads();
        check(before.t);
    }
    if (row0 >= sq.len) return;
#pragma unroll
    for (int s = 0; s < TL::US; ++s)
#pragma unroll
        for (int db = 0; db < TL::DB; ++db) o[db] = P::mma(AHEAD ? va[AHEAD ? s * TL::DB + db : 0] : TL::comps_piece(vat(before), cplace, db, s), pf[s], o[db]);
    look(before.t, before.u);
    l = halves_sum(l);
    T* orow = real ? out + (long long)sq.tb * A.os[0] + (long long)h * A.os[1] + (long long)(sq.first + row) * A.os[2] : nullptr;
    store_row<T, D>(orow, o, 1.f / l, lane);
    if (lse && real && hh == 0) lse[((long long)sq.tb * A.Hq + h) * A.n + sq.first + row] = (m + log2f(l)) * LN2;
}

template <typename T, int D, bool CAP>
hipError_t launch_cap(const WindowArgs& A, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st)
{
    const int G = A.Hq / A.Hkv, blocks = (A.span_max + 31) / 32;
    const long long groups = work_groups((long long)A.B * A.Hkv * ((blocks * G + 3) / 4));
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
