// Attention of a sliding window with sinks, forward: row i sees key j iff j <= i and (i - j < window or j < sinks).
//
// One pass over the keys a tile of rows can see, with a running reference and sum of the softmax:
//   S^T = K Q^T  (A = keys by rows, B = the wavefront's 32 queries, held in registers)
//   P^T = exp2(scale' S^T - m), one row of the softmax per lane (and half-wave), so its maximum and sum are sums in a lane
//   O^T += V^T P^T (A = values by components; P^T is the B operand as the first product left it, focus_window.h)
// A work-group is four wavefronts of 32 rows each that share the staged keys: of up to four query heads of one KV head (the same rows: the
// four walk in step and the walk is as short as the window allows), else of consecutive rows.  Keys come through registers
// (the next tile's loads are on their way during the products of this one); values are turned there (16 v_perm per 4 x 8 components), so
// no copy of them in another order is needed and the call is one launch without workspace.
// The reference m of a row moves only when its maximum has risen by more than 8 (log2 units): O is rarely rescaled, and the
// probabilities stay below 2^8.  IEEE halves lose bits below 2^-14: there the reference lies 6 lower, so what is dropped is below 2^-31 of the
// largest, 2^-11 of the sum over 2^20 keys.
#include "focus_window.h"

namespace focus {

using namespace window;

namespace {

template <typename T, int D> constexpr int key_tile() { return sizeof(T) == 4 || D > 128 ? 32 : 64; }
// wavefronts per SIMD: the queries and the output of 256 components (fp32: above 96) alone fill half of the registers
template <typename T, int D> constexpr int fwd_waves() { return D * (int)sizeof(T) > 384 ? 1 : 2; }

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(WTHR, (fwd_waves<T, D>())) void window_fwd_kernel(WindowArgs A, int tiles, int heads, const T* __restrict__ q,
                                                                             const T* __restrict__ k, const T* __restrict__ v,
                                                                             T* __restrict__ out, float* __restrict__ lse)
{
    constexpr int R = key_tile<T, D>();
    typedef Tile<T, D, R> TL;
    typedef Piece<T> P;
    __shared__ __attribute__((aligned(16))) char s_k[TL::RBYTES];
    __shared__ __attribute__((aligned(16))) char s_v[TL::TBYTES];
    __shared__ unsigned s_bad[2][2];
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // (b, KV head, tile of rows, share of the query heads), the last one fastest
    const int G = A.Hq / A.Hkv, shares = G / heads, subs = 4 / heads;
    const long long w = work_of((long long)A.B * A.Hkv * tiles * shares);
    if (w < 0) return;
    const int share = (int)(w % shares), tile = (int)(w / shares % tiles), hk = (int)(w / shares / tiles % A.Hkv);
    const int b = (int)(w / shares / tiles / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    const int tile0 = tile * 32 * subs;                       // first row of the work-group, of the wavefront
    if (tile0 >= sq.len) return;
    const int row0 = tile0 + 32 * (wave % subs);
    const int h = hk * G + share * heads + wave / subs;
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
    constexpr float LOWER = sizeof(T) == 4 ? 0.f : P::EXP == 0x7c007c00u ? 6.f : 0.f;       // IEEE halves, see above
    float m = -1e30f, l = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;

    // tiles with sinks, then those from the first key of the window on
    const int last = min(tile0 + 32 * subs, sq.len) - 1;
    const int sink_tiles = (min(A.sinks, last + 1) + R - 1) / R;
    const int near0 = max(sink_tiles, max(0, tile0 - A.window + 1) / R);
    const int count = sink_tiles + max(0, last / R - near0 + 1);
    auto tile_at = [&](int t) { return (t < sink_tiles ? t : near0 + t - sink_tiles) * R; };

    if (threadIdx.x < 4) s_bad[threadIdx.x >> 1][threadIdx.x & 1] = 0u;
    Stage<T, D, R> st;
    st.load(kb, A.ks[2], vb, A.ks[2], tile_at(0), sq.len);
    for (int t = 0; t < count; ++t) {
        const int key0 = tile_at(t);
        const bool edge = key0 + R - 1 > tile0 || (last - key0 >= A.window && key0 + R - 1 >= A.sinks);
        __syncthreads();                                      // the tile before has been read
        if (edge) st.take_out_not_finite(s_bad[t & 1]);
        if (threadIdx.x < 2) s_bad[(t + 1) & 1][threadIdx.x] = 0u;
        st.store(s_k, nullptr, nullptr, s_v);
        __syncthreads();
        if (t + 1 < count) st.load(kb, A.ks[2], vb, A.ks[2], tile_at(t + 1), sq.len);

#pragma unroll 1
        for (int u = 0; u < R / 32; ++u) {
            const Block kind = block_kind(row0, key0 + 32 * u, A.window, A.sinks);
            if (kind == HIDDEN) continue;
            f32x16 x = 0.f;
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) x = P::mma(TL::rows_piece(s_k, u, s, lane), qf[s], x);
            if (CAP) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = tanhf(x[i] * ci);
            }
            if (kind == EDGE) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[i] = visible(row, key0 + 32 * u + 8 * (i / 4) + 4 * hh + i % 4, A.window, A.sinks) ? x[i] : -INFINITY;
            }
            float top = x[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
            top = fmaxf(top, other_half(top)) * c;
            if (__any(top > m + LOWER + 8.f)) {
                const float to = fmaxf(m, top - LOWER), f = exp2f(m - to);
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
            u32x4 pf[TL::US];
#pragma unroll
            for (int s = 0; s < TL::US; ++s) pf[s] = P::pack(p + s * P::E);
#pragma unroll
            for (int s = 0; s < TL::US; ++s)
#pragma unroll
                for (int db = 0; db < TL::DB; ++db) o[db] = P::mma(TL::comps_piece(s_v, db, u, s, lane), pf[s], o[db]);
            const unsigned marks = s_bad[t & 1][u];
            if (edge && marks != 0u && spoiled_by<true>(marks, row, key0 + 32 * u, hh, A.window, A.sinks)) l = __builtin_nanf("");
        }
    }
    l += other_half(l);
    T* orow = real ? out + (long long)sq.tb * A.os[0] + (long long)h * A.os[1] + (long long)(sq.first + row) * A.os[2] : nullptr;
    store_row<T, D>(orow, o, 1.f / l, lane);
    if (lse && real && hh == 0) lse[((long long)sq.tb * A.Hq + h) * A.n + sq.first + row] = (m + log2f(l)) * LN2;
}

template <typename T, int D, bool CAP>
hipError_t launch_cap(const WindowArgs& A, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st)
{
    const int G = A.Hq / A.Hkv, heads = G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1, rows = 32 * (4 / heads);
    const int tiles = (A.span_max + rows - 1) / rows;
    const long long groups = work_groups((long long)A.B * A.Hkv * tiles * (G / heads));
    if (groups > 0x7fffffffll) return hipErrorInvalidConfiguration;
    window_fwd_kernel<T, D, CAP><<<(unsigned)groups, WTHR, 0, st>>>(A, tiles, heads, (const T*)q, (const T*)k, (const T*)v, (T*)out, lse);
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
