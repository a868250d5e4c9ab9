// Attention of a sliding window with sinks, gradients.  With P = exp(x - lse) and delta_i = sum_d dout_i out_i:
//   dS = P (dout V^T - delta) (1 - tanh^2) scale      dQ = dS K      dK = dS^T Q      dV = P^T dout
// Two passes find P again rather than keep it (a score is two products of a block; kept in memory it would be a hundred times the traffic):
//   dq    a wavefront owns 32 queries and walks over the keys as the forward pass does (S^T = K Q^T, dP^T = V dout^T,
//         dQ^T += K^T dS^T); it also leaves delta for the next one
//   dkv   a wavefront owns 32 keys and walks over the rows that see them, of every query head of the KV head in turn
//         (S = Q K^T, dP = dout V^T, dV^T += dout^T P, dK^T += Q^T dS), so the sums over rows and heads have one order and need
//         no atomics: seven products of a block instead of the five that a sum into dQ would take, and the same bits every time.
// The first `sinks` keys are seen by every row.  The rows behind their window are far too many for the wavefronts that own these keys:
// work-groups of their own (far) take them in chunks, leave sums in 32 bits, and the last launch adds them to the owners' in order.
// The products' operands are laid out as in the forward pass (focus_window.h): what is the A operand twice, by rows and by
// components, is turned in registers on its way into LDS.
#include "focus_window.h"

#include <algorithm>

namespace focus {

using namespace window;

namespace {

template <typename T, int D> constexpr int bwd_tile() { return sizeof(T) == 4 || D > 128 ? 32 : 64; }
template <typename T, int D> constexpr int dq_waves() { return D * (int)sizeof(T) > 256 ? 1 : 2; }
template <typename T, int D> constexpr int dkv_waves() { return D * (int)sizeof(T) > 128 ? 1 : 2; }

constexpr int KEYS = 128;                   // keys of a dkv work-group
constexpr int FAR_KEYS = 64;                // ... of a far one: two blocks of 32, each by two wavefronts that share the rows

// Where the sums of the sinks lie in the workspace, and how the far rows are cut.
struct FarPlan {
    int any;                                // some rows may see sinks behind their window
    int near_tiles;                         // key tiles of 128 that hold sinks
    int blocks;                             // blocks of 64 sinks
    int chunk, chunks;                      // rows of a chunk (a multiple of 64); chunks of the longest span
    size_t off_near, off_far, total;        // [B,Hkv,near_tiles][2][128][d], [B,Hkv,blocks,G,chunks,2][2][64][d], bytes from the workspace's base
};

FarPlan far_plan(const WindowArgs& A)
{
    FarPlan f = {};
    const size_t rows = (size_t)(A.packed ? 1 : A.B) * A.Hq * A.n;
    size_t off = (rows * sizeof(float) + 255) & ~(size_t)255;          // delta
    f.any = A.sinks > 0 && A.span_max > A.window;
    if (f.any) {
        const int G = A.Hq / A.Hkv;
        f.near_tiles = (std::min(A.sinks, A.span_max) + KEYS - 1) / KEYS;
        f.blocks = (std::min(A.sinks, A.span_max) + FAR_KEYS - 1) / FAR_KEYS;
        // about two work-groups for each compute unit, of 512 rows at least
        const long long whole = (long long)A.B * A.Hq * f.blocks;
        const int want = (int)std::max(1ll, 512 / std::max(1ll, whole));
        f.chunk = std::max(512, round_up((A.span_max + want - 1) / want, 64));
        f.chunks = (A.span_max + f.chunk - 1) / f.chunk;
        f.off_near = off;
        off += (size_t)A.B * A.Hkv * f.near_tiles * 2 * KEYS * A.d * sizeof(float);
        f.off_far = off;
        off += (size_t)A.B * A.Hkv * f.blocks * G * f.chunks * 2 * 2 * FAR_KEYS * A.d * sizeof(float);
    }
    f.total = off;
    return f;
}

// first far row of the keys of near tile `tile`: the near walk ends with the row tile that holds the last row of the window
template <int R> __host__ __device__ int far_start(int tile, int window) { return ((tile * KEYS + KEYS - 1 + window - 1) / R + 1) * R; }

// P and dS of one lane's 16 pairs: x holds the scores, dp the products of dout and V; seen: pairs that are not visible give zeros
template <bool CAP>
__device__ inline float prob(float x, float c, float ci, float lse2, float* t)
{
    if (CAP) {
        *t = tanhf(x * ci);
        return __builtin_amdgcn_exp2f(fmaf(*t, c, -lse2));
    }
    return __builtin_amdgcn_exp2f(fmaf(x, c, -lse2));
}

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(WTHR, (dq_waves<T, D>())) void window_dq_kernel(WindowArgs A, int tiles, int heads, const T* __restrict__ q,
                                                                           const T* __restrict__ k, const T* __restrict__ v,
                                                                           const T* __restrict__ out, const float* __restrict__ lse,
                                                                           const T* __restrict__ dout, float* __restrict__ delta,
                                                                           T* __restrict__ dq)
{
    constexpr int R = bwd_tile<T, D>();
    typedef Tile<T, D, R> TL;
    typedef Piece<T> P;
    __shared__ __attribute__((aligned(16))) char s_k[TL::RBYTES];
    __shared__ __attribute__((aligned(16))) char s_kc[TL::TBYTES];
    __shared__ __attribute__((aligned(16))) char s_v[TL::RBYTES];
    __shared__ unsigned s_bad[2][2];
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = A.Hq / A.Hkv, shares = G / heads, subs = 4 / heads;
    const long long w = work_of((long long)A.B * A.Hkv * tiles * shares);
    if (w < 0) return;
    const int share = (int)(w % shares), tile = (int)(w / shares % tiles), hk = (int)(w / shares / tiles % A.Hkv);
    const int b = (int)(w / shares / tiles / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    const int tile0 = tile * 32 * subs;
    if (tile0 >= sq.len) return;
    const int row0 = tile0 + 32 * (wave % subs);
    const int h = hk * G + share * heads + wave / subs;
    const int row = row0 + (lane & 31);
    const bool real = row < sq.len;
    const int at = sq.first + (real ? row : sq.len - 1);
    const long long qoff = (long long)sq.tb * A.qs[0] + (long long)h * A.qs[1] + (long long)at * A.qs[2];
    const long long ooff = (long long)sq.tb * A.os[0] + (long long)h * A.os[1] + (long long)at * A.os[2];
    const T* kb = k + (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)sq.first * A.ks[2];
    const T* vb = v + (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)sq.first * A.ks[2];
    const long long li = ((long long)sq.tb * A.Hq + h) * A.n + at;

    u32x4 qf[TL::KS], gf[TL::KS];
    float del = 0.f;
#pragma unroll
    for (int s = 0; s < TL::KS; ++s) {
        qf[s] = load_piece(q + qoff, 2 * s + hh);
        gf[s] = load_piece(dout + ooff, 2 * s + hh);
        del += P::dot(gf[s], load_piece(out + ooff, 2 * s + hh));
    }
    del += other_half(del);
    if (real && hh == 0) delta[li] = del;
    const float lse2 = lse[li] * LOG2E;
    float spoiled = 0.f;                                      // or NaN
    f32x16 acc[TL::DB];
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) acc[i] = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;

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
        __syncthreads();
        if (edge) st.take_out_not_finite(s_bad[t & 1]);
        if (threadIdx.x < 2) s_bad[(t + 1) & 1][threadIdx.x] = 0u;
        st.store(s_k, s_kc, s_v, nullptr);
        __syncthreads();
        if (t + 1 < count) st.load(kb, A.ks[2], vb, A.ks[2], tile_at(t + 1), sq.len);
#pragma unroll 1
        for (int u = 0; u < R / 32; ++u) {
            const Block kind = block_kind(row0, key0 + 32 * u, A.window, A.sinks);
            if (kind == HIDDEN) continue;
            f32x16 x = 0.f, dp = 0.f;
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) {
                x = P::mma(TL::rows_piece(s_k, u, s, lane), qf[s], x);
                dp = P::mma(TL::rows_piece(s_v, u, s, lane), gf[s], dp);
            }
            float ds[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float th = 0.f;
                const float p = prob<CAP>(x[i], c, ci, lse2, &th);
                ds[i] = p * (dp[i] - del);
                if (CAP) ds[i] *= 1.f - th * th;
                if (kind == EDGE)
                    ds[i] = visible(row, key0 + 32 * u + 8 * (i / 4) + 4 * hh + i % 4, A.window, A.sinks) ? ds[i] : 0.f;
            }
#pragma unroll
            for (int s = 0; s < TL::US; ++s) {
                const u32x4 pf = P::pack(ds + s * P::E);
#pragma unroll
                for (int db = 0; db < TL::DB; ++db) acc[db] = P::mma(TL::comps_piece(s_kc, db, u, s, lane), pf, acc[db]);
            }
            const unsigned marks = s_bad[t & 1][u];
            if (edge && marks != 0u && spoiled_by<true>(marks, row, key0 + 32 * u, hh, A.window, A.sinks)) spoiled = __builtin_nanf("");
        }
    }
    spoiled += other_half(spoiled);
    store_row<T, D>(real ? dq + qoff : nullptr, acc, A.scale + spoiled, lane);
}

// FAR: the rows behind the window of 64 sinks, one query head and one chunk of rows per work-group; sums in 32 bits to `part`.
// Otherwise the rows from a key tile's own to the end of its window, of every query head; to dk and dv, or, where far rows
// follow, in 32 bits to `part`.
template <typename T, int D, bool CAP, bool FAR>
__global__ __launch_bounds__(WTHR, (dkv_waves<T, D>())) void window_dkv_kernel(WindowArgs A, FarPlan F, int tiles, const T* __restrict__ q,
                                                                             const T* __restrict__ k, const T* __restrict__ v,
                                                                             const float* __restrict__ lse, const T* __restrict__ dout,
                                                                             const float* __restrict__ delta, float* __restrict__ part,
                                                                             T* __restrict__ dk, T* __restrict__ dv)
{
    constexpr int R = bwd_tile<T, D>();
    typedef Tile<T, D, R> TL;
    typedef Piece<T> P;
    // the keys' and values' operands stay in registers where they fit; above 256 bytes a row they are read again from L1 for every block
    constexpr bool KEEP = D * (int)sizeof(T) <= 256;
    __shared__ __attribute__((aligned(16))) char s_q[TL::RBYTES];
    __shared__ __attribute__((aligned(16))) char s_qc[TL::TBYTES];
    __shared__ __attribute__((aligned(16))) char s_g[TL::RBYTES];
    __shared__ __attribute__((aligned(16))) char s_gc[TL::TBYTES];
    __shared__ __attribute__((aligned(16))) float s_lse[R], s_del[R];
    __shared__ unsigned s_bad[2][2];
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = A.Hq / A.Hkv;
    int b, hk, key0, h0, h1, from, to;                        // keys of the wavefront; heads; rows [from, to) of the walk
    Sequence sq;
    float* slot = nullptr;                                    // [2][KEYS or FAR_KEYS][D] of the work-group
    int slot_row = 0;                                         // first key of the wavefront in it
    if constexpr (FAR) {
        const long long w = work_of((long long)A.B * A.Hkv * F.blocks * G * F.chunks);
        if (w < 0) return;
        const int chunk = (int)(w % F.chunks), g = (int)(w / F.chunks % G), blk = (int)(w / F.chunks / G % F.blocks);
        hk = (int)(w / F.chunks / G / F.blocks % A.Hkv);
        b = (int)(w / F.chunks / G / F.blocks / A.Hkv);
        sq = sequence_of(A, b);
        key0 = blk * FAR_KEYS + 32 * (wave >> 1);
        h0 = hk * G + g;
        h1 = h0 + 1;
        from = max(chunk * F.chunk, far_start<R>(blk * FAR_KEYS / KEYS, A.window));
        to = min((chunk + 1) * F.chunk, sq.len);
        if (from >= to) return;
        slot = part + F.off_far / sizeof(float) + ((size_t)w * 2 + (wave & 1)) * 2 * FAR_KEYS * D;
        slot_row = 32 * (wave >> 1);
    } else {
        const long long w = work_of((long long)A.B * A.Hkv * tiles);
        if (w < 0) return;
        const int tile = (int)(w % tiles);
        hk = (int)(w / tiles % A.Hkv);
        b = (int)(w / tiles / A.Hkv);
        sq = sequence_of(A, b);
        if (tile * KEYS >= sq.len) return;
        key0 = tile * KEYS + 32 * wave;
        h0 = hk * G;
        h1 = h0 + G;
        from = tile * KEYS / R * R;
        to = min(far_start<R>(tile, A.window), sq.len);
        if (F.any && tile < F.near_tiles) {
            slot = part + F.off_near / sizeof(float) + (((size_t)b * A.Hkv + hk) * F.near_tiles + tile) * 2 * KEYS * D;
            slot_row = 32 * wave;
        }
    }
    const int key = key0 + (lane & 31);
    const bool real = key < sq.len;
    const long long koff = (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)(sq.first + (real ? key : sq.len - 1)) * A.ks[2];

    u32x4 kf[KEEP ? TL::KS : 1], vf[KEEP ? TL::KS : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int s = 0; s < TL::KS; ++s) {
            kf[s] = load_piece(k + koff, 2 * s + hh);
            vf[s] = load_piece(v + koff, 2 * s + hh);
        }
    }
    float spoiled = 0.f;                                      // or NaN
    f32x16 ak[TL::DB], av[TL::DB];
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) ak[i] = av[i] = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;
    if (threadIdx.x < 4) s_bad[threadIdx.x >> 1][threadIdx.x & 1] = 0u;

    const int per_head = (to - from + R - 1) / R, count = per_head * (h1 - h0);
    Stage<T, D, R> st;
    float nlse = 0.f, ndel = 0.f;
    auto fetch = [&](int t) {
        const int h = h0 + t / per_head, r0 = from + t % per_head * R;
        st.load(q + (long long)sq.tb * A.qs[0] + (long long)h * A.qs[1] + (long long)sq.first * A.qs[2], A.qs[2],
                dout + (long long)sq.tb * A.os[0] + (long long)h * A.os[1] + (long long)sq.first * A.os[2], A.os[2], r0, to);
        if (threadIdx.x < R) {
            const int r = r0 + threadIdx.x;
            const long long li = ((long long)sq.tb * A.Hq + h) * A.n + sq.first + r;
            nlse = r < to ? lse[li] * LOG2E : INFINITY;       // a row that is not there has probabilities of zero
            ndel = r < to ? delta[li] : 0.f;
        }
    };
    fetch(0);
    for (int t = 0; t < count; ++t) {
        const int row0 = from + t % per_head * R;
        const bool edge = FAR ? true : row0 < key0 - 32 * wave + KEYS || row0 + R - 1 - (key0 - 32 * wave) >= A.window;
        __syncthreads();
        if (edge) st.take_out_not_finite(s_bad[t & 1]);
        if (threadIdx.x < 2) s_bad[(t + 1) & 1][threadIdx.x] = 0u;
        st.store(s_q, s_qc, s_g, s_gc);
        if (threadIdx.x < R) { s_lse[threadIdx.x] = nlse; s_del[threadIdx.x] = ndel; }
        __syncthreads();
        if (t + 1 < count) fetch(t + 1);
        // far: the two wavefronts of a block of keys take the blocks of rows in turn
        const int u0 = FAR && R == 64 ? wave & 1 : 0, u1 = FAR ? (R == 64 ? u0 + 1 : 1 - ((t ^ wave) & 1)) : R / 32;
#pragma unroll 1
        for (int u = u0; u < u1; ++u) {
            const int r0 = row0 + 32 * u;
            const Block kind = block_kind(r0, key0, A.window, A.sinks);
            if (kind == HIDDEN) continue;
            f32x16 x = 0.f, dp = 0.f;
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) {
                const u32x4 kk = KEEP ? kf[KEEP ? s : 0] : load_piece(k + koff, 2 * s + hh);
                const u32x4 vv = KEEP ? vf[KEEP ? s : 0] : load_piece(v + koff, 2 * s + hh);
                x = P::mma(TL::rows_piece(s_q, u, s, lane), kk, x);
                dp = P::mma(TL::rows_piece(s_g, u, s, lane), vv, dp);
            }
            float p[16], ds[16];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const float4 l4 = *(const float4*)(s_lse + 32 * u + 8 * m + 4 * hh), d4 = *(const float4*)(s_del + 32 * u + 8 * m + 4 * hh);
                const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * m + j;
                    float th = 0.f;
                    p[i] = prob<CAP>(x[i], c, ci, ls[j], &th);
                    ds[i] = p[i] * (dp[i] - dl[j]);
                    if (CAP) ds[i] *= 1.f - th * th;
                    if (kind == EDGE) {
                        const int row = r0 + 8 * m + 4 * hh + j;
                        const bool seen = row < to && visible(row, key, A.window, A.sinks);
                        p[i] = seen ? p[i] : 0.f;
                        ds[i] = seen ? ds[i] : 0.f;
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < TL::US; ++s) {
                const u32x4 pf = P::pack(p + s * P::E), df = P::pack(ds + s * P::E);
#pragma unroll
                for (int db = 0; db < TL::DB; ++db) {
                    av[db] = P::mma(TL::comps_piece(s_gc, db, u, s, lane), pf, av[db]);
                    ak[db] = P::mma(TL::comps_piece(s_qc, db, u, s, lane), df, ak[db]);
                }
            }
            const unsigned marks = s_bad[t & 1][u];
            if (edge && marks != 0u && spoiled_by<false>(marks, key, r0, hh, A.window, A.sinks)) spoiled = __builtin_nanf("");
        }
    }
    spoiled += other_half(spoiled);
    if (slot) {
        // (what is at and behind the sinks of a far slot, or behind the sequence, is not read)
        const bool keep = real && (!FAR || key < A.sinks);
        float* at = slot + (size_t)(slot_row + (lane & 31)) * D;
        store_row<float, D>(keep ? at : nullptr, ak, A.scale + spoiled, lane);
        store_row<float, D>(keep ? at + (size_t)(FAR ? FAR_KEYS : KEYS) * D : nullptr, av, 1.f + spoiled, lane);
    } else {
        store_row<T, D>(real ? dk + koff : nullptr, ak, A.scale + spoiled, lane);
        store_row<T, D>(real ? dv + koff : nullptr, av, 1.f + spoiled, lane);
    }
}

// dk and dv of the key tiles that hold sinks: the owner's sums, then the far chunks' head by head and chunk by chunk.
// One work-group per (b, KV head, key), a thread per component of dk, then of dv.
template <typename T, int R>
__global__ __launch_bounds__(WTHR) void window_join_kernel(WindowArgs A, FarPlan F, const float* __restrict__ part, T* __restrict__ dk,
                                                          T* __restrict__ dv)
{
    const int keys = F.near_tiles * KEYS;
    const int key = (int)(blockIdx.x % keys), hk = (int)(blockIdx.x / keys % A.Hkv), b = (int)(blockIdx.x / keys / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    if (key >= sq.len) return;
    const int G = A.Hq / A.Hkv, d = A.d, blk = key / FAR_KEYS;
    const int start = far_start<R>(key / KEYS, A.window);
    const float* near = part + F.off_near / sizeof(float) + (((size_t)b * A.Hkv + hk) * F.near_tiles + key / KEYS) * 2 * KEYS * d;
    const float* far = part + F.off_far / sizeof(float) + (((size_t)b * A.Hkv + hk) * F.blocks + blk) * G * F.chunks * 2 * 2 * FAR_KEYS * d;
    const long long off = (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)(sq.first + key) * A.ks[2];
    for (int i = threadIdx.x; i < 2 * d; i += WTHR) {
        const int which = i >= d, comp = which ? i - d : i;
        float sum = near[((size_t)which * KEYS + key % KEYS) * d + comp];
        if (key < A.sinks)
            for (int g = 0; g < G; ++g)
                for (int c = 0; c < F.chunks; ++c) {
                    if (max(c * F.chunk, start) >= min((c + 1) * F.chunk, sq.len)) continue;
                    for (int half = 0; half < 2; ++half)
                        sum += far[((((size_t)g * F.chunks + c) * 2 + half) * 2 + which) * FAR_KEYS * d + (size_t)(key % FAR_KEYS) * d + comp];
                }
        T* to = (which ? dv : dk) + off + comp;
        const float x[8] = {sum, sum, sum, sum, sum, sum, sum, sum};
        const u32x4 p = Piece<T>::pack(x);
        __builtin_memcpy(to, &p, sizeof(T));
    }
}

template <typename T, int D, bool CAP>
hipError_t launch_cap(const WindowArgs& A, const void* q_, const void* k_, const void* v_, const void* out_, const float* lse, const void* dout_,
                      char* ws, void* dq, void* dk_, void* dv_, hipStream_t st)
{
    const T *q = (const T*)q_, *k = (const T*)k_, *v = (const T*)v_, *out = (const T*)out_, *dout = (const T*)dout_;
    T *dk = (T*)dk_, *dv = (T*)dv_;
    constexpr int R = bwd_tile<T, D>();
    const FarPlan F = far_plan(A);
    float *delta = (float*)ws, *part = (float*)ws;
    const int G = A.Hq / A.Hkv, heads = G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1, rows = 32 * (4 / heads);
    const int tiles = (A.span_max + rows - 1) / rows, ktiles = (A.span_max + KEYS - 1) / KEYS;
    const long long g1 = work_groups((long long)A.B * A.Hkv * tiles * (G / heads)), g2 = work_groups((long long)A.B * A.Hkv * ktiles);
    const long long g3 = F.any ? work_groups((long long)A.B * A.Hkv * F.blocks * G * F.chunks) : 0;
    const long long g4 = F.any ? (long long)A.B * A.Hkv * F.near_tiles * KEYS : 0;
    if (std::max(std::max(g1, g2), std::max(g3, g4)) > 0x7fffffffll) return hipErrorInvalidConfiguration;
    window_dq_kernel<T, D, CAP><<<(unsigned)g1, WTHR, 0, st>>>(A, tiles, heads, q, k, v, out, lse, dout, delta, (T*)dq);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    window_dkv_kernel<T, D, CAP, false><<<(unsigned)g2, WTHR, 0, st>>>(A, F, ktiles, q, k, v, lse, dout, delta, part, dk, dv);
    e = hipGetLastError();
    if (e != hipSuccess || !F.any) return e;
    window_dkv_kernel<T, D, CAP, true><<<(unsigned)g3, WTHR, 0, st>>>(A, F, ktiles, q, k, v, lse, dout, delta, part, dk, dv);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    window_join_kernel<T, R><<<(unsigned)g4, WTHR, 0, st>>>(A, F, part, dk, dv);
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

size_t window_bwd_workspace(const WindowArgs& A) { return far_plan(A).total; }

hipError_t launch_window_bwd(const WindowArgs& A, const void* q, const void* k, const void* v, const void* out, const float* lse,
                             const void* dout, char* ws, void* dq, void* dk, void* dv, hipStream_t st)
{
    if (A.dtype == 0) return launch_t<float>(A, q, k, v, out, lse, dout, ws, dq, dk, dv, st);
    if (A.dtype == 1) return launch_t<uint16_t>(A, q, k, v, out, lse, dout, ws, dq, dk, dv, st);
    return launch_t<f16_bits>(A, q, k, v, out, lse, dout, ws, dq, dk, dv, st);
}

}  // namespace focus
