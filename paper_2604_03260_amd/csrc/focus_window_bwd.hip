// Attention of a sliding window with sinks, gradients.  With P = exp(x - lse) and delta_i = sum_d dout_i out_i:
//   dS = P (dout V^T - delta) (1 - tanh^2) scale      dQ = dS K      dK = dS^T Q      dV = P^T dout
// Two passes find P again rather than keep it (a score is two products of a block; kept in memory it would be a hundred times the traffic):
//   dq    a wavefront owns 32 queries and walks over the keys as the forward pass does (S^T = K Q^T, dP^T = V dout^T,
//         dQ^T += K^T dS^T); it also leaves delta for the next one
//   dkv   a wavefront owns 32 keys and walks over the rows that see them, of every query head of the KV head in turn
//         (S = Q K^T, dP = dout V^T, dV^T += dout^T P, dK^T += Q^T dS), so the sums over rows and heads have one order and need
//         no atomics: the same bits every time, for seven or eight products of a block (dkv_split) in place of the five that one walk would take.
// The first `sinks` keys are seen by every row.  The rows behind their window are far too many for the wavefronts that own these keys:
// work-groups of their own (far) take them in chunks, leave sums in 32 bits, and the last launch adds them to the owners' in order.
// The products' operands lie in LDS as in the forward pass (focus_window.h): what is a first operand twice, by rows and by components, is copied
// once and turned by the LDS reads.  The walk over the keys is the forward kernel's too: two buffers, one barrier per tile of 32, and the
// wavefronts of a SIMD hide each other's waits (two at 128 components of 16 bits; 16384 tokens of 32/8 heads, window 1024: 520 us.  With one
// that found its scores a block ahead and summed a block behind: 606).
#include "focus_window.h"

#include <algorithm>

namespace focus {

using namespace window;

namespace {

// Rows of a dkv tile: what its wavefronts fill evenly.
template <typename T, int D> constexpr int dkv_tile() { return D * (int)sizeof(T) > 512 || (sizeof(T) == 4 && (D == 64 || D == 128)) ? 32 : 64; }
template <typename T, int D> constexpr int dq_waves() { return D * (int)sizeof(T) > 256 ? 1 : D * (int)sizeof(T) > 128 ? 2 : 3; }

constexpr int KEYS = 128;                   // keys of a dkv work-group
constexpr int FAR_KEYS = 32;                // ... of a far one, whose wavefronts share the rows

// Where the sums of the sinks lie in the workspace, and how the far rows are cut.
struct FarPlan {
    int any;                                // some rows may see sinks behind their window
    int near_tiles;                         // key tiles of 128 that hold sinks
    int blocks;                             // blocks of 32 sinks
    int chunk, chunks;                      // rows of a chunk (a multiple of 64); chunks of the longest span
    size_t off_near, off_far, total;        // [B,Hkv,near_tiles][2][128][d], [B,Hkv,blocks,G,chunks][2][32][d], bytes from the workspace's base
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
        // about two work-groups for each compute unit, of 256 rows at least
        const long long whole = (long long)A.B * A.Hq * f.blocks;
        const int want = (int)std::max(1ll, 512 / std::max(1ll, whole));
        f.chunk = std::max(256, round_up((A.span_max + want - 1) / want, 64));
        f.chunks = (A.span_max + f.chunk - 1) / f.chunk;
        f.off_near = off;
        off += (size_t)A.B * A.Hkv * f.near_tiles * 2 * KEYS * A.d * sizeof(float);
        f.off_far = off;
        off += (size_t)A.B * A.Hkv * f.blocks * G * f.chunks * 2 * FAR_KEYS * A.d * sizeof(float);
    }
    f.total = off;
    return f;
}

// first far row of the keys of near tile `tile`: the near walk ends with the block of 32 rows that holds the last row of the window
__host__ __device__ inline int far_start(int tile, int window) { return ((tile * KEYS + KEYS - 1 + window - 1) / 32 + 1) * 32; }

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(WTHR, (dq_waves<T, D>())) void window_dq_kernel(WindowArgs A, int blocks, const T* __restrict__ q,
                                                                           const T* __restrict__ k, const T* __restrict__ v,
                                                                           const T* __restrict__ out, const float* __restrict__ lse,
                                                                           const T* __restrict__ dout, float* __restrict__ delta,
                                                                           T* __restrict__ dq)
{
    constexpr int R = 32;
    typedef Tile<T, D, R> TL;
    typedef Piece<T> P;
    __shared__ __attribute__((aligned(256))) char s_k[2][TL::BYTES], s_v[2][TL::BYTES];
    __shared__ unsigned s_bad[2];
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = A.Hq / A.Hkv, fours = (blocks * G + 3) / 4;
    const long long w = work_of((long long)A.B * A.Hkv * fours);
    if (w < 0) return;
    const int four = (int)(w % fours), hk = (int)(w / fours % A.Hkv), b = (int)(w / fours / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    const int tile0 = four * 4 / G * 32;
    if (tile0 >= sq.len) return;
    const int row0 = (four * 4 + wave) / G * 32;
    const int h = hk * G + (four * 4 + wave) % G;
    const bool idle = row0 >= sq.len;
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
    del = halves_sum(del);
    if (real && hh == 0) delta[li] = del;
    const float lse2 = lse[li] * LOG2E;
    float spoiled = 0.f;                                      // or NaN
    f32x16 acc[TL::DB];
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) acc[i] = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;

    const int rplace = TL::rows_place(lane), cplace = TL::comps_place(lane);
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
    landed(gf);
#pragma unroll 1
    for (int t = 0; t < W.tiles; ++t) {
        const int buf = t & 1, key0 = W.key_at(t);
        dma_wait();
        __syncthreads();
        const bool edge = W.edge(key0, A);
        if (edge) {
            scrub<T, D, R>(s_k[buf], &s_bad[buf], threadIdx.x, WTHR);
            __syncthreads();
        }
        if (t + 1 < W.tiles) fetch(t + 1);
        const Block kind = idle ? HIDDEN : block_kind(row0, key0, A.window, A.sinks);
        if (kind != HIDDEN) {
            const int rp = opaque(rplace), cp = opaque(cplace);
            f32x16 x = 0.f, dx = 0.f;
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) {
                x = P::mma(TL::rows_piece(s_k[buf], rp, s), qf[s], x);
                dx = P::mma(TL::rows_piece(s_v[buf], rp, s), gf[s], dx);
            }
            settle<T>();
            if (CAP) tanh_scores<T>(x, ci);
            if (kind == EDGE) {                               // hidden: an exponent of -inf, and dP = delta
                const int key = opaque(key0 + 4 * hh);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool seen = visible(row, key + 8 * (i / 4) + i % 4, A.window, A.sinks);
                    x[i] = seen ? x[i] : CAP ? -1e30f : -INFINITY;
                    dx[i] = seen ? dx[i] : 0.f;
                }
            }
            u32x4 pf[TL::US];
#pragma unroll
            for (int s = 0; s < TL::US; ++s) {
                float ds[8];
#pragma unroll
                for (int j = 0; j < P::E; ++j) {
                    const float z = x[s * P::E + j];
                    ds[j] = __builtin_amdgcn_exp2f(fmaf(z, c, -lse2)) * (dx[s * P::E + j] - del);
                    if (CAP) ds[j] = z > -2.f ? ds[j] * (1.f - z * z) : 0.f;
                }
                pf[s] = P::pack(ds);
            }
#pragma unroll
            for (int s = 0; s < TL::US; ++s)
#pragma unroll
                for (int db = 0; db < TL::DB; ++db) acc[db] = P::mma(TL::comps_piece(s_k[buf], cp, db, s), pf[s], acc[db]);
            settle<T>();
            if (edge) {
                const unsigned marks = s_bad[buf];
                if (marks != 0u && spoiled_by<true>(marks, row, key0, hh, A.window, A.sinks)) spoiled = __builtin_nanf("");
            }
        }
        if (edge) {                                           // (the marks have been seen by all before they go)
            __syncthreads();
            if (threadIdx.x == 0) s_bad[buf] = 0u;
        }
    }
    if (idle) return;
    spoiled = halves_sum(spoiled);
    store_row<T, D>(real ? dq + qoff : nullptr, acc, A.scale + spoiled, lane);
}

// P of a lane's 16 pairs from its scores (tanh of them with a softcap), or dS from these and dP (grad), packed as operands.  ls, dl: the
// log-sum-exps (log2 units) and deltas of the 16 rows, in LDS.  A pair that is hidden has a score of -inf (softcap: -1e30) and dP = 0.
template <typename T, bool CAP>
__device__ inline void probabilities(const f32x16& x, const f32x16& dp, float c, const float* ls, const float* dl, int hh, bool grad, u32x4* out)
{
    typedef Piece<T> P;
    constexpr int US = 16 / P::E;
    float p[16];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const float4 l4 = *(const float4*)(ls + 8 * m + 4 * hh);
        const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) p[4 * m + j] = __builtin_amdgcn_exp2f(fmaf(x[4 * m + j], c, -lv[j]));
    }
    if (grad) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const float4 d4 = *(const float4*)(dl + 8 * m + 4 * hh);
            const float dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = 4 * m + j;
                p[i] *= dp[i] - dv[j];
                if (CAP) p[i] = x[i] > -2.f ? p[i] * (1.f - x[i] * x[i]) : 0.f;
            }
        }
    }
#pragma unroll
    for (int s = 0; s < US; ++s) out[s] = P::pack(p + s * P::E);
}

// The rows from a key tile's own to the end of its window, of every query head; to dk and dv, or, where far rows follow, in 32 bits to `part`.
// Two wavefronts fit a SIMD if the sums of one are those of dK or of dV (dkv_split; not at 64 components of 16 bits): eight wavefronts, two for
// each 32 keys.  Both find the scores (ten products of a block in place of eight), but with one that held all sums, every wait, barrier and
// vector instruction was in the way of the products (16384 tokens of 32/8 heads of 128, window 1024: 1214 us, split 995; at 64 components,
// 8 x 4096 tokens of 12 heads, window 256: 165 us with both, split 277).
template <typename T, int D> constexpr bool dkv_split() { return D * (int)sizeof(T) > 128; }
template <typename T, int D> constexpr int dkv_threads() { return dkv_split<T, D>() ? 512 : 256; }
template <typename T, int D, bool CAP>
__global__ __launch_bounds__((dkv_threads<T, D>()), 2) void window_dkv_kernel(WindowArgs A, FarPlan F, int tiles, const T* __restrict__ q, const T* __restrict__ k,
                                                              const T* __restrict__ v, const float* __restrict__ lse,
                                                              const T* __restrict__ dout, const float* __restrict__ delta,
                                                              float* __restrict__ part, T* __restrict__ dk, T* __restrict__ dv)
{
    constexpr int R = dkv_tile<T, D>(), U = R / 32;
    typedef Tile<T, D, R> TL;
    typedef Piece<T> P;
    // the keys' and values' operands stay in registers where they fit; above 256 bytes a row they are read again from L1 for every block
    constexpr bool KEEP = D * (int)sizeof(T) <= 256, SPLIT = dkv_split<T, D>();
    __shared__ __attribute__((aligned(256))) char s_q[2][TL::BYTES], s_g[2][TL::BYTES];
    __shared__ __attribute__((aligned(16))) float s_lse[2][R], s_del[2][R];
    __shared__ unsigned s_bad[2][2], s_lost[2][2];
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool sum_k = !SPLIT || wave >= 4, sum_v = !SPLIT || wave < 4;
    const int G = A.Hq / A.Hkv;
    const long long w = work_of((long long)A.B * A.Hkv * tiles);
    if (w < 0) return;
    const int tile = (int)(w % tiles), hk = (int)(w / tiles % A.Hkv), b = (int)(w / tiles / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    if (tile * KEYS >= sq.len) return;
    const int tkey = tile * KEYS, key0 = tkey + 32 * (wave & 3);        // keys of the work-group, of the wavefront
    const int from = tkey, to = min(far_start(tile, A.window), sq.len);
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
    f32x16 acc[TL::DB], both[SPLIT ? 1 : TL::DB];             // dK or dV; dV beside dK
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) acc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < (SPLIT ? 1 : TL::DB); ++i) both[i] = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;

    // the walk: tiles of R rows, head after head, th of each head (rows behind `to` in the last one are hidden)
    const int th = (to - from + R - 1) / R, ntiles = th * G;
    // a tile of the walk: first row (from + j R), and where its rows and sums lie
    struct Cursor {
        int t, j, row;
        const T *q, *g;
        long long sums;
    };
    const long long qhead = A.qs[1], ghead = A.os[1], qstep = (long long)R * A.qs[2], gstep = (long long)R * A.os[2];
    Cursor next;                                              // the next tile to be fetched
    next.t = next.j = 0;
    next.row = from;
    next.q = q + (long long)sq.tb * A.qs[0] + (long long)hk * G * qhead + (long long)(sq.first + from) * A.qs[2];
    next.g = dout + (long long)sq.tb * A.os[0] + (long long)hk * G * ghead + (long long)(sq.first + from) * A.os[2];
    next.sums = ((long long)sq.tb * A.Hq + hk * G) * A.n + sq.first + from;
    auto advance = [&](Cursor& c) WINDOW_INLINE {
        ++c.t;
        if (++c.j < th) {
            c.row += R;
            c.q += qstep;
            c.g += gstep;
            c.sums += R;
        } else {
            const int back = th - 1;
            c.j = 0;
            c.row = from;
            c.q += qhead - back * qstep;
            c.g += ghead - back * gstep;
            c.sums += A.n - (long long)back * R;
        }
    };
    const int qpitch = (int)(A.qs[2] * (long long)sizeof(T)), gpitch = (int)(A.os[2] * (long long)sizeof(T));
    Dma<T, D, R, SPLIT ? 8 : 4> qdma, gdma;
    qdma.init(wave, lane, qpitch);
    gdma.init(wave, lane, gpitch);
    auto edge_row = [&](int row) WINDOW_INLINE { return row < tkey + KEYS || row + R - 1 - tkey >= A.window; };
    float nlse = 0.f, ndel = 0.f;
    auto fetch = [&]() WINDOW_INLINE {                         // rows, log-sum-exps and deltas of a tile
        const int buf = next.t & 1;
        qdma.load(next.q, qpitch, to - next.row, s_q[buf], wave, lane);
        gdma.load(next.g, gpitch, to - next.row, s_g[buf], wave, lane);
        if (wave == 0 && lane < R) {
            const bool there = next.row + lane < to;
            nlse = there ? lse[next.sums + lane] * LOG2E : INFINITY;    // a row that is not there has probabilities of zero
            ndel = there ? delta[next.sums + lane] : 0.f;
        }
    };
    // (a row whose sums are not finite would spoil keys that do not see it: in a tile with hidden pairs it is taken out and marked)
    auto put_sums = [&](int t, int row) WINDOW_INLINE {
        if (wave != 0) return;
        bool lost = false;
        if (edge_row(row)) {
            lost = lane < R && row + lane < to && !(fabsf(nlse) < INFINITY && fabsf(ndel) < INFINITY);
            nlse = lost ? INFINITY : nlse;
            ndel = lost ? 0.f : ndel;
        }
        const unsigned long long all = __ballot(lost);
        if (lane == 0) { s_lost[t & 1][0] = (unsigned)all; s_lost[t & 1][1] = (unsigned)(all >> 32); }
        if (lane < R) { s_lse[t & 1][lane] = nlse; s_del[t & 1][lane] = ndel; }
    };
    if (threadIdx.x < 4) s_bad[threadIdx.x >> 1][threadIdx.x & 1] = 0u;
    fetch();
    if constexpr (KEEP) {
        landed(kf);
        landed(vf);
    }
    const int rplace = TL::rows_place(lane), cplace = TL::comps_place(lane);
#pragma unroll 1
    for (int t = 0; t < ntiles; ++t) {
        const int row_t = next.row, buf = t & 1;
        put_sums(t, row_t);                                   // (read two tiles ago, before a barrier)
        dma_wait();
        __syncthreads();
        const bool edge = edge_row(row_t);
        if (edge) {
            scrub<T, D, R>(s_q[buf], s_bad[buf], threadIdx.x, dkv_threads<T, D>());
            scrub<T, D, R>(s_g[buf], s_bad[buf], threadIdx.x, dkv_threads<T, D>());
            __syncthreads();
        }
        advance(next);
        if (t + 1 < ntiles) fetch();
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
            const int row0 = row_t + 32 * u;
            const Block kind = row0 >= to ? HIDDEN : block_kind(row0, key0, A.window, A.sinks);
            if (kind == HIDDEN) continue;
            const char *qb = s_q[buf] + TL::BLOCK * u, *gb = s_g[buf] + TL::BLOCK * u;
            const int rp = opaque(rplace), cp = opaque(cplace);
            f32x16 x = 0.f, dx = 0.f;
#pragma unroll
            for (int s = 0; s < TL::KS; ++s) x = P::mma(TL::rows_piece(qb, rp, s), KEEP ? kf[KEEP ? s : 0] : load_piece(k + koff, 2 * s + hh), x);
            if (sum_k) {
#pragma unroll
                for (int s = 0; s < TL::KS; ++s) dx = P::mma(TL::rows_piece(gb, rp, s), KEEP ? vf[KEEP ? s : 0] : load_piece(v + koff, 2 * s + hh), dx);
            }
            if (CAP) tanh_scores<T>(x, ci);
            if (kind == EDGE || row0 + 32 > to) {
                const int row = opaque(row0 + 4 * hh);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = row + 8 * (i / 4) + i % 4;
                    const bool seen = (bool)((int)(r < to) & (int)visible(r, key, A.window, A.sinks));
                    x[i] = seen ? x[i] : CAP ? -1e30f : -INFINITY;
                    dx[i] = seen ? dx[i] : 0.f;
                }
            }
            const float *ls = &s_lse[buf][32 * u], *dl = &s_del[buf][32 * u];
            u32x4 w4[TL::US];
            if constexpr (SPLIT) {
                probabilities<T, CAP>(x, dx, c, ls, dl, hh, sum_k, w4);
                const char* tb = sum_k ? qb : gb;
#pragma unroll
                for (int s = 0; s < TL::US; ++s)
#pragma unroll
                    for (int db = 0; db < TL::DB; ++db) acc[db] = P::mma(TL::comps_piece(tb, cp, db, s), w4[s], acc[db]);
            } else {
                u32x4 p4[TL::US];
                probabilities<T, CAP>(x, dx, c, ls, dl, hh, false, p4);
                probabilities<T, CAP>(x, dx, c, ls, dl, hh, true, w4);
#pragma unroll
                for (int s = 0; s < TL::US; ++s)
#pragma unroll
                    for (int db = 0; db < TL::DB; ++db) {
                        both[db] = P::mma(TL::comps_piece(gb, cp, db, s), p4[s], both[db]);
                        acc[db] = P::mma(TL::comps_piece(qb, cp, db, s), w4[s], acc[db]);
                    }
            }
            if (edge) {
                const unsigned marks = s_bad[buf][u] | s_lost[buf][u];
                if (marks != 0u && spoiled_by<false>(marks, key, row0, hh, A.window, A.sinks)) spoiled = __builtin_nanf("");
            }
        }
        if (edge) {                                           // (the marks have been seen by all before they go)
            __syncthreads();
            if (threadIdx.x < 2) s_bad[buf][threadIdx.x] = 0u;
        }
    }
    spoiled = halves_sum(spoiled);
    const bool sum_here = F.any && tile < F.near_tiles;
    float* at = part + F.off_near / sizeof(float) + (((size_t)b * A.Hkv + hk) * F.near_tiles + tile) * 2 * KEYS * D + (size_t)(key - tkey) * D;
    if (sum_k) {
        if (sum_here) store_row<float, D>(real ? at : nullptr, acc, A.scale + spoiled, lane);
        else store_row<T, D>(real ? dk + koff : nullptr, acc, A.scale + spoiled, lane);
    }
    if (sum_v) {
        const f32x16* sums = SPLIT ? acc : both;
        if (sum_here) store_row<float, D>(real ? at + (size_t)KEYS * D : nullptr, sums, 1.f + spoiled, lane);
        else store_row<T, D>(real ? dv + koff : nullptr, sums, 1.f + spoiled, lane);
    }
}

// The rows behind the window of 32 sinks, one query head and one chunk of rows per work-group: its wavefronts take blocks of 32 rows in turn, each
// by itself, through LDS of its own, and join their sums in LDS, in order.
template <typename T, int D> constexpr int far_waves() { return D > 128 ? 2 : 4; }     // (what fits LDS)
template <typename T, int D, bool CAP>
__global__ __launch_bounds__((64 * far_waves<T, D>()), 1) void window_far_kernel(WindowArgs A, FarPlan F, const T* __restrict__ q,
                                                                             const T* __restrict__ k, const T* __restrict__ v,
                                                                             const float* __restrict__ lse, const T* __restrict__ dout,
                                                                             const float* __restrict__ delta, float* __restrict__ part)
{
    typedef Tile<T, D, 32> TL;
    typedef Piece<T> P;
    constexpr int WAVES = far_waves<T, D>();
    constexpr bool KEEP = D * (int)sizeof(T) <= 256;
    constexpr int PER = 2 * TL::BYTES + 256;                  // of a wavefront: Q and dout, lse and delta of the rows
    constexpr int JOIN = 2 * FAR_KEYS * (D + 4) * 4;
    __shared__ __attribute__((aligned(256))) char smem[WAVES * PER > JOIN ? WAVES * PER : JOIN];
    const int lane = threadIdx.x & 63, hh = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = A.Hq / A.Hkv;
    const long long w = work_of((long long)A.B * A.Hkv * F.blocks * G * F.chunks);
    if (w < 0) return;
    const int chunk = (int)(w % F.chunks), g = (int)(w / F.chunks % G), blk = (int)(w / F.chunks / G % F.blocks);
    const int hk = (int)(w / F.chunks / G / F.blocks % A.Hkv), b = (int)(w / F.chunks / G / F.blocks / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    const int from = max(chunk * F.chunk, far_start(blk * FAR_KEYS / KEYS, A.window)), to = min((chunk + 1) * F.chunk, sq.len);
    if (from >= to) return;
    const int h = hk * G + g, key = blk * FAR_KEYS + col;
    const bool sink = key < A.sinks;                          // (from > every key of the block: a sink is seen by all these rows)
    const long long koff = (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)(sq.first + (sink ? key : A.sinks - 1)) * A.ks[2];
    const T* qb = q + (long long)sq.tb * A.qs[0] + (long long)h * A.qs[1] + (long long)sq.first * A.qs[2];
    const T* gb = dout + (long long)sq.tb * A.os[0] + (long long)h * A.os[1] + (long long)sq.first * A.os[2];
    const long long lb = ((long long)sq.tb * A.Hq + h) * A.n + sq.first;
    char *qt = smem + wave * PER, *gt = qt + TL::BYTES;
    float *ls = (float*)(gt + TL::BYTES), *dl = ls + 32;
    const int qpitch = (int)(A.qs[2] * (long long)sizeof(T)), gpitch = (int)(A.os[2] * (long long)sizeof(T));
    Dma<T, D, 32, 1> qdma, gdma;
    qdma.init(0, lane, qpitch);
    gdma.init(0, lane, gpitch);

    u32x4 kf[KEEP ? TL::KS : 1], vf[KEEP ? TL::KS : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int s = 0; s < TL::KS; ++s) {
            kf[s] = load_piece(k + koff, 2 * s + hh);
            vf[s] = load_piece(v + koff, 2 * s + hh);
        }
    }
    f32x16 ak[TL::DB], av[TL::DB];
#pragma unroll
    for (int i = 0; i < TL::DB; ++i) ak[i] = av[i] = 0.f;
    const float c = CAP ? A.softcap * LOG2E : A.scale * LOG2E;
    const float ci = CAP ? A.scale / A.softcap : 0.f;
    const int rplace = TL::rows_place(lane), cplace = TL::comps_place(lane);
    for (int row0 = from + 32 * wave; row0 < to; row0 += 32 * WAVES) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the block before has been read
        qdma.load(qb + (long long)row0 * A.qs[2], qpitch, to - row0, qt, 0, lane);
        gdma.load(gb + (long long)row0 * A.os[2], gpitch, to - row0, gt, 0, lane);
        const int r = min(row0 + col, to - 1);
        const float l1 = row0 + col < to ? lse[lb + r] * LOG2E : INFINITY, d1 = row0 + col < to ? delta[lb + r] : 0.f;
        if (hh == 0) { ls[col] = l1; dl[col] = d1; }
        dma_wait();
        own_fence();
        f32x16 x = 0.f, dx = 0.f;
#pragma unroll
        for (int s = 0; s < TL::KS; ++s) {
            const u32x4 kk = KEEP ? kf[KEEP ? s : 0] : load_piece(k + koff, 2 * s + hh);
            const u32x4 vv = KEEP ? vf[KEEP ? s : 0] : load_piece(v + koff, 2 * s + hh);
            x = P::mma(TL::rows_piece(qt, rplace, s), kk, x);
            dx = P::mma(TL::rows_piece(gt, rplace, s), vv, dx);
        }
        if (CAP) tanh_scores<T>(x, ci);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool there = row0 + 8 * (i / 4) + 4 * hh + i % 4 < to;
            x[i] = there ? x[i] : CAP ? -1e30f : -INFINITY;
            dx[i] = there ? dx[i] : 0.f;
        }
        u32x4 pf[TL::US], df[TL::US];
        probabilities<T, CAP>(x, dx, c, ls, dl, hh, false, pf);
        probabilities<T, CAP>(x, dx, c, ls, dl, hh, true, df);
#pragma unroll
        for (int s = 0; s < TL::US; ++s)
#pragma unroll
            for (int db = 0; db < TL::DB; ++db) {
                av[db] = P::mma(TL::comps_piece(gt, cplace, db, s), pf[s], av[db]);
                ak[db] = P::mma(TL::comps_piece(qt, cplace, db, s), df[s], ak[db]);
            }
    }
    float* sum = (float*)smem;                                // [2][32][D + 4]
    for (int turn = 0; turn < WAVES; ++turn) {
        __syncthreads();
        if (wave != turn) continue;
#pragma unroll
        for (int db = 0; db < TL::DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int comp = 32 * db + 8 * (i / 4) + 4 * hh + i % 4;
                if (comp >= D) continue;
                float *a = sum + col * (D + 4) + comp, *z = a + FAR_KEYS * (D + 4);
                *a = (turn ? *a : 0.f) + ak[db][i] * A.scale;
                *z = (turn ? *z : 0.f) + av[db][i];
            }
    }
    __syncthreads();
    float* slot = part + F.off_far / sizeof(float) + (size_t)w * 2 * FAR_KEYS * D;
    const int sinks = min(FAR_KEYS, A.sinks - blk * FAR_KEYS);          // (what lies behind them is not read)
    for (int i = threadIdx.x; i < 2 * sinks * D; i += 64 * WAVES) {
        const int which = i / (sinks * D), j = i % (sinks * D);
        slot[(size_t)which * FAR_KEYS * D + j] = sum[(which * FAR_KEYS + j / D) * (D + 4) + j % D];
    }
}

// dk and dv of the key tiles that hold sinks: the owner's sums, then the far chunks' head by head and chunk by chunk.  A sink takes a work-group, its
// far sums in 16 shares that are joined in order; the other keys of these tiles 16 to a work-group, rounded.
constexpr int JOIN_THR = 1024;
template <typename T>
__global__ __launch_bounds__(JOIN_THR) void window_join_kernel(WindowArgs A, FarPlan F, const float* __restrict__ part, T* __restrict__ dk,
                                                              T* __restrict__ dv)
{
    __shared__ float s_sum[16][64];
    const int keys = F.near_tiles * KEYS, sinks = min(A.sinks, keys), groups = sinks + (keys - sinks + 15) / 16;
    const int g = (int)(blockIdx.x % groups), hk = (int)(blockIdx.x / groups % A.Hkv), b = (int)(blockIdx.x / groups / A.Hkv);
    const Sequence sq = sequence_of(A, b);
    const int share = threadIdx.x >> 6, c0 = threadIdx.x & 63, G = A.Hq / A.Hkv, d = A.d;
    const bool sink = g < sinks;
    const int key = sink ? g : sinks + (g - sinks) * 16 + share;
    const bool there = key < keys && key < sq.len;
    if (sink && !there) return;
    const int start = far_start(key / KEYS, A.window);
    // far chunks that have rows: from the one that holds `start` on
    const int c1 = start / F.chunk, n = sink && start < sq.len ? (sq.len - 1) / F.chunk - c1 + 1 : 0;
    const float* near = part + F.off_near / sizeof(float) + (((size_t)b * A.Hkv + hk) * F.near_tiles + key / KEYS) * 2 * KEYS * d;
    const float* far = part + F.off_far / sizeof(float) + ((((size_t)b * A.Hkv + hk) * F.blocks + key / FAR_KEYS) * G * F.chunks * 2 * FAR_KEYS +
                                                          key % FAR_KEYS) * d;
    const long long off = (long long)sq.tb * A.ks[0] + (long long)hk * A.ks[1] + (long long)(sq.first + key) * A.ks[2];
    for (int i = c0; i < round_up(2 * d, 64); i += 64) {
        const int which = i >= d, comp = which ? i - d : i;
        const bool mine = there && i < 2 * d;
        float sum = mine && (!sink || share == 0) ? near[((size_t)which * KEYS + key % KEYS) * d + comp] : 0.f;
        if (sink) {
            if (mine) {
#pragma unroll 4
                for (int j = share * G * n / 16; j < (share + 1) * G * n / 16; ++j)
                    sum += far[((size_t)(j / n) * F.chunks + c1 + j % n) * 2 * FAR_KEYS * d + (size_t)which * FAR_KEYS * d + comp];
            }
            s_sum[share][c0] = sum;
            __syncthreads();
            sum = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) sum += s_sum[j][c0];
            __syncthreads();
        }
        if (mine && (!sink || share == 0)) {
            const float y[8] = {sum, sum, sum, sum, sum, sum, sum, sum};
            const u32x4 p = Piece<T>::pack(y);
            __builtin_memcpy((which ? dv : dk) + off + comp, &p, sizeof(T));
        }
    }
}

template <typename T, int D, bool CAP>
hipError_t launch_cap(const WindowArgs& A, const void* q_, const void* k_, const void* v_, const void* out_, const float* lse, const void* dout_,
                      char* ws, void* dq, void* dk_, void* dv_, hipStream_t st)
{
    const T *q = (const T*)q_, *k = (const T*)k_, *v = (const T*)v_, *out = (const T*)out_, *dout = (const T*)dout_;
    T *dk = (T*)dk_, *dv = (T*)dv_;
    const FarPlan F = far_plan(A);
    float *delta = (float*)ws, *part = (float*)ws;
    const int G = A.Hq / A.Hkv, blocks = (A.span_max + 31) / 32, ktiles = (A.span_max + KEYS - 1) / KEYS;
    const long long g1 = work_groups((long long)A.B * A.Hkv * ((blocks * G + 3) / 4)), g2 = work_groups((long long)A.B * A.Hkv * ktiles);
    const long long g3 = F.any ? work_groups((long long)A.B * A.Hkv * F.blocks * G * F.chunks) : 0;
    const int near_keys = F.near_tiles * KEYS, sinks = std::min(A.sinks, near_keys);
    const long long g4 = F.any ? (long long)A.B * A.Hkv * (sinks + (near_keys - sinks + 15) / 16) : 0;
    if (std::max(std::max(g1, g2), std::max(g3, g4)) > 0x7fffffffll) return hipErrorInvalidConfiguration;
    window_dq_kernel<T, D, CAP><<<(unsigned)g1, WTHR, 0, st>>>(A, blocks, q, k, v, out, lse, dout, delta, (T*)dq);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    window_dkv_kernel<T, D, CAP><<<(unsigned)g2, dkv_threads<T, D>(), 0, st>>>(A, F, ktiles, q, k, v, lse, dout, delta, part, dk, dv);
    e = hipGetLastError();
    if (e != hipSuccess || !F.any) return e;
    window_far_kernel<T, D, CAP><<<(unsigned)g3, 64 * far_waves<T, D>(), 0, st>>>(A, F, q, k, v, lse, dout, delta, part);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    window_join_kernel<T><<<(unsigned)g4, JOIN_THR, 0, st>>>(A, F, part, dk, dv);
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
