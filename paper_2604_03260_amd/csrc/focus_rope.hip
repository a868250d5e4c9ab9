// Positions and head norms in front of the attention, q and k in one launch:
//   rotation       y = m R(pos) x          pairs (a, b) of a head: (a c - b s, b c + a s), c + i s = exp(2 pi i pos turns_i)
//   norm, rotation y = m R(pos) (w * xh)   xh = x / sqrt(mean x^2 + eps) over the d components of a head
//   its gradient   g = m R(pos)^T dy, u = w * g, dx = (u - xh mean(u xh)) / sqrt(mean x^2 + eps), dw = sum of g * xh over all rows
// (m scales the rotated components only; a head whose first `rot` components are rotated keeps the others.)
//
// Memory bounds all three: a row of d components is read (twice in the gradient) and written once, with about ten operations per
// component.  A row belongs to LPR lanes, d / 16 of them at work; each holds two chunks of 8 components that contain both partners
// of its pairs: 16-byte loads and stores, and the sums of a row take log2(LPR) steps through the registers of a lane's neighbours.
// The lanes keep their token and walk over the heads of a chunk, so the angles (a 64-bit product, sine and cosine for 8 pairs)
// are found once for up to HEADS rows; HU rows are on their way at a time.  The angle is taken in turns, pos * turns_i in 64 bits, and
// its whole turns are dropped there: at position 10^6 a product in 32 bits would be off by up to 0.06 radians.
#include "focus_internal.h"

#include <algorithm>

namespace focus {

namespace {

constexpr int RTHR = 256;
constexpr int HEADS = 8;              // most heads a lane group walks over with one set of angles

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16v8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16v8 __attribute__((ext_vector_type(8)));

// eight components in memory: one 16-byte access of a 16-bit type, two of fp32
template <typename T> struct Chunk;
template <> struct Chunk<uint16_t> {
    bf16v8 v;
    __device__ f32x8 f() const { return __builtin_convertvector(v, f32x8); }
    __device__ void set(f32x8 x) { v = __builtin_convertvector(x, bf16v8); }
};
template <> struct Chunk<f16_bits> {
    f16v8 v;
    __device__ f32x8 f() const { return __builtin_convertvector(v, f32x8); }
    __device__ void set(f32x8 x) { v = __builtin_convertvector(x, f16v8); }
};
template <> struct Chunk<float> {
    f32x8 v;
    __device__ f32x8 f() const { return v; }
    __device__ void set(f32x8 x) { v = x; }
};

__device__ inline float one_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ inline float one_f32(f16_bits b) { return f16_bits_to_f32(b.v); }
__device__ inline float one_f32(float b) { return b; }
__device__ inline void one_set(uint16_t* p, float f)
{
    const __bf16 h = (__bf16)f;
    __builtin_memcpy(p, &h, 2);
}
__device__ inline void one_set(f16_bits* p, float f) { p->v = f32_to_f16_bits(f); }
__device__ inline void one_set(float* p, float f) { *p = f; }

// which components lie where
constexpr int INTERLEAVED = 0;        // pairs (2i, 2i+1): a lane's chunks start at 8c and d/2 + 8c
constexpr int HALVES = 1;             // pairs (i, i + rot/2), rot % 16 == 0: both chunks in 16-byte pieces
constexpr int HALVES_ODD = 2;         // the same for any even rot: components one by one

// First component of a lane's two chunks (HALVES_ODD: of the two runs that its pairs p = 8c .. 8c+7 come from, see pair_at).
__device__ inline void chunk_starts(int lay, int c, int d, int rot, int* a, int* b)
{
    if (lay == INTERLEAVED) { *a = 8 * c; *b = d / 2 + 8 * c; return; }
    const int p = 8 * c;
    if (p < rot / 2) { *a = p; *b = rot / 2 + p; }
    else { *a = rot / 2 + p; *b = d / 2 + p; }          // rot + (p - rot/2), and (d - rot)/2 further on
}
__device__ inline void pair_at(int p, int d, int rot, int* a, int* b)
{
    if (p < rot / 2) { *a = p; *b = rot / 2 + p; }
    else { *a = rot / 2 + p; *b = d / 2 + p; }
}

// sum over the LPR lanes of a row (LPR 4, 8 or 16 consecutive lanes), the same value in all of them
template <int LPR>
__device__ inline float row_sum(float x)
{
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xf, 0xf, true));     // lane ^ 1
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xf, 0xf, true));     // lane ^ 2
    if (LPR >= 8) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xf, 0xf, true));    // the other half of 8
    if (LPR >= 16) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xf, 0xf, true));   // the other half of 16
    return x;
}

template <int LAY, typename T>
struct Row {
    Chunk<T> a, b;
    __device__ void load(const T* p, int ca, int cb, int c, int d, int rot)
    {
        if constexpr (LAY == HALVES_ODD) {
            f32x8 fa, fb;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                int ia, ib;
                pair_at(8 * c + j, d, rot, &ia, &ib);
                fa[j] = one_f32(p[ia]);
                fb[j] = one_f32(p[ib]);
            }
            a.set(fa);
            b.set(fb);
        } else {
            a = *(const Chunk<T>*)(p + ca);
            b = *(const Chunk<T>*)(p + cb);
        }
    }
    __device__ static void store(T* p, f32x8 fa, f32x8 fb, int ca, int cb, int c, int d, int rot)
    {
        if constexpr (LAY == HALVES_ODD) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                int ia, ib;
                pair_at(8 * c + j, d, rot, &ia, &ib);
                one_set(p + ia, fa[j]);
                one_set(p + ib, fb[j]);
            }
        } else {
            Chunk<T> x, y;
            x.set(fa);
            y.set(fb);
            *(Chunk<T>*)(p + ca) = x;
            *(Chunk<T>*)(p + cb) = y;
        }
    }
};

// (a, b) rotated by the lane's eight angles: pair j of the halves is (a_j, b_j); interleaved, angles 0..3 belong to the pairs of a,
// 4..7 to those of b
template <int LAY>
__device__ inline void rotate(f32x8& a, f32x8& b, const f32x8& co, const f32x8& si)
{
    if constexpr (LAY == INTERLEAVED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = a[2 * j], y = a[2 * j + 1], z = b[2 * j], w = b[2 * j + 1];
            a[2 * j] = x * co[j] - y * si[j];
            a[2 * j + 1] = y * co[j] + x * si[j];
            b[2 * j] = z * co[4 + j] - w * si[4 + j];
            b[2 * j + 1] = w * co[4 + j] + z * si[4 + j];
        }
    } else {
        const f32x8 x = a, y = b;
        a = x * co - y * si;
        b = y * co + x * si;
    }
}

// OP: 0 rotation (a.invert: by the negative angle), 1 norm and rotation, 2 the gradient of 1.
// blockIdx.y is a chunk of at most a.heads heads, those of q first, then those of k.
template <int OP, typename T, int LAY, int LPR>
__global__ __launch_bounds__(RTHR) void rope_kernel(RopeArgs A)
{
    constexpr int TPB = RTHR / LPR;              // tokens of a work-group at a time
    constexpr int HU = (sizeof(T) == 4 || OP == 2) ? 2 : 4;     // rows of a lane group on their way
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    const int qchunks = (A.Hq + A.heads - 1) / A.heads;
    const bool isk = (int)blockIdx.y >= qchunks;
    const int h0 = ((int)blockIdx.y - (isk ? qchunks : 0)) * A.heads;
    const int h1 = min(h0 + A.heads, isk ? A.Hkv : A.Hq);
    const int d = A.d, rot = A.rot;
    const bool active = lane < d / 16;
    const int c = active ? lane : 0;
    const RopeSide S = isk ? A.k : A.q;
    const T* x = (const T*)S.x;
    int ca, cb;
    chunk_starts(LAY, c, d, rot, &ca, &cb);

    f32x8 wa, wb, da = 0.f, db = 0.f;
    if constexpr (OP != 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            int ia = ca + j, ib = cb + j;
            if (LAY == HALVES_ODD) pair_at(8 * c + j, d, rot, &ia, &ib);
            wa[j] = S.w[ia];
            wb[j] = S.w[ib];
        }
    }
    const long long tokens = (long long)A.B * A.n;
    for (long long t0 = (long long)blockIdx.x * TPB; t0 < tokens; t0 += (long long)gridDim.x * TPB) {
        const long long tok = t0 + group;
        const bool live = active && tok < tokens;
        const long long tk = tok < tokens ? tok : 0;
        const int b = (int)(tk / A.n), t = (int)(tk % A.n);
        f32x8 co = 1.f, si = 0.f;
        if (rot > 0 && live) {
            const double pos = (double)(A.positions ? A.positions[tk] : t);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = LAY == INTERLEAVED ? (j < 4 ? ca / 2 + j : cb / 2 + j - 4) : 8 * c + j;
                if (e < rot / 2) {
                    const double turn = pos * A.turns[e];
                    float s0, c0;
                    sincospif(2.f * (float)(turn - rint(turn)), &s0, &c0);
                    co[j] = A.magnitude * c0;
                    si[j] = A.magnitude * ((OP == 2) != (A.invert != 0) ? -s0 : s0);
                }
            }
        }
        const T* px = x + (long long)b * S.xs[0] + (long long)t * S.xs[2];
        T* py = (T*)S.y + (long long)b * S.ys[0] + (long long)t * S.ys[2];
        for (int h = h0; h < h1; h += HU) {
            Row<LAY, T> rx[HU], rg[OP == 2 ? HU : 1];
#pragma unroll
            for (int u = 0; u < HU; ++u)
                if (live && h + u < h1) {
                    rx[u].load(px + (long long)(h + u) * S.xs[1], ca, cb, c, d, rot);
                    if constexpr (OP == 2)
                        rg[u].load((const T*)S.g + (long long)b * S.ys[0] + (long long)t * S.ys[2] + (long long)(h + u) * S.ys[1],
                                   ca, cb, c, d, rot);
                }
#pragma unroll
            for (int u = 0; u < HU; ++u) {
                f32x8 a = 0.f, bb = 0.f;
                const bool mine = live && h + u < h1;
                if (mine) { a = rx[u].a.f(); bb = rx[u].b.f(); }
                if constexpr (OP == 0) {
                    rotate<LAY>(a, bb, co, si);
                } else {
                    float ss = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) ss += a[j] * a[j] + bb[j] * bb[j];
                    ss = row_sum<LPR>(ss);
                    const float rstd = rsqrtf(ss / (float)d + A.eps);
                    a *= rstd;                                     // xh
                    bb *= rstd;
                    if constexpr (OP == 1) {
                        a *= wa;
                        bb *= wb;
                        rotate<LAY>(a, bb, co, si);
                    } else {
                        f32x8 ga = 0.f, gb = 0.f;
                        if (mine) { ga = rg[u].a.f(); gb = rg[u].b.f(); }
                        rotate<LAY>(ga, gb, co, si);
                        float dot = 0.f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            da[j] += ga[j] * a[j];
                            db[j] += gb[j] * bb[j];
                            ga[j] *= wa[j];
                            gb[j] *= wb[j];
                            dot += ga[j] * a[j] + gb[j] * bb[j];
                        }
                        dot = row_sum<LPR>(dot) / (float)d;
                        a = rstd * (ga - a * dot);
                        bb = rstd * (gb - bb * dot);
                    }
                }
                if (mine) {
                    if constexpr (OP == 2)
                        Row<LAY, T>::store((T*)S.dx + (long long)b * S.xs[0] + (long long)t * S.xs[2] + (long long)(h + u) * S.xs[1],
                                           a, bb, ca, cb, c, d, rot);
                    else
                        Row<LAY, T>::store(py + (long long)(h + u) * S.ys[1], a, bb, ca, cb, c, d, rot);
                }
            }
        }
    }
    if constexpr (OP == 2) {
        // the weights' gradients: lanes of equal c of a wavefront, then the four wavefronts, in one order
        __shared__ float s_dw[RTHR / 64][256];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int m = LPR; m < 64; m *= 2) {
                da[j] += __shfl_xor(da[j], m);
                db[j] += __shfl_xor(db[j], m);
            }
        if ((threadIdx.x & 63) < LPR && active) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                int ia = ca + j, ib = cb + j;
                if (LAY == HALVES_ODD) pair_at(8 * c + j, d, rot, &ia, &ib);
                s_dw[threadIdx.x >> 6][ia] = da[j];
                s_dw[threadIdx.x >> 6][ib] = db[j];
            }
        }
        __syncthreads();
        float* slot = A.partial + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * d;
        for (int i = threadIdx.x; i < d; i += RTHR) slot[i] = (s_dw[0][i] + s_dw[1][i]) + (s_dw[2][i] + s_dw[3][i]);
    }
}

// dw[i] = sum of the partial sums of q's (blockIdx.y 0) or k's slots, in 64 bits and in one order: 16 components per work-group, 64 shares of
// the slots for each.
constexpr int DW_THR = 1024;
__global__ __launch_bounds__(DW_THR) void rope_dw_kernel(const float* __restrict__ partial, int qslots, int kslots, int d,
                                                        float* __restrict__ dwq, float* __restrict__ dwk)
{
    __shared__ double s[64][16];
    const int c = threadIdx.x % 16, i = blockIdx.x * 16 + c, part = threadIdx.x / 16;
    const int first = blockIdx.y ? qslots : 0, count = blockIdx.y ? kslots : qslots;
    double sum = 0.0;
#pragma unroll 8
    for (int j = part; j < count; j += 64) sum += (double)partial[(size_t)(first + j) * d + i];
    s[part][c] = sum;
    __syncthreads();
    for (int half = 32; half > 0; half /= 2) {
        if (part < half) s[part][c] += s[part + half][c];
        __syncthreads();
    }
    if (part == 0) (blockIdx.y ? dwk : dwq)[i] = (float)s[0][c];
}

template <int OP, typename T, int LAY>
hipError_t launch_lanes(const RopeArgs& A, dim3 grid, hipStream_t st)
{
    if (A.d <= 64) rope_kernel<OP, T, LAY, 4><<<grid, RTHR, 0, st>>>(A);
    else if (A.d <= 128) rope_kernel<OP, T, LAY, 8><<<grid, RTHR, 0, st>>>(A);
    else rope_kernel<OP, T, LAY, 16><<<grid, RTHR, 0, st>>>(A);
    return hipGetLastError();
}

template <int OP, typename T>
hipError_t launch_layout(const RopeArgs& A, dim3 grid, hipStream_t st)
{
    if (A.interleaved) return launch_lanes<OP, T, INTERLEAVED>(A, grid, st);
    if (A.rot % 16 == 0) return launch_lanes<OP, T, HALVES>(A, grid, st);
    return launch_lanes<OP, T, HALVES_ODD>(A, grid, st);
}

template <int OP>
hipError_t launch_type(const RopeArgs& A, dim3 grid, hipStream_t st)
{
    if (A.dtype == 0) return launch_layout<OP, float>(A, grid, st);
    if (A.dtype == 1) return launch_layout<OP, uint16_t>(A, grid, st);
    return launch_layout<OP, f16_bits>(A, grid, st);
}

int lanes_per_row(int d) { return d <= 64 ? 4 : d <= 128 ? 8 : 16; }

// Heads of a chunk: as many as share a set of angles while the rows still make two work-groups for each of 256 compute units.
int heads_per_chunk(const RopeArgs& A)
{
    const long long tpb = RTHR / lanes_per_row(A.d), blocks = ((long long)A.B * A.n + tpb - 1) / tpb;
    int heads = HEADS;
    while (heads > 1 && blocks * ((A.Hq + heads - 1) / heads + (A.Hkv + heads - 1) / heads) < 512) heads /= 2;
    return heads;
}

}  // namespace

// work-groups along the tokens of the gradient's launch: each leaves one partial sum of the weights' gradients per chunk of heads
static int bwd_blocks(const RopeArgs& A, int chunks)
{
    const long long tpb = RTHR / lanes_per_row(A.d), blocks = ((long long)A.B * A.n + tpb - 1) / tpb;
    return (int)std::max(1ll, std::min(blocks, (long long)std::max(1, 1024 / chunks)));
}

size_t rope_bwd_workspace(const RopeArgs& A0)
{
    RopeArgs A = A0;
    A.heads = heads_per_chunk(A);
    const int chunks = (A.Hq + A.heads - 1) / A.heads + (A.Hkv + A.heads - 1) / A.heads;
    return (size_t)chunks * bwd_blocks(A, chunks) * A.d * sizeof(float);
}

hipError_t launch_rope(const RopeArgs& A0, int op, hipStream_t st)
{
    RopeArgs A = A0;
    A.heads = heads_per_chunk(A);
    const int qchunks = (A.Hq + A.heads - 1) / A.heads, chunks = qchunks + (A.Hkv + A.heads - 1) / A.heads;
    if (op == 2) {
        const int bx = bwd_blocks(A, chunks);
        hipError_t e = launch_type<2>(A, dim3(bx, chunks), st);
        if (e != hipSuccess) return e;
        rope_dw_kernel<<<dim3(A.d / 16, A.Hkv > 0 ? 2 : 1), DW_THR, 0, st>>>(A.partial, qchunks * bx, (chunks - qchunks) * bx, A.d,
                                                                          A.q.dw, A.k.dw);
        return hipGetLastError();
    }
    const long long tpb = RTHR / lanes_per_row(A.d), blocks = ((long long)A.B * A.n + tpb - 1) / tpb;
    const dim3 grid((unsigned)std::min(blocks, 1ll << 20), chunks);
    return op == 0 ? launch_type<0>(A, grid, st) : launch_type<1>(A, grid, st);
}

}  // namespace focus
