// What the kernels of the sliding window with sinks share: operands of the matrix products in 16-byte pieces, tiles of rows in LDS
// in two orders, the mask.
//
// All products are 32 x 32 blocks.  An operand piece is 16 bytes of a lane, taken from 32 consecutive bytes of a row: lanes 0..31 hold
// the first half for their row or column, lanes 32..63 the second.  For 16-bit types that is the operand of one v_mfma 32x32x16; for
// fp32 its four components go into four v_mfma 32x32x2, whose two contracted indices are then 4 apart, on both operands alike.
// The result holds, in lane l and register i, column l % 32 and row 8 (i/4) + 4 (l/32) + i % 4.  A result can therefore be
// the next product's second operand as it is, if the first operand's contracted index is taken in that order (comps_piece).
#pragma once
#include "focus_internal.h"

namespace focus {
namespace window {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define WINDOW_INLINE __attribute__((always_inline))     // of lambdas: a call would go through memory

constexpr int WTHR = 256;                   // threads of a work-group: four wavefronts
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__host__ __device__ constexpr int round_up(int x, int m) { return (x + m - 1) / m * m; }

template <typename T> struct Piece;
template <> struct Piece<uint16_t> {
    static constexpr int E = 8;             // components of a piece
    static constexpr unsigned EXP = 0x7f807f80u;       // the exponents of infinities and NaN
    static __device__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    // eight fp32 values, rounded to the type (probabilities and their gradients: one rounding, as the products need)
    static __device__ u32x4 pack(const float* x)
    {
        bf16x8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (__bf16)x[i];
        return __builtin_bit_cast(u32x4, r);
    }
    static __device__ float dot(u32x4 a, u32x4 b)
    {
        const bf16x8 x = __builtin_bit_cast(bf16x8, a), y = __builtin_bit_cast(bf16x8, b);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += (float)x[i] * (float)y[i];
        return s;
    }
};
template <> struct Piece<f16_bits> {
    static constexpr int E = 8;
    static constexpr unsigned EXP = 0x7c007c00u;
    static __device__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ u32x4 pack(const float* x)
    {
        f16x8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (_Float16)x[i];
        return __builtin_bit_cast(u32x4, r);
    }
    static __device__ float dot(u32x4 a, u32x4 b)
    {
        const f16x8 x = __builtin_bit_cast(f16x8, a), y = __builtin_bit_cast(f16x8, b);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += (float)x[i] * (float)y[i];
        return s;
    }
};
template <> struct Piece<float> {
    static constexpr int E = 4;
    static constexpr unsigned EXP = 0x7f800000u;
    static __device__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
    static __device__ u32x4 pack(const float* x)
    {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(x[i]);
        return r;
    }
    static __device__ float dot(u32x4 a, u32x4 b)
    {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) s += __uint_as_float(a[i]) * __uint_as_float(b[i]);
        return s;
    }
};

// Rows of 16-byte pieces in global memory
template <typename T>
__device__ inline u32x4 load_piece(const T* row, int piece) { return *(const u32x4*)((const char*)row + 16 * piece); }

// A register whose value the compiler cannot see through: addresses derived from it are found where they are used (a few additions)
// instead of being kept, which cost the kernels below up to 70 spilled registers.
__device__ inline int opaque(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Operands loaded before a loop have arrived.  Otherwise the compiler waits for them at their use in the loop, every time around, and with them
// for every load issued since: the copy of the next tile, which it does not count.
template <int N>
__device__ inline void landed(u32x4 (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// The wait between a matrix product and the first read of its result by another instruction, in the source.  The compiler puts in what it has counted, but
// where the read is a copy behind the end of a conditional part it has been seen to count along one of the two ways only, and a row's last
// components came out wrong (5 of the 12 states that a 32x32x16 product needs; 18 for 32x32x2).  With it the listings
// have the full count on all ways; it takes 1 to 3% of the time of a long 16-bit call.
template <typename T>
__device__ inline void settle()
{
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (sizeof(T) == 4) asm volatile("s_nop 15\n\ts_nop 1");
    else asm volatile("s_nop 11");
    __builtin_amdgcn_sched_barrier(0);
}

// A tile of R rows of D components in LDS, the first operand of both kinds of product: by rows (its rows are the product's rows), and by components
// (its components are; its rows are contracted, four at a time from the LDS reads that turn 4 x 16 values of 16 bits around, one by one for fp32).
// Row r lies at r * RPITCH, its 16-byte piece c at place c ^ turn(r), so that neither kind of read meets a bank twice: the 16 consecutive rows
// of a read by rows have 16 different turns (8, where two rows share 256 bytes), and the four rows of a read by components differ
// in the bits of the turn that choose among the 64-byte quarters.  Tiles start at multiples of 256 bytes.
template <typename T, int D, int R>
struct Tile {
    static constexpr int ES = (int)sizeof(T), E = Piece<T>::E;
    static constexpr int PIECES = D / E;                       // 16-byte pieces of a row
    static constexpr int KS = PIECES / 2;                      // steps of a product over the components
    static constexpr int DB = (D + 31) / 32;                   // blocks of 32 components
    static constexpr int US = 32 / (2 * E);                    // steps of a product over 32 rows
    static constexpr int RPITCH = round_up(PIECES, 8) * 16, BLOCK = 32 * RPITCH;       // bytes of a row, of 32 rows
    static constexpr int BYTES = R * RPITCH;
    static constexpr int SWAP = RPITCH % 256 == 0 ? 15 : 7;    // places among which a row's pieces change

    static __device__ int turn_of_row(int r) { return SWAP == 15 ? (r & 3) << 2 | ((r >> 2) & 3) : (r & 2) << 1 | ((r >> 2) & 3); }
    // A lane's place for reads by rows of a block of 32 rows, and the operand of step s over the components: pieces 2s and 2s + 1
    static __device__ int rows_place(int lane)
    {
        const int r = lane & 31, hh = lane >> 5;
        return r * RPITCH + ((hh ^ turn_of_row(r)) << 4);
    }
    static __device__ u32x4 rows_piece(const char* block, int place, int s)
    {
        return *(const u32x4*)(block + ((place ^ ((2 * s & SWAP) << 4)) + 16 * (2 * s & ~SWAP)));
    }
    // The same by components: the operand of components 32 db .. and step s over the 32 rows.  16-bit types: v_mfma slots 0 .. 7 of half-wave h
    // are rows 16 s + 4 h + {0 .. 3, 8 .. 11}, the order in which a result holds its rows; fp32: row 8 s + 4 h + j for product j.
    static __device__ int comps_place(int lane)
    {
        const int hh = lane >> 5, l = lane & 15;
        if (ES == 4) return 4 * hh * RPITCH + ((((lane & 31) >> 2) ^ hh) << 4) + 4 * (lane & 3);
        const int r = 4 * hh + l / 4, c = 2 * ((lane >> 4) & 1) + (l & 3) / 2;
        return r * RPITCH + ((c ^ turn_of_row(r)) << 4) + 8 * (l & 1);
    }
    static __device__ u32x4 comps_piece(const char* block, int place, int db, int s)
    {
        u32x4 x;
        if constexpr (ES == 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int turn = (SWAP == 15 ? j << 2 : (j & 2) << 1) | 2 * (s & 1);
                x[j] = *(const unsigned*)(block + ((place ^ ((turn ^ (8 * db & SWAP)) << 4)) + 16 * (8 * db & ~SWAP) + (8 * s + j) * RPITCH));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const char* at = block + ((place ^ (((4 * db & SWAP) ^ 2 * j) << 4)) + 16 * (4 * db & ~SWAP) + (16 * s + 8 * j) * RPITCH);
                const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
                x[2 * j] = y.x;
                x[2 * j + 1] = y.y;
            }
        }
        return x;
    }
};

// A tile straight from global memory to LDS, 16 bytes a lane: a wavefront's loads fill LDS in order, so a lane fetches the piece that belongs in its
// place.  WAVES wavefronts share the tile.  Rows behind the last one are that row again (they are hidden by position).  Complete when vmcnt
// is 0 (dma_wait).  64 rows span less than 2^31 bytes (checked by the host).
template <typename T, int D, int R, int WAVES>
struct Dma {
    typedef Tile<T, D, R> TL;
    static constexpr int N = TL::BYTES / (1024 * WAVES);      // 1-KB loads of a wavefront
    static_assert(TL::BYTES % (1024 * WAVES) == 0, "the wavefronts fill a tile with equal numbers of loads");
    int off[N];                                               // of a lane in a whole tile

    static __device__ int source(int i, int wave, int lane, int pitch, int left)
    {
        constexpr int PLACES = TL::RPITCH / 16;
        const int id = 64 * (wave * N + i) + lane, row = id / PLACES, at = id % PLACES;
        int piece = at ^ TL::turn_of_row(row);
        if (TL::PIECES % 8 != 0 && piece >= TL::PIECES) piece = 0;      // (a place that matters to no result)
        return min(row, left - 1) * pitch + 16 * piece;
    }
    __device__ void init(int wave, int lane, int pitch)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) off[i] = source(i, wave, lane, pitch, R);
    }
    // rows of `pitch` bytes from `rows` on, `left` of them
    __device__ void load(const T* rows, int pitch, int left, char* tile, int wave, int lane) const
    {
        const unsigned to = __builtin_amdgcn_readfirstlane(lds_addr_of(tile) + 1024 * N * wave);
        const uintptr_t from = (uintptr_t)rows;               // (the same in all lanes, in scalar registers)
        const char* base = (const char*)((uintptr_t)(unsigned)__builtin_amdgcn_readfirstlane((int)from) |
                                         (uintptr_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(from >> 32)) << 32);
        if (left >= R) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds_dma16(base, off[i], to + 1024 * i);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) lds_dma16(base, source(i, wave, opaque(lane), pitch, left), to + 1024 * i);
        }
    }
};
__device__ inline void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Values that are not finite, in a tile that some row does not see as a whole: the weight of what is hidden is zero, but 0 * inf is not.  They
// become zeros, and their rows are marked (bit r of the words at bad): whoever sees such a row is spoiled as a whole (spoiled_by).
// By `threads` threads, of which this is one: the work-group's between two barriers, or a wavefront's in a tile of its own.
template <typename T, int D, int R>
__device__ inline void scrub(char* tile, unsigned* bad, int thread, int threads)
{
    typedef Tile<T, D, R> TL;
    for (int id = thread; id < TL::BYTES / 16; id += threads) {
        u32x4 v = *(const u32x4*)(tile + 16 * id);
        bool found = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const unsigned x = v[c] & Piece<T>::EXP;
            unsigned keep = (x & 0xffff0000u) == (Piece<T>::EXP & 0xffff0000u) ? 0u : 0xffffffffu;
            if constexpr (TL::ES == 2) keep = (keep & 0xffff0000u) | ((x & 0xffffu) == (Piece<T>::EXP & 0xffffu) ? 0u : 0xffffu);
            found |= keep != 0xffffffffu;
            v[c] &= keep;
        }
        if (found) {
            const int row = id / (TL::RPITCH / 16);
            *(u32x4*)(tile + 16 * id) = v;
            atomicOr(&bad[row >> 5], 1u << (row & 31));
        }
    }
}

// A wavefront's LDS accesses take effect in order: between its own writes and reads only the compiler has to be kept to it.
__device__ inline void own_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A sequence of a call: its length and the element offsets of its first row.
struct Sequence {
    int len, first, tb;        // rows; first row; batch row of the tensors
};
__device__ inline Sequence sequence_of(const WindowArgs& A, int b)
{
    Sequence s;
    s.first = 0;
    s.len = A.n;
    if (A.spans) {
        const int2 sp = A.spans[b];
        s.first = sp.x;
        s.len = sp.x < 0 || sp.x >= A.n || sp.y < 0 ? 0 : min(sp.y, A.n - sp.x);
    }
    s.len = min(s.len, A.span_max);
    s.tb = A.packed ? 0 : b;
    return s;
}

// Lanes l and l ^ 32 hold halves of one column: the largest, the sum of their values
__device__ inline float halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float halves_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a block of 32 rows and 32 keys (positions row0.., key0..) needs
enum Block { HIDDEN, OPEN, EDGE };
__device__ inline Block block_kind(int row0, int key0, int window, int sinks)
{
    if (key0 > row0 + 31) return HIDDEN;
    if (row0 - (key0 + 31) >= window && key0 >= sinks) return HIDDEN;
    if (key0 + 31 <= row0 && (row0 + 31 - key0 < window || key0 + 31 < sinks)) return OPEN;
    return EDGE;
}
__device__ inline bool visible(int row, int key, int window, int sinks)
{
    // (bitwise: as a chain of conditions it became branches, 32 of them in a block)
    return (bool)((int)((unsigned)(row - key) < (unsigned)window) | ((int)(key < sinks) & (int)(key <= row)));
}

// Does a lane's row (or key) see a marked one of the 32 keys (rows) at `other`?  marks: the 32 bits of that block; kept by the half-wave that holds
// them, so the two halves' answers have to be joined.
template <bool KEYS_MARKED>
__device__ inline bool spoiled_by(unsigned marks, int mine, int other, int hh, int window, int sinks)
{
    bool hit = false;
    mine = opaque(mine);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int at = 8 * (i / 4) + 4 * hh + i % 4;
        const bool seen = KEYS_MARKED ? visible(mine, other + at, window, sinks) : visible(other + at, mine, window, sinks);
        hit |= (bool)((int)seen & (int)((marks >> at) & 1u));
    }
    return hit;
}

// Stores a result held by components: lane l has row l % 32 (at `row`, null: not stored), blocks db of 32 components; times f.
template <typename T, int D>
__device__ inline void store_row(T* row, const f32x16* acc, float f, int lane)
{
    const int hh = lane >> 5;
#pragma unroll
    for (int db = 0; db < (D + 31) / 32; ++db)
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (32 * db + 8 * m >= D) continue;
            float x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = x[4 + i] = acc[db][4 * m + i] * f;
            if (!row) continue;
            const u32x4 p = Piece<T>::pack(x);
            T* at = row + 32 * db + 8 * m + 4 * hh;
            if constexpr (sizeof(T) == 4) *(u32x4*)at = p;
            else { uint2 y; y.x = p[0]; y.y = p[1]; *(uint2*)at = y; }
        }
}

// The keys that rows first .. last can see, in tiles of 32: the sinks', then those from the first key of the window on
struct Walk {
    int first, last, sink_tiles, base, tiles;
    int open0;                  // keys from here to the first row hide nothing
    __device__ Walk(const WindowArgs& A, int first_, int last_)
    {
        first = first_;
        last = last_;
        sink_tiles = (min(A.sinks, last + 1) + 31) / 32;
        base = max(32 * sink_tiles, max(0, first - A.window + 1) & ~31);
        tiles = sink_tiles + max(0, last / 32 - base / 32 + 1);
        open0 = last - A.window + 1;
    }
    __device__ int key_at(int t) const { return t < sink_tiles ? 32 * t : base + 32 * (t - sink_tiles); }
    // may a pair of the rows and keys key0 .. key0 + 31 be hidden?
    __device__ bool edge(int key0, const WindowArgs& A) const { return key0 + 31 > first || (key0 < open0 && key0 + 31 >= A.sinks); }
};

// tanh of 16 scores times f: its series to z^9 while all are below 0.3 in magnitude (the next term is 1.6e-8 there, half a step of fp32
// relative to z: six operations in place of an exponential and a reciprocal), else from exp(-2 |z|); fp32 takes the library's there.
template <typename T>
__device__ inline void tanh_scores(f32x16& x, float f)
{
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] *= f;
        big = fmaxf(big, fabsf(x[i]));
    }
    if (!__any(!(big <= 0.3f))) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float z = x[i], w = z * z;
            x[i] = fmaf(z * w, fmaf(w, fmaf(w, fmaf(w, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), z);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = tanhf(x[i]);
            else {
                const float e = __builtin_amdgcn_exp2f(-2.f * LOG2E * fabsf(x[i]));
                x[i] = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), x[i]);
            }
        }
    }
}

// The place of a work-group: consecutive ones go to the eight XCDs in turn, and each XCD gets a contiguous share of the work, so that
// neighbours that read the same keys (the query heads of a KV head, neighbouring tiles) meet in one L2.  -1: behind the end.
__device__ inline long long work_of(long long total)
{
    const long long share = (total + 7) / 8, x = blockIdx.x, w = (x % 8) * share + x / 8;
    return x / 8 < share && w < total ? w : -1;
}
inline long long work_groups(long long total) { return (total + 7) / 8 * 8; }

}  // namespace window
}  // namespace focus
