// What the kernels of the sliding window with sinks share: operands of the matrix products in 16-byte pieces, tiles of rows in LDS
// in two orders, the mask.
//
// All products are 32 x 32 blocks.  An operand piece is 16 bytes of a lane, taken from 32 consecutive bytes of a row: lanes 0..31 hold
// the first half for their row or column, lanes 32..63 the second.  For 16-bit types that is the operand of one v_mfma 32x32x16; for
// fp32 its four components go into four v_mfma 32x32x2, whose two contracted indices are then 4 apart, on both operands alike.
// The result holds, in lane l and register i, column l % 32 and row 8 (i/4) + 4 (l/32) + i % 4.  A result can therefore be
// the next product's second operand as it is, if the first operand's contracted index is stored in that order (slot_of_row).
#pragma once
#include "focus_internal.h"

namespace focus {
namespace window {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

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

// A tile of R rows of D components in LDS.
//   by rows       row r at r * RPITCH, its 16-byte piece c at place c ^ f(r), f(r) = (r ^ r >> 2) & 7: the eight lanes that a 16-byte access serves
//                 at a time touch all 32 banks, when they read eight consecutive rows and when they write every fourth one
//   by components component d at d * TPITCH, the R rows in operand order; 16 bytes of padding do the same there
template <typename T, int D, int R>
struct Tile {
    static constexpr int ES = (int)sizeof(T), E = Piece<T>::E;
    static constexpr int PIECES = D / E;                       // 16-byte pieces of a row
    static constexpr int KS = PIECES / 2;                      // steps of a product over the components
    static constexpr int DB = (D + 31) / 32;                   // blocks of 32 components
    static constexpr int US = 32 / (2 * E);                    // steps of a product over 32 rows
    static constexpr int RPITCH = round_up(PIECES, 8) * 16;
    static constexpr int TPITCH = R * ES + 16;
    static constexpr int RBYTES = R * RPITCH, TBYTES = DB * 32 * TPITCH;
    static constexpr int BLOCKS = R / 4 * PIECES;              // blocks of 4 rows by one piece: what a thread moves at a time

    static __device__ int row_at(int r, int piece) { return r * RPITCH + (piece >> 3) * 128 + (((piece & 7) ^ ((r ^ (r >> 2)) & 7)) << 4); }
    // first of four consecutive rows 4g .. 4g+3 in operand order (in rows)
    static __device__ int slot_of_rows(int g) { return ES == 4 ? 4 * g : (g >> 2) * 16 + (g & 1) * 8 + ((g >> 1) & 1) * 4; }

    // operand of 32 rows (from row 32 * unit), step s over the components
    static __device__ u32x4 rows_piece(const char* tile, int unit, int s, int lane)
    {
        return *(const u32x4*)(tile + row_at(32 * unit + (lane & 31), 2 * s + (lane >> 5)));
    }
    // operand of 32 components (block db), step s over the rows of 32-row unit `unit`
    static __device__ u32x4 comps_piece(const char* tile, int db, int unit, int s, int lane)
    {
        return *(const u32x4*)(tile + (32 * db + (lane & 31)) * TPITCH + 32 * ES * unit + 32 * s + 16 * (lane >> 5));
    }
};

// Two tiles on their way from global memory to LDS: every thread holds blocks of 4 rows by 16 bytes.
template <typename T, int D, int R>
struct Stage {
    typedef Tile<T, D, R> TL;
    static constexpr int N = (2 * TL::BLOCKS + WTHR - 1) / WTHR;
    u32x4 r[N][4];

    static __device__ void place(int i, int* which, int* rows, int* piece)
    {
        int id = (int)threadIdx.x + WTHR * i;
        *which = id >= TL::BLOCKS;
        id -= *which ? TL::BLOCKS : 0;
        *rows = id % (R / 4);
        *piece = id / (R / 4);
    }
    // rows row0 .. row0 + R - 1 of a and b (row strides as, bs); zeros at and behind row len
    __device__ void load(const T* a, long long as, const T* b, long long bs, int row0, int len)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int which, g, piece;
            place(i, &which, &g, &piece);
            if ((2 * TL::BLOCKS) % WTHR != 0 && piece >= TL::PIECES) continue;      // behind the last block
            const T* p = which ? b : a;
            const long long st = which ? bs : as;
            const int row = row0 + 4 * g;
            p += (long long)row * st;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4 x = {0u, 0u, 0u, 0u};
                if (row + j < len) x = load_piece(p + j * st, piece);
                r[i][j] = x;
            }
        }
    }
    // tile `which` by rows and by components (null: not in that order)
    __device__ void store(char* arows, char* acomps, char* brows, char* bcomps) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int which, g, piece;
            place(i, &which, &g, &piece);
            if ((2 * TL::BLOCKS) % WTHR != 0 && piece >= TL::PIECES) continue;
            char* rows = which ? brows : arows;
            char* comps = which ? bcomps : acomps;
            if (rows) {
#pragma unroll
                for (int j = 0; j < 4; ++j) *(u32x4*)(rows + TL::row_at(4 * g + j, piece)) = r[i][j];
            }
            if (comps) {
                char* at = comps + piece * TL::E * TL::TPITCH + TL::slot_of_rows(g) * TL::ES;
                if constexpr (TL::ES == 4) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const u32x4 x = {r[i][0][c], r[i][1][c], r[i][2][c], r[i][3][c]};
                        *(u32x4*)(at + c * TL::TPITCH) = x;
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint2 lo, hi;                                    // components 2c and 2c + 1 of the four rows
                        lo.x = __builtin_amdgcn_perm(r[i][1][c], r[i][0][c], 0x05040100u);
                        lo.y = __builtin_amdgcn_perm(r[i][3][c], r[i][2][c], 0x05040100u);
                        hi.x = __builtin_amdgcn_perm(r[i][1][c], r[i][0][c], 0x07060302u);
                        hi.y = __builtin_amdgcn_perm(r[i][3][c], r[i][2][c], 0x07060302u);
                        *(uint2*)(at + 2 * c * TL::TPITCH) = lo;
                        *(uint2*)(at + (2 * c + 1) * TL::TPITCH) = hi;
                    }
                }
            }
        }
    }
    // Values that are not finite, in a tile with hidden pairs: a hidden pair's weight is zero, but 0 * inf is not.  They become zeros, and
    // their rows are marked (bit r of the two words at bad): whoever sees such a row is spoiled as a whole (spoiled_by).
    __device__ void take_out_not_finite(unsigned* bad)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int which, g, piece;
            place(i, &which, &g, &piece);
            if ((2 * TL::BLOCKS) % WTHR != 0 && piece >= TL::PIECES) continue;
            unsigned rows = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const unsigned x = r[i][j][c] & Piece<T>::EXP;
                    unsigned keep = (x & 0xffff0000u) == (Piece<T>::EXP & 0xffff0000u) ? 0u : 0xffffffffu;
                    if constexpr (TL::ES == 2) keep = (keep & 0xffff0000u) | ((x & 0xffffu) == (Piece<T>::EXP & 0xffffu) ? 0u : 0xffffu);
                    r[i][j][c] &= keep;
                    rows |= keep != 0xffffffffu ? 1u << j : 0u;
                }
            if (rows) atomicOr(&bad[g >> 3], rows << (4 * (g & 7)));
        }
    }
};

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

// The other half-wave's value: lanes l and l ^ 32 hold halves of one column
__device__ inline float other_half(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
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
    return (unsigned)(row - key) < (unsigned)window || (key < sinks && key <= row);
}

// Does a lane's row (or key) see a marked one of the 32 keys (rows) at `other`?  marks: the 32 bits of that block; kept by the half-wave that holds
// them, so the two halves' answers have to be joined.
template <bool KEYS_MARKED>
__device__ inline bool spoiled_by(unsigned marks, int mine, int other, int hh, int window, int sinks)
{
    bool hit = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int at = 8 * (i / 4) + 4 * hh + i % 4;
        const bool seen = KEYS_MARKED ? visible(mine, other + at, window, sinks) : visible(other + at, mine, window, sinks);
        hit |= seen && ((marks >> at) & 1u);
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
