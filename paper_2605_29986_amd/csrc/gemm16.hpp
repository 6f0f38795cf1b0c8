// Products of 16-bit matrices in tiles on the matrix cores, for the vocabulary projection's loss and gradients (gfx950).
//
//     acc[m][n] = sum_k A[m][k] B[n][k]      A, B bf16 or fp16, acc fp32
//
// A workgroup makes BM x BN of it, in steps of 64 along k.  Either operand may lie in memory with k next to k ("rows") or with
// m (n) next to m ("columns", the transposed use of a row-major matrix).  Both are copied to LDS as they lie, in units of 16
// bytes, by loads that write LDS without passing registers, into one of two buffers while the other is multiplied; fragments of
// "columns" come out of LDS transposed (ds_read_b64_tr_b16: of a group of 16 lanes, lane i hands in four elements of row i / 4
// and gets one column's four).  Units are permuted within their row on the way in so that the 64 lanes of a fragment read spread
// over all banks: unit c of row r lies at c ^ (r & 7) (rows of 128 bytes), the 32-byte pair c of a column-major row k at
// c ^ (k & 3 | (k >> 3 & 1) << 2).
#pragma once

#include "common.hpp"

namespace cfgzip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

struct Bf16 {
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint16_t round(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
    static __device__ __forceinline__ float value(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
};
struct Fp16 {
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint16_t round(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
    static __device__ __forceinline__ float value(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
};

template <typename T>
__device__ __forceinline__ u32x2 round4(f32x4 x) {
    u32x2 y;
    y[0] = T::round(x[0]) | (uint32_t)T::round(x[1]) << 16;
    y[1] = T::round(x[2]) | (uint32_t)T::round(x[3]) << 16;
    return y;
}

// One operand of a product.  A thread's offsets from the tile's first element stay below 2^32 bytes: the host refuses strides
// of 2^22 elements and more.
struct Operand {
    const uint16_t *p;
    int64_t ld;    // elements from one row of memory to the next
    int32_t rows;  // extent in m or n
    int32_t k;     // extent in k
};

constexpr int kStepK = 64;
constexpr int64_t kMaxStride = 1 << 22;

static __device__ const u32x4 kZeros = {0, 0, 0, 0};  // what lanes behind the end of k load

// R: the tile's extent in m or n.  COLUMNS: m (n) next to m in memory.  DIRECT: the base and the rows of memory lie at multiples
// of 16 bytes and hold whole units of 8 elements; then lanes load to LDS directly, else through registers, the units at the end
// of a row element by element.
template <int R, int THREADS, bool COLUMNS, bool DIRECT>
struct Tile {
    static constexpr int kUnits = R * kStepK / 8;
    static constexpr int kPer = (kUnits + THREADS - 1) / THREADS;  // units of a thread
    static constexpr int kRowUnits = COLUMNS ? R / 8 : kStepK / 8;
    static constexpr int kPairMask = R / 16 >= 8 ? 7 : R / 16 - 1;  // of the permutation of a column-major row's pairs
    static constexpr int kBytes = kUnits * 16;

    const uint16_t *base;  // uniform: the tile's first element at the present k
    int64_t ld;
    int32_t rows_left, k_left;
    uint32_t at[kPer];     // byte offsets from base
    u32x4 held[DIRECT ? 1 : kPer];

    static __device__ __forceinline__ int pair_swizzle(int k) { return ((k & 3) | ((k >> 3) & 1) << 2) & kPairMask; }

    static __device__ __forceinline__ void place(int unit, int &r, int &c) {  // memory row of the tile and unit in it
        r = unit / kRowUnits;
        c = unit % kRowUnits;
        if (COLUMNS) c = (((c >> 1) ^ pair_swizzle(r)) << 1) | (c & 1);
        else c ^= r & 7;
    }

    __device__ __forceinline__ void init(const Operand &o, int32_t row0, int32_t k0) {
        ld = o.ld;
        rows_left = o.rows - row0;
        k_left = o.k - k0;
        base = COLUMNS ? o.p + k0 * o.ld + row0 : o.p + row0 * o.ld + k0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            int r, c;
            place(i * THREADS + (int)threadIdx.x, r, c);
            // rows (units of a column-major row) behind the end load the last one; what comes of them is not stored
            if (COLUMNS) {
                if (DIRECT && c * 8 >= rows_left) c = rows_left / 8 - 1;
            } else {
                if (r >= rows_left) r = rows_left - 1;
            }
            at[i] = (uint32_t)(r * ld + c * 8) * 2u;
        }
    }

    __device__ __forceinline__ bool has_unit(int i) const {
        return kUnits % THREADS == 0 || i * THREADS + (int)threadIdx.x < kUnits;
    }

    // begins the load of the next 64 k into `lds`
    __device__ __forceinline__ void load(char *lds) {
        const char *b = reinterpret_cast<const char *>(base);
        if constexpr (DIRECT) {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
            if (k_left >= kStepK) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (has_unit(i))
                        __builtin_amdgcn_global_load_lds((global_void *)(b + at[i]),
                                                         (lds_void *)(lds + (i * THREADS + wave * kWave) * 16), 16, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (has_unit(i)) {
                        int r, c;
                        place(i * THREADS + (int)threadIdx.x, r, c);
                        const bool there = COLUMNS ? r < k_left : c * 8 < k_left;
                        const char *p = there ? b + at[i] : reinterpret_cast<const char *>(&kZeros);
                        __builtin_amdgcn_global_load_lds((global_void *)p,
                                                         (lds_void *)(lds + (i * THREADS + wave * kWave) * 16), 16, 0, 0);
                    }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (!has_unit(i)) continue;
                int r, c;
                place(i * THREADS + (int)threadIdx.x, r, c);
                const int left = COLUMNS ? (r < k_left ? rows_left - c * 8 : 0) : k_left - c * 8;  // elements of the unit that exist
                u32x4 v = {0, 0, 0, 0};
                if (left >= 8) {
                    v = *reinterpret_cast<const u32x4_any *>(b + at[i]);
                } else {
                    const uint16_t *e = reinterpret_cast<const uint16_t *>(b + at[i]);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < left) v[j / 2] |= (uint32_t)e[j] << (j % 2 * 16);
                }
                held[i] = v;
            }
        }
        base += COLUMNS ? kStepK * ld : (int64_t)kStepK;
        k_left -= kStepK;
    }

    // what load() holds in registers goes to LDS; the caller puts a barrier behind it
    __device__ __forceinline__ void commit(char *lds) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (has_unit(i)) *reinterpret_cast<u32x4 *>(lds + (i * THREADS + (int)threadIdx.x) * 16) = held[i];
        }
    }

    // fragment of 16 rows from row0 + 16 f (row0 of the wave) and 32 k from 32 kk: lane l has row l & 15, k = 8 (l >> 4) + 0..7
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int row0, int f, int kk, int lane) {
        const int i = lane & 15, g = lane >> 4;
        if constexpr (COLUMNS) {
            const int pair = ((row0 / 16 + f) ^ pair_swizzle(8 * g + (i >> 2)));
            const char *p = lds + (8 * g + (i >> 2)) * (R * 2) + pair * 32 + (i & 3) * 8 + kk * 32 * R * 2;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * R * 2)));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            const char *p = lds + (row0 + i) * 128 + ((g ^ (i & 7)) ^ (kk * 4)) * 16 + f * 16 * 128;
            return *reinterpret_cast<const u32x4 *>(p);
        }
    }
};

// BM x BN by WM x WN waves
template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kThreads = WM * WN * kWave;
    static constexpr int TM = BM / WM, TN = BN / WN;  // a wave's part
    static constexpr int FM = TM / 16, FN = TN / 16;  // in fragments
    static constexpr int kLds = (BM + BN) * kStepK * 2;  // one buffer
};

// acc[i][j][r]: lane l has m = 16 i + 4 (l >> 4) + r, n = 16 j + (l & 15) of its wave's part
template <typename T, typename S, typename TileA, typename TileB>
__device__ __forceinline__ void multiply_step(const char *lds, int wm, int wn, int lane, f32x4 (&acc)[S::FM][S::FN]) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
        u32x4 a[S::FM], b[S::FN];
#pragma unroll
        for (int i = 0; i < S::FM; ++i) a[i] = TileA::fragment(lds, wm * S::TM, i, kk, lane);
#pragma unroll
        for (int j = 0; j < S::FN; ++j) b[j] = TileB::fragment(lds + TileA::kBytes, wn * S::TN, j, kk, lane);
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) acc[i][j] = T::mma(a[i], b[j], acc[i][j]);
    }
}

// the tile's sum over k0 <= k < k1 (k1 - k0 rounded up to whole steps; operands are 0 behind their k).  Two LDS buffers of
// S::kLds bytes, objects of their own, so that the compiler sees that a buffer in use is not the one being filled.
template <typename T, typename S, typename TileA, typename TileB>
__device__ __forceinline__ void multiply(const Operand &A, const Operand &B, int32_t m0, int32_t n0, int32_t k0, int32_t k1,
                                         char *lds0, char *lds1, f32x4 (&acc)[S::FM][S::FN]) {
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wm = wave / S::WN, wn = wave % S::WN;
    TileA ta;
    TileB tb;
    ta.init(A, m0, k0);
    tb.init(B, n0, k0);
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    int steps = (k1 - k0 + kStepK - 1) / kStepK;
    ta.load(lds0);
    tb.load(lds0 + TileA::kBytes);
    ta.commit(lds0);
    tb.commit(lds0 + TileA::kBytes);
    __syncthreads();
    while (true) {
        if (steps > 1) {
            ta.load(lds1);
            tb.load(lds1 + TileA::kBytes);
        }
        multiply_step<T, S, TileA, TileB>(lds0, wm, wn, lane, acc);
        if (steps == 1) break;
        ta.commit(lds1);
        tb.commit(lds1 + TileA::kBytes);
        __syncthreads();
        if (steps > 2) {
            ta.load(lds0);
            tb.load(lds0 + TileA::kBytes);
        }
        multiply_step<T, S, TileA, TileB>(lds1, wm, wn, lane, acc);
        if (steps == 2) break;
        ta.commit(lds0);
        tb.commit(lds0 + TileA::kBytes);
        __syncthreads();
        steps -= 2;
    }
}

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn, and each XCD has an L2 of its own: workgroup
// b is number b / 8 of XCD b % 8, an XCD's workgroups take tiles next to each other, in panels of kPanel tiles of m and all of
// n, so that those running at a time share both operands' tiles.
constexpr int kPanel = 4;
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t total, int32_t tiles_m, int32_t tiles_n, int32_t &tm, int32_t &tn) {
    const uint32_t per = total / 8, more = total % 8, x = b % 8;
    const uint32_t t = x * per + (x < more ? x : more) + b / 8;
    const uint32_t panel = t / (kPanel * tiles_n), in = t % (kPanel * tiles_n);
    const uint32_t width = panel * kPanel + kPanel <= (uint32_t)tiles_m ? kPanel : tiles_m - panel * kPanel;
    tm = panel * kPanel + in % width;
    tn = in / width;
}

}  // namespace cfgzip
