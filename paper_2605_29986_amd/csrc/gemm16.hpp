// Products of 16-bit matrices in tiles on the matrix cores, for the vocabulary projection's loss and gradients, and by the same loop
// of 4-bit ones for its logits (gfx950).
//
//     acc[m][n] = sum_k A[m][k] B[n][k]      A, B bf16 or fp16, acc fp32
//
// A workgroup makes BM x BN of it at a time, in steps of 64 along k.  Either operand may lie in memory with k next to k ("rows") or
// with m (n) next to m ("columns", the transposed use of a row-major matrix).  Both are copied to LDS as they lie, in units of 16
// bytes, by loads that write LDS without passing registers, into one of several buffers while another is multiplied; fragments of
// "columns" come out of LDS transposed (ds_read_b64_tr_b16: of a group of 16 lanes, lane i hands in four elements of row i / 4
// and gets one column's four).  Units are permuted within their row on the way in so that the 64 lanes of a fragment read spread
// over all banks: unit c of row r lies at c ^ (r & 7), the 32-byte pair c of a column-major row k at c ^ (k & 3 | (k >> 3 & 1) << 2).
#pragma once

#include <utility>

#include "common.hpp"

namespace cfgzip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) char lds_char;
typedef const __attribute__((address_space(1))) void global_void;

#define CFGZIP_INLINE __attribute__((always_inline))

// f(0), .., f(N - 1) with the number as a constant: what is indexed by it stays in registers
template <typename F, int... I>
__device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F &&f) {
    each_of(f, std::make_integer_sequence<int, N>{});
}

// x, and nothing known about it: what is worked out from it is worked out where it is written, and kept in no registers beyond that
__device__ __forceinline__ int afresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

struct Bf16 {
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    // Four products with one a, their sums in accumulation registers: 256 of them the compiler moves about and spills.  It does not see
    // the products in here, so the two wait states between a vector instruction and a product that reads what it wrote are part of
    // the text, and those behind the last product are settle()'s.
    static __device__ __forceinline__ void mma4(u32x4 a, u32x4 b0, u32x4 b1, u32x4 b2, u32x4 b3, f32x4 &c0, f32x4 &c1, f32x4 &c2, f32x4 &c3) {
        asm volatile(
            "s_nop 1\n\t"
            "v_mfma_f32_16x16x32_bf16 %0, %4, %5, %0\n\t"
            "v_mfma_f32_16x16x32_bf16 %1, %4, %6, %1\n\t"
            "v_mfma_f32_16x16x32_bf16 %2, %4, %7, %2\n\t"
            "v_mfma_f32_16x16x32_bf16 %3, %4, %8, %3"
            : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3)
            : "v"(a), "v"(b0), "v"(b1), "v"(b2), "v"(b3));
    }
    static __device__ __forceinline__ uint16_t round(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
    static __device__ __forceinline__ uint32_t round2(float x, float y) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
    }
    static __device__ __forceinline__ float value(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
};
struct Fp16 {
    static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    // Four products with one a, their sums in accumulation registers: 256 of them the compiler moves about and spills.  It does not see
    // the products in here, so the two wait states between a vector instruction and a product that reads what it wrote are part of
    // the text, and those behind the last product are settle()'s.
    static __device__ __forceinline__ void mma4(u32x4 a, u32x4 b0, u32x4 b1, u32x4 b2, u32x4 b3, f32x4 &c0, f32x4 &c1, f32x4 &c2, f32x4 &c3) {
        asm volatile(
            "s_nop 1\n\t"
            "v_mfma_f32_16x16x32_f16 %0, %4, %5, %0\n\t"
            "v_mfma_f32_16x16x32_f16 %1, %4, %6, %1\n\t"
            "v_mfma_f32_16x16x32_f16 %2, %4, %7, %2\n\t"
            "v_mfma_f32_16x16x32_f16 %3, %4, %8, %3"
            : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3)
            : "v"(a), "v"(b0), "v"(b1), "v"(b2), "v"(b3));
    }
    static __device__ __forceinline__ uint16_t round(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
    static __device__ __forceinline__ uint32_t round2(float x, float y) { return round(x) | (uint32_t)round(y) << 16; }
    static __device__ __forceinline__ float value(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
};

template <typename T>
__device__ __forceinline__ u32x2 round4(f32x4 x) {
    return u32x2{T::round2(x[0], x[1]), T::round2(x[2], x[3])};
}

// One operand of a product.  A thread's offsets from the tile's first element stay below 2^32 bytes: the host refuses strides of
// 2^22 elements and more.
struct Operand {
    const uint16_t *p;
    int64_t ld;     // elements from one row of memory to the next
    int64_t block;  // columns: elements from 64 elements of a row to the next 64; 64 where rows are contiguous
    int64_t step;   // elements from one step along k to the next
    int32_t rows;   // extent in m or n
};
constexpr int kStepK = 64;
constexpr int64_t kMaxStride = 1 << 22;

__host__ __device__ inline Operand by_rows(const uint16_t *p, int64_t ld, int32_t rows) { return Operand{p, ld, 64, kStepK, rows}; }
__host__ __device__ inline Operand by_columns(const uint16_t *p, int64_t ld, int32_t columns) { return Operand{p, ld, 64, kStepK * ld, columns}; }

// R: the tile's extent in m or n.  COLUMNS: m (n) next to m in memory.  DIRECT: the base and the rows of memory lie at multiples
// of 16 bytes and hold whole units of 8 elements; then lanes load to LDS directly, else through registers, the units at the end
// of a row element by element.
// END: what a tile holds where k has ended within a step.  ZERO: zeros.  ANY: something that is there and finite if the operand is, for
// the other operand holds zeros there.  PADDED: memory itself goes on with zeros to the end of the step.  (Zeros are put in place
// behind the loads to LDS, which costs two waits for memory a tile: the logits of 777 x 50,003 x 1,000 took 170 us for 160 without.)
enum : int { ZERO = 0, ANY = 1, PADDED = 2 };

template <int R, int THREADS, bool COLUMNS, bool DIRECT, int END>
struct Tile {
    static constexpr bool kDirect = DIRECT;
    static constexpr int kUnits = R * kStepK / 8;
    static constexpr int kPer = (kUnits + THREADS - 1) / THREADS;  // units of a thread; of fewer than threads some have the same
    static_assert(kUnits % THREADS == 0 || THREADS % kUnits == 0, "every wave loads as often");
    static constexpr int kRowUnits = COLUMNS ? R / 8 : kStepK / 8;
    static constexpr int kPairMask = R / 16 >= 8 ? 7 : R / 16 - 1;  // of the permutation of a column-major row's pairs
    static constexpr int kBytes = kUnits * 16;

    const uint16_t *base;  // uniform: the tile's first element at the present step
    int64_t ld, block, step;
    int32_t rows_left;
    int32_t wave_at;       // where the wave's first unit lies in LDS
    uint32_t at[kPer];     // byte offsets from base
    u32x4 held[DIRECT ? 1 : kPer];

    static __device__ __forceinline__ int pair_swizzle(int k) { return ((k & 3) | ((k >> 3) & 1) << 2) & kPairMask; }

    static __device__ __forceinline__ void place(int unit, int &r, int &c) {  // memory row of the tile and unit in it
        if (kUnits < THREADS) unit %= kUnits;
        r = unit / kRowUnits;
        c = unit % kRowUnits;
        if (COLUMNS) c = (((c >> 1) ^ pair_swizzle(r)) << 1) | (c & 1);
        else c ^= r & 7;
    }

    __device__ __forceinline__ uint32_t offset(int r, int c) const {
        // rows (units of a column-major row) behind the end load the last one; what comes of them is not stored
        if (COLUMNS) {
            if (DIRECT && c * 8 >= rows_left) c = rows_left / 8 - 1;
            return ((uint32_t)r * (uint32_t)ld + (uint32_t)(c >> 3) * (uint32_t)block + (c & 7) * 8) * 2u;
        }
        return ((uint32_t)(r < rows_left ? r : rows_left - 1) * (uint32_t)ld + c * 8) * 2u;
    }

    // the tile from row0 (unit-aligned column row0) on, k from step0 steps on
    __device__ __forceinline__ void init(const Operand &o, int32_t row0, int32_t step0) {
        ld = o.ld, block = o.block, step = o.step;
        rows_left = o.rows - row0;
        wave_at = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave) % (kUnits / kWave) * (kWave * 16);
        base = o.p + step0 * o.step + (COLUMNS ? (row0 / 64) * o.block + row0 % 64 : row0 * o.ld);
        const int thread = afresh(threadIdx.x);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            int r, c;
            place(i * THREADS + thread, r, c);
            at[i] = offset(r, c);
        }
    }

    // the elements of a unit that exist, from memory at any alignment; `left` of them in front of an end
    static __device__ __forceinline__ u32x4 unit_of(const char *p, int left) {
        u32x4 v = {0, 0, 0, 0};
        if (left >= 8) {
            v = *reinterpret_cast<const u32x4_any *>(p);
        } else {
            const uint16_t *e = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) v[j / 2] |= (uint32_t)e[j] << (j % 2 * 16);
        }
        return v;
    }

    // Loads to LDS are not conditional, so that nothing branches among the products: where not all of a step's k are there (`whole`
    // of them) they fetch units that are, and commit() puts what belongs there in its place.
    __device__ __forceinline__ void not_whole(int whole) {
        if constexpr (DIRECT) {
            if (END == PADDED && whole > 0) return;
            const int thread = afresh(threadIdx.x);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                int r, c;
                place(i * THREADS + thread, r, c);
                at[i] = END != ANY ? 0 : COLUMNS ? offset(r < whole ? r : 0, c) : offset(r, c * 8 < whole ? c : 0);
            }
        }
    }
    template <int I>
    __device__ __forceinline__ void load_one(lds_char *lds, int whole) {
        if constexpr (DIRECT) {
            const uint32_t from = COLUMNS ? at[I] : (uint32_t)afresh((int)at[I]);  // (else some are kept in 64 bits)
            __builtin_amdgcn_global_load_lds((global_void *)(reinterpret_cast<const char *>(base) + from),
                                             (lds_void *)(lds + (I * THREADS * 16 + wave_at)), 16, 0, 0);
        } else {
            int r, c;
            place(I * THREADS + (int)threadIdx.x, r, c);
            held[I] = unit_of(reinterpret_cast<const char *>(base) + at[I], COLUMNS ? (r < whole ? rows_left - c * 8 : 0) : whole - c * 8);
        }
    }
    __device__ __forceinline__ void commit(lds_char *lds, int whole) {
        typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
        if constexpr (DIRECT) {
            if (END == ANY || whole == kStepK || (END == PADDED && whole > 0)) return;
            __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): what the loads to LDS left is replaced
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                int unit = i * THREADS + afresh(threadIdx.x);
                if (kUnits < THREADS) unit %= kUnits;
                int r, c;
                place(unit, r, c);
                u32x4 v = {0, 0, 0, 0};
                if (COLUMNS ? r < whole : c * 8 < whole)
                    v = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(base) + offset(r, c));
                *reinterpret_cast<lds_u32x4 *>(lds + unit * 16) = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                *reinterpret_cast<lds_u32x4 *>(lds + (i * THREADS + (int)threadIdx.x % kUnits) * 16) = held[i];
        }
    }

    // Fragment of 16 rows from row0 + 16 f (row0 of the wave) and 32 k from 32 kk: lane l has row l & 15, k = 8 (l >> 4) + 0..7.
    // The address is one offset from the buffer, so that the compiler knows which buffer a read is from (else it would have every
    // transposing read wait for the loads in flight into the other one).
    static __device__ __forceinline__ u32x4 fragment(lds_char *lds, int row0, int f, int kk, int lane) {
        const int i = lane & 15, g = lane >> 4;
        if constexpr (COLUMNS) {
            const int pair = ((row0 / 16 + f) ^ pair_swizzle(8 * g + (i >> 2)));
            const int at = (8 * g + (i >> 2)) * (R * 2) + pair * 32 + (i & 3) * 8 + kk * 32 * R * 2;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + at)));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + (at + 4 * R * 2))));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            const int at = (row0 + i) * 128 + ((g ^ (i & 7)) ^ (kk * 4)) * 16 + f * 16 * 128;
            return *reinterpret_cast<__attribute__((address_space(3))) const u32x4 *>(lds + at);
        }
    }
};

// BM x BN by WM x WN waves, STAGES buffers in LDS
template <int BM_, int BN_, int WM_, int WN_, int STAGES = 2>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kThreads = WM * WN * kWave;
    static constexpr int TM = BM / WM, TN = BN / WN;  // a wave's part
    static constexpr int FM = TM / 16, FN = TN / 16;  // in fragments
    static constexpr int kStages = STAGES;
    static constexpr int kGroup = FM * FN == 64 ? 4 : 1;  // products at a time
    static constexpr int kBytesA = BM * kStepK * 2, kBytesB = BN * kStepK * 2;  // one buffer
    static constexpr int kLds = kBytesA + kBytesB;
};

// The buffers of a kernel, an object of its own for each operand's part of each: so the compiler sees that one that is read is not one
// that is being filled, and does not have every read wait for all loads.
struct Stage {
    lds_char *a, *b;
};
#define CFGZIP_STAGES(S, name)                                                                                                     \
    __shared__ __attribute__((aligned(16))) char name##a0[S::kBytesA], name##a1[S::kBytesA], name##a2[S::kStages > 2 ? S::kBytesA : 16], \
        name##a3[S::kStages > 3 ? S::kBytesA : 16], name##b0[S::kBytesB], name##b1[S::kBytesB],                                    \
        name##b2[S::kStages > 2 ? S::kBytesB : 16], name##b3[S::kStages > 3 ? S::kBytesB : 16];                                    \
    const Stage name[4] = {{(lds_char *)name##a0, (lds_char *)name##b0},                                                           \
                           {(lds_char *)name##a1, (lds_char *)name##b1},                                                           \
                           {(lds_char *)name##a2, (lds_char *)name##b2},                                                           \
                           {(lds_char *)name##a3, (lds_char *)name##b3}}

template <typename T, typename S, typename TileA, typename TileB>
struct Fragments {
    u32x4 a[S::FM], b[S::FN];
    template <int Q>
    __device__ __forceinline__ void read_one(const Stage &lds, int wm, int wn, int kk, int lane) {
        if constexpr (Q < S::FN) b[Q] = TileB::fragment(lds.b, wn * S::TN, Q, kk, lane);
        else a[Q - S::FN] = TileA::fragment(lds.a, wm * S::TM, Q - S::FN, kk, lane);
    }
    // acc[i][j][r]: lane l has m = 16 i + 4 (l >> 4) + r, n = 16 j + (l & 15) of its wave's part; group P of the FM * FN products
    template <int P, int BYTE, typename X>
    __device__ __forceinline__ void multiply_some(f32x4 (&acc)[S::FM][S::FN], const X &scales) const {
        constexpr int i = P * S::kGroup / S::FN, j = P * S::kGroup % S::FN;
        if constexpr (X::kScaled)
            T::template mma4<BYTE>(a[i], b[j], b[j + 1], b[j + 2], b[j + 3], acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3],
                                   scales.a[i], scales.b[j], scales.b[j + 1], scales.b[j + 2], scales.b[j + 3]);
        else if constexpr (S::kGroup == 4)
            T::mma4(a[i], b[j], b[j + 1], b[j + 2], b[j + 3], acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3]);
        else acc[i][j] = T::mma(a[i], b[j], acc[i][j]);
    }
};

// behind the last of mma4's products: their sums may be read by what the compiler writes.  Read only: with something added to them in place
// in lanes that a condition picks the compiler moved them about between the products, and results were wrong.
template <typename S>
__device__ __forceinline__ void settle(f32x4 (&acc)[S::FM][S::FN]) {
    if constexpr (S::kGroup == 4) {
        asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) asm volatile("" : "+a"(acc[i][j]));
    }
}

// the first of `count` things, spread evenly over `groups` groups, that comes behind group p - 1
constexpr int from(int p, int count, int groups) { return p >= groups ? count : (p * count + groups - 1) / groups; }

// The products of `now`; the fragments `next` are read in three quarters of their time, and LOADS loads begun and then `last`, evenly
// among them.  The order is the one written here: the compiler's own gathers the reads, and the matrix cores wait.
template <typename S, int LOADS, int BYTE, typename F, typename L, typename M, typename X>
__device__ __forceinline__ void multiply_and_read(const F &now, F &next, const Stage &lds, int wm, int wn, int kk, int lane,
                                                  f32x4 (&acc)[S::FM][S::FN], L &&load_one, M &&last, const X &scales) {
    constexpr int kGroups = S::FM * S::FN / S::kGroup, kFragments = S::FM + S::FN, kLast = kGroups * 3 / 4 ? kGroups * 3 / 4 : 1;
    each<kGroups>([&](auto p) CFGZIP_INLINE {
        now.template multiply_some<p.value, BYTE>(acc, scales);
        constexpr int q0 = from(p.value, kFragments, kLast), q1 = from(p.value + 1, kFragments, kLast);
        each<q1 - q0>([&](auto q) CFGZIP_INLINE { next.template read_one<q0 + q.value>(lds, wm, wn, kk, lane); });
        constexpr int l0 = from(p.value, LOADS + 1, kGroups), l1 = from(p.value + 1, LOADS + 1, kGroups);
        each<l1 - l0>([&](auto l) CFGZIP_INLINE {
            if constexpr (l0 + l.value < LOADS) load_one(std::integral_constant<int, l0 + l.value>{});
            else last();
        });
        if constexpr (kGroups > 4) __builtin_amdgcn_sched_barrier(0);
    });
}

// Waits until at most `LEFT` of the wave's loads are on their way, and for everybody.  What is read from or loaded into LDS stays on its
// side.
template <int LEFT>
__device__ __forceinline__ void wait_for_loads() {
    static_assert(LEFT < 64, "as far as the counter goes");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 0x70);  // vmcnt(LEFT) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What a workgroup multiplies: for each of its tiles, A's and B's first rows and the steps along k.
struct Work {
    int32_t m0, n0, step0, k;  // k elements from step0 steps on
};

// Scales of what is multiplied, for operands that have them: those of two steps at a time (kStages of them), kept by the lane that has
// the fragment.  begin(w) asks memory for a tile's first ones, ask() for those of the next two steps, put() leaves them in LDS, take()
// fetches the lane's own from there.  With scales a workgroup has one tile (the registers do not suffice for a next one's beginning).
struct NoScales {
    static constexpr bool kScaled = false;
    __device__ void begin(const Work &) {}
    __device__ void ask() {}
    __device__ void put() {}
    __device__ void take(int, int, int) {}
};

// Makes tile after tile: work(i, Work &) says whether there is an i-th one and which, store(i, acc, ..) takes its sums.  While
// the sums of one are stored the first steps of the next are on their way into LDS.
template <typename T, typename S, typename TileA, typename TileB, typename W, typename E, typename X>
__device__ __forceinline__ void multiply(const Operand &A, const Operand &B, const Stage (&lds)[4], W &&work, E &&store, X &&scales) {
    constexpr bool kScaled = std::remove_reference_t<X>::kScaled;
    static_assert(!kScaled || S::kStages == 2, "scales of two steps at a time");
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wm = wave / S::WN, wn = wave % S::WN;
    constexpr int kStages = S::kStages, kLoads = TileA::kPer + TileB::kPer;
    constexpr int kToLds = (TileA::kDirect ? TileA::kPer : 0) + (TileB::kDirect ? TileB::kPer : 0);
    TileA ta;
    TileB tb;
    Work w;
    if (!work(0, w)) return;
    // of the loads: k from the step to be loaded next on; how many of them that step has; and of the step loaded last
    int32_t k_left, whole, loaded;
    auto look = [&]() CFGZIP_INLINE {
        whole = kStepK;
        if (k_left < kStepK) {
            whole = k_left > 0 ? k_left : 0;
            ta.not_whole(whole);
            tb.not_whole(whole);
        }
    };
    auto advance = [&]() CFGZIP_INLINE {
        loaded = whole;
        if (k_left > kStepK) {  // else the base stays at elements that are there
            ta.base += ta.step;
            tb.base += tb.step;
        }
        k_left -= kStepK;
        look();
    };
    auto start = [&]() CFGZIP_INLINE {
        ta.init(A, w.m0, w.step0);
        tb.init(B, w.n0, w.step0);
        k_left = w.k;
        look();
    };
    auto load_into = [&](const Stage &to) CFGZIP_INLINE {
        return [&](auto i) CFGZIP_INLINE {
            if constexpr (i.value < TileA::kPer) ta.template load_one<i.value>(to.a, whole);
            else tb.template load_one<i.value - TileA::kPer>(to.b, whole);
        };
    };
    auto commit = [&](const Stage &to) CFGZIP_INLINE {
        ta.commit(to.a, loaded);
        tb.commit(to.b, loaded);
    };
    start();
    each<kStages>([&](auto s) CFGZIP_INLINE {
        each<kLoads>(load_into(lds[s.value]));
        advance();
        if constexpr (s.value + 1 < kStages) commit(lds[s.value]);
    });
    if constexpr (kScaled) {
        scales.begin(w);
        scales.put();
    }
    wait_for_loads<(kStages - 1) * kToLds>();
    if constexpr (kScaled) scales.take(wm, wn, lane);
    Fragments<T, S, TileA, TileB> f0, f1;
    const auto no_load = [](auto) CFGZIP_INLINE {};
    const auto nothing = []() CFGZIP_INLINE {};
    f32x4 acc[S::FM][S::FN];
    for (int32_t tile = 0;; ++tile) {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
        // (again for every tile: its registers are the sums' way out in between)
        each<S::FM + S::FN>([&](auto q) CFGZIP_INLINE { f0.template read_one<q.value>(lds[0], wm, wn, 0, lane); });
        bool more = false;
        // Half a step is multiplied at a time, while the fragments of the next half are read.  Where those are of the next step, its
        // loads have to have come in for everybody; then this step's buffer has been read by everybody, and is loaded again with
        // what lies kStages steps ahead.  kStages steps in a row without a way out in between (the sums would be moved about):
        // behind a tile's last step follow some of zeros.
        const int32_t steps = (w.k + kStepK - 1) / kStepK;
        int32_t left = (steps + kStages - 1) / kStages;
        do {
            each<kStages>([&](auto s) CFGZIP_INLINE {
                const Stage &here = lds[s.value], &next = lds[(s.value + 1) % kStages];
                multiply_and_read<S, 0, 2 * s.value>(f0, f1, here, wm, wn, 1, lane, acc, no_load, nothing, scales);
                commit(lds[(s.value + kStages - 1) % kStages]);
                if constexpr (kScaled && s.value == 1) scales.put();
                wait_for_loads<(kStages - 2) * kToLds>();
                if constexpr (s.value == 0) {
                    if constexpr (kScaled) {
                        scales.ask();
                    } else if (left == 1) {  // from here on it is the next tile's steps that are loaded
                        more = work(tile + 1, w);
                        if (more) start();
                    }
                }
                multiply_and_read<S, kLoads, 2 * s.value + 1>(f1, f0, next, wm, wn, 0, lane, acc, load_into(here), advance, scales);
            });
            if constexpr (kScaled) scales.take(wm, wn, lane);
        } while (--left > 0);
        settle<S>(acc);
        store(tile, acc, wm, wn, afresh(lane));
        if (!more) break;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): nothing is on its way into LDS that may soon be another workgroup's
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
