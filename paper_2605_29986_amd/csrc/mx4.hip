// Blocks of 32 values in 4 bits with a shared power of two: quantisation, reading back, and the vocabulary projection's logits
// from weights so kept, under a grammar's masks.
//
// A block has the scale 2^e, e = floor(log2 max|x|) - 2 >= -127, kept as the byte e + 127; a value is the nearest of
// +-{0, 1/2, 1, 3/2, 2, 3, 4, 6} to x / 2^e, ties to the even code.  Row r has its codes at codes[r][16 * blocks], the earlier
// value in a byte's low half, and its scales at scales[r][blocks].  A block that holds an infinity or a NaN has the scale byte
// 255, which makes all of its values NaN.
//
// In the product a 4-bit value times its scale is exact in bf16, so weights become bf16 in registers and are multiplied there
// with bf16 hidden states; fp16 hidden states go in as the sum of two bf16 numbers, which is exact too.  Hidden states in 4 bits
// are multiplied as they are, by the matrix instruction that takes both sides' scales.  Sums are fp32.

#include "gemm16.hpp"

namespace cfgzip {
namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_bytes __attribute__((ext_vector_type(4), aligned(1)));
typedef uint16_t u16_bytes __attribute__((aligned(1)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

constexpr uint32_t kNan = 0x7FC00000u;
constexpr float kInf = __builtin_inff();

// the scale of a byte as a float's bits: byte 0 is 2^-127, which is subnormal, byte 255 NaN
__device__ __forceinline__ uint32_t scale_bits(uint32_t byte) {
    const uint32_t b = byte << 23;
    return byte == 255 ? kNan : b > 0x00400000u ? b : 0x00400000u;
}

// ---------------------------------------------------------------- quantisation

// eight values of a row from element c on, 0 behind its end
template <int DTYPE>
__device__ __forceinline__ void load8(const void *x, int64_t at, int32_t left, float (&v)[8]) {
    if constexpr (DTYPE == CFGZIP_DTYPE_F32) {
        const float *p = static_cast<const float *>(x) + at;
        if (left >= 8) {
            const f32x4 a = *reinterpret_cast<const f32x4_any *>(p), b = *reinterpret_cast<const f32x4_any *>(p + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < left ? p[j] : 0.0f;
        }
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(x) + at;
        uint16_t e[8];
        if (left >= 8) {
            const u32x4 a = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = (uint16_t)(a[j / 2] >> (j % 2 * 16));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : (uint16_t)0;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = DTYPE == CFGZIP_DTYPE_BF16 ? Bf16::value(e[j]) : Fp16::value(e[j]);
    }
}

constexpr int kUnroll = 4;

// Units of eight values; four lanes next to each other have a block.  A wave takes 64 units next to each other at a time and
// kUnroll times that in all, whole rows after each other.
template <int DTYPE>
__global__ __launch_bounds__(256) void quantize_kernel(const void *x, int64_t x_ld, int64_t R, int32_t K, int32_t nb, uint32_t *codes,
                                                       uint8_t *scales) {
    const int32_t per = nb * 4;
    const int64_t units = R * per;
    const int64_t first = ((int64_t)blockIdx.x * 256 + threadIdx.x / kWave * kWave) * kUnroll + threadIdx.x % kWave;
    int64_t row = first / per;
    int32_t u = (int32_t)(first - row * per);
    float v[kUnroll][8];
    int64_t rows[kUnroll];
    int32_t us[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        rows[i] = row, us[i] = u;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
        if (row < R) load8<DTYPE>(x, row * x_ld + u * 8, K - u * 8, v[i]);
        for (u += kWave; u >= per; u -= per) ++row;
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        uint32_t most = 0;  // of the values' bits without sign: NaN above infinity above the rest
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = __builtin_bit_cast(uint32_t, v[i][j]) & 0x7FFFFFFFu;
            most = b > most ? b : most;
        }
        uint32_t other = __shfl_xor(most, 1);
        most = other > most ? other : most;
        other = __shfl_xor(most, 2);
        most = other > most ? other : most;
        const uint32_t e = most >> 23;
        const uint32_t byte = e == 255 ? 255 : e > 2 ? e - 2 : 0;
        const float scale = __builtin_bit_cast(float, scale_bits(byte));
        uint32_t code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[i][0], v[i][1], scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[i][2], v[i][3], scale, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[i][4], v[i][5], scale, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[i][6], v[i][7], scale, 3);
        if (rows[i] < R) {
            const int64_t at = rows[i] * per + us[i];
            codes[at] = byte == 255 ? 0u : code;
            if (us[i] % 4 == 0) scales[at / 4] = (uint8_t)byte;
        }
    }
    (void)units;
}

template <int DTYPE>
__global__ __launch_bounds__(256) void values_kernel(const uint32_t *codes, const uint8_t *scales, int64_t R, int32_t K, int32_t nb,
                                                     void *x, int64_t x_ld) {
    const int32_t per = nb * 4;
    const int64_t first = ((int64_t)blockIdx.x * 256 + threadIdx.x / kWave * kWave) * kUnroll + threadIdx.x % kWave;
    int64_t row = first / per;
    int32_t u = (int32_t)(first - row * per);
    uint32_t code[kUnroll], byte[kUnroll];
    int64_t rows[kUnroll];
    int32_t us[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        rows[i] = row, us[i] = u;
        code[i] = byte[i] = 0;
        if (row < R) {
            const int64_t at = row * per + u;
            code[i] = codes[at];
            byte[i] = scales[at / 4];
        }
        for (u += kWave; u >= per; u -= per) ++row;
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const int32_t left = K - us[i] * 8;
        if (rows[i] >= R || left <= 0) continue;
        const float scale = __builtin_bit_cast(float, scale_bits(byte[i]));
        f32x2 v[4];
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], scale, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], scale, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], scale, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], scale, 3);
        if (byte[i] == 255)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = f32x2{__builtin_nanf(""), __builtin_nanf("")};
        const int64_t at = rows[i] * x_ld + us[i] * 8;
        if constexpr (DTYPE == CFGZIP_DTYPE_F32) {
            float *p = static_cast<float *>(x) + at;
            if (left >= 8) {
                *reinterpret_cast<f32x4_any *>(p) = f32x4{v[0][0], v[0][1], v[1][0], v[1][1]};
                *reinterpret_cast<f32x4_any *>(p + 4) = f32x4{v[2][0], v[2][1], v[3][0], v[3][1]};
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) p[j] = v[j / 2][j % 2];
            }
        } else {
            uint16_t *p = static_cast<uint16_t *>(x) + at;
            uint16_t e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                e[j] = DTYPE == CFGZIP_DTYPE_BF16 ? Bf16::round(v[j / 2][j % 2]) : Fp16::round(v[j / 2][j % 2]);
            if (left >= 8) {
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
                *reinterpret_cast<u32x4_any *>(p) = w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) p[j] = e[j];
            }
        }
    }
}

// ---------------------------------------------------------------- logits

struct Weights {
    const uint8_t *codes;   // [V][16 * nb]
    const uint8_t *scales;  // [V][nb]
    int32_t V, nb;
};

struct Logits {
    void *p;
    int64_t ld;
    int32_t B;
    bool f32;
};

// eight weights (a quarter of a block) as bf16
__device__ __forceinline__ u32x4 weights8(uint32_t code, float scale) {
    u32x4 w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
    return w;
}

__device__ __forceinline__ f32x4 multiply4(u32x4 a, u32x4 b, f32x4 c, uint32_t scale_a, uint32_t scale_b) {
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)scale_a, 0, (int)scale_b);
}

// logits of four tokens from v on in row b; bit r of ok: token v + r is admitted
__device__ __forceinline__ void store_logits(const Logits &o, int32_t b, int32_t v, int32_t V, f32x4 z, uint32_t ok) {
    const int32_t left = V - v;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (!(ok >> r & 1)) z[r] = -kInf;
    if (o.f32) {
        float *p = static_cast<float *>(o.p) + b * o.ld + v;
        if (left >= 4) {
            *reinterpret_cast<f32x4_any *>(p) = z;
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < left) p[r] = z[r];
        }
    } else {
        uint16_t *p = static_cast<uint16_t *>(o.p) + b * o.ld + v;
        if (left >= 4) {
            *reinterpret_cast<u32x2_any *>(p) = round4<Bf16>(z);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < left) p[r] = Bf16::round(z[r]);
        }
    }
}

// Few rows: reading the weights is what counts.  Hidden states lie in LDS; a wave takes 16 tokens (or a share of the blocks of 16
// tokens, joined through LDS where tokens are few) straight from memory, 64 bytes of a token at a load and kAhead loads at a
// time.  Tokens that no row admits are not read.
struct FewArgs {
    Weights w;
    const void *x;          // [B] rows, x_ld elements apart (codes: 16 nb bytes)
    int64_t x_ld;
    const uint8_t *x_scales;  // 4 bits
    int32_t K;
    Logits out;
    const int32_t *bits;  // masks over classes (class_of_token given) or tokens, or null
    int64_t words;
    const int32_t *class_of_token;
    int32_t share;        // waves of a tile: 1, 2, 4, 8 or 16
    int32_t lds_row;      // bytes from one row of hidden states to the next
};

enum : int { X_BF16 = 0, X_F16 = 1, X_4 = 2 };

constexpr int kFewThreads = 1024;
constexpr int kFewWaves = kFewThreads / kWave;
constexpr int kAhead = 8;  // loads of 64 bytes a token: a KB and four blocks each

// ROWS: LDS rows of hidden states in fragments of 16.  fp16 has two bf16 rows of each: the rest lies 8 rows behind (up to 8 rows,
// one fragment) or 16.
template <int X, int FRAGMENTS>
__global__ __launch_bounds__(kFewThreads) void few_rows_kernel(FewArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int m = lane & 15, g = lane >> 4;
    const int32_t nb = a.w.nb, B = a.out.B, V = a.w.V;
    const int rest = FRAGMENTS == 2 ? 16 : 8;  // where the rests of fp16 lie

    // hidden states to LDS; what lies behind K is 0
    if constexpr (X == X_4) {
        for (int32_t k = threadIdx.x; k < B * nb; k += kFewThreads) {
            const int32_t b = k / nb, c = k % nb;
            *reinterpret_cast<u32x4 *>(lds + b * a.lds_row + c * 16) =
                *reinterpret_cast<const u32x4_bytes *>(static_cast<const uint8_t *>(a.x) + b * a.x_ld + c * 16);
            lds[b * a.lds_row + nb * 16 + c] = (char)a.x_scales[(int64_t)b * nb + c];
        }
    } else {
        const uint16_t *x = static_cast<const uint16_t *>(a.x);
        const int32_t units = nb * 4;
        for (int32_t k = threadIdx.x; k < B * units; k += kFewThreads) {
            const int32_t b = k / units, c = k % units, left = a.K - c * 8;
            uint16_t e[8];
            if (left >= 8) {
                const u32x4 v = *reinterpret_cast<const u32x4_any *>(x + b * a.x_ld + c * 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = (uint16_t)(v[j / 2] >> (j % 2 * 16));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = j < left ? x[b * a.x_ld + c * 8 + j] : (uint16_t)0;
            }
            u32x4 hi = {0, 0, 0, 0}, lo = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t h = e[j], l = 0;
                if constexpr (X == X_F16) {
                    const float f = Fp16::value(e[j]);
                    h = Bf16::round(f);
                    const float d = f - Bf16::value((uint16_t)h);
                    l = fabsf(f) < kInf ? Bf16::round(d) : 0;
                }
                hi[j / 2] |= h << (j % 2 * 16);
                lo[j / 2] |= l << (j % 2 * 16);
            }
            *reinterpret_cast<u32x4 *>(lds + b * a.lds_row + c * 16) = hi;
            if constexpr (X == X_F16) *reinterpret_cast<u32x4 *>(lds + (rest + b) * a.lds_row + c * 16) = lo;
        }
    }
    __syncthreads();

    // lanes of rows that are not there read one that is
    const char *xs[FRAGMENTS];
    if constexpr (X == X_F16) {
        const int b = m < 8 || FRAGMENTS == 2 ? m : m - 8;
        const int row = b < B ? b : B - 1;
        xs[0] = lds + (FRAGMENTS == 1 && m >= 8 ? rest + row : row) * a.lds_row;
        if (FRAGMENTS == 2) xs[FRAGMENTS - 1] = lds + (rest + row) * a.lds_row;
    } else {
#pragma unroll
        for (int f = 0; f < FRAGMENTS; ++f) {
            const int row = f * 16 + m;
            xs[f] = lds + (row < B ? row : B - 1) * a.lds_row;
        }
    }

    const int tiles_here = kFewWaves / a.share;
    const int part = wave % a.share;
    const int32_t loads = (nb + 3) / 4;
    const int32_t l0 = (int32_t)((int64_t)loads * part / a.share), l1 = (int32_t)((int64_t)loads * (part + 1) / a.share);
    const int32_t tiles = (V + 15) / 16;
    f32x4 *joined = reinterpret_cast<f32x4 *>(lds + (size_t)(X == X_F16 ? rest + B : B) * a.lds_row);

    // which rows admit token v: bit b
    auto admitting = [&](int32_t tile) -> uint32_t {
        const int32_t v = tile * 16 + m;
        uint32_t ok = 0;
        if (tile < tiles && v < V) {
            if (!a.bits) {
                ok = 0xFFFFFFFFu;
            } else {
                const int32_t k = a.class_of_token ? a.class_of_token[v] : v;
                for (int32_t b = g; b < B; b += 4) ok |= (uint32_t)(a.bits[b * a.words + (k >> 5)] >> (k & 31) & 1) << b;
            }
        }
        ok |= __shfl_xor(ok, 16);
        ok |= __shfl_xor(ok, 32);
        return ok;
    };

    int32_t tile = blockIdx.x * tiles_here + wave / a.share;
    const int32_t stride = gridDim.x * tiles_here;
    // every wave of a workgroup goes around equally often: there is a barrier in the way where tiles are shared
    const int32_t rounds = (tiles - (int32_t)blockIdx.x * tiles_here + stride - 1) / stride;
    uint32_t ok = admitting(tile);
    for (int32_t round = 0; round < rounds; ++round, tile += stride) {
        const uint32_t ok_next = round + 1 < rounds ? admitting(tile + stride) : 0;
        f32x4 acc[FRAGMENTS];
#pragma unroll
        for (int f = 0; f < FRAGMENTS; ++f) acc[f] = f32x4{0, 0, 0, 0};
        const int32_t v = tile * 16 + m;
        const uint8_t *codes = a.w.codes + (int64_t)v * nb * 16, *scales = a.w.scales + (int64_t)v * nb;
        for (int32_t l = l0; l < l1; l += kAhead) {
            u32x4 code[kAhead];
            uint32_t byte[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int32_t block = (l + i) * 4 + g;
                code[i] = u32x4{0, 0, 0, 0};
                byte[i] = 127;
                if (ok != 0 && l + i < l1 && block < nb) {
                    code[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes + block * 16));
                    byte[i] = scales[block];
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int32_t last = nb - 1, block = (l + i) * 4 + g < nb ? (l + i) * 4 + g : last;
                if (l + i >= l1) break;
                if constexpr (X == X_4) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(xs[0] + block * 16);
                    acc[0] = multiply4(code[i], x, acc[0], byte[i], (uint8_t)xs[0][nb * 16 + block]);
                } else {
                    const float scale = __builtin_bit_cast(float, scale_bits(byte[i]));
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const u32x4 w = weights8(code[i][q], scale);
#pragma unroll
                        for (int f = 0; f < FRAGMENTS; ++f)
                            acc[f] = Bf16::mma(w, *reinterpret_cast<const u32x4 *>(xs[f] + block * 64 + q * 16), acc[f]);
                    }
                }
            }
        }
        if (a.share > 1) {
            __syncthreads();  // the round before has been read
#pragma unroll
            for (int f = 0; f < FRAGMENTS; ++f) joined[(f * kFewWaves + wave) * kWave + lane] = acc[f];
            __syncthreads();
            if (part == 0) {
                for (int s = 1; s < a.share; ++s)
#pragma unroll
                    for (int f = 0; f < FRAGMENTS; ++f) acc[f] += joined[(f * kFewWaves + wave + s) * kWave + lane];
            }
        }
        if constexpr (X == X_F16) {
            if (FRAGMENTS == 2) {
                acc[0] += acc[FRAGMENTS - 1];
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[0][r] += __shfl_xor(acc[0][r], 8);
            }
        }
        uint32_t oks[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) oks[r] = __shfl(ok, 4 * g + r);
        if (part == 0 && tile < tiles && tile * 16 + 4 * g < V) {
            constexpr int kOut = X == X_F16 ? 1 : FRAGMENTS;
#pragma unroll
            for (int f = 0; f < kOut; ++f) {
                const int32_t b = f * 16 + m;
                if (b >= B) continue;
                const uint32_t four = (oks[0] >> b & 1) | (oks[1] >> b & 1) << 1 | (oks[2] >> b & 1) << 2 | (oks[3] >> b & 1) << 3;
                store_logits(a.out, b, tile * 16 + 4 * g, V, acc[f], four);
            }
        }
        ok = ok_next;
    }
}

// ---------------------------------------------------------------- many rows

static __device__ const u32x4 kZeros = {0, 0, 0, 0};  // what lanes behind the end of a row load

// Rows of UNITS units of 16 bytes of a step, to LDS directly; unit c of row r lies where the 16 lanes of a read spread over all banks
template <int R, int THREADS, int UNITS>
struct Rows {
    static constexpr int kPer = R * UNITS / THREADS;
    static_assert(R * UNITS % THREADS == 0, "whole units");
    static constexpr int kBytes = R * UNITS * 16;
    const char *base;
    int32_t left;  // units of a row from the present step on
    uint32_t at[kPer];

    static __device__ __forceinline__ int swizzle(int r) { return UNITS == 4 ? r >> 2 & 3 : r & (UNITS - 1); }

    __device__ __forceinline__ void init(const void *p, int64_t row_bytes, int32_t rows_left, int32_t units) {
        base = static_cast<const char *>(p);
        left = units;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int u = i * THREADS + (int)threadIdx.x, r = u / UNITS, c = (u % UNITS) ^ swizzle(r);
            at[i] = (uint32_t)((r < rows_left ? r : rows_left - 1) * row_bytes) + c * 16;
        }
    }
    __device__ __forceinline__ void load(char *lds) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int u = i * THREADS + (int)threadIdx.x, r = u / UNITS, c = (u % UNITS) ^ swizzle(r);
            const char *p = base + at[i];
            if (left < UNITS && c >= left) p = reinterpret_cast<const char *>(&kZeros);
            __builtin_amdgcn_global_load_lds((global_void *)p, (lds_void *)(lds + (i * THREADS + wave * kWave) * 16), 16, 0, 0);
        }
        base += UNITS * 16;
        left -= UNITS;
    }
    static __device__ __forceinline__ u32x4 read(const char *lds, int r, int c) {
        return *reinterpret_cast<const u32x4 *>(lds + r * (UNITS * 16) + (c ^ swizzle(r)) * 16);
    }
};

struct ManyArgs {
    Weights w;
    const char *x;         // 16 bits: [parts][B] rows; 4 bits: [B][16 nb]
    int64_t x_row_bytes;
    int64_t x_part_bytes;  // from one part to the next
    int32_t parts;         // 2 for fp16: bf16 and rest
    int32_t x_units;       // of 16 bytes in a row
    const uint8_t *x_scales;
    Logits out;
    const int32_t *bits;  // over tokens, or null
    int64_t words;
    int32_t tiles_m, tiles_n;
};

template <typename S>
__device__ __forceinline__ void store_tile(const ManyArgs &a, int32_t tm, int32_t tn, int wm, int wn, int lane,
                                           const f32x4 (&acc)[S::FM][S::FN]) {
    const int g = lane >> 4;
    const int32_t first = tm * S::BM + wm * S::TM;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int32_t b = tn * S::BN + wn * S::TN + 16 * j + (lane & 15);
        if (b >= a.out.B) continue;
        uint32_t words[(S::TM + 31) / 32];
#pragma unroll
        for (int w = 0; w < (S::TM + 31) / 32; ++w) {
            const int64_t k = (first >> 5) + w;
            words[w] = !a.bits ? 0xFFFFFFFFu : k < a.words ? (uint32_t)a.bits[b * a.words + k] : 0u;
        }
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            const int32_t v = first + 16 * i + 4 * g;
            if (v < a.w.V) store_logits(a.out, b, v, a.w.V, acc[i][j], words[i / 2] >> (v & 31));
        }
    }
}

// 16-bit hidden states.  A step has 128 k: lane (r, g) of a fragment has block g of its token, 32 weights, as four fragments of
// eight, and the hidden states of the same k.
template <typename S>
__global__ __launch_bounds__(S::kThreads) void many_rows_kernel(ManyArgs a) {
    using RowsW = Rows<S::BM, S::kThreads, 4>;
    using RowsX = Rows<S::BN, S::kThreads, 16>;
    constexpr int kBuffer = RowsW::kBytes + RowsX::kBytes;
    __shared__ __attribute__((aligned(16))) char lds0[kBuffer], lds1[kBuffer];
    int32_t tm, tn;
    tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wm = wave / S::WN, wn = wave % S::WN, r = lane & 15, g = lane >> 4;
    const int32_t m0 = tm * S::BM, n0 = tn * S::BN;
    f32x4 acc[S::FM][S::FN];
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    const uint8_t *scale_row[S::FM];
#pragma unroll
    for (int i = 0; i < S::FM; ++i) {
        const int32_t v = m0 + wm * S::TM + 16 * i + r;
        scale_row[i] = a.w.scales + (int64_t)(v < a.w.V ? v : a.w.V - 1) * a.w.nb;
    }
    for (int part = 0; part < a.parts; ++part) {
        RowsW tw;
        RowsX tx;
        tw.init(a.w.codes + (int64_t)m0 * a.w.nb * 16, (int64_t)a.w.nb * 16, a.w.V - m0, a.w.nb);
        tx.init(a.x + part * a.x_part_bytes + n0 * a.x_row_bytes, a.x_row_bytes, a.out.B - n0, a.x_units);
        uint32_t byte[S::FM];
        int32_t block = g;
        auto load = [&](char *lds) {
            tw.load(lds);
            tx.load(lds + RowsW::kBytes);
        };
        auto scales = [&]() {
#pragma unroll
            for (int i = 0; i < S::FM; ++i) byte[i] = block < a.w.nb ? scale_row[i][block] : 127;
            block += 4;
        };
        auto step = [&](const char *lds) {
            u32x4 code[S::FM];
            float scale[S::FM];
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                code[i] = RowsW::read(lds, wm * S::TM + 16 * i + r, g);
                scale[i] = __builtin_bit_cast(float, scale_bits(byte[i]));
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                u32x4 x[S::FN];
#pragma unroll
                for (int j = 0; j < S::FN; ++j) x[j] = RowsX::read(lds + RowsW::kBytes, wn * S::TN + 16 * j + r, g * 4 + q);
#pragma unroll
                for (int i = 0; i < S::FM; ++i) {
                    const u32x4 w = weights8(code[i][q], scale[i]);
#pragma unroll
                    for (int j = 0; j < S::FN; ++j) acc[i][j] = Bf16::mma(w, x[j], acc[i][j]);
                }
            }
        };
        int32_t steps = (a.w.nb + 3) / 4;
        __syncthreads();  // the part before has been read
        load(lds0);
        scales();
        __syncthreads();
        while (true) {
            if (steps > 1) load(lds1);
            step(lds0);
            if (steps == 1) break;
            scales();
            __syncthreads();
            if (steps > 2) load(lds0);
            step(lds1);
            if (steps == 2) break;
            scales();
            __syncthreads();
            steps -= 2;
        }
    }
    store_tile<S>(a, tm, tn, wm, wn, lane, acc);
}

// Hidden states in 4 bits.  A step has 256 k; lane (r, g) of a fragment has block 2 g + kk, so that its two scales lie side by side.
template <typename S>
__global__ __launch_bounds__(S::kThreads) void many_rows4_kernel(ManyArgs a) {
    using RowsW = Rows<S::BM, S::kThreads, 8>;
    using RowsX = Rows<S::BN, S::kThreads, 8>;
    constexpr int kBuffer = RowsW::kBytes + RowsX::kBytes;
    __shared__ __attribute__((aligned(16))) char lds0[kBuffer], lds1[kBuffer];
    int32_t tm, tn;
    tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wm = wave / S::WN, wn = wave % S::WN, r = lane & 15, g = lane >> 4;
    const int32_t m0 = tm * S::BM, n0 = tn * S::BN, nb = a.w.nb;
    f32x4 acc[S::FM][S::FN];
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    RowsW tw;
    RowsX tx;
    tw.init(a.w.codes + (int64_t)m0 * nb * 16, (int64_t)nb * 16, a.w.V - m0, nb);
    tx.init(a.x + n0 * a.x_row_bytes, a.x_row_bytes, a.out.B - n0, nb);
    const uint8_t *base_w = a.w.scales + (int64_t)m0 * nb, *base_x = a.x_scales + (int64_t)n0 * nb;
    uint32_t at_w[S::FM], at_x[S::FN];
#pragma unroll
    for (int i = 0; i < S::FM; ++i) {
        const int32_t v = wm * S::TM + 16 * i + r;
        at_w[i] = (uint32_t)(m0 + v < a.w.V ? v : a.w.V - 1 - m0) * nb;
    }
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int32_t b = wn * S::TN + 16 * j + r;
        at_x[j] = (uint32_t)(n0 + b < a.out.B ? b : a.out.B - 1 - n0) * nb;
    }
    uint32_t next_w[S::FM], next_x[S::FN];
    int32_t block = 2 * g;
    auto pair = [&](const uint8_t *p) -> uint32_t {
        return block + 1 < nb ? *reinterpret_cast<const u16_bytes *>(p) : block < nb ? p[0] : 0;
    };
    auto scales = [&]() {
#pragma unroll
        for (int i = 0; i < S::FM; ++i) next_w[i] = pair(base_w + at_w[i] + block);
#pragma unroll
        for (int j = 0; j < S::FN; ++j) next_x[j] = pair(base_x + at_x[j] + block);
        block += 8;
    };
    auto load = [&](char *lds) {
        tw.load(lds);
        tx.load(lds + RowsW::kBytes);
    };
    auto step = [&](const char *lds, bool more) {
        uint32_t sw[S::FM], sx[S::FN];
#pragma unroll
        for (int i = 0; i < S::FM; ++i) sw[i] = next_w[i];
#pragma unroll
        for (int j = 0; j < S::FN; ++j) sx[j] = next_x[j];
        if (more) scales();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 x[S::FN];
#pragma unroll
            for (int j = 0; j < S::FN; ++j) x[j] = RowsX::read(lds + RowsW::kBytes, wn * S::TN + 16 * j + r, 2 * g + kk);
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const u32x4 w = RowsW::read(lds, wm * S::TM + 16 * i + r, 2 * g + kk);
                const i32x8 wide = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < S::FN; ++j) {
                    const i32x8 y = {(int)x[j][0], (int)x[j][1], (int)x[j][2], (int)x[j][3], 0, 0, 0, 0};
                    acc[i][j] = kk == 0 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide, y, acc[i][j], 4, 4, 0, (int)sw[i], 0, (int)sx[j])
                                        : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide, y, acc[i][j], 4, 4, 1, (int)sw[i], 1, (int)sx[j]);
                }
            }
        }
    };
    int32_t steps = (nb + 7) / 8;
    load(lds0);
    scales();
    __syncthreads();
    while (true) {
        if (steps > 1) load(lds1);
        step(lds0, steps > 1);
        if (steps == 1) break;
        __syncthreads();
        if (steps > 2) load(lds0);
        step(lds1, steps > 2);
        if (steps == 2) break;
        __syncthreads();
        steps -= 2;
    }
    store_tile<S>(a, tm, tn, wm, wn, lane, acc);
}

// Hidden states as bf16 in rows of whole blocks, zeros behind K; of fp16 the rests behind all rows
template <bool F16>
__global__ __launch_bounds__(256) void split_kernel(const uint16_t *x, int64_t x_ld, int32_t B, int32_t K, int32_t y_ld, uint16_t *y) {
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int32_t units = y_ld / 8;
    if (k >= (int64_t)B * units) return;
    const int32_t b = (int32_t)(k / units), c = (int32_t)(k % units) * 8;
    u32x4 hi = {0, 0, 0, 0}, lo = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t h = c + j < K ? x[b * x_ld + c + j] : 0, l = 0;
        if constexpr (F16) {
            const float f = Fp16::value((uint16_t)h);
            h = Bf16::round(f);
            l = fabsf(f) < kInf ? Bf16::round(f - Bf16::value((uint16_t)h)) : 0;
        }
        hi[j / 2] |= h << (j % 2 * 16);
        lo[j / 2] |= l << (j % 2 * 16);
    }
    *reinterpret_cast<u32x4 *>(y + (int64_t)b * y_ld + c) = hi;
    if constexpr (F16) *reinterpret_cast<u32x4 *>(y + (int64_t)(B + b) * y_ld + c) = lo;
}

// ---------------------------------------------------------------- host

constexpr size_t kLdsBytes = 160 * 1024;
constexpr int32_t kMaxBlocks = 1 << 17;  // K <= 2^22: offsets of a tile's rows stay below 2^32

int32_t blocks_of(int32_t K) { return (int32_t)ceil_div(K, 32); }

// Rows in LDS of the kernel for few rows and the bytes of one, so that 16 of them spread over all banks; 0 bytes: does not fit
size_t few_lds(int x, int32_t B, int32_t nb, int32_t &row, int &fragments) {
    row = x == X_4 ? (int32_t)align_up((size_t)nb * 17, 16) + (nb * 17 % 256 <= 240 ? 16 : 0) : nb * 64 + 16;
    int64_t rows = B;
    fragments = B <= 16 ? 1 : 2;
    if (x == X_F16) {
        fragments = B <= 8 ? 1 : 2;
        rows = (fragments == 2 ? 16 : 8) + B;
    }
    if (x == X_F16 ? B > 16 : x == X_4 ? B > 16 : B > 32) return 0;
    const size_t bytes = (size_t)rows * row + (size_t)fragments * kFewWaves * kWave * 16;
    return bytes <= kLdsBytes ? bytes : 0;
}

template <int X, int FRAGMENTS>
int launch_few(const FewArgs &a, size_t lds, hipStream_t stream) {
    const int64_t tiles = ceil_div(a.w.V, 16);
    const int64_t at_a_time = lds * 2 <= kLdsBytes ? 512 : 256;
    const int64_t groups = ceil_div(tiles, kFewWaves / a.share);
    const void *kernel = reinterpret_cast<const void *>(&few_rows_kernel<X, FRAGMENTS>);
    CFGZIP_TRY(check_hip(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)));
    hipLaunchKernelGGL((few_rows_kernel<X, FRAGMENTS>), dim3((uint32_t)(groups < at_a_time ? groups : at_a_time)), dim3(kFewThreads),
                       lds, stream, a);
    return check_launch();
}

using Many64 = Shape<128, 64, 4, 1>;
using Many128 = Shape<256, 128, 4, 2>;
using Many4_64 = Shape<256, 64, 4, 1>;
using Many4_256 = Shape<256, 256, 2, 4>;

template <typename S, bool FOUR>
int launch_many(ManyArgs a, hipStream_t stream) {
    a.tiles_m = (int32_t)ceil_div(a.w.V, S::BM);
    a.tiles_n = (int32_t)ceil_div(a.out.B, S::BN);
    const int64_t grid = (int64_t)a.tiles_m * a.tiles_n;
    if (grid > 0x7FFFFFFF) return CFGZIP_E_TOO_LARGE;
    if constexpr (FOUR) hipLaunchKernelGGL((many_rows4_kernel<S>), dim3((uint32_t)grid), dim3(S::kThreads), 0, stream, a);
    else hipLaunchKernelGGL((many_rows_kernel<S>), dim3((uint32_t)grid), dim3(S::kThreads), 0, stream, a);
    return check_launch();
}

int x_kind(int32_t dtype) { return dtype == CFGZIP_DTYPE_BF16 ? X_BF16 : dtype == CFGZIP_DTYPE_F16 ? X_F16 : X_4; }

struct LogitsWorkspace {
    int32_t *tok_bits;
    uint16_t *x;
    size_t bytes;
};
LogitsWorkspace logits_workspace(void *ws, int32_t dtype, int32_t B, int32_t V, int32_t K, int32_t bits_kind) {
    Carver c(ws);
    LogitsWorkspace w{};
    int32_t row;
    int fragments;
    if (!few_lds(x_kind(dtype), B, blocks_of(K), row, fragments)) {
        if (bits_kind == CFGZIP_BITS_CLASS) w.tok_bits = c.take<int32_t>((size_t)B * words_for(V));
        if (dtype != CFGZIP_DTYPE_MX4) w.x = c.take<uint16_t>((size_t)B * blocks_of(K) * 32 * (dtype == CFGZIP_DTYPE_F16 ? 2 : 1));
    }
    w.bytes = c.used;
    return w;
}

bool logits_sizes_ok(int32_t dtype, int32_t B, int32_t V, int32_t K, int32_t bits_kind) {
    return B >= 0 && V > 0 && K > 0 &&
           (dtype == CFGZIP_DTYPE_BF16 || dtype == CFGZIP_DTYPE_F16 || dtype == CFGZIP_DTYPE_MX4) &&
           (bits_kind == CFGZIP_BITS_TOKEN || bits_kind == CFGZIP_BITS_CLASS || bits_kind == CFGZIP_BITS_NONE);
}

}  // namespace
}  // namespace cfgzip

using namespace cfgzip;

extern "C" int cfgzip_mx4_quantize(const void *x, int32_t dtype, int64_t R, int32_t K, int64_t x_stride, uint8_t *codes, uint8_t *scales,
                                   void *stream) {
    if (R < 0 || K <= 0) return CFGZIP_E_INVALID;
    if (dtype != CFGZIP_DTYPE_F32 && dtype != CFGZIP_DTYPE_BF16 && dtype != CFGZIP_DTYPE_F16) return CFGZIP_E_INVALID;
    if (R == 0) return CFGZIP_OK;
    if (!x || !codes || !scales || x_stride < K || !aligned_to(x, dtype == CFGZIP_DTYPE_F32 ? 4 : 2) || !aligned_to(codes, 16))
        return CFGZIP_E_INVALID;
    const int32_t nb = blocks_of(K);
    if (nb > kMaxBlocks) return CFGZIP_E_TOO_LARGE;
    const int64_t grid = ceil_div(R * nb * 4, 256 * kUnroll);
    if (grid > 0x7FFFFFFF) return CFGZIP_E_TOO_LARGE;
    const dim3 g((uint32_t)grid), t(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint32_t *c = reinterpret_cast<uint32_t *>(codes);
    switch (dtype) {
        case CFGZIP_DTYPE_F32: hipLaunchKernelGGL(quantize_kernel<CFGZIP_DTYPE_F32>, g, t, 0, s, x, x_stride, R, K, nb, c, scales); break;
        case CFGZIP_DTYPE_BF16: hipLaunchKernelGGL(quantize_kernel<CFGZIP_DTYPE_BF16>, g, t, 0, s, x, x_stride, R, K, nb, c, scales); break;
        default: hipLaunchKernelGGL(quantize_kernel<CFGZIP_DTYPE_F16>, g, t, 0, s, x, x_stride, R, K, nb, c, scales); break;
    }
    return check_launch();
}

extern "C" int cfgzip_mx4_values(const uint8_t *codes, const uint8_t *scales, int64_t R, int32_t K, void *x, int32_t dtype,
                                 int64_t x_stride, void *stream) {
    if (R < 0 || K <= 0) return CFGZIP_E_INVALID;
    if (dtype != CFGZIP_DTYPE_F32 && dtype != CFGZIP_DTYPE_BF16 && dtype != CFGZIP_DTYPE_F16) return CFGZIP_E_INVALID;
    if (R == 0) return CFGZIP_OK;
    if (!x || !codes || !scales || x_stride < K || !aligned_to(x, dtype == CFGZIP_DTYPE_F32 ? 4 : 2) || !aligned_to(codes, 16))
        return CFGZIP_E_INVALID;
    const int32_t nb = blocks_of(K);
    if (nb > kMaxBlocks) return CFGZIP_E_TOO_LARGE;
    const int64_t grid = ceil_div(R * nb * 4, 256 * kUnroll);
    if (grid > 0x7FFFFFFF) return CFGZIP_E_TOO_LARGE;
    const dim3 g((uint32_t)grid), t(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint32_t *c = reinterpret_cast<const uint32_t *>(codes);
    switch (dtype) {
        case CFGZIP_DTYPE_F32: hipLaunchKernelGGL(values_kernel<CFGZIP_DTYPE_F32>, g, t, 0, s, c, scales, R, K, nb, x, x_stride); break;
        case CFGZIP_DTYPE_BF16: hipLaunchKernelGGL(values_kernel<CFGZIP_DTYPE_BF16>, g, t, 0, s, c, scales, R, K, nb, x, x_stride); break;
        default: hipLaunchKernelGGL(values_kernel<CFGZIP_DTYPE_F16>, g, t, 0, s, c, scales, R, K, nb, x, x_stride); break;
    }
    return check_launch();
}

extern "C" size_t cfgzip_mx4_logits_workspace_bytes(int32_t hidden_dtype, int32_t B, int32_t V, int32_t K, int32_t bits_kind) {
    if (!logits_sizes_ok(hidden_dtype, B, V, K, bits_kind) || B == 0 || blocks_of(K) > kMaxBlocks) return 0;
    return logits_workspace(nullptr, hidden_dtype, B, V, K, bits_kind).bytes;
}

extern "C" int cfgzip_mx4_logits(const void *hidden, int32_t hidden_dtype, int64_t hidden_stride, const uint8_t *hidden_scales,
                                 const uint8_t *codes, const uint8_t *scales, int32_t B, int32_t V, int32_t K, const int32_t *bits,
                                 int32_t bits_kind, const int32_t *class_of_token, int32_t C, void *logits, int32_t dtype,
                                 int64_t row_stride, void *ws, size_t ws_bytes, void *stream) {
    if (!logits_sizes_ok(hidden_dtype, B, V, K, bits_kind)) return CFGZIP_E_INVALID;
    if (dtype != CFGZIP_DTYPE_F32 && dtype != CFGZIP_DTYPE_BF16) return CFGZIP_E_INVALID;
    if (B == 0) return CFGZIP_OK;
    const bool four = hidden_dtype == CFGZIP_DTYPE_MX4;
    const int32_t nb = blocks_of(K);
    if (!hidden || !codes || !scales || !logits || row_stride < V) return CFGZIP_E_INVALID;
    if (four ? (!hidden_scales || hidden_stride != (int64_t)nb * 16 || !aligned_to(hidden, 16)) : (hidden_stride < K || !aligned_to(hidden, 2)))
        return CFGZIP_E_INVALID;
    if (!aligned_to(codes, 16) || !aligned_to(logits, dtype == CFGZIP_DTYPE_F32 ? 4 : 2)) return CFGZIP_E_INVALID;
    if (bits_kind != CFGZIP_BITS_NONE && (!bits || !aligned_to(bits, 4))) return CFGZIP_E_INVALID;
    if (bits_kind == CFGZIP_BITS_CLASS && (!class_of_token || C <= 0 || !aligned_to(class_of_token, 4))) return CFGZIP_E_INVALID;
    if (nb > kMaxBlocks || V > 0x7FFFFC00) return CFGZIP_E_TOO_LARGE;
    const LogitsWorkspace w = logits_workspace(ws, hidden_dtype, B, V, K, bits_kind);
    if (w.bytes && (!ws || !aligned_to(ws, 256) || ws_bytes < w.bytes)) return CFGZIP_E_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Weights weights{codes, scales, V, nb};
    const Logits out{logits, row_stride, B, dtype == CFGZIP_DTYPE_F32};
    const int x = x_kind(hidden_dtype);

    FewArgs few{};
    int fragments;
    if (const size_t lds = few_lds(x, B, nb, few.lds_row, fragments)) {
        few.w = weights;
        few.x = hidden;
        few.x_ld = hidden_stride;
        few.x_scales = hidden_scales;
        few.K = K;
        few.out = out;
        few.bits = bits_kind == CFGZIP_BITS_NONE ? nullptr : bits;
        few.words = bits_kind == CFGZIP_BITS_CLASS ? words_for(C) : words_for(V);
        few.class_of_token = bits_kind == CFGZIP_BITS_CLASS ? class_of_token : nullptr;
        // 4,096 waves are at work at a time; a share below kAhead loads would not fill what is in flight
        few.share = 1;
        while (few.share < kFewWaves && ceil_div(V, 16) * few.share * 2 <= 4096 && nb / 4 >= few.share * 2 * 2) few.share *= 2;
        switch (x * 2 + fragments) {
            case X_BF16 * 2 + 1: return launch_few<X_BF16, 1>(few, lds, s);
            case X_BF16 * 2 + 2: return launch_few<X_BF16, 2>(few, lds, s);
            case X_F16 * 2 + 1: return launch_few<X_F16, 1>(few, lds, s);
            case X_F16 * 2 + 2: return launch_few<X_F16, 2>(few, lds, s);
            default: return launch_few<X_4, 1>(few, lds, s);
        }
    }

    ManyArgs a{};
    a.w = weights;
    a.out = out;
    a.parts = 1;
    a.words = words_for(V);
    if (bits_kind == CFGZIP_BITS_TOKEN) a.bits = bits;
    if (bits_kind == CFGZIP_BITS_CLASS) {
        CFGZIP_TRY(cfgzip_expand_mask(bits, B, C, class_of_token, V, w.tok_bits, stream));
        a.bits = w.tok_bits;
    }
    if (four) {
        a.x = static_cast<const char *>(hidden);
        a.x_row_bytes = (int64_t)nb * 16;
        a.x_scales = hidden_scales;
        a.x_units = nb;
        return B <= 64 ? launch_many<Many4_64, true>(a, s) : launch_many<Many4_256, true>(a, s);
    }
    if (x == X_BF16 && K % 8 == 0 && hidden_stride % 8 == 0 && hidden_stride < kMaxStride && aligned_to(hidden, 16)) {
        a.x = static_cast<const char *>(hidden);
        a.x_row_bytes = hidden_stride * 2;
        a.x_units = K / 8;
    } else {
        const dim3 g((uint32_t)ceil_div((int64_t)B * nb * 4, 256)), t(256);
        const uint16_t *h = static_cast<const uint16_t *>(hidden);
        if (x == X_F16) hipLaunchKernelGGL(split_kernel<true>, g, t, 0, s, h, hidden_stride, B, K, nb * 32, w.x);
        else hipLaunchKernelGGL(split_kernel<false>, g, t, 0, s, h, hidden_stride, B, K, nb * 32, w.x);
        CFGZIP_TRY(check_launch());
        a.x = reinterpret_cast<const char *>(w.x);
        a.x_row_bytes = (int64_t)nb * 64;
        a.x_part_bytes = (int64_t)B * nb * 64;
        a.x_units = nb * 4;
        a.parts = x == X_F16 ? 2 : 1;
    }
    return B <= 64 ? launch_many<Many64, false>(a, s) : launch_many<Many128, false>(a, s);
}
