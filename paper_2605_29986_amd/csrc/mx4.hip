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
// kUnroll times that in all, whole rows after each other.  Bound by memory: 128,256 x 4,096 bf16 values to 4 bits and back move
// 2.7 GB in 472 us, 5.6 TB/s, beyond the rate of a large copy (4.9).
template <int DTYPE>
__global__ __launch_bounds__(256) void quantize_kernel(const void *x, int64_t x_ld, int64_t R, int32_t K, int32_t nb, uint32_t *codes,
                                                       uint8_t *scales) {
    const int32_t per = nb * 4;
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

// logits of four tokens (WHOLE: all of them there) from v on in row b; bit r of ok: token v + r is admitted
template <bool WHOLE, bool F32>
__device__ __forceinline__ void store_logits(const Logits &o, int32_t b, int32_t v, int32_t V, f32x4 z, uint32_t ok) {
    const int32_t left = WHOLE ? 4 : V - v;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (!(ok >> r & 1)) z[r] = -kInf;
    if (F32) {
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

// Few rows: reading the weights is what counts: 5.4 TB/s for four rows of 128,256 x 4,096 (52 us; with a mask that leaves half of the
// tokens 34 us, 4.1 TB/s of what it leaves: rows of weights here and there).  Hidden states lie in LDS; a wave takes 16 tokens (or a share of the blocks of 16
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

// Blocks of a row in LDS.  Where a load's four go beyond the last one, lanes have codes of 0 there, and one more block, of zeros, to multiply
// with them: of an infinity they would make a NaN.
__host__ __device__ inline int32_t lds_blocks(int32_t nb) { return nb % 4 ? nb + 1 : nb; }

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
    const int32_t there = lds_blocks(nb);
    if constexpr (X == X_4) {
        for (int32_t k = threadIdx.x; k < B * there; k += kFewThreads) {
            const int32_t b = k / there, c = k % there;
            u32x4 v = {0, 0, 0, 0};
            uint8_t scale = 0;
            if (c < nb) {
                v = *reinterpret_cast<const u32x4_bytes *>(static_cast<const uint8_t *>(a.x) + b * a.x_ld + c * 16);
                scale = a.x_scales[(int64_t)b * nb + c];
            }
            *reinterpret_cast<u32x4 *>(lds + b * a.lds_row + c * 16) = v;
            lds[b * a.lds_row + there * 16 + c] = (char)scale;
        }
    } else {
        const uint16_t *x = static_cast<const uint16_t *>(a.x);
        const int32_t units = there * 4;
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
            // All there: the scales of 32 blocks in two loads (byte by byte, a load for every load of codes, one row of 128,256 x
            // 4,096 took 43.5 us for 34.4).  Nothing is marked as not to be kept: a line's second half is asked for by the next load.
            if (l + kAhead <= l1 && (l + kAhead) * 4 <= nb) {
                u32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
                for (int i = 0; i < kAhead; ++i) code[i] = u32x4{0, 0, 0, 0};
                if (ok != 0) {
                    s[0] = *reinterpret_cast<const u32x4_bytes *>(scales + l * 4);
                    s[1] = *reinterpret_cast<const u32x4_bytes *>(scales + l * 4 + 16);
#pragma unroll
                    for (int i = 0; i < kAhead; ++i)
                        code[i] = *reinterpret_cast<const u32x4 *>(codes + ((l + i) * 4 + g) * 16);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) byte[i] = s[i / 4][i % 4] >> (8 * g) & 255;
            } else {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int32_t block = (l + i) * 4 + g;
                    code[i] = u32x4{0, 0, 0, 0};
                    byte[i] = 127;
                    if (ok != 0 && l + i < l1 && block < nb) {
                        code[i] = *reinterpret_cast<const u32x4 *>(codes + block * 16);
                        byte[i] = scales[block];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int32_t block = (l + i) * 4 + g < nb ? (l + i) * 4 + g : nb;
                if (l + i >= l1) break;
                if constexpr (X == X_4) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(xs[0] + block * 16);
                    acc[0] = multiply4(code[i], x, acc[0], byte[i], (uint8_t)xs[0][there * 16 + block]);
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
                if (a.out.f32) store_logits<false, true>(a.out, b, tile * 16 + 4 * g, V, acc[f], four);
                else store_logits<false, false>(a.out, b, tile * 16 + 4 * g, V, acc[f], four);
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
    int32_t part_steps;    // of 128 values in a part's row, where those are whole pairs of steps
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
    constexpr int kWords = (S::TM + 31) / 32;
    const int32_t b0 = tn * S::BN + wn * S::TN + (lane & 15);
    uint32_t words[S::FN][kWords];  // all of them are asked for before the first is used
    each<S::FN>([&](auto j) CFGZIP_INLINE {
        each<kWords>([&](auto w) CFGZIP_INLINE { words[j.value][w.value] = ~0u; });
        if (a.bits) {
            const int32_t b = b0 + 16 * j.value;
            const int32_t *const bits = a.bits + (b < a.out.B ? b : a.out.B - 1) * a.words;
            each<kWords>([&](auto w) CFGZIP_INLINE {  // (tokens behind the last word are not stored)
                const int64_t k = (first >> 5) + w.value < a.words ? (first >> 5) + w.value : a.words - 1;
                words[j.value][w.value] = (uint32_t)bits[k];
            });
        }
    });
    auto store = [&](auto whole, auto f32) CFGZIP_INLINE {
        each<S::FN>([&](auto j) CFGZIP_INLINE {
            const int32_t b = b0 + 16 * j.value;
            if (b >= a.out.B) return;
            each<S::FM>([&](auto i) CFGZIP_INLINE {
                const int32_t v = first + 16 * i.value + 4 * g;
                if (whole.value || v < a.w.V)
                    store_logits<whole.value, f32.value>(a.out, b, v, a.w.V, acc[i.value][j.value], words[j.value][i.value / 2] >> (v & 31));
            });
        });
    };
    // (asked once a tile and not once for every four logits)
    const std::true_type yes;
    const std::false_type no;
    if (first + S::TM > a.w.V) {
        if (a.out.f32) store(no, yes);
        else store(no, no);
    } else {
        if (a.out.f32) store(yes, yes);
        else store(yes, no);
    }
}

// 16-bit hidden states.  A step has 128 k: lane (r, g) of a fragment has block g of its token, 32 weights, as four fragments of
// eight, and the hidden states of the same k.  Every barrier that hands on what was loaded to LDS waits for the wave's own loads
// first: the compiler need not know that they write it.
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
        wait_for_loads<0>();  // (none yet:) the part before has been read
        load(lds0);
        scales();
        wait_for_loads<0>();
        while (true) {
            if (steps > 1) load(lds1);
            step(lds0);
            if (steps == 1) break;
            scales();
            wait_for_loads<0>();
            if (steps > 2) load(lds0);
            step(lds1);
            if (steps == 2) break;
            scales();
            wait_for_loads<0>();
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
    wait_for_loads<0>();
    while (true) {
        if (steps > 1) load(lds1);
        step(lds0, steps > 1);
        if (steps == 1) break;
        wait_for_loads<0>();
        if (steps > 2) load(lds0);
        step(lds1, steps > 2);
        if (steps == 2) break;
        wait_for_loads<0>();
        steps -= 2;
    }
    store_tile<S>(a, tm, tn, wm, wn, lane, acc);
}

// 16-bit hidden states, many rows: tiles of 256 x 256 by four waves.  A step has 128 k: lane (r, g) of a fragment has block g of its
// token, 32 weights, as four fragments of eight that become bf16 while the products of the row before are at work, and the hidden
// states of the same k.  Hidden states lie in whole pairs of steps, zeros behind K; those of fp16 have a row's rests behind
// its first numbers, and the weights are gone through twice.  Products a wave: 256 a step; out of LDS 8 KB of codes and 32 of hidden
// states.
// 256 x 128,256 x 4,096: 248 us, 1.09 PFLOP/s (a library product of bf16 weights 1.2 to 1.4); 128 x 64 a wave, eight waves, weights made
// bf16 in front of their products: 332.
using Large16 = Shape<256, 256, 2, 2, 2>;
constexpr int32_t kPairK = 256;

// four products with one fragment of weights, while the next one's `to` is made of eight codes
__device__ __forceinline__ void mma4_and_convert(u32x4 a, u32x4 b0, u32x4 b1, u32x4 b2, u32x4 b3, f32x4 &c0, f32x4 &c1, f32x4 &c2, f32x4 &c3,
                                                 u32x4 &to, uint32_t codes, float scale) {
    uint32_t t0, t1, t2, t3;
    asm volatile(
        "s_nop 1\n\t"
        "v_mfma_f32_16x16x32_bf16 %0, %8, %9, %0\n\t"
        "v_cvt_scalef32_pk_bf16_fp4 %4, %13, %14\n\t"
        "v_mfma_f32_16x16x32_bf16 %1, %8, %10, %1\n\t"
        "v_cvt_scalef32_pk_bf16_fp4 %5, %13, %14 op_sel:[1,0,0]\n\t"
        "v_mfma_f32_16x16x32_bf16 %2, %8, %11, %2\n\t"
        "v_cvt_scalef32_pk_bf16_fp4 %6, %13, %14 op_sel:[0,1,0]\n\t"
        "v_mfma_f32_16x16x32_bf16 %3, %8, %12, %3\n\t"
        "v_cvt_scalef32_pk_bf16_fp4 %7, %13, %14 op_sel:[1,1,0]"
        : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3), "=&v"(t0), "=&v"(t1), "=&v"(t2), "=&v"(t3)
        : "v"(a), "v"(b0), "v"(b1), "v"(b2), "v"(b3), "v"(codes), "v"(scale));
    to = u32x4{t0, t1, t2, t3};
}

__global__ __launch_bounds__(Large16::kThreads) void large16_kernel(ManyArgs a) {
    using S = Large16;
    constexpr int kThreads = S::kThreads, kUnitsW = 4, kUnitsX = 16;  // of 16 bytes of a row and step
    constexpr int kPerW = S::BM * kUnitsW / kThreads, kPerX = S::BN * kUnitsX / kThreads, kLoads = kPerW + kPerX;
    typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
    __shared__ __attribute__((aligned(16))) char w0[S::BM * kUnitsW * 16], w1[S::BM * kUnitsW * 16], x0[S::BN * kUnitsX * 16],
        x1[S::BN * kUnitsX * 16];
    const Stage lds[2] = {{(lds_char *)w0, (lds_char *)x0}, {(lds_char *)w1, (lds_char *)x1}};
    int32_t tm, tn;
    tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wm = wave / S::WN, wn = wave % S::WN, r = lane & 15, g = lane >> 4;
    const int32_t m0 = tm * S::BM, n0 = tn * S::BN, nb = a.w.nb;
    const int32_t part_steps = a.part_steps;  // even

    // The loads of a step.  Unit c of a row lies where the 16 lanes of a fragment's read spread over all banks.  Behind the end of a
    // row of codes its step's first unit is loaded, which is multiplied with zeros.
    const char *base_w = reinterpret_cast<const char *>(a.w.codes) + (int64_t)m0 * nb * 16, *base_x = a.x + n0 * a.x_row_bytes;
    const char *const first_w = base_w;
    uint32_t at_w[kPerW], at_x[kPerX];
    const int32_t c_w = ((int)threadIdx.x & 3) ^ ((int)threadIdx.x >> 4 & 3);
    each<kPerW>([&](auto i) CFGZIP_INLINE {
        const int32_t row = i.value * (kThreads / kUnitsW) + (int)threadIdx.x / kUnitsW, last = a.w.V - m0 - 1;
        at_w[i.value] = (uint32_t)afresh((int)((uint32_t)(row < last ? row : last) * (uint32_t)nb * 16u + c_w * 16));
    });
    each<kPerX>([&](auto i) CFGZIP_INLINE {
        const int32_t row = i.value * (kThreads / kUnitsX) + (int)threadIdx.x / kUnitsX, last = a.out.B - n0 - 1;
        const int32_t c = ((int)threadIdx.x & 15) ^ (row & 15);
        at_x[i.value] = (uint32_t)afresh((int)((uint32_t)(row < last ? row : last) * (uint32_t)a.x_row_bytes + c * 16));
    });
    int32_t steps_left = part_steps * a.parts;  // of those to be loaded
    int32_t step_w = 0;                         // of the weights, of the next to be loaded
    uint32_t skip_w = 0;                        // what takes the thread's unit back to the step's first where it is not there
    auto look = [&]() CFGZIP_INLINE {
        const int32_t there = nb - (base_w == first_w ? 0 : (int32_t)((base_w - first_w) / 64)) * 4;
        skip_w = c_w >= there ? (uint32_t)c_w * 16u : 0u;
    };
    look();
    auto load_into = [&](const Stage &to) CFGZIP_INLINE {
        return [&](auto i) CFGZIP_INLINE {
            if constexpr (i.value < kPerW) {
                const uint32_t from = (uint32_t)afresh((int)(at_w[i.value] - skip_w));
                __builtin_amdgcn_global_load_lds((global_void *)(base_w + from), (lds_void *)(to.a + (i.value * kThreads + wave * kWave) * 16),
                                                 16, 0, 0);
            } else {
                const uint32_t from = (uint32_t)afresh((int)at_x[i.value - kPerW]);
                __builtin_amdgcn_global_load_lds((global_void *)(base_x + from),
                                                 (lds_void *)(to.b + ((i.value - kPerW) * kThreads + wave * kWave) * 16), 16, 0, 0);
            }
        };
    };
    auto advance = [&]() CFGZIP_INLINE {
        ++step_w;
        if (step_w == part_steps) {
            step_w = 0;
            base_w = first_w;
        } else if (step_w * 4 < nb) {  // else the base stays at blocks that are there
            base_w += kUnitsW * 16;
        }
        if (--steps_left > 0) base_x += kUnitsX * 16;
        look();
    };

    // a lane's scales: those of the step at hand, and the next one's bytes on their way
    const uint8_t *const scale_base = a.w.scales + (int64_t)m0 * nb;
    uint32_t at_s[S::FM], bytes[S::FM];
    each<S::FM>([&](auto i) CFGZIP_INLINE {
        const int32_t row = wm * S::TM + 16 * i.value + r, last = a.w.V - m0 - 1;
        at_s[i.value] = (uint32_t)(row < last ? row : last) * (uint32_t)nb;
    });
    int32_t block = g;
    auto ask = [&]() CFGZIP_INLINE {
        const uint32_t from = block < nb ? block : nb - 1;
        each<S::FM>([&](auto i) CFGZIP_INLINE { bytes[i.value] = scale_base[at_s[i.value] + from]; });
    };
    float scale[S::FM];
    auto take = [&]() CFGZIP_INLINE {  // (a block that is not there: what is loaded in its place is finite, and so has to be its scale)
        each<S::FM>([&](auto i) CFGZIP_INLINE { scale[i.value] = __builtin_bit_cast(float, block < nb ? scale_bits(bytes[i.value]) : 0x3F800000u); });
        block += 4;
        if (block >= part_steps * 4) block = g;
    };

    // fragments
    const int32_t from_w = (wm * S::TM + r) * (kUnitsW * 16) + (g ^ (r >> 2 & 3)) * 16;
    const int32_t from_x = (wn * S::TN + r) * (kUnitsX * 16) + ((4 * g) ^ r) * 16;
    u32x4 codes[S::FM], next_codes[S::FM], x[2][S::FN];
    auto read_w = [&](const Stage &from, auto i) CFGZIP_INLINE {
        next_codes[i.value] = *reinterpret_cast<lds_u32x4 *>(from.a + from_w + i.value * (16 * kUnitsW * 16));
    };
    auto read_x = [&](const Stage &from, auto q, auto j) CFGZIP_INLINE {
        x[q.value & 1][j.value] = *reinterpret_cast<lds_u32x4 *>(from.b + (from_x ^ (q.value * 16)) + j.value * (16 * kUnitsX * 16));
    };
    f32x4 acc[S::FM][S::FN];
    each<S::FM>([&](auto i) CFGZIP_INLINE {
        each<S::FN>([&](auto j) CFGZIP_INLINE { acc[i.value][j.value] = f32x4{0, 0, 0, 0}; });
    });

    each<kLoads>(load_into(lds[0]));
    advance();
    each<kLoads>(load_into(lds[1]));
    advance();
    ask();
    wait_for_loads<0>();
    const std::integral_constant<int, 0> zero;
    each<S::FM>([&](auto i) CFGZIP_INLINE { read_w(lds[0], i); });
    each<S::FN>([&](auto j) CFGZIP_INLINE { read_x(lds[0], zero, j); });
    u32x4 w;
    int32_t left = part_steps * a.parts / 2;
    do {
        each<2>([&](auto s) CFGZIP_INLINE {
            const Stage &here = lds[s.value], &next = lds[1 - s.value];
            take();
            each<S::FM>([&](auto i) CFGZIP_INLINE { codes[i.value] = next_codes[i.value]; });
            w = weights8(codes[0][0], scale[0]);
            each<4>([&](auto q) CFGZIP_INLINE {
                if constexpr (q.value == 1) ask();
                // The next step's loads have come in and this one's have been read by everybody: its buffers are loaded again with what
                // lies two steps ahead.
                if constexpr (q.value == 3) wait_for_loads<0>();
                each<2 * S::FM>([&](auto p) CFGZIP_INLINE {
                    constexpr int i = p.value / 2, j = p.value % 2 * 4;
                    u32x4 (&y)[S::FN] = x[q.value & 1];
                    if constexpr (j == 0) {
                        Bf16::mma4(w, y[0], y[1], y[2], y[3], acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
                    } else if constexpr (i + 1 < S::FM || q.value < 3) {
                        constexpr int i1 = (i + 1) % S::FM, q1 = i + 1 < S::FM ? q.value : q.value + 1;
                        u32x4 to;
                        mma4_and_convert(w, y[4], y[5], y[6], y[7], acc[i][4], acc[i][5], acc[i][6], acc[i][7], to, codes[i1][q1], scale[i1]);
                        w = to;
                    } else {
                        Bf16::mma4(w, y[4], y[5], y[6], y[7], acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
                    }
                    constexpr int kLast = 12;
                    constexpr int kReads = S::FN + (q.value == 3 ? S::FM : 0);
                    constexpr int f0 = from(p.value, kReads, kLast), f1 = from(p.value + 1, kReads, kLast);
                    each<f1 - f0>([&](auto f) CFGZIP_INLINE {
                        constexpr int n = f0 + f.value;
                        if constexpr (n < S::FN) {
                            if constexpr (q.value < 3) read_x(here, std::integral_constant<int, q.value + 1>{}, std::integral_constant<int, n>{});
                            else read_x(next, std::integral_constant<int, 0>{}, std::integral_constant<int, n>{});
                        } else {
                            read_w(next, std::integral_constant<int, n - S::FN>{});
                        }
                    });
                    if constexpr (q.value == 3) {
                        constexpr int l0 = from(p.value, kLoads + 1, 16), l1 = from(p.value + 1, kLoads + 1, 16);
                        each<l1 - l0>([&](auto l) CFGZIP_INLINE {
                            if constexpr (l0 + l.value < kLoads) load_into(here)(std::integral_constant<int, l0 + l.value>{});
                            else advance();
                        });
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        });
    } while (--left > 0);
    settle<S>(acc);
    store_tile<S>(a, tm, tn, wm, wn, lane, acc);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): nothing is on its way into LDS that may soon be another workgroup's
}

// Products of 4-bit operands by the loop of the 16-bit ones: a step of 64 16-bit elements is 256 values, lane (r, g) of a fragment has
// block 4 kk + g of its row in half kk of a step, 16 bytes like eight 16-bit elements.
struct Mx4 {
    template <int BYTE>
    static __device__ __forceinline__ void mma4(u32x4 a, u32x4 b0, u32x4 b1, u32x4 b2, u32x4 b3, f32x4 &c0, f32x4 &c1, f32x4 &c2, f32x4 &c3,
                                                uint32_t sa, uint32_t s0, uint32_t s1, uint32_t s2, uint32_t s3) {
        // (four products with one a and the wait states in front of them as in the 16-bit forms; BYTE: of the scales)
#define CFGZIP_MMA4(op_sel, op_sel_hi)                                                                                                      \
    asm volatile(                                                                                                                           \
        "s_nop 1\n\t"                                                                                                                       \
        "v_mfma_scale_f32_16x16x128_f8f6f4 %0, %4, %5, %0, %9, %10 op_sel:" op_sel " op_sel_hi:" op_sel_hi " cbsz:4 blgp:4\n\t"             \
        "v_mfma_scale_f32_16x16x128_f8f6f4 %1, %4, %6, %1, %9, %11 op_sel:" op_sel " op_sel_hi:" op_sel_hi " cbsz:4 blgp:4\n\t"             \
        "v_mfma_scale_f32_16x16x128_f8f6f4 %2, %4, %7, %2, %9, %12 op_sel:" op_sel " op_sel_hi:" op_sel_hi " cbsz:4 blgp:4\n\t"             \
        "v_mfma_scale_f32_16x16x128_f8f6f4 %3, %4, %8, %3, %9, %13 op_sel:" op_sel " op_sel_hi:" op_sel_hi " cbsz:4 blgp:4"                  \
        : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3)                                                                                            \
        : "v"(a), "v"(b0), "v"(b1), "v"(b2), "v"(b3), "v"(sa), "v"(s0), "v"(s1), "v"(s2), "v"(s3))
        if constexpr (BYTE == 0) CFGZIP_MMA4("[0,0,0]", "[0,0,0]");
        if constexpr (BYTE == 1) CFGZIP_MMA4("[1,1,0]", "[0,0,0]");
        if constexpr (BYTE == 2) CFGZIP_MMA4("[0,0,0]", "[1,1,0]");
        if constexpr (BYTE == 3) CFGZIP_MMA4("[1,1,0]", "[1,1,0]");
#undef CFGZIP_MMA4
    }
};

// Scales of a tile's rows, of two steps (16 blocks) at a time.  Thread t has row t of the tile's tokens and row t of its hidden states:
// it loads a row's 16 bytes at once, and leaves the four that lane group g needs, blocks g, 4 + g, 8 + g and 12 + g, next to each
// other.  (Two bytes a fragment, step and lane straight from memory take sixteen loads of sixteen pieces a step instead of one load of
// 64, and as long in the caches as the codes.)
template <typename S>
struct TileScales {
    static constexpr bool kScaled = true;
    static_assert(S::kThreads == S::BM && S::kThreads == S::BN, "a row of either side to a thread");
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    typedef __attribute__((address_space(3))) const uint32_t lds_u32;
    static constexpr int kBytes = (S::BM + S::BN) * 16;  // of one of two buffers

    const uint8_t *w, *x;
    int32_t V, B, nb;
    lds_char *lds;
    int32_t at = 0;        // of the buffer to be filled
    int32_t left;          // blocks of a row from those asked for on
    int32_t m0, n0;        // the tile's first rows
    u32x4 asked[2];
    uint32_t a[S::FM], b[S::FN];

    // Blocks of a row from its `left`-last on, sixteen bytes.  No branch, and nothing behind the array is read: there its last sixteen
    // are, which whole() moves down.
    static __device__ __forceinline__ int32_t moved(int32_t row, int32_t rows, int32_t nb, int32_t left) {
        const int64_t behind = (int64_t)(rows - 1 - row) * nb + left;  // blocks up to the array's end
        return behind < 16 ? 16 - (int32_t)(behind > 0 ? behind : 1) : 0;
    }
    static __device__ __forceinline__ u32x4 sixteen(const uint8_t *base, int32_t row, int32_t rows, int32_t nb, int32_t left) {
        const int64_t all = (int64_t)rows * nb, at = (int64_t)row * nb + (nb - left);
        return *reinterpret_cast<const u32x4_bytes *>(base + (at < all - 16 ? at : all - 16));
    }
    // What belongs to the row, and 0 behind its end (a scale that is a NaN would make its products with the zeros there NaN).
    static __device__ __forceinline__ u32x4 whole(u32x4 v, int32_t moved, int32_t left) {
        const uint32_t down = moved * 8;
        uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
        const uint64_t over = hi << 1 << (63 - (down & 63));
        lo = down & 64 ? hi >> (down & 63) : lo >> (down & 63) | over;
        hi = down & 64 ? 0 : hi >> (down & 63);
        u32x4 out = {(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int32_t here = left - 4 * d;
            out[d] &= here >= 4 ? ~0u : here <= 0 ? 0u : (1u << (8 * here)) - 1u;
        }
        return out;
    }
    static __device__ __forceinline__ u32x4 transposed(u32x4 v) {
        const uint32_t lo01 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400), hi01 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602);
        const uint32_t lo23 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400), hi23 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602);
        return u32x4{__builtin_amdgcn_perm(lo23, lo01, 0x05040100), __builtin_amdgcn_perm(lo23, lo01, 0x07060302),
                     __builtin_amdgcn_perm(hi23, hi01, 0x05040100), __builtin_amdgcn_perm(hi23, hi01, 0x07060302)};
    }
    __device__ __forceinline__ int32_t v() const { return clamped(m0, V); }
    __device__ __forceinline__ int32_t r() const { return clamped(n0, B); }
    static __device__ __forceinline__ int32_t clamped(int32_t first, int32_t rows) {
        const int32_t row = first + afresh(threadIdx.x);
        return row < rows ? row : rows - 1;
    }
    __device__ __forceinline__ void load() {
        asked[0] = sixteen(w, v(), V, nb, left);
        asked[1] = sixteen(x, r(), B, nb, left);
    }
    __device__ __forceinline__ void begin(const Work &work) {
        m0 = work.m0, n0 = work.n0, left = nb;
        load();
    }
    __device__ __forceinline__ void ask() {
        left -= 16;
        load();
    }
    __device__ __forceinline__ void put() {
        const int32_t t = (int32_t)afresh(threadIdx.x) * 16 + at;
        u32x4 s = asked[0], z = asked[1];
        if (left < 16) {
            s = whole(s, moved(v(), V, nb, left), left);
            z = whole(z, moved(r(), B, nb, left), left);
        }
        *reinterpret_cast<lds_u32x4 *>(lds + t) = transposed(s);
        *reinterpret_cast<lds_u32x4 *>(lds + (t + S::BM * 16)) = transposed(z);
    }
    __device__ __forceinline__ void take(int wm, int wn, int lane) {
        const int32_t from = at + (lane & 15) * 16 + (lane >> 4) * 4;
        each<S::FM>([&](auto i) CFGZIP_INLINE { a[i.value] = *reinterpret_cast<lds_u32 *>(lds + (from + (wm * S::TM + 16 * i.value) * 16)); });
        each<S::FN>([&](auto j) CFGZIP_INLINE {
            b[j.value] = *reinterpret_cast<lds_u32 *>(lds + (from + (S::BM + wn * S::TN + 16 * j.value) * 16));
        });
        at ^= kBytes;
    }
};

// Both sides in 4 bits, many rows of both: tiles of 256 x 256 by four waves.  1,024 x 128,256 x 4,096: 397 us, 2.7 PFLOP/s (128 x 64 a wave,
// eight waves, scales straight from memory: 690).  By calls of K = 1,024 to 16,384 a step of 256 values takes 2.0 us (0.85 at the products'
// peak; reading its fragments keeps LDS busy for three quarters of that, and its loads have one step to arrive), and a tile's
// beginning and end, which nothing runs beside, 17, of which the round's logits are 7: of a round of 49 us 16 steps are 33.
using Large4 = Shape<256, 256, 2, 2, 2>;
__global__ __launch_bounds__(Large4::kThreads) void large4_kernel(ManyArgs a) {
    using S = Large4;
    // behind a row's end both sides hold some codes, with scales of 2^-127 each: products far below the smallest number
    using TileW = Tile<S::BM, S::kThreads, false, true, ANY>;
    using TileX = Tile<S::BN, S::kThreads, false, true, ANY>;
    CFGZIP_STAGES(S, lds);
    __shared__ __attribute__((aligned(16))) char scales_lds[2 * TileScales<S>::kBytes];
    const int32_t elements = a.w.nb * 8;  // 16-bit ones of a row
    int32_t tm, tn;
    tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
    auto work = [&](int32_t, Work &w) CFGZIP_INLINE {
        w = Work{tm * S::BM, tn * S::BN, 0, elements};
        return true;
    };
    auto store = [&](int32_t, f32x4(&acc)[S::FM][S::FN], int wm, int wn, int lane) CFGZIP_INLINE { store_tile<S>(a, tm, tn, wm, wn, lane, acc); };
    TileScales<S> scales;
    scales.w = a.w.scales;
    scales.x = a.x_scales;
    scales.V = a.w.V;
    scales.B = a.out.B;
    scales.nb = a.w.nb;
    scales.lds = (lds_char *)scales_lds;
    multiply<Mx4, S, TileW, TileX>(by_rows(reinterpret_cast<const uint16_t *>(a.w.codes), elements, a.w.V),
                                   by_rows(reinterpret_cast<const uint16_t *>(a.x), elements, a.out.B), lds, work, store, scales);
}

// Hidden states as bf16 in rows of whole pairs of steps, zeros behind K; of fp16 a row's rests behind its first numbers
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
    y += (int64_t)b * y_ld * (F16 ? 2 : 1) + c;
    *reinterpret_cast<u32x4 *>(y) = hi;
    if constexpr (F16) *reinterpret_cast<u32x4 *>(y + y_ld) = lo;
}

// ---------------------------------------------------------------- host

constexpr size_t kLdsBytes = 160 * 1024;
constexpr int32_t kMaxBlocks = 1 << 17;  // K <= 2^22: offsets of a tile's rows stay below 2^32

int32_t blocks_of(int32_t K) { return (int32_t)ceil_div(K, 32); }
int32_t whole_pairs(int32_t K) { return (int32_t)ceil_div(K, kPairK) * kPairK; }  // K in whole pairs of steps

// Rows in LDS of the kernel for few rows and the bytes of one, so that 16 of them spread over all banks; 0 bytes: does not fit
size_t few_lds(int x, int32_t B, int32_t nb, int32_t &row, int &fragments) {
    nb = lds_blocks(nb);
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
    const int64_t at_a_time = 256;  // a workgroup's registers fill a compute unit
    const int64_t groups = ceil_div(tiles, kFewWaves / a.share);
    const void *kernel = reinterpret_cast<const void *>(&few_rows_kernel<X, FRAGMENTS>);
    CFGZIP_TRY(check_hip(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)));
    hipLaunchKernelGGL((few_rows_kernel<X, FRAGMENTS>), dim3((uint32_t)(groups < at_a_time ? groups : at_a_time)), dim3(kFewThreads),
                       lds, stream, a);
    return check_launch();
}

using Many64 = Shape<128, 64, 4, 1>;
using Many4_64 = Shape<256, 64, 4, 1>;

int launch_large16(ManyArgs a, hipStream_t stream) {
    a.tiles_m = (int32_t)ceil_div(a.w.V, Large16::BM);
    a.tiles_n = (int32_t)ceil_div(a.out.B, Large16::BN);
    const int64_t work = (int64_t)a.tiles_m * a.tiles_n;
    if (work > 0x7FFFFFFF) return CFGZIP_E_TOO_LARGE;
    hipLaunchKernelGGL(large16_kernel, dim3((uint32_t)work), dim3(Large16::kThreads), 0, stream, a);
    return check_launch();
}

int launch_large4(ManyArgs a, hipStream_t stream) {
    a.tiles_m = (int32_t)ceil_div(a.w.V, Large4::BM);
    a.tiles_n = (int32_t)ceil_div(a.out.B, Large4::BN);
    const int64_t work = (int64_t)a.tiles_m * a.tiles_n;
    if (work > 0x7FFFFFFF) return CFGZIP_E_TOO_LARGE;
    hipLaunchKernelGGL(large4_kernel, dim3((uint32_t)work), dim3(Large4::kThreads), 0, stream, a);
    return check_launch();
}

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
        if (dtype != CFGZIP_DTYPE_MX4) w.x = c.take<uint16_t>((size_t)B * whole_pairs(K) * (dtype == CFGZIP_DTYPE_F16 ? 2 : 1));
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
        return B <= 64 || (int64_t)V * nb < 16 ? launch_many<Many4_64, true>(a, s) : launch_large4(a, s);
    }
    a.parts = x == X_F16 ? 2 : 1;
    a.part_steps = whole_pairs(K) / 128;
    if (x == X_BF16 && K % kPairK == 0 && hidden_stride % 8 == 0 && hidden_stride < kMaxStride && aligned_to(hidden, 16)) {
        a.x = static_cast<const char *>(hidden);
        a.x_row_bytes = hidden_stride * 2;
    } else {
        const int32_t ld = whole_pairs(K);
        const dim3 g((uint32_t)ceil_div((int64_t)B * (ld / 8), 256)), t(256);
        const uint16_t *h = static_cast<const uint16_t *>(hidden);
        if (x == X_F16) hipLaunchKernelGGL(split_kernel<true>, g, t, 0, s, h, hidden_stride, B, K, ld, w.x);
        else hipLaunchKernelGGL(split_kernel<false>, g, t, 0, s, h, hidden_stride, B, K, ld, w.x);
        CFGZIP_TRY(check_launch());
        a.x = reinterpret_cast<const char *>(w.x);
        a.x_part_bytes = (int64_t)ld * 2;
        a.x_row_bytes = a.x_part_bytes * a.parts;
    }
    a.x_units = nb * 4;
    if (B > 64) return launch_large16(a, s);
    return launch_many<Many64, false>(a, s);
}
