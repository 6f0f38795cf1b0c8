// The vocabulary projection's loss under a grammar's masks, and its gradients, without the logits in memory (but for gradients of few
// rows).
//
//     z[i][v] = sum_d hidden[i][d] weight[v][d]
//     lse[i] = log sum over admitted v of exp z[i][v],   loss[i] = lse[i] - z[i][target[i]]
//     dz[i][v] = grad_loss[i] (exp(z[i][v] - lse[i]) - [v = target[i]]) for admitted v
//     grad_hidden = dz weight,   grad_weight = dz^T hidden
//
// Forward: a tile of logits stays in the accumulators of the product that makes it; each wave leaves the maximum of its part of
// every row and the sum of exponentials against that maximum, and a second kernel joins them.  Backward: the logits are made
// again, for a piece of the vocabulary at a time, turned into dz in the accumulators, and stored in 16 bits; the two products
// that read the piece follow, where it is one of several while most of it is in the last-level cache.  All sums are fp32.
//
// What bounds it: with many rows the matrix cores.  Tiles of 256 x 256 by four waves, whose sums are in the 256 accumulation registers
// of each, need 64 KB of operands for every 8.4 MFLOP; loss of 2,048 x 128,256 x 2,048 860 us, 1.25 PFLOP/s, as a large library
// product of that shape (1.23).  With few rows it is reading the weights (one row of 32,000 x 2,048: 6.1 TB/s from the caches, the
// rest of the call's 40 us three launches and the host), with small sizes the chain of launches, 4 to 14 us each.

#include <algorithm>

#include "gemm16.hpp"

namespace cfgzip {
namespace {

using Shape16 = Shape<64, 16, 4, 1, 4>;  // few rows: reading the weights is what counts, many small workgroups
using Shape64 = Shape<128, 64, 4, 1, 3>;
using Shape128 = Shape<256, 128, 4, 2, 3>;
using Shape256 = Shape<256, 256, 2, 2, 2>;
using ShapeFlat = Shape<128, 256, 2, 4, 3>;  // weight gradients of small hidden sizes

// workgroups that are at work at a time: as many to a compute unit as its LDS holds
template <typename S>
constexpr int64_t slots() {
    return 256 * (160 * 1024 / (S::kStages * S::kLds));
}

// What a product's tiles take, in microseconds: rounds of as many as are at work at a time, of so many steps each and a beginning and an
// end.  (Estimates from traces of whole calls, to choose between tiles by; not measured one by one.)
template <typename S>
constexpr double kStepTime = S::BM * S::BN == 65536 ? 1.6 : S::BM * S::BN == 32768 ? 1.0 : S::BM * S::BN == 8192 ? 0.6 : 0.35;
template <typename S>
constexpr double kEndsTime = S::BM * S::BN == 65536 ? 10.0 : S::BM * S::BN == 32768 ? 6.0 : 4.0;
template <typename S>
double time_of(int64_t m, int64_t n, int64_t steps) {
    return (double)ceil_div(ceil_div(m, S::BM) * ceil_div(n, S::BN), slots<S>()) * ((double)steps * kStepTime<S> + kEndsTime<S>);
}

// Of dz, and of bf16 weights in fp16 or fp16 rows' rests beside it, in memory at a time: seven eighths of the last-level cache, so that the
// products that read them find them there.  But each piece adds to grad_hidden's sums anew and has ends of its own: where rows times
// hidden size are few, as many tokens as make that little beside the products, if dz alone still fits there and both take up to three
// times as much (777 rows of 128,256 x 4,096 in eight pieces 4.36 ms, in two 4.00, in one 3.95).
constexpr int64_t kPieceBytes = (int64_t)224 << 20;
constexpr double kPieceProducts = 2e11;  // rows * hidden size * tokens
// Up to so many rows dz is kept in two 16-bit numbers, and its probabilities come from the row's maximum and sum beside lse, which
// large logits round to few digits behind the point: a few rows' roundings do not average out, and reading the weights takes longer
// than the products, which are twice as many.  With more rows dz is one fp16 number, for which bf16 weights are read and written once
// more.  Gradients of 200 bf16 rows of 32,000 x 2,048 take 298 us so and 244 as two numbers, of 128,256 x 4,096 1,840 and 1,607; of 50,003 x
// 333, whose rows lie at no multiples of 16 bytes until they are fp16, 181 and 249.  fp16 rows would be faster in one number as well (200 of
// 50,003 x 1,000 163 us for 247): there it is the precision.
template <typename T>
int32_t few_rows_of(int32_t D) { return std::is_same_v<T, Bf16> && D % 8 ? 128 : 256; }
constexpr int32_t kPieceLeast = 2048;              // tokens
constexpr int32_t kSplitLeast = 256;               // tokens of grad_hidden's sum that a workgroup takes at the least
constexpr int32_t kMaxRows = 1 << 22;               // offsets in a tile of dz stay below 2^32
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

struct Masks {
    const int32_t *bits;  // [N][words], over tokens; null: every token is admitted
    int64_t words;
};

// Of dz in one number for fp16 results its largest element, the target's, is kept to the last bit: what its rounding leaves goes to
// grad_hidden as rest * weight[target], and to the token's row of grad_weight as the sum of rest * hidden over the token's rows, in their
// order.  (Without, 777 rows of 50,003 x 1,000 were 1.7 times as far from 64 bits as their own rounding makes them.)
struct Rests {
    float *rest;       // [N]
    int32_t *first;    // [V]: the first row whose target the token is
    int32_t *count;    // [V]: how many there are
    float *sums;       // [N + 1][ld]: at a token's first row; zeros at the last
    int32_t ld;
};
constexpr int32_t kNoRow = 0x7FFFFFFF;

struct LogitsArgs {
    Operand W, H;  // [V][D], [N][D]
    int32_t V, N, D;
    int32_t v0;        // first token of W
    int32_t tiles_m, tiles_n;
    Masks masks;
    const int32_t *target;
    // forward
    f32x2 *parts;  // [parts][N]: maximum and sum
    float *z_target;
    // backward
    const float *lse;
    const float *factor;       // of a row's dz; 0: it has no gradient
    const float *common;       // of all
    Rests rests;               // fp16
    uint16_t *dz;              // [piece / 64][dz_rows][64]
    int64_t dz_rows;
    float *z;                  // [tokens / 64][N][64], -inf where not admitted
};

// what becomes of a tile of logits: maxima and sums; those and the logits themselves, of few rows; dz
enum : int { STATISTICS = 0, KEPT = 1, GRADIENT = 2 };

// exp(z - shift) grad, the same bits wherever it stands: the product is not fused with what is taken from it
__device__ __forceinline__ float probability(float z, float shift, float grad) {
#pragma clang fp contract(off)
    return __builtin_amdgcn_exp2f((z - shift) * kLog2e) * grad;
}

template <typename T, typename S, bool DIRECT, int WHAT>
__global__ __launch_bounds__(S::kThreads) void logits_kernel(LogitsArgs a) {
    using TileA = Tile<S::BM, S::kThreads, false, DIRECT, ANY>;
    using TileB = Tile<S::BN, S::kThreads, false, true, PADDED>;
    CFGZIP_STAGES(S, lds);
    auto work = [&](int32_t i, Work &w) CFGZIP_INLINE {
        const uint32_t total = (uint32_t)a.tiles_m * a.tiles_n, t = blockIdx.x + i * gridDim.x;
        if (t >= total) return false;
        int32_t tm, tn;
        tile_of(t, total, a.tiles_m, a.tiles_n, tm, tn);
        w = Work{tm * S::BM, tn * S::BN, 0, a.D};
        return true;
    };
    auto store = [&](int32_t i, f32x4(&acc)[S::FM][S::FN], int wm, int wn, int lane) CFGZIP_INLINE {
        int32_t tm, tn;
        tile_of(blockIdx.x + i * gridDim.x, (uint32_t)a.tiles_m * a.tiles_n, a.tiles_m, a.tiles_n, tm, tn);
        const int g = lane >> 4;
        const int32_t first = tm * S::BM + wm * S::TM;  // in the piece
        const int32_t v_first = a.v0 + first;
        const bool masked = a.masks.bits || v_first + S::TM > a.V;
        // What belongs to the rows is asked for before the first of it is used: a load from memory takes as long as hundreds of
        // the elements' instructions (with a wait for each row in turn dz of 777 x 50,003 x 1,000 took 191 us for 174).
        constexpr int kWords = (S::TM + 31) / 32;
        const int32_t k_first = v_first >> 5;
        uint32_t words[S::FN][kWords];
        int32_t targets[S::FN];
        float shifts[S::FN], grads[S::FN];
        each<S::FN>([&](auto j) CFGZIP_INLINE {
            const int32_t row = tn * S::BN + wn * S::TN + 16 * j.value + (lane & 15), at = row < a.N ? row : a.N - 1;
            targets[j.value] = a.target[at];
            if constexpr (WHAT == GRADIENT) {
                grads[j.value] = a.factor[at] * *a.common;
                shifts[j.value] = a.lse[at];
            }
            each<kWords>([&](auto w) CFGZIP_INLINE { words[j.value][w.value] = ~0u; });
            if (a.masks.bits) {
                const int32_t *const bits = a.masks.bits + at * a.masks.words;
                each<kWords>([&](auto w) CFGZIP_INLINE {  // (what lies behind the last word is cut off below)
                    const int64_t k = k_first + w.value < a.masks.words ? k_first + w.value : a.masks.words - 1;
                    words[j.value][w.value] = (uint32_t)bits[k];
                });
            }
        });
        each<S::FN>([&](auto jj) CFGZIP_INLINE {
            constexpr int j = jj.value;
            const int32_t row = tn * S::BN + wn * S::TN + 16 * j + (lane & 15);
            const bool in = row < a.N;
            if (masked) {  // what a row does not admit becomes -inf, whatever it was
                each<kWords>([&](auto ww) CFGZIP_INLINE {
                    uint32_t word = words[j][ww.value];
                    const int64_t left = a.V - (int64_t)(k_first + ww.value) * 32;  // tokens from the word's first on
                    if (left < 32) word &= left > 0 ? (1u << left) - 1u : 0u;
                    each<(S::TM < 32 ? S::FM : 2)>([&](auto ii) CFGZIP_INLINE {
                        constexpr int i = ww.value * 2 + ii.value;
                        const int32_t four = (int32_t)(word >> (((v_first & 31) + 16 * ii.value + 4 * g) & 31));
                        each<4>([&](auto r) CFGZIP_INLINE {
                            const uint32_t keep = (uint32_t)((int32_t)((uint32_t)four << (31 - r.value)) >> 31);
                            const float z = acc[i][j][r.value];  // (a cast of the element itself takes the first one's bits)
                            acc[i][j][r.value] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, z) & keep) | (0xFF800000u & ~keep));
                        });
                    });
                });
            }
            const int32_t mark = targets[j] - v_first - 4 * g;  // the target is element mark % 16 of fragment mark / 16
            const bool marked = __builtin_amdgcn_ballot_w64(in && mark >= 0 && mark < S::TM) != 0;  // seldom
            if constexpr (WHAT != GRADIENT) {
                float most = -kInf;
                each<S::FM>([&](auto i) CFGZIP_INLINE {
                    most = fmaxf(fmaxf(most, acc[i.value][j][0]), acc[i.value][j][1]);
                    most = fmaxf(fmaxf(most, acc[i.value][j][2]), acc[i.value][j][3]);
                });
                if (WHAT == STATISTICS && marked) {
                    float z = 0.0f;
                    bool mine = false;
                    each<S::FM * 4>([&](auto e) CFGZIP_INLINE {
                        const bool here = mark == e.value / 4 * 16 + e.value % 4;
                        z = here ? acc[e.value / 4][j][e.value % 4] : z;
                        mine |= here;
                    });
                    if (in && mine) a.z_target[row] = z;
                }
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                const float shift = most == -kInf ? 0.0f : most;
                float sum = 0.0f;
                each<S::FM * 4>([&](auto e) CFGZIP_INLINE {
                    sum += __builtin_amdgcn_exp2f((acc[e.value / 4][j][e.value % 4] - shift) * kLog2e);
                });
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                if (g == 0 && in) a.parts[(int64_t)(tm * S::WM + wm) * a.N + row] = f32x2{most, sum};
                if (WHAT == KEPT && in) {
                    float *const out = a.z + ((int64_t)(first >> 6) * a.N + row) * 64 + (first & 63) + 4 * g;
                    each<S::FM>([&](auto i) CFGZIP_INLINE {
                        *reinterpret_cast<f32x4 *>(out + (int64_t)(i.value / 4) * a.N * 64 + i.value % 4 * 16) = acc[i.value][j];
                    });
                }
            } else {
                const float grad = in ? grads[j] : 0.0f;
                // rows without a gradient have hidden states of 0 here, so logits of 0 or -inf, and exp(-inf) * 0
                const float shift = grad != 0.0f ? shifts[j] : kInf;
                uint16_t *const out = a.dz + row * 64 + (first >> 6) * (a.dz_rows * 64) + (first & 63) + 4 * g;
                each<S::FM>([&](auto i) CFGZIP_INLINE {
                    f32x4 d;
                    each<4>([&](auto r) CFGZIP_INLINE {
                        d[r.value] = probability(acc[i.value][j][r.value], shift, grad);
                    });
                    if (marked) {
                        each<4>([&](auto r) CFGZIP_INLINE {
                            if (mark == 16 * i.value + r.value && acc[i.value][j][r.value] > -kInf) d[r.value] -= grad;
                        });
                    }
                    *reinterpret_cast<u32x2 *>(out + (i.value / 4) * (a.dz_rows * 64) + i.value % 4 * 16) = round4<Fp16>(d);
                });
                if constexpr (std::is_same_v<T, Fp16>) {
                    if (marked) {  // the target's dz once more (among the elements it took the kernel 22 us of 150)
                        float z = -kInf;
                        each<S::FM * 4>([&](auto e) CFGZIP_INLINE {
                            const bool here = mark == e.value / 4 * 16 + e.value % 4;
                            z = here ? acc[e.value / 4][j][e.value % 4] : z;
                        });
                        const float d = probability(z, shift, grad) - grad;
                        if (grad != 0.0f && z > -kInf) {
                            a.rests.rest[row] = d - Fp16::value(Fp16::round(d));
                            atomicMin(&a.rests.first[targets[j]], row);
                            atomicAdd(&a.rests.count[targets[j]], 1);
                        }
                    }
                }
            }
        });
    };
    multiply<T, S, TileA, TileB>(a.W, a.H, lds, work, store, NoScales{});
}

// Joins the parts of a row: lse and loss; or (`whole` given) its maximum and sum, so that exp(z - maximum) / sum is exp(z - lse) of the lse
// that the caller gave, without its rounding where it is the row's own.  A workgroup has ROWS rows and splits the parts over the other
// lanes; a lane asks for eight parts before it uses the first.
template <int ROWS>
__global__ __launch_bounds__(1024) void join_kernel(const f32x2 *parts, int32_t count, int32_t N, int32_t V, Masks masks,
                                                    const int32_t *target, const float *z_target, float *loss, float *lse,
                                                    f32x2 *whole) {  // lse: out, with `whole` in
    constexpr int kShares = 1024 / ROWS;
    struct Part {
        float most;
        double sum;  // the sum of a row that is certain is 1 and very little, and that little is its gradient
    };
    __shared__ Part shared[kShares][ROWS + 1];
    const int r = threadIdx.x % ROWS, s = threadIdx.x / ROWS;
    const int32_t row = blockIdx.x * ROWS + r;
    float most = -kInf;
    double sum = 0.0;
    auto take = [&](float m, double x) {
        const float top = fmaxf(most, m);
        // a part without admitted tokens has the maximum -inf and the sum 0 (or NaN, of logits that are)
        sum = (most == -kInf ? sum : sum * __expf(most - top)) + (m == -kInf ? x : x * __expf(m - top));
        most = top;
    };
    if (row < N) {
        for (int32_t p = s; p < count; p += 8 * kShares) {
            f32x2 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p + i * kShares < count ? parts[(int64_t)(p + i * kShares) * N + row] : f32x2{-kInf, 0.0f};
#pragma unroll
            for (int i = 0; i < 8; ++i) take(x[i][0], x[i][1]);
        }
    }
    shared[s][r] = Part{most, sum};
    for (int half = kShares / 2; half > 0; half /= 2) {
        __syncthreads();
        if (s < half) {
            take(shared[s + half][r].most, shared[s + half][r].sum);
            shared[s][r] = Part{most, sum};
        }
    }
    if (s != 0 || row >= N) return;
    const float l = (most == -kInf ? 0.0f : most) + logf((float)sum);
    if (whole) {
        float apart = l - lse[row];
        if (fabsf(apart) <= 0x1p-22f * fabsf(l)) apart = 0.0f;  // the same number, by sums of other parts or their roundings
        whole[row] = f32x2{most - apart, (float)sum};
        return;
    }
    const int32_t t = target[row];
    float out = 0.0f;
    if (t >= 0 && t < V) {
        const bool ok = !masks.bits || (masks.bits[row * masks.words + (t >> 5)] >> (t & 31) & 1);
        out = ok ? l - z_target[row] : kInf;
    }
    lse[row] = l;
    loss[row] = out;
}

// Row i's gradient; 0 if its target is none or not admitted.
struct Rows {
    const float *grad_loss;
    const int32_t *target;
    int32_t N, V;
    Masks masks;
    __device__ __forceinline__ float grad(int32_t i) const {
        const int32_t t = target[i];
        if (t < 0 || t >= V) return 0.0f;
        if (masks.bits && !(masks.bits[i * masks.words + (t >> 5)] >> (t & 31) & 1)) return 0.0f;
        return grad_loss[i];
    }
    // The largest finite gradient.  For all threads of a workgroup, whose waves leave their maxima in `shared`.
    __device__ float largest(float *shared) const {
        float most = 0.0f;
        for (int32_t i = threadIdx.x; i < N; i += blockDim.x) {
            const float x = fabsf(grad(i));
            if (x < kInf) most = fmaxf(most, x);
        }
        for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = most;
        __syncthreads();
        for (int i = 0; i < (int)blockDim.x / kWave; ++i) most = fmaxf(most, shared[i]);
        return most;
    }
    // The factor that makes it 2^14, for dz in bf16, whose range holds what the clamps leave beyond that and rows of any size beside each other.
    __device__ float scale(float *shared) const { return 0x1p14f / fminf(fmaxf(largest(shared), 0x1p-86f), 0x1p114f); }
};

// floor(log2 |x|) of a finite x other than 0
__device__ __forceinline__ int32_t exponent_of(float x) { return __builtin_amdgcn_frexp_expf(x) - 1; }

// dz in fp16.  Its range holds a row's probabilities beside the row's own gradient, but not those of a row beside a gradient that is
// 2^28 times as large, nor every gradient that there is.  So a row's gradient is digits * 2^(power + 14) with digits of 1 to 2: dz has
// the digits times 2^14, the power of two multiplies the row of grad_hidden on its way out and, for grad_weight's sum over the rows,
// the row's hidden states as they become fp16 with a common power of two.
struct RowFactors {
    float *dz;       // 0: the row has no gradient
    int32_t *power;
    // [0] takes from the digits what they have in common, so that where all rows have the same gradient, as that of a mean, a row that is
    // certain and wrong has dz without a rounding; [1] its inverse.  null where two numbers make up dz.
    float *common;
};

// dz of few rows from their logits, as the sum of two 16-bit numbers: rows 0 .. N - 1 of dz are the first ones, N .. 2 N - 1 what they
// leave, the rest 0.  A thread has four tokens.
template <typename T>
__global__ __launch_bounds__(256) void few_rows_dz_kernel(Rows rows, const float *z, int32_t blocks, const f32x2 *whole, uint16_t *dz,
                                                          int32_t dz_rows, const float *factors, float *unscale) {
    float factor = 1.0f;
    if constexpr (std::is_same_v<T, Bf16>) {
        __shared__ float shared[4];
        factor = rows.scale(shared);
        if (blockIdx.x == 0 && threadIdx.x == 0) *unscale = 1.0f / factor;
    }
    const int32_t N = rows.N, span = dz_rows - N;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int32_t q = (int32_t)(k & 15), r = (int32_t)((k >> 4) % span);
    const int64_t block = (k >> 4) / span;
    if (block >= blocks) return;
    uint16_t *const out = dz + block * dz_rows * 64 + q * 4;
    u32x2 hi = {0, 0}, lo = {0, 0};
    if (r < N) {
        const float grad = std::is_same_v<T, Bf16> ? rows.grad(r) * factor : factors[r];
        if (grad != 0.0f) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(z + (block * N + r) * 64 + q * 4);
            const f32x2 w = whole[r];
            const int32_t mark = rows.target[r] - (int32_t)(block * 64 + q * 4);
            f32x4 d, rest;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = __expf(x[j] - w[0]) / w[1];
                d[j] = x[j] == -kInf ? 0.0f : (p - (j == mark ? 1.0f : 0.0f)) * grad;
                rest[j] = d[j] - T::value(T::round(d[j]));
            }
            hi = round4<T>(d);
            lo = round4<T>(rest);
        }
        *reinterpret_cast<u32x2 *>(out + (int64_t)(N + r) * 64) = lo;
        *reinterpret_cast<u32x2 *>(out + (int64_t)r * 64) = hi;
    } else {
        *reinterpret_cast<u32x2 *>(out + (int64_t)(N + r) * 64) = hi;
    }
}

// Hidden states in rows of whole steps of 64 elements (zeros behind D), `times` times over, and rows of zeros behind them up to `all`;
// but for `whole`, zeros in those that have no gradient, whatever they hold.
__global__ __launch_bounds__(256) void copy_rows_kernel(const uint16_t *x, int64_t x_ld, int32_t N, int32_t D, int32_t times, int32_t all,
                                                        bool whole, Rows rows, uint16_t *y, int32_t y_ld) {
    const int32_t units = y_ld / 8;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= (int64_t)(N + all - N * times) * units) return;
    const int32_t row = (int32_t)(k / units), c = (int32_t)(k % units) * 8;
    u32x4 v = {0, 0, 0, 0};
    if (row >= N) {
        *reinterpret_cast<u32x4 *>(y + ((int64_t)N * (times - 1) + row) * y_ld + c) = v;
        return;
    }
    if (whole || rows.grad(row) != 0.0f) {
        const uint16_t *p = x + row * x_ld + c;
        if (c + 8 <= D) {
            v = *reinterpret_cast<const u32x4_any *>(p);
        } else {
            for (int j = 0; c + j < D; ++j) v[j / 2] |= (uint32_t)p[j] << (j % 2 * 16);
        }
    }
    for (int32_t i = 0; i < times; ++i) *reinterpret_cast<u32x4 *>(y + ((int64_t)i * N + row) * y_ld + c) = v;
}

// four results next to each other at any element alignment, the last of a row one by one
template <typename T>
__device__ __forceinline__ void store4(uint16_t *row, int32_t c, int32_t n, f32x4 x) {
    if (c + 4 <= n) {
        *reinterpret_cast<u32x2_any *>(row + c) = round4<T>(x);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (c + r < n) row[c + r] = T::round(x[r]);
    }
}

constexpr int32_t kNone = -100000;  // floor(log2 0)

// The largest finite |x| of 16-bit numbers as bits
template <typename T>
__device__ __forceinline__ void take_largest(uint32_t &most, uint32_t bits) {
    bits &= 0x7FFFu;
    most = bits > most && bits < (std::is_same_v<T, Bf16> ? 0x7F80u : 0x7C00u) ? bits : most;
}
// The largest of a workgroup's WAVES waves, for thread 0
template <int WAVES>
__device__ __forceinline__ int32_t largest_of(int32_t x, int32_t *shared) {
    for (int d = 1; d < kWave; d *= 2) {
        const int32_t other = __shfl_xor(x, d);
        x = other > x ? other : x;
    }
    if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < WAVES; ++i) x = shared[i] > x ? shared[i] : x;
    return x;
}

// For dz in fp16: the rows' factors, their hidden states in rows of whole steps of 64 elements (zeros behind D, and in those without a
// gradient, whatever they hold), and floor(log2) of the largest |hidden| times its row's power of two, which workgroup b leaves of the
// rows that it took in largest[b], kNone where all is 0.  A wave takes a row at a time; the last workgroup has the digits' common part.
constexpr int kRowsOfBlock = 16, kRowBlocks = 256;
template <typename T>
__global__ __launch_bounds__(kRowsOfBlock *kWave) void rows_kernel(Rows rows, const uint16_t *x, int64_t x_ld, int32_t D, uint16_t *y, int32_t y_ld,
                                                                   RowFactors f, Rests rests, int32_t *largest) {
    __shared__ int32_t shared[kRowsOfBlock];
    if (rests.rest) {
        for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows.V; i += (int64_t)gridDim.x * blockDim.x)
            rests.first[i] = kNoRow, rests.count[i] = 0;
        for (int32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < rests.ld; i += gridDim.x * blockDim.x)
            rests.sums[(int64_t)rows.N * rests.ld + i] = 0.0f;
    }
    const int32_t blocks = gridDim.x - 1;
    if ((int32_t)blockIdx.x == blocks) {
        if (!f.common) return;
        const float most = rows.largest(reinterpret_cast<float *>(shared));
        if (threadIdx.x == 0) {
            const float digits = most == 0.0f ? 1.0f : ldexpf(most, -exponent_of(most));
            f.common[0] = 1.0f / digits;
            f.common[1] = digits;
        }
        return;
    }
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int32_t most = kNone;
    for (int32_t row = blockIdx.x * kRowsOfBlock + wave; row < rows.N; row += blocks * kRowsOfBlock) {
        const float grad = rows.grad(row);
        const bool finite = fabsf(grad) < kInf && grad != 0.0f;
        const int32_t e = finite ? exponent_of(grad) : 0, power = e - 14;
        const float digits = finite ? ldexpf(grad, -e) : grad;
        if (lane == 0) {
            f.dz[row] = digits * 0x1p14f;
            f.power[row] = power;
            if (rests.rest) rests.rest[row] = 0.0f;
        }
        const uint16_t *const p = x + row * x_ld;
        uint16_t *const to = y + (int64_t)row * y_ld;
        uint32_t bits = 0;
        constexpr int kUnits = 4;  // on their way at a time
        for (int32_t c = lane * 8; c < y_ld; c += kWave * 8 * kUnits) {
            u32x4 v[kUnits];
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int32_t at = c + i * kWave * 8;
                v[i] = u32x4{0, 0, 0, 0};
                if (grad != 0.0f && at + 8 <= D) {
                    v[i] = *reinterpret_cast<const u32x4_any *>(p + at);
                } else if (grad != 0.0f) {
                    for (int j = 0; at + j < D; ++j) v[i][j / 2] |= (uint32_t)p[at + j] << (j % 2 * 16);
                }
            }
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int32_t at = c + i * kWave * 8;
                if (at < y_ld) *reinterpret_cast<u32x4 *>(to + at) = v[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) take_largest<T>(bits, v[i][j]), take_largest<T>(bits, v[i][j] >> 16);
            }
        }
        if (bits) {
            const int32_t here = exponent_of(T::value((uint16_t)bits)) + power;
            most = here > most ? here : most;
        }
    }
    most = largest_of<kRowsOfBlock>(most, shared);
    if (threadIdx.x == 0) largest[blockIdx.x] = most;
}

// floor(log2) of the largest finite |x| of bf16 weights: workgroup b leaves that of the rows it took in largest[b], kNone where all is 0.
// A wave takes a row at a time.  (One word and atomic maxima took 250 us for 128,256 x 4,096: as many waves, one after the other.)
constexpr int kWeightBlocks = 1024;
struct Matrix16 {
    const uint16_t *x;
    int64_t ld;
    int32_t rows, D;
};
__global__ __launch_bounds__(256) void largest_kernel(Matrix16 m, int32_t *largest) {
    __shared__ int32_t shared[4];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint32_t bits = 0;
    constexpr int kUnits = 8;  // on their way at a time
    for (int64_t row = (int64_t)blockIdx.x * 4 + wave; row < m.rows; row += kWeightBlocks * 4) {
        const uint16_t *const p = m.x + row * m.ld;
        for (int32_t c = lane * 8; c < m.D; c += kWave * 8 * kUnits) {
            u32x4 v[kUnits];
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int32_t at = c + i * kWave * 8;
                v[i] = u32x4{0, 0, 0, 0};
                if (at + 8 <= m.D) {
                    v[i] = *reinterpret_cast<const u32x4_any *>(p + at);
                } else {
                    for (int32_t j = at; j < m.D; ++j) take_largest<Bf16>(bits, p[j]);
                }
            }
#pragma unroll
            for (int i = 0; i < kUnits; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) take_largest<Bf16>(bits, v[i][j]), take_largest<Bf16>(bits, v[i][j] >> 16);
        }
    }
    const int32_t most = largest_of<4>(bits ? exponent_of(Bf16::value((uint16_t)bits)) : kNone, shared);
    if (threadIdx.x == 0) largest[blockIdx.x] = most;
}

// 2^e in two factors: one alone may be too much for fp32, and what is beyond both is 0 in 16 bits.  (ldexp is half as fast as a product.)
struct PowerOfTwo {
    float a, b;
    __device__ __forceinline__ explicit PowerOfTwo(int32_t e) {
        const int32_t first = e < -126 ? -126 : e > 127 ? 127 : e, rest = e - first;
        a = __builtin_bit_cast(float, (uint32_t)(127 + first) << 23);
        b = __builtin_bit_cast(float, (uint32_t)(127 + (rest < -126 ? -126 : rest > 127 ? 127 : rest)) << 23);
    }
};

// 16-bit rows as fp16, times a row's power of two where there is one and the one that brings the largest of the `count` to 2^14 to 2^15:
// bf16 within 2^31 of the largest keeps its eight bits, what is smaller is 2^-39 of the largest or less off.  The rows `times` times over,
// y_ld elements each, zeros behind D and behind the last up to `all`.  Leaves the power of two that takes that back in `back`.  A thread has
// four units of eight.
template <typename T>
__global__ __launch_bounds__(256) void halves_kernel(Matrix16 x, const int32_t *powers, const int32_t *largest, int32_t count, int32_t times,
                                                     uint16_t *y, int32_t y_ld, int32_t all, int32_t *back) {
    __shared__ int32_t shared[5];
    int32_t most = kNone;
    for (int32_t i = threadIdx.x; i < count; i += 256) most = largest[i] > most ? largest[i] : most;
    most = largest_of<4>(most, shared);
    if (threadIdx.x == 0) shared[4] = most;
    __syncthreads();
    most = shared[4];
    const int32_t power = most == kNone ? 0 : 14 - most;
    if (blockIdx.x == 0 && threadIdx.x == 0) *back = -power;
    const int32_t units = y_ld / 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t at = ((int64_t)blockIdx.x * 4 + i) * 256 + threadIdx.x;
        if (at >= (int64_t)all * units) break;
        const int32_t to = (int32_t)(at / units), c = (int32_t)(at % units) * 8, row = times == 2 && to >= x.rows ? to - x.rows : to;
        u32x4 v = {0, 0, 0, 0};
        int32_t e = power;
        if (row < x.rows) {
            const uint16_t *const p = x.x + row * x.ld + c;
            if (c + 8 <= x.D) {
                v = *reinterpret_cast<const u32x4_any *>(p);
            } else {
                for (int j = 0; c + j < x.D; ++j) v[j / 2] |= (uint32_t)p[j] << (j % 2 * 16);
            }
            if (powers) e += powers[row];
        }
        const PowerOfTwo scale(e);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = Fp16::round2(T::value((uint16_t)v[j]) * scale.a * scale.b, T::value((uint16_t)(v[j] >> 16)) * scale.a * scale.b);
        *reinterpret_cast<u32x4 *>(y + (int64_t)to * y_ld + c) = v;
    }
}

// The sums of rest * hidden of the tokens v0 .. v0 + tokens - 1, in the order of their rows.  A workgroup has a row, and works if it is its
// token's first, until it has met them all; most tokens have one.  A thread has four columns.
__global__ __launch_bounds__(256) void rests_kernel(RowFactors f, Rests rests, const int32_t *target, int32_t N, int64_t v0, int32_t tokens,
                                                    const uint16_t *hidden16) {
    __shared__ uint64_t same[4];
    const int32_t row = blockIdx.x, t = target[row], lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    if (f.dz[row] == 0.0f || t < v0 || t - v0 >= tokens || rests.first[t] != row) return;
    const int32_t c = (blockIdx.y * 256 + threadIdx.x) * 4;
    int32_t left = rests.count[t];
    f32x4 sum = {0, 0, 0, 0};
    for (int32_t first = row; left > 0 && first < N; first += 256) {
        const int32_t j = first + threadIdx.x;
        const uint64_t here = __builtin_amdgcn_ballot_w64(j < N && target[j] == t && f.dz[j] != 0.0f);
        __syncthreads();
        if (lane == 0) same[wave] = here;
        __syncthreads();
        for (int w = 0; w < 4; ++w) {
            for (uint64_t more = same[w]; more; more &= more - 1, --left) {
                const int32_t k = first + w * kWave + __builtin_ctzll(more);
                if (c >= rests.ld) continue;
                const float rest = rests.rest[k];
                const u32x2 h = *reinterpret_cast<const u32x2 *>(hidden16 + (int64_t)k * rests.ld + c);
                sum += rest * f32x4{Fp16::value((uint16_t)h[0]), Fp16::value((uint16_t)(h[0] >> 16)), Fp16::value((uint16_t)h[1]),
                                    Fp16::value((uint16_t)(h[1] >> 16))};
            }
        }
    }
    if (c < rests.ld) *reinterpret_cast<f32x4 *>(rests.sums + (int64_t)row * rests.ld + c) = sum;
}

// What a result takes back of the factors of dz and of the product's other operand, each null where there is none.
struct Factors {
    const float *all;      // of all results
    const int32_t *power;  // of a row
    const int32_t *back;   // of all results
    __device__ __forceinline__ f32x2 of(int32_t row) const {
        const PowerOfTwo scale((power ? power[row] : 0) + (back ? *back : 0));
        return f32x2{scale.a, scale.b * (all ? *all : 1.0f)};
    }
};

struct GradArgs {
    Operand A, B;  // A: m = hidden size; B: n = rows (grad_hidden) or tokens (grad_weight)
    int32_t n, D;  // extents of the result
    int32_t k, k_split, splits;
    int32_t tiles_m, tiles_n;
    Factors factors;
    uint16_t *out;  // [n][out_ld]
    int64_t out_ld;
    float *sums;  // [splits][n][sums_ld], sums_ld = D rounded up to 4; null: the result goes to `out` at once
    int32_t sums_ld;
    int32_t add;  // to what is in `sums`
    const int32_t *first;  // grad_weight in fp16: the tokens' rows with rests; or null
    const float *rests;
    int32_t rests_ld, rests_rows;
};

// grad_hidden: A = weight by columns, B = dz by rows.  grad_weight: A = hidden, B = dz, both by columns.
// T: the operands' type, O: the results'.
// RESTS: of grad_weight, what dz's rounding left is added.
template <typename T, typename O, typename S, bool DIRECT, bool B_COLUMNS, bool RESTS>
__global__ __launch_bounds__(S::kThreads) void grad_kernel(GradArgs a) {
    // (weights end where the vocabulary does; hidden states and dz go on with zeros)
    using TileA = Tile<S::BM, S::kThreads, true, DIRECT, B_COLUMNS ? PADDED : ZERO>;
    using TileB = Tile<S::BN, S::kThreads, B_COLUMNS, true, PADDED>;
    CFGZIP_STAGES(S, lds);
    auto place = [&](int32_t i, int32_t &tm, int32_t &tn, int32_t &split) CFGZIP_INLINE {
        const uint32_t total = (uint32_t)a.tiles_m * a.tiles_n * a.splits, t = blockIdx.x + i * gridDim.x;
        if (t >= total) return false;
        tile_of(t, total, a.tiles_m, a.tiles_n * a.splits, tm, tn);
        split = tn / a.tiles_n;
        tn -= split * a.tiles_n;
        return true;
    };
    auto work = [&](int32_t i, Work &w) CFGZIP_INLINE {
        int32_t tm, tn, split;
        if (!place(i, tm, tn, split)) return false;
        const int32_t k0 = split * a.k_split;
        w = Work{tm * S::BM, tn * S::BN, k0 / kStepK, a.k - k0 < a.k_split ? a.k - k0 : a.k_split};
        return true;
    };
    auto store = [&](int32_t i, f32x4(&acc)[S::FM][S::FN], int wm, int wn, int lane) CFGZIP_INLINE {
        int32_t tm = 0, tn = 0, split = 0;
        place(i, tm, tn, split);
        f32x2 factor = {1.0f, 1.0f};
        if (B_COLUMNS) factor = a.factors.of(0);  // (asked for once: 32,000 x 2,048 with 64 rows 69 us for 79)
        each<S::FN>([&](auto j) CFGZIP_INLINE {
            const int32_t n = tn * S::BN + wn * S::TN + 16 * j.value + (lane & 15);
            if (n >= a.n) return;
            if (!B_COLUMNS && !a.sums) factor = a.factors.of(n);
            auto store_some = [&](auto with, const float *rests) CFGZIP_INLINE {
                each<S::FM>([&](auto i) CFGZIP_INLINE {
                    const int32_t c = tm * S::BM + wm * S::TM + 16 * i.value + 4 * (lane >> 4);
                    if (c >= a.D) return;
                    f32x4 x = acc[i.value][j.value];
                    if constexpr (with.value) x += *reinterpret_cast<const f32x4 *>(rests + c);
                    if (!RESTS && a.sums) {
                        f32x4 *p = reinterpret_cast<f32x4 *>(a.sums + ((int64_t)split * a.n + n) * a.sums_ld + c);
                        *p = a.add ? *p + x : x;
                    } else {
                        store4<O>(a.out + n * a.out_ld, c, a.D, x * factor[0] * factor[1]);
                    }
                });
            };
            if constexpr (RESTS) {
                // whose sum of rests belongs to the token; the last one's is 0
                // (the loop twice, behind a condition of the whole wave: one load that each lane's own condition guards took the kernel
                // 263 us for 151, its loads' addresses out of the registers)
                const int32_t row = a.first[n];
                if (__builtin_amdgcn_ballot_w64(row != kNoRow) != 0)  // (few tokens are a row's target)
                    store_some(std::true_type{}, a.rests + (int64_t)(row != kNoRow ? row : a.rests_rows) * a.rests_ld);
                else store_some(std::false_type{}, nullptr);
            } else {
                store_some(std::false_type{}, nullptr);
            }
        });
    };
    multiply<T, S, TileA, TileB>(a.A, a.B, lds, work, store, NoScales{});
}

// Joins grad_hidden's shares of the sum (and the two numbers of few rows' dz, or what is left of dz in one).
template <typename T>
__global__ __launch_bounds__(kWave) void finish_kernel(const float *sums, int32_t count, int32_t n, int32_t D, int32_t sums_ld,
                                                         Factors factors, const float *rest, const int32_t *target, const uint16_t *weight,
                                                         int64_t weight_ld, uint16_t *out, int64_t out_ld) {
    const int32_t units = sums_ld / 4;
    const int64_t k = (int64_t)blockIdx.x * kWave + threadIdx.x;
    if (k >= (int64_t)n * units) return;
    const int32_t row = (int32_t)(k / units), c = (int32_t)(k % units) * 4;
    const f32x2 factor = factors.of(row);
    const float *p = sums + (int64_t)row * sums_ld + c;
    const int64_t step = (int64_t)n * sums_ld;
    f32x4 x = {0, 0, 0, 0};
    for (int32_t s = 0; s < count; s += 16) {  // 16 loads on their way at a time: with each waited for 32 sums took 9.4 us
        f32x4 y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = s + i < count ? *reinterpret_cast<const f32x4 *>(p + (s + i) * step) : f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) x += y[i];
    }
    if (rest && rest[row] != 0.0f) {
        const uint16_t *const w = weight + target[row] * weight_ld + c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < D) x[i] += rest[row] * T::value(w[i]);
    }
    store4<T>(out + row * out_ld, c, D, x * factor[0] * factor[1]);
}

__global__ __launch_bounds__(256) void zero_rows_kernel(uint16_t *out, int64_t out_ld, int32_t n, int32_t D) {
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x)
        for (int32_t c = threadIdx.x; c < D; c += 256) out[row * out_ld + c] = 0;
}

// ---------------------------------------------------------------- host

int64_t pad(int64_t x, int64_t to) { return ceil_div(x, to) * to; }

// Rows of a tile.  Above 64 the larger tile reaches the higher rate, the smaller one wastes less of a last tile.
int rows_of_tile(int32_t N) {
    if (N <= 16) return 16;
    if (N <= 64) return 64;
    return pad(N, 128) * 4 < pad(N, 256) * 3 ? 128 : 256;
}
int32_t columns_of_tile(int rows) { return rows == 16 ? 64 : rows == 64 ? 128 : 256; }

struct Plan {
    int logits_rows;    // of a tile of logits
    int32_t parts;      // 16-bit numbers that make up a value of dz
    int rows;           // of a tile of dz
    int32_t rows_pad;   // rows of dz in whole tiles and steps
    int32_t d_pad;      // hidden size in whole steps
    int32_t piece;      // tokens of a piece of dz
    int32_t splits;     // of grad_hidden's sum over a piece
    int32_t sums_ld;
    bool direct_out;    // grad_hidden in one go
};

// halves: bf16 weights are written in fp16, a piece at a time
Plan plan_of(int32_t N, int32_t V, int32_t D, int32_t few_rows, bool halves) {
    Plan p{};
    p.parts = N <= few_rows ? 2 : 1;
    p.logits_rows = p.parts == 2 ? std::min(rows_of_tile(N), 128) : rows_of_tile(N);
    p.d_pad = (int32_t)pad(D, kStepK);
    const int32_t rows_dz = N * p.parts;
    // (tiles of logits leave zeros behind N as well, and grad_weight's sum goes over whole steps of rows)
    // A piece is a whole number of rounds of 256 tiles of logits, one to a compute unit, and one round at the least.
    const int64_t bytes = (pad(rows_dz, 256) + (halves && p.parts == 1 ? pad(D, 8) : 0)) * 2;  // of a token
    const int64_t rests = halves ? 0 : (int64_t)N * p.d_pad * 4 + (int64_t)V * 8;
    const int64_t there = std::max(kPieceBytes - rests, kPieceBytes / 2);
    const int64_t round = std::max<int64_t>(slots<Shape256>() / ceil_div(N, p.logits_rows), 1) * Shape256::BM;
    const int64_t fit = std::min(there / (pad(rows_dz, 256) * 2), 3 * there / bytes) / round;
    const int64_t products = std::min((int64_t)std::min(kPieceProducts / N / D / (double)round + 0.5, 1e9), fit);
    const int64_t least = std::max<int64_t>(ceil_div(kPieceLeast, round), 1);
    const int64_t rounds = std::max(std::max(there / bytes / round, products), least);
    const int64_t pieces = p.parts == 2 ? 1 : ceil_div(V, rounds * round);
    p.piece = (int32_t)(pieces == 1 ? pad(V, 256) : ceil_div(ceil_div(V, round), pieces) * round);
    // grad_hidden's sum runs over the vocabulary: it is split so that its tiles fill the chip, which costs a pass over the shares
    const int64_t first = V < p.piece ? V : p.piece;
    double best = 0;
    int64_t best_split = 0;
    auto look = [&](auto shape, int rows) {
        using S = decltype(shape);
        const int64_t tiles = ceil_div(D, S::BM) * ceil_div(rows_dz, S::BN);
        for (int64_t s = 1; s == 1 || (s * kSplitLeast <= p.piece && tiles * s <= slots<S>() * 2); ++s) {
            const int64_t k_split = pad(ceil_div(p.piece, s), kStepK);
            // a launch, and the shares written and read at 4 TB/s
            const double shares = s > 1 || pieces > 1 || p.parts > 1 ? 4.0 + (double)s * rows_dz * D * 8.0 / 4e6 : 0.0;
            const double tiles_time = (double)ceil_div(tiles * s, slots<S>()) * ((double)(k_split / kStepK) * kStepTime<S> + kEndsTime<S>);
            // (or reading the weights at 4.5 TB/s, which rows of several tiles read more than once, half of it from the caches, and
            // which takes twice as long through registers)
            const double time = std::max(tiles_time, (double)first * D * 2.0 / 4.5e6 * (0.5 + 0.5 * (double)ceil_div(rows_dz, S::BN)) * (D % 8 ? 2 : 1)) + shares;
            if (best == 0 || time < best) {
                best = time;
                p.rows = rows;
                best_split = k_split;
            }
        }
    };
    if (rows_dz <= 16) look(Shape16{}, 16);
    if (rows_dz <= 512) look(Shape64{}, 64);
    look(Shape128{}, 128);
    look(Shape256{}, 256);
    p.rows_pad = (int32_t)pad(rows_dz, std::max(std::max(p.rows, p.logits_rows), (int)kStepK));
    p.splits = (int32_t)ceil_div(first, best_split);  // of the first piece; later ones add to them
    p.sums_ld = (int32_t)pad(D, 4);
    p.direct_out = halves && pieces == 1 && p.splits == 1 && p.parts == 1;  // (fp16 rows: the rests are added behind it)
    return p;
}

bool kind_ok(int32_t bits_kind) {
    return bits_kind == CFGZIP_BITS_TOKEN || bits_kind == CFGZIP_BITS_CLASS || bits_kind == CFGZIP_BITS_NONE;
}

struct LossCall {
    const void *hidden;
    int64_t hidden_stride;
    const void *weight;
    int64_t weight_stride;
    int32_t dtype, N, V, D;
    const int32_t *target, *bits;
    int32_t bits_kind;
    const int32_t *class_of_token;
    int32_t C;
};

int check_call(const LossCall &c) {
    if (c.N < 0 || c.V <= 0 || c.D <= 0) return CFGZIP_E_INVALID;
    if (c.dtype != CFGZIP_DTYPE_BF16 && c.dtype != CFGZIP_DTYPE_F16) return CFGZIP_E_INVALID;
    if (!kind_ok(c.bits_kind)) return CFGZIP_E_INVALID;
    if (!c.weight || !aligned_to(c.weight, 2) || c.weight_stride < c.D) return CFGZIP_E_INVALID;
    if (c.N > 0) {
        if (!c.hidden || !c.target || !aligned_to(c.hidden, 2) || !aligned_to(c.target, 4) || c.hidden_stride < c.D)
            return CFGZIP_E_INVALID;
        if (c.bits_kind != CFGZIP_BITS_NONE && (!c.bits || !aligned_to(c.bits, 4))) return CFGZIP_E_INVALID;
        if (c.bits_kind == CFGZIP_BITS_CLASS && (!c.class_of_token || c.C <= 0 || !aligned_to(c.class_of_token, 4)))
            return CFGZIP_E_INVALID;
    }
    if (c.V > 0x7FFFFC00 || c.N > kMaxRows) return CFGZIP_E_TOO_LARGE;
    if (c.weight_stride >= kMaxStride || c.D >= kMaxStride - 8) return CFGZIP_E_TOO_LARGE;
    return CFGZIP_OK;
}

bool whole_units(const void *p, int64_t stride, int32_t D) { return aligned_to(p, 16) && stride % 8 == 0 && D % 8 == 0; }

// token-level masks of a call, expanded into the workspace from masks over classes
int masks_of(const LossCall &c, Carver &ws, hipStream_t stream, Masks &m, bool launch) {
    m = Masks{nullptr, words_for(c.V)};
    if (c.bits_kind == CFGZIP_BITS_TOKEN) m.bits = c.bits;
    if (c.bits_kind == CFGZIP_BITS_CLASS) {
        int32_t *tok = ws.take<int32_t>((size_t)c.N * m.words);
        m.bits = tok;
        if (launch) return cfgzip_expand_mask(c.bits, c.N, c.C, c.class_of_token, c.V, tok, stream);
    }
    return CFGZIP_OK;
}

template <typename T, typename S, int WHAT>
int launch_logits_of(const LogitsArgs &a, bool direct, hipStream_t stream) {
    const int64_t work = (int64_t)a.tiles_m * a.tiles_n, grid = work < slots<S>() ? work : slots<S>();
    if (work > 0x7FFFFFFF - slots<S>()) return CFGZIP_E_TOO_LARGE;
    if (direct) hipLaunchKernelGGL((logits_kernel<T, S, true, WHAT>), dim3((uint32_t)grid), dim3(S::kThreads), 0, stream, a);
    else hipLaunchKernelGGL((logits_kernel<T, S, false, WHAT>), dim3((uint32_t)grid), dim3(S::kThreads), 0, stream, a);
    return check_launch();
}

template <typename T, int WHAT>
int launch_logits(int rows, LogitsArgs a, int32_t tokens, bool direct, hipStream_t stream) {
    a.tiles_m = (int32_t)ceil_div(tokens, columns_of_tile(rows));
    a.tiles_n = (int32_t)ceil_div(a.N, rows);
    switch (rows) {
        case 16: return launch_logits_of<T, Shape16, WHAT>(a, direct, stream);
        case 64: return launch_logits_of<T, Shape64, WHAT>(a, direct, stream);
        case 128: return launch_logits_of<T, Shape128, WHAT>(a, direct, stream);
        default:
            if constexpr (WHAT == KEPT) return CFGZIP_E_INVALID;  // (not that few rows)
            else return launch_logits_of<T, Shape256, WHAT>(a, direct, stream);
    }
}

template <typename T, typename O, typename S, bool DIRECT, bool B_COLUMNS, bool RESTS = false>
int launch_grad_of(GradArgs a, hipStream_t stream) {
    a.tiles_m = (int32_t)ceil_div(a.D, S::BM);
    a.tiles_n = (int32_t)ceil_div(a.n, S::BN);
    const int64_t work = (int64_t)a.tiles_m * a.tiles_n * a.splits, grid = work < slots<S>() ? work : slots<S>();
    if (work > 0x7FFFFFFF - slots<S>()) return CFGZIP_E_TOO_LARGE;
    hipLaunchKernelGGL((grad_kernel<T, O, S, DIRECT, B_COLUMNS, RESTS>), dim3((uint32_t)grid), dim3(S::kThreads), 0, stream, a);
    return check_launch();
}

template <typename T, typename O, bool DIRECT>
int launch_grad_hidden(int rows, const GradArgs &a, hipStream_t stream) {
    switch (rows) {
        case 16: return launch_grad_of<T, O, Shape16, DIRECT, false>(a, stream);
        case 64: return launch_grad_of<T, O, Shape64, DIRECT, false>(a, stream);
        case 128: return launch_grad_of<T, O, Shape128, DIRECT, false>(a, stream);
        default: return launch_grad_of<T, O, Shape256, DIRECT, false>(a, stream);
    }
}

template <typename T, typename O, bool RESTS>
int launch_grad_weight_of(const GradArgs &a, hipStream_t stream) {
    const int32_t steps = (int32_t)ceil_div(a.k, kStepK);
    const double large = time_of<Shape256>(a.D, a.n, steps), middle = time_of<Shape128>(a.D, a.n, steps),
                 flat = time_of<ShapeFlat>(a.D, a.n, steps), small = time_of<Shape64>(a.D, a.n, steps);
    if (large <= middle && large <= flat && large <= small) return launch_grad_of<T, O, Shape256, true, true, RESTS>(a, stream);
    if (flat <= middle && flat <= small) return launch_grad_of<T, O, ShapeFlat, true, true, RESTS>(a, stream);
    return middle <= small ? launch_grad_of<T, O, Shape128, true, true, RESTS>(a, stream) : launch_grad_of<T, O, Shape64, true, true, RESTS>(a, stream);
}
template <typename T, typename O>
int launch_grad_weight(const GradArgs &a, hipStream_t stream) {
    if constexpr (std::is_same_v<O, Fp16>)
        if (a.first) return launch_grad_weight_of<T, O, true>(a, stream);
    return launch_grad_weight_of<T, O, false>(a, stream);
}

int copy_rows(const LossCall &c, int32_t times, int32_t all, bool whole, const Rows &rows, uint16_t *y, int32_t y_ld,
              hipStream_t stream) {
    const int64_t units = (int64_t)(c.N + all - c.N * times) * (y_ld / 8);
    hipLaunchKernelGGL(copy_rows_kernel, dim3((uint32_t)ceil_div(units, 256)), dim3(256), 0, stream,
                       static_cast<const uint16_t *>(c.hidden), c.hidden_stride, c.N, c.D, times, all, whole, rows, y, y_ld);
    return check_launch();
}

int join(const f32x2 *parts, int32_t count, const LossCall &c, const Masks &masks, const float *z_target, float *loss, float *lse,
         f32x2 *whole, hipStream_t stream) {
    if (c.N <= 64)
        hipLaunchKernelGGL(join_kernel<1>, dim3(c.N), dim3(1024), 0, stream, parts, count, c.N, c.V, masks, c.target, z_target, loss, lse,
                           whole);
    else
        hipLaunchKernelGGL(join_kernel<16>, dim3((uint32_t)ceil_div(c.N, 16)), dim3(1024), 0, stream, parts, count, c.N, c.V, masks,
                           c.target, z_target, loss, lse, whole);
    return check_launch();
}

int32_t part_count(int rows, int32_t V) {  // one from each wave along the tokens
    const int waves = rows == 16 || rows == 64 || rows == 128 ? 4 : 2;
    return (int32_t)ceil_div(V, columns_of_tile(rows)) * waves;
}

template <typename T>
int forward(const LossCall &c, float *loss, float *lse, Carver &ws, hipStream_t stream, bool launch) {
    const int rows = rows_of_tile(c.N);
    const int32_t d_pad = (int32_t)pad(c.D, kStepK), parts = part_count(rows, c.V);
    LogitsArgs a{};
    CFGZIP_TRY(masks_of(c, ws, stream, a.masks, launch));
    a.parts = ws.take<f32x2>((size_t)parts * c.N);
    a.z_target = ws.take<float>(c.N);
    uint16_t *copy = ws.take<uint16_t>((size_t)c.N * d_pad);
    if (!launch) return CFGZIP_OK;
    const bool as_it_is = whole_units(c.hidden, c.hidden_stride, c.D) && c.D % kStepK == 0 && c.hidden_stride < kMaxStride;
    if (!as_it_is) CFGZIP_TRY(copy_rows(c, 1, c.N, true, Rows{}, copy, d_pad, stream));
    a.W = by_rows(static_cast<const uint16_t *>(c.weight), c.weight_stride, c.V);
    a.H = as_it_is ? by_rows(static_cast<const uint16_t *>(c.hidden), c.hidden_stride, c.N) : by_rows(copy, d_pad, c.N);
    a.V = c.V;
    a.N = c.N;
    a.D = c.D;
    a.target = c.target;
    CFGZIP_TRY((launch_logits<T, STATISTICS>(rows, a, c.V, whole_units(c.weight, c.weight_stride, c.D), stream)));
    return join(a.parts, parts, c, a.masks, a.z_target, loss, lse, nullptr, stream);
}

template <typename T>
int backward(const LossCall &c, const float *lse, const float *grad_loss, uint16_t *grad_hidden, int64_t gh_stride,
             uint16_t *grad_weight, int64_t gw_stride, Carver &ws, hipStream_t stream, bool launch) {
    const Plan p = plan_of(c.N, c.V, c.D, few_rows_of<T>(c.D), std::is_same_v<T, Bf16>);
    Masks masks;
    CFGZIP_TRY(masks_of(c, ws, stream, masks, launch));
    const bool few = p.parts == 2;
    // Of many rows dz is one fp16 number, whose eleven bits leave bf16 gradients as near to the truth as their own rounding does (in bf16
    // dz's largest element, the target's, was off by as much as all of that); of fp16 ones the target's element is kept whole.  The
    // products' other sides, where they are bf16, become fp16 too.
    constexpr bool kBf16 = std::is_same_v<T, Bf16>;
    const bool halves = kBf16 && !few, fp16_dz = !kBf16 || !few;
    const int32_t rows_dz = c.N * p.parts, count = part_count(p.logits_rows, c.V);
    float *unscale = ws.take<float>(1);  // of dz in two bf16 numbers
    RowFactors of_rows{};                // of dz in fp16
    int32_t *back = ws.take<int32_t>(2);  // of weights in fp16; of hidden states times their rows' factors
    int32_t *largest_w = ws.take<int32_t>(kWeightBlocks), *largest_h = ws.take<int32_t>(kRowBlocks);
    Rests rests{};                       // of dz in one number for fp16
    if (fp16_dz) {
        of_rows.dz = ws.take<float>(c.N);
        of_rows.power = ws.take<int32_t>(c.N);
        if (!few) of_rows.common = ws.take<float>(2);
        if (!few && !kBf16) {
            rests.rest = ws.take<float>(c.N);
            rests.first = ws.take<int32_t>(c.V);
            rests.count = ws.take<int32_t>(c.V);
            rests.ld = p.d_pad;
            rests.sums = ws.take<float>((size_t)(c.N + 1) * p.d_pad);
        }
    }
    const int32_t copy_rows_pad = (int32_t)pad(rows_dz, kStepK), w_pad = (int32_t)pad(c.D, 8);
    // hidden states, 0 where a row has no gradient: for the logits, and for grad_weight as dz needs them
    uint16_t *copy = ws.take<uint16_t>((size_t)(fp16_dz ? c.N : copy_rows_pad) * p.d_pad);
    uint16_t *copy16 = fp16_dz ? ws.take<uint16_t>((size_t)copy_rows_pad * p.d_pad) : copy;
    uint16_t *weight16 = halves ? ws.take<uint16_t>((size_t)std::min(p.piece, c.V) * w_pad) : nullptr;
    uint16_t *dz = ws.take<uint16_t>((size_t)p.rows_pad * p.piece);
    float *sums = ws.take<float>((size_t)p.splits * rows_dz * p.sums_ld);
    float *z = few ? ws.take<float>((size_t)c.N * p.piece) : nullptr;
    f32x2 *parts = few ? ws.take<f32x2>((size_t)count * c.N) : nullptr, *whole = few ? ws.take<f32x2>(c.N) : nullptr;
    if (!launch) return CFGZIP_OK;
    const Rows rows{grad_loss, c.target, c.N, c.V, masks};
    auto to_halves = [&](const Matrix16 &x, const int32_t *powers, const int32_t *most, int32_t many, int32_t times, uint16_t *y, int32_t y_ld,
                         int32_t all, int32_t *to) {
        hipLaunchKernelGGL(halves_kernel<T>, dim3((uint32_t)ceil_div((int64_t)all * (y_ld / 8), 1024)), dim3(256), 0, stream, x, powers,
                           most, many, times, y, y_ld, all, to);
        return check_launch();
    };
    if (fp16_dz) {
        const int32_t blocks = std::min((int32_t)ceil_div(c.N, kRowsOfBlock), kRowBlocks);
        hipLaunchKernelGGL(rows_kernel<T>, dim3(blocks + 1), dim3(kRowsOfBlock * kWave), 0, stream, rows,
                           static_cast<const uint16_t *>(c.hidden), c.hidden_stride, c.D, copy, p.d_pad, of_rows, rests, largest_h);
        CFGZIP_TRY(check_launch());
        if (grad_weight)
            CFGZIP_TRY(to_halves(Matrix16{copy, p.d_pad, c.N, c.D}, of_rows.power, largest_h, blocks, p.parts, copy16, p.d_pad, copy_rows_pad,
                                 back + 1));
    } else {
        CFGZIP_TRY(copy_rows(c, p.parts, copy_rows_pad, false, rows, copy, p.d_pad, stream));
    }
    if (halves && grad_hidden) {
        hipLaunchKernelGGL(largest_kernel, dim3(kWeightBlocks), dim3(256), 0, stream,
                           Matrix16{static_cast<const uint16_t *>(c.weight), c.weight_stride, c.V, c.D}, largest_w);
        CFGZIP_TRY(check_launch());
    }
    const float *const all = !fp16_dz ? unscale : few ? nullptr : of_rows.common + 1;
    const Factors factors_h{all, of_rows.power, halves ? back : nullptr}, factors_w{all, nullptr, fp16_dz ? back + 1 : nullptr};
    const uint16_t *weight = static_cast<const uint16_t *>(c.weight);
    const bool direct = whole_units(c.weight, c.weight_stride, c.D);
    for (int64_t v0 = 0; v0 < c.V; v0 += p.piece) {
        const int32_t tokens = (int32_t)(c.V - v0 < p.piece ? c.V - v0 : p.piece);
        const uint16_t *const first = weight + v0 * c.weight_stride;
        LogitsArgs a{};
        a.W = by_rows(first, c.weight_stride, tokens);
        a.H = by_rows(copy, p.d_pad, c.N);
        a.V = c.V;
        a.N = c.N;
        a.D = c.D;
        a.v0 = (int32_t)v0;
        a.masks = masks;
        a.target = c.target;
        a.lse = lse;
        a.factor = of_rows.dz;
        a.common = of_rows.common;
        a.rests = rests;
        a.dz = dz;
        a.dz_rows = p.rows_pad;
        a.parts = parts;
        a.z = z;
        if (few) {
            CFGZIP_TRY((launch_logits<T, KEPT>(p.logits_rows, a, tokens, direct, stream)));
            CFGZIP_TRY(join(parts, count, c, masks, nullptr, nullptr, const_cast<float *>(lse), whole, stream));
            const int32_t blocks = (int32_t)(pad(tokens, 64) / 64);
            const int64_t threads = (int64_t)blocks * (p.rows_pad - c.N) * 16;
            hipLaunchKernelGGL((few_rows_dz_kernel<T>), dim3((uint32_t)ceil_div(threads, 256)), dim3(256), 0, stream, rows, z, blocks, whole,
                               dz, p.rows_pad, of_rows.dz, unscale);
            CFGZIP_TRY(check_launch());
        } else {
            CFGZIP_TRY((launch_logits<T, GRADIENT>(p.logits_rows, a, tokens, direct, stream)));
        }
        if (grad_hidden) {
            GradArgs g{};
            g.A = halves ? by_columns(weight16, w_pad, w_pad) : by_columns(first, c.weight_stride, c.D);
            g.B = Operand{dz, 64, 64, (int64_t)p.rows_pad * 64, p.rows_pad};
            g.n = rows_dz;
            g.D = c.D;
            g.k = tokens;
            g.k_split = (int32_t)pad(ceil_div(tokens, p.splits), kStepK);
            g.factors = factors_h;
            g.out = grad_hidden;
            g.out_ld = gh_stride;
            g.sums = p.direct_out ? nullptr : sums;
            g.sums_ld = p.sums_ld;
            g.add = v0 > 0;
            g.splits = (int32_t)ceil_div(tokens, g.k_split);
            if (halves) {
                const Matrix16 w{first, c.weight_stride, tokens, c.D};
                CFGZIP_TRY(to_halves(w, nullptr, largest_w, kWeightBlocks, 1, weight16, w_pad, tokens, back));
                CFGZIP_TRY((launch_grad_hidden<Fp16, T, true>(p.rows, g, stream)));
            } else {
                CFGZIP_TRY(direct ? (launch_grad_hidden<T, T, true>(p.rows, g, stream))
                                  : (launch_grad_hidden<T, T, false>(p.rows, g, stream)));
            }
        }
        if (grad_weight) {
            GradArgs g{};
            g.A = by_columns(copy16, p.d_pad, p.d_pad);
            g.B = Operand{dz, 64, (int64_t)p.rows_pad * 64, kStepK * 64, p.piece};
            g.n = tokens;
            g.D = c.D;
            g.k = rows_dz;
            g.k_split = (int32_t)pad(rows_dz, kStepK);
            g.splits = 1;
            g.factors = factors_w;
            if (rests.rest) {
                hipLaunchKernelGGL(rests_kernel, dim3(c.N, (uint32_t)ceil_div(p.d_pad, 1024)), dim3(256), 0, stream, of_rows, rests, c.target,
                                   c.N, v0, tokens, copy16);
                CFGZIP_TRY(check_launch());
                g.first = rests.first + v0;
                g.rests = rests.sums;
                g.rests_ld = rests.ld;
                g.rests_rows = c.N;
            }
            g.out = grad_weight + v0 * gw_stride;
            g.out_ld = gw_stride;
            CFGZIP_TRY(halves ? (launch_grad_weight<Fp16, T>(g, stream)) : (launch_grad_weight<T, T>(g, stream)));
        }
    }
    if (grad_hidden && !p.direct_out) {
        const int64_t units = (int64_t)c.N * (p.sums_ld / 4);
        hipLaunchKernelGGL((finish_kernel<T>), dim3((uint32_t)ceil_div(units, kWave)), dim3(kWave), 0, stream, sums, p.splits * p.parts, c.N,
                           c.D, p.sums_ld, factors_h, rests.rest, c.target, weight, c.weight_stride, grad_hidden, gh_stride);
        CFGZIP_TRY(check_launch());
    }
    return CFGZIP_OK;
}

}  // namespace
}  // namespace cfgzip

using namespace cfgzip;

extern "C" size_t cfgzip_head_loss_workspace_bytes(int32_t N, int32_t V, int32_t D, int32_t bits_kind) {
    if (N <= 0 || V <= 0 || D <= 0 || N > kMaxRows || V > 0x7FFFFC00 || D >= kMaxStride - 8 || !kind_ok(bits_kind)) return 0;
    LossCall c{};
    c.N = N, c.V = V, c.D = D, c.bits_kind = bits_kind;
    Carver ws(nullptr);
    forward<Bf16>(c, nullptr, nullptr, ws, nullptr, false);
    return ws.used;
}

extern "C" size_t cfgzip_head_loss_grad_workspace_bytes(int32_t N, int32_t V, int32_t D, int32_t bits_kind) {
    if (N <= 0 || V <= 0 || D <= 0 || N > kMaxRows || V > 0x7FFFFC00 || D >= kMaxStride - 8 || !kind_ok(bits_kind)) return 0;
    LossCall c{};
    c.N = N, c.V = V, c.D = D, c.bits_kind = bits_kind;
    Carver bf16(nullptr), fp16(nullptr);  // (the call's type is not asked for: the larger)
    backward<Bf16>(c, nullptr, nullptr, nullptr, 0, nullptr, 0, bf16, nullptr, false);
    backward<Fp16>(c, nullptr, nullptr, nullptr, 0, nullptr, 0, fp16, nullptr, false);
    return std::max(bf16.used, fp16.used);
}

extern "C" int cfgzip_head_loss(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                                int32_t dtype, int32_t N, int32_t V, int32_t D, const int32_t *target, const int32_t *bits,
                                int32_t bits_kind, const int32_t *class_of_token, int32_t C, float *loss, float *lse, void *ws,
                                size_t ws_bytes, void *stream) {
    const LossCall c{hidden, hidden_stride, weight, weight_stride, dtype, N, V, D, target, bits, bits_kind, class_of_token, C};
    CFGZIP_TRY(check_call(c));
    if (N == 0) return CFGZIP_OK;
    if (!loss || !lse || !aligned_to(loss, 4) || !aligned_to(lse, 4)) return CFGZIP_E_INVALID;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cfgzip_head_loss_workspace_bytes(N, V, D, bits_kind)) return CFGZIP_E_WORKSPACE;
    Carver carve(ws);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == CFGZIP_DTYPE_BF16 ? forward<Bf16>(c, loss, lse, carve, s, true) : forward<Fp16>(c, loss, lse, carve, s, true);
}

extern "C" int cfgzip_head_loss_grad(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                                     int32_t dtype, int32_t N, int32_t V, int32_t D, const int32_t *target, const int32_t *bits,
                                     int32_t bits_kind, const int32_t *class_of_token, int32_t C, const float *lse,
                                     const float *grad_loss, void *grad_hidden, int64_t grad_hidden_stride, void *grad_weight,
                                     int64_t grad_weight_stride, void *ws, size_t ws_bytes, void *stream) {
    const LossCall c{hidden, hidden_stride, weight, weight_stride, dtype, N, V, D, target, bits, bits_kind, class_of_token, C};
    CFGZIP_TRY(check_call(c));
    if (grad_hidden && (!aligned_to(grad_hidden, 2) || grad_hidden_stride < D)) return CFGZIP_E_INVALID;
    if (grad_weight && (!aligned_to(grad_weight, 2) || grad_weight_stride < D)) return CFGZIP_E_INVALID;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (N == 0) {
        if (!grad_weight) return CFGZIP_OK;
        hipLaunchKernelGGL(zero_rows_kernel, dim3(V < 4096 ? V : 4096), dim3(256), 0, s, static_cast<uint16_t *>(grad_weight),
                           grad_weight_stride, V, D);
        return check_launch();
    }
    if ((!grad_hidden && !grad_weight) || !lse || !grad_loss || !aligned_to(lse, 4) || !aligned_to(grad_loss, 4))
        return CFGZIP_E_INVALID;
    if (!ws || !aligned_to(ws, 256) || ws_bytes < cfgzip_head_loss_grad_workspace_bytes(N, V, D, bits_kind))
        return CFGZIP_E_WORKSPACE;
    Carver carve(ws);
    uint16_t *gh = static_cast<uint16_t *>(grad_hidden), *gw = static_cast<uint16_t *>(grad_weight);
    return dtype == CFGZIP_DTYPE_BF16
               ? backward<Bf16>(c, lse, grad_loss, gh, grad_hidden_stride, gw, grad_weight_stride, carve, s, true)
               : backward<Fp16>(c, lse, grad_loss, gh, grad_hidden_stride, gw, grad_weight_stride, carve, s, true);
}
