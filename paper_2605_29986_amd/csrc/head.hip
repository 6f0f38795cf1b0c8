// The vocabulary projection's loss under a grammar's masks, and its gradients, without the logits in memory.
//
//     z[i][v] = sum_d hidden[i][d] weight[v][d]
//     lse[i] = log sum over admitted v of exp z[i][v],   loss[i] = lse[i] - z[i][target[i]]
//     dz[i][v] = grad_loss[i] (exp(z[i][v] - lse[i]) - [v = target[i]]) for admitted v
//     grad_hidden = dz weight,   grad_weight = dz^T hidden
//
// Forward: a tile of logits stays in the accumulators of the product that makes it; each wave leaves the maximum of its part of
// every row and the sum of exponentials against that maximum, and a second kernel joins them.  Backward: the logits are made
// again, for a piece of the vocabulary at a time, turned into dz in the accumulators, and stored in 16 bits; the two products
// that read the piece follow while it is in the last-level cache.  All sums are fp32.

#include "gemm16.hpp"

namespace cfgzip {
namespace {

using Shape16 = Shape<64, 16, 4, 1>;     // few rows: reading the weights is what counts, many small workgroups
using Shape64 = Shape<128, 64, 4, 1>;
using Shape128 = Shape<256, 128, 4, 2>;
using Shape256 = Shape<256, 256, 2, 4>;
using ShapeFlat = Shape<128, 256, 2, 4>;  // weight gradients of small hidden sizes

constexpr size_t kPieceBytes = (size_t)256 << 20;  // of dz in memory at a time: the size of the last-level cache
constexpr int32_t kPieceLeast = 2048;              // columns
constexpr float kInf = __builtin_inff();

struct Masks {
    const int32_t *bits;  // [N][words], over tokens; null: every token is admitted
    int64_t words;
};

// bit r: whether token v + r is admitted, for the four tokens from v on (v a multiple of 4)
__device__ __forceinline__ uint32_t admitted4(const Masks &m, uint32_t word, int32_t v, int32_t V) {
    const int32_t left = V - v;
    const uint32_t there = left >= 4 ? 15u : left <= 0 ? 0u : (1u << left) - 1u;
    return m.bits ? (word >> (v & 31)) & there : there;
}

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
    const float *scaled_grad;  // 0: the row has no gradient
    uint16_t *dz;              // [rows][ld]
    int64_t dz_ld;
};

enum : int { STATISTICS = 0, GRADIENT = 1 };

template <typename T, typename S, bool DIRECT, int WHAT>
__global__ __launch_bounds__(S::kThreads) void logits_kernel(LogitsArgs a) {
    using TileA = Tile<S::BM, S::kThreads, false, DIRECT>;
    using TileB = Tile<S::BN, S::kThreads, false, true>;
    __shared__ __attribute__((aligned(16))) char lds0[S::kLds], lds1[S::kLds];
    int32_t tm, tn;
    tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
    f32x4 acc[S::FM][S::FN];
    multiply<T, S, TileA, TileB>(a.W, a.H, tm * S::BM, tn * S::BN, 0, a.D, lds0, lds1, acc);

    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wm = wave / S::WN, wn = wave % S::WN, g = lane >> 4;
    const int32_t first = tm * S::BM + wm * S::TM;  // in the piece
    const int32_t v_first = a.v0 + first;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int32_t row = tn * S::BN + wn * S::TN + 16 * j + (lane & 15);
        const bool in = row < a.N;
        const int32_t at = in ? row : a.N - 1;
        const int32_t target = a.target[at];
        uint32_t words[(S::TM + 31) / 32] = {};
        if (a.masks.bits) {
#pragma unroll
            for (int w = 0; w < (S::TM + 31) / 32; ++w) {
                const int64_t k = (v_first >> 5) + w;
                words[w] = k < a.masks.words ? (uint32_t)a.masks.bits[at * a.masks.words + k] : 0u;
            }
        }
        if constexpr (WHAT == STATISTICS) {
            float most = -kInf;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int32_t v = v_first + 16 * i + 4 * g;
                const uint32_t ok = admitted4(a.masks, words[i / 2], v, a.V);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (ok >> r & 1) most = fmaxf(most, acc[i][j][r]);
                    if (in && v + r == target) a.z_target[row] = acc[i][j][r];
                }
            }
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const float shift = most == -kInf ? 0.0f : most;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const uint32_t ok = admitted4(a.masks, words[i / 2], v_first + 16 * i + 4 * g, a.V);
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += ok >> r & 1 ? __expf(acc[i][j][r] - shift) : 0.0f;
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (g == 0 && in) a.parts[(int64_t)(tm * S::WM + wm) * a.N + row] = f32x2{most, sum};
        } else {
            const float lse = a.lse[at], grad = in ? a.scaled_grad[at] : 0.0f;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int32_t v = v_first + 16 * i + 4 * g;
                const uint32_t ok = grad != 0.0f ? admitted4(a.masks, words[i / 2], v, a.V) : 0u;
                f32x4 d;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __expf(acc[i][j][r] - lse) - (v + r == target ? 1.0f : 0.0f);
                    d[r] = ok >> r & 1 ? p * grad : 0.0f;
                }
                *reinterpret_cast<u32x2 *>(a.dz + row * a.dz_ld + first + 16 * i + 4 * g) = round4<T>(d);
            }
        }
    }
}

// Joins the parts of 16 rows: lse and loss.
__global__ __launch_bounds__(256) void join_kernel(const f32x2 *parts, int32_t count, int32_t N, int32_t V, Masks masks,
                                                   const int32_t *target, const float *z_target, float *loss, float *lse) {
    __shared__ f32x2 shared[16][17];
    const int r = threadIdx.x & 15, s = threadIdx.x >> 4;
    const int32_t row = blockIdx.x * 16 + r;
    float most = -kInf, sum = 0.0f;
    auto take = [&](f32x2 p) {
        const float m = fmaxf(most, p[0]);
        // a part without admitted tokens has the maximum -inf and the sum 0 (or NaN, of logits that are)
        sum = (most == -kInf ? sum : sum * __expf(most - m)) + (p[0] == -kInf ? p[1] : p[1] * __expf(p[0] - m));
        most = m;
    };
    if (row < N)
        for (int32_t p = s; p < count; p += 16) take(parts[(int64_t)p * N + row]);
    shared[s][r] = f32x2{most, sum};
    __syncthreads();
    if (s != 0 || row >= N) return;
    for (int p = 1; p < 16; ++p) take(shared[p][r]);
    const float l = (most == -kInf ? 0.0f : most) + logf(sum);
    const int32_t t = target[row];
    float out = 0.0f;
    if (t >= 0 && t < V) {
        const bool ok = !masks.bits || (masks.bits[row * masks.words + (t >> 5)] >> (t & 31) & 1);
        out = ok ? l - z_target[row] : kInf;
    }
    lse[row] = l;
    loss[row] = out;
}

// The rows' gradients times a power of two that brings the largest to at most 2^14, so that dz fills the range of fp16 (bf16
// would not need it), and 2 to minus that; 0 for rows whose target is none or not admitted.  One workgroup.
__global__ __launch_bounds__(1024) void rows_kernel(const float *grad_loss, const int32_t *target, int32_t N, int32_t V, Masks masks,
                                                    float *scaled, float *unscale) {
    __shared__ float shared[16];
    auto grad_of = [&](int32_t i) {
        const int32_t t = target[i];
        if (t < 0 || t >= V) return 0.0f;
        if (masks.bits && !(masks.bits[i * masks.words + (t >> 5)] >> (t & 31) & 1)) return 0.0f;
        return grad_loss[i];
    };
    float most = 0.0f;
    for (int32_t i = threadIdx.x; i < N; i += 1024) {
        const float x = fabsf(grad_of(i));
        if (x < kInf) most = fmaxf(most, x);
    }
    for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = most;
    __syncthreads();
    for (int i = 0; i < 16; ++i) most = fmaxf(most, shared[i]);
    int e = 0;
    if (most > 0.0f) {
        frexpf(most, &e);  // most < 2^e
        e = 14 - e;
        e = e > 100 ? 100 : e < -100 ? -100 : e;
    }
    for (int32_t i = threadIdx.x; i < N; i += 1024) scaled[i] = ldexpf(grad_of(i), e);
    if (threadIdx.x == 0) *unscale = ldexpf(1.0f, -e);
}

// hidden states in rows of whole units of 8 elements; zeros in rows that have no gradient (`scaled`, or null), whatever they hold
__global__ __launch_bounds__(256) void copy_rows_kernel(const uint16_t *x, int64_t x_ld, int32_t N, int32_t D, const float *scaled,
                                                        uint16_t *y, int32_t y_ld) {
    const int32_t units = y_ld / 8;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= (int64_t)N * units) return;
    const int32_t row = (int32_t)(k / units), c = (int32_t)(k % units) * 8;
    u32x4 v = {0, 0, 0, 0};
    if (!scaled || scaled[row] != 0.0f) {
        const uint16_t *p = x + row * x_ld + c;
        if (c + 8 <= D) {
            v = *reinterpret_cast<const u32x4_any *>(p);
        } else {
            for (int j = 0; c + j < D; ++j) v[j / 2] |= (uint32_t)p[j] << (j % 2 * 16);
        }
    }
    *reinterpret_cast<u32x4 *>(y + (int64_t)row * y_ld + c) = v;
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

struct GradArgs {
    Operand A, B;  // A: m = hidden size; B: n = rows (grad_hidden) or tokens (grad_weight)
    int32_t n, D;  // extents of the result
    int32_t k, k_split;
    int32_t tiles_m, tiles_n;
    const float *unscale;
    uint16_t *out;  // [n][out_ld]
    int64_t out_ld;
    float *sums;  // [splits][n][sums_ld], sums_ld = D rounded up to 4; null: the result goes to `out` at once
    int32_t sums_ld;
    int32_t add;  // to what is in `sums`
};

// grad_hidden: A = weight by columns, B = dz by rows.  grad_weight: A = hidden, B = dz, both by columns.
template <typename T, typename S, bool DIRECT, bool B_COLUMNS>
__global__ __launch_bounds__(S::kThreads) void grad_kernel(GradArgs a) {
    using TileA = Tile<S::BM, S::kThreads, true, DIRECT>;
    using TileB = Tile<S::BN, S::kThreads, B_COLUMNS, true>;
    __shared__ __attribute__((aligned(16))) char lds0[S::kLds], lds1[S::kLds];
    int32_t tm, tn;
    tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
    const int32_t k0 = blockIdx.y * a.k_split, k1 = k0 + a.k_split < a.k ? k0 + a.k_split : a.k;
    f32x4 acc[S::FM][S::FN];
    multiply<T, S, TileA, TileB>(a.A, a.B, tm * S::BM, tn * S::BN, k0, k1, lds0, lds1, acc);

    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wm = wave / S::WN, wn = wave % S::WN;
    const float unscale = *a.unscale;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int32_t n = tn * S::BN + wn * S::TN + 16 * j + (lane & 15);
        if (n >= a.n) continue;
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            const int32_t c = tm * S::BM + wm * S::TM + 16 * i + 4 * (lane >> 4);
            if (c >= a.D) continue;
            if (a.sums) {
                f32x4 *p = reinterpret_cast<f32x4 *>(a.sums + ((int64_t)blockIdx.y * a.n + n) * a.sums_ld + c);
                *p = a.add ? *p + acc[i][j] : acc[i][j];
            } else {
                store4<T>(a.out + n * a.out_ld, c, a.D, acc[i][j] * unscale);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void finish_kernel(const float *sums, int32_t splits, int32_t n, int32_t D, int32_t sums_ld,
                                                     const float *unscale, uint16_t *out, int64_t out_ld) {
    const int32_t units = sums_ld / 4;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= (int64_t)n * units) return;
    const int32_t row = (int32_t)(k / units), c = (int32_t)(k % units) * 4;
    f32x4 x = {0, 0, 0, 0};
    for (int32_t s = 0; s < splits; ++s) x += *reinterpret_cast<const f32x4 *>(sums + ((int64_t)s * n + row) * sums_ld + c);
    store4<T>(out + row * out_ld, c, D, x * *unscale);
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
    int rows;           // of a tile
    int32_t rows_pad;   // N in whole tiles
    int32_t d_pad;      // hidden size in units of 8
    int32_t piece;      // tokens of a piece of dz
    int32_t splits, k_split;
    int32_t sums_ld;
    bool direct_out;    // grad_hidden in one go
};

Plan plan_of(int32_t N, int32_t V, int32_t D) {
    Plan p{};
    p.rows = rows_of_tile(N);
    p.rows_pad = (int32_t)pad(N, p.rows);
    p.d_pad = (int32_t)pad(D, 8);
    int64_t most = (int64_t)(kPieceBytes / 2 / p.rows_pad) / 256 * 256;
    if (most < kPieceLeast) most = kPieceLeast;
    const int64_t pieces = ceil_div(V, most);
    p.piece = (int32_t)pad(ceil_div(V, pieces), 256);
    // grad_hidden's sum runs over the vocabulary: it is split so that its tiles fill the chip
    const int64_t tiles = ceil_div(D, columns_of_tile(p.rows)) * ceil_div(N, p.rows);
    const int64_t at_a_time = p.rows == 256 ? 256 : p.rows == 128 ? 256 : p.rows == 64 ? 768 : 1024;
    int64_t best = 1;
    double best_use = 0;
    for (int64_t s = 1; s <= 1024 && s * 256 <= p.piece; ++s) {
        const int64_t rounds = ceil_div(tiles * s, at_a_time);
        const double use = (double)(tiles * s) / (double)(rounds * at_a_time);
        if (use > best_use + 0.05) {
            best_use = use;
            best = s;
        }
        if (tiles * s >= at_a_time * 2) break;
    }
    p.k_split = (int32_t)pad(ceil_div(p.piece, best), kStepK);
    p.splits = (int32_t)ceil_div(p.piece, p.k_split);
    p.sums_ld = (int32_t)pad(D, 4);
    p.direct_out = pieces == 1 && p.splits == 1;
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
    if (c.V > 0x7FFFFC00 || c.N > 0x7FFFFC00) return CFGZIP_E_TOO_LARGE;
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
    const int64_t grid = (int64_t)a.tiles_m * a.tiles_n;
    if (grid > 0x7FFFFFFF) return CFGZIP_E_TOO_LARGE;
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
        default: return launch_logits_of<T, Shape256, WHAT>(a, direct, stream);
    }
}

template <typename T, typename S, bool DIRECT, bool B_COLUMNS>
int launch_grad_of(GradArgs a, int32_t splits, hipStream_t stream) {
    a.tiles_m = (int32_t)ceil_div(a.D, S::BM);
    a.tiles_n = (int32_t)ceil_div(a.n, S::BN);
    const int64_t grid = (int64_t)a.tiles_m * a.tiles_n;
    if (grid > 0x7FFFFFFF) return CFGZIP_E_TOO_LARGE;
    hipLaunchKernelGGL((grad_kernel<T, S, DIRECT, B_COLUMNS>), dim3((uint32_t)grid, splits), dim3(S::kThreads), 0, stream, a);
    return check_launch();
}

template <typename T, bool DIRECT>
int launch_grad_hidden(int rows, const GradArgs &a, int32_t splits, hipStream_t stream) {
    switch (rows) {
        case 16: return launch_grad_of<T, Shape16, DIRECT, false>(a, splits, stream);
        case 64: return launch_grad_of<T, Shape64, DIRECT, false>(a, splits, stream);
        case 128: return launch_grad_of<T, Shape128, DIRECT, false>(a, splits, stream);
        default: return launch_grad_of<T, Shape256, DIRECT, false>(a, splits, stream);
    }
}

template <typename T>
int copy_rows(const LossCall &c, const float *scaled, uint16_t *y, int32_t y_ld, hipStream_t stream) {
    const int64_t units = (int64_t)c.N * (y_ld / 8);
    hipLaunchKernelGGL(copy_rows_kernel, dim3((uint32_t)ceil_div(units, 256)), dim3(256), 0, stream,
                       static_cast<const uint16_t *>(c.hidden), c.hidden_stride, c.N, c.D, scaled, y, y_ld);
    return check_launch();
}

int32_t part_count(int rows, int32_t V) {  // one from each wave along the tokens
    const int waves = rows == 16 || rows == 64 || rows == 128 ? 4 : 2;
    return (int32_t)ceil_div(V, columns_of_tile(rows)) * waves;
}

template <typename T>
int forward(const LossCall &c, float *loss, float *lse, Carver &ws, hipStream_t stream, bool launch) {
    const int rows = rows_of_tile(c.N);
    const int32_t d_pad = (int32_t)pad(c.D, 8), parts = part_count(rows, c.V);
    LogitsArgs a{};
    CFGZIP_TRY(masks_of(c, ws, stream, a.masks, launch));
    a.parts = ws.take<f32x2>((size_t)parts * c.N);
    a.z_target = ws.take<float>(c.N);
    uint16_t *copy = ws.take<uint16_t>((size_t)c.N * d_pad);
    if (!launch) return CFGZIP_OK;
    const bool as_it_is = whole_units(c.hidden, c.hidden_stride, c.D) && c.hidden_stride < kMaxStride;
    if (!as_it_is) CFGZIP_TRY(copy_rows<T>(c, nullptr, copy, d_pad, stream));
    a.W = Operand{static_cast<const uint16_t *>(c.weight), c.weight_stride, c.V, c.D};
    a.H = as_it_is ? Operand{static_cast<const uint16_t *>(c.hidden), c.hidden_stride, c.N, c.D}
                   : Operand{copy, d_pad, c.N, d_pad};
    a.V = c.V;
    a.N = c.N;
    a.D = c.D;
    a.target = c.target;
    CFGZIP_TRY((launch_logits<T, STATISTICS>(rows, a, c.V, whole_units(c.weight, c.weight_stride, c.D), stream)));
    hipLaunchKernelGGL(join_kernel, dim3((uint32_t)ceil_div(c.N, 16)), dim3(256), 0, stream, a.parts, parts, c.N, c.V, a.masks,
                       c.target, a.z_target, loss, lse);
    return check_launch();
}

template <typename T>
int backward(const LossCall &c, const float *lse, const float *grad_loss, uint16_t *grad_hidden, int64_t gh_stride,
             uint16_t *grad_weight, int64_t gw_stride, Carver &ws, hipStream_t stream, bool launch) {
    const Plan p = plan_of(c.N, c.V, c.D);
    Masks masks;
    CFGZIP_TRY(masks_of(c, ws, stream, masks, launch));
    float *unscale = ws.take<float>(1);
    float *scaled = ws.take<float>(c.N);
    uint16_t *copy = ws.take<uint16_t>((size_t)c.N * p.d_pad);
    uint16_t *dz = ws.take<uint16_t>((size_t)p.rows_pad * p.piece);
    float *sums = ws.take<float>((size_t)p.splits * c.N * p.sums_ld);
    if (!launch) return CFGZIP_OK;
    hipLaunchKernelGGL(rows_kernel, dim3(1), dim3(1024), 0, stream, grad_loss, c.target, c.N, c.V, masks, scaled, unscale);
    CFGZIP_TRY(check_launch());
    CFGZIP_TRY(copy_rows<T>(c, scaled, copy, p.d_pad, stream));
    const uint16_t *weight = static_cast<const uint16_t *>(c.weight);
    const bool direct = whole_units(c.weight, c.weight_stride, c.D);
    for (int64_t v0 = 0; v0 < c.V; v0 += p.piece) {
        const int32_t tokens = (int32_t)(c.V - v0 < p.piece ? c.V - v0 : p.piece);
        const Operand W{weight + v0 * c.weight_stride, c.weight_stride, tokens, c.D};
        LogitsArgs a{};
        a.W = W;
        a.H = Operand{copy, p.d_pad, c.N, p.d_pad};
        a.V = c.V;
        a.N = c.N;
        a.D = c.D;
        a.v0 = (int32_t)v0;
        a.masks = masks;
        a.target = c.target;
        a.lse = lse;
        a.scaled_grad = scaled;
        a.dz = dz;
        a.dz_ld = p.piece;
        CFGZIP_TRY((launch_logits<T, GRADIENT>(p.rows, a, tokens, direct, stream)));
        if (grad_hidden) {
            GradArgs g{};
            g.A = Operand{W.p, W.ld, c.D, tokens};  // by columns
            g.B = Operand{dz, p.piece, p.rows_pad, (int32_t)pad(tokens, 8)};
            g.n = c.N;
            g.D = c.D;
            g.k = tokens;
            g.k_split = p.k_split;
            g.unscale = unscale;
            g.out = grad_hidden;
            g.out_ld = gh_stride;
            g.sums = p.direct_out ? nullptr : sums;
            g.sums_ld = p.sums_ld;
            g.add = v0 > 0;
            const int32_t splits = (int32_t)ceil_div(tokens, p.k_split);
            CFGZIP_TRY(direct ? (launch_grad_hidden<T, true>(p.rows, g, splits, stream))
                              : (launch_grad_hidden<T, false>(p.rows, g, splits, stream)));
        }
        if (grad_weight) {
            GradArgs g{};
            g.A = Operand{copy, p.d_pad, p.d_pad, c.N};
            g.B = Operand{dz, p.piece, p.piece, c.N};
            g.n = tokens;
            g.D = c.D;
            g.k = c.N;
            g.k_split = (int32_t)pad(c.N, kStepK);
            g.unscale = unscale;
            g.out = grad_weight + v0 * gw_stride;
            g.out_ld = gw_stride;
            CFGZIP_TRY(c.D > 128 ? (launch_grad_of<T, Shape256, true, true>(g, 1, stream))
                                 : (launch_grad_of<T, ShapeFlat, true, true>(g, 1, stream)));
        }
    }
    if (grad_hidden && !p.direct_out) {
        const int64_t units = (int64_t)c.N * (p.sums_ld / 4);
        hipLaunchKernelGGL((finish_kernel<T>), dim3((uint32_t)ceil_div(units, 256)), dim3(256), 0, stream, sums, p.splits, c.N, c.D,
                           p.sums_ld, unscale, grad_hidden, gh_stride);
        CFGZIP_TRY(check_launch());
    }
    return CFGZIP_OK;
}

}  // namespace
}  // namespace cfgzip

using namespace cfgzip;

extern "C" size_t cfgzip_head_loss_workspace_bytes(int32_t N, int32_t V, int32_t D, int32_t bits_kind) {
    if (N <= 0 || V <= 0 || D <= 0 || N > 0x7FFFFC00 || V > 0x7FFFFC00 || D >= kMaxStride - 8 || !kind_ok(bits_kind)) return 0;
    LossCall c{};
    c.N = N, c.V = V, c.D = D, c.bits_kind = bits_kind;
    Carver ws(nullptr);
    forward<Bf16>(c, nullptr, nullptr, ws, nullptr, false);
    return ws.used;
}

extern "C" size_t cfgzip_head_loss_grad_workspace_bytes(int32_t N, int32_t V, int32_t D, int32_t bits_kind) {
    if (N <= 0 || V <= 0 || D <= 0 || N > 0x7FFFFC00 || V > 0x7FFFFC00 || D >= kMaxStride - 8 || !kind_ok(bits_kind)) return 0;
    LossCall c{};
    c.N = N, c.V = V, c.D = D, c.bits_kind = bits_kind;
    Carver ws(nullptr);
    backward<Bf16>(c, nullptr, nullptr, nullptr, 0, nullptr, 0, ws, nullptr, false);
    return ws.used;
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
