// Softmax cross entropy of a last dense layer over many classes, and its gradient, in pieces of the vocabulary.
//   1. logits' statistics: z = x W + b a tile at a time; a tile leaves, per row, its largest logit and the sum of exp of the
//      distances to it, the label's logit where the tile holds it, and z itself where it stays for step 3.
//   2. per row: the tiles' pairs joined to its max and sum; row losses max - z_label + log(sum), their mean and 1 / (labelled
//      rows).
//   3. for every piece of the vocabulary: z again, G = exp(z - max) / sum - onehot into a buffer of [rows][piece], then
//      dx += G W^T (shares of the contraction side by side, added in a fixed order) and dW = x^T G.  Where one piece holds the vocabulary, the
//      logits of step 1 stay for it: always with few rows, with more where forming them again costs more than their bytes (Plan::keep).
// A row without a label has G = 0 and its x is read as zeros.
#include <cmath>
#include <type_traits>

#include "direct_product.h"

namespace hadfl {
namespace head {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// exp of a number that is not positive, off by |t| / 2 units in the last place at most: what a rounding of t itself does
__device__ __forceinline__ float exp_down(float t) { return __builtin_amdgcn_exp2f(t * kLog2e); }

// whether z * log2(e) is a float for every logit z of a row up to its largest, but for those that exp makes zero: else the difference first
__device__ __forceinline__ bool folds(float largest) { return __builtin_fabsf(largest) <= 0x1p126f; }

// logits z of a wave's block of 32 rows (lanes along m), with the bias, -inf beyond the classes; n0: the first column's class
template <int TM, int TN>
__device__ __forceinline__ void logits_of(const Tile<TM, TN>& t, int i, int n0, int classes, const float* bias, float (&z)[TN][16])
{
    if (!bias && n0 + 32 * TN <= classes) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) z[j][e] = t.acc[i][j][e];
        return;
    }
    float b[TN][16] = {};
    if (bias) {                    // beyond the classes: the last one's, unused
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) b[j][e] = bias[min(n0 + 32 * j + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4, classes - 1)];
    }
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int c = n0 + 32 * j + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4;
            z[j][e] = c < classes ? t.acc[i][j][e] + b[j][e] : -INFINITY;
        }
}
// f(j, e) for the column of class y, in the lane that holds it; few waves hold any of their rows' labels
template <int TN, class F> __device__ __forceinline__ void at_label(int lane, int n0, int y, F&& f)
{
    if (!__any(y >= n0 && y < n0 + 32 * TN)) return;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (y == n0 + 32 * j + 8 * (e / 4) + 4 * (lane >> 5) + e % 4) f(j, e);
}

__device__ __forceinline__ void join(float2& have, const float2& v)
{
    const float top = fmaxf(have.x, v.x);
    if (top == -INFINITY) { have.y += v.y; return; }           // nothing yet: zero, or a NaN that stays
    have = float2{top, have.y * exp_down(have.x - top) + v.y * exp_down(v.x - top)};
}

// The statistics of a tile: per wave and row, then joined over the WN waves that share rows.  z: the logits too (few rows), or null.
// EXACT (32-bit operands): the distance to the largest first, then exp; else both in one multiply-add, off by 2^-24 |z| at most, which is far below
// what bf16 operands leave of z.  128 values a lane, some 3 us a tile that no product overlaps: 2 x 4096 x 2048 x 65536 bf16 1.85 ms with the
// product, 1190 TFLOP/s, the matrix cores busy 61 % of the time; 8 x 512 x 512 x 32000, where a tile's product is a quarter as long, 178 us, 755
// TFLOP/s, 43 %.
template <bool EXACT, int BM, int BN, int WN> struct Statistics {
    static constexpr bool kLaneM = true, kStaged = true, kSums = false;
    const float* bias;
    long long bias_rep;
    const int32_t* labels;
    float2* part;                  // [replicas][parts][rows]
    float* z_label;                // [replicas][rows]
    float* z;                      // [replicas][rows][ld]
    int rows, c0, classes, parts, ld;           // column 0 is class c0
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t, char* lds) const
    {
        const float* b = bias ? bias + t.rep * bias_rep : nullptr;
        const int n0 = c0 + t.n0;
        float2* got = (float2*)lds;                            // [WN][BM]
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = t.m0 + 32 * i + (t.lane & 31);
            const int y = m < rows ? labels[(long long)t.rep * rows + m] : -1;
            float v[TN][16], top = -INFINITY;
            logits_of(t, i, n0, classes, b, v);
            if (z && m < rows) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *(f4*)(z + ((long long)t.rep * rows + m) * ld + n0 + 32 * j + 8 * q + 4 * (t.lane >> 5)) =
                            f4{v[j][4 * q], v[j][4 * q + 1], v[j][4 * q + 2], v[j][4 * q + 3]};
            }
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = __builtin_fmaxf(top, v[j][e]);          // NaNs show in the sum
            at_label<TN>(t.lane, n0, y < classes ? y : -1, [&](int j, int e) { z_label[(long long)t.rep * rows + m] = v[j][e]; });
            top = __builtin_fmaxf(top, other<32>(top));
            float sum = 0.f;
            const float base = top == -INFINITY ? 0.f : top;   // a row of -inf alone: every term is zero
            if (EXACT || b || !folds(base)) {                  // the difference first: a bias may be the type's lowest value
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += exp_down(v[j][e] - base);
            } else {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(v[j][e], kLog2e, -base * kLog2e));
            }
            sum += other<32>(sum);
            if (t.lane < 32) got[(t.n0 - t.bn) / (32 * TN) * BM + m - t.bm] = float2{top, sum};
        }
        __syncthreads();
        const int m = t.bm + threadIdx.x;
        if (threadIdx.x >= BM || m >= rows) return;
        float2 have = got[threadIdx.x];
#pragma unroll
        for (int w = 1; w < WN; ++w) join(have, got[w * BM + threadIdx.x]);
        part[((long long)t.rep * parts + (c0 + t.bn) / BN) * rows + m] = have;
    }
};

// The pairs of a row's tiles joined: `shares` threads a row, each its tiles in ascending order, eight loads in flight; then the
// shares pairwise.  Where one workgroup has all rows of a replica it also takes their mean (loss, factor; else null).  Bound by latency: one row of
// 250 pairs 4.0 us, 128 rows of 79 pairs 4.9, 2 x 4096 rows of 256 pairs (17 MB) 7.4.
template <int NT> __device__ __forceinline__ void mean_of_rows(float sum, int count, float* sums, int* counts, float* loss, float* factor)
{
    __syncthreads();
    sums[threadIdx.x] = sum;
    counts[threadIdx.x] = count;
    for (int d = NT / 2; d > 0; d /= 2) {
        __syncthreads();
        if (threadIdx.x < d) { sums[threadIdx.x] += sums[threadIdx.x + d]; counts[threadIdx.x] += counts[threadIdx.x + d]; }
    }
    if (threadIdx.x == 0) {
        *factor = counts[0] ? 1.f / (float)counts[0] : 0.f;
        *loss = counts[0] ? sums[0] / (float)counts[0] : 0.f;
    }
}
template <int NT>
__global__ __launch_bounds__(NT) void row_loss_kernel(const float2* part, const float* z_label, const int32_t* labels, int rows, int classes,
                                                       int parts, int shares, float2* norm, float* row_loss, float* loss, float* factor)
{
    constexpr int U = 8;
    __shared__ float2 got[NT];
    const int per = NT / shares, r = threadIdx.x % per, share = threadIdx.x / per, k = blockIdx.y, t = blockIdx.x * per + r;
    const float2* src = part + (long long)k * parts * rows + t;
    float2 have{-INFINITY, 0.f};
    if (t < rows)
        for (int p = share; p < parts; p += U * shares) {
            float2 v[U];
            float top = have.x;
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = p + u * shares < parts ? src[(long long)(p + u * shares) * rows] : float2{-INFINITY, 0.f};
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, v[u].x);
            const float base = top == -INFINITY ? 0.f : top;
            have.y *= exp_down(have.x - base);
#pragma unroll
            for (int u = 0; u < U; ++u) have.y += v[u].y * exp_down(v[u].x - base);
            have.x = top;                                      // all -inf so far: the sums are zeros, or NaNs that stay
        }
    got[threadIdx.x] = have;
    for (int d = shares / 2; d > 0; d /= 2) {
        __syncthreads();
        if (share < d) { join(have, got[threadIdx.x + d * per]); got[threadIdx.x] = have; }
    }
    float value = 0.f;
    int live = 0;
    if (share == 0 && t < rows) {
        const long long at = (long long)k * rows + t;
        norm[at] = have;
        live = (unsigned)labels[at] < (unsigned)classes;
        value = live ? (have.x - z_label[at]) + logf(have.y) : 0.f;
        row_loss[at] = value;
    }
    if (!loss) return;
    __shared__ float sums[NT];
    __shared__ int counts[NT];
    mean_of_rows<NT>(value, live, sums, counts, loss + k, factor + k);
}

// a replica's mean loss and the factor 1 / (labelled rows), 0 without any (4096 rows: 4.8 us, a launch)
__global__ __launch_bounds__(256) void mean_loss_kernel(const float* row_loss, const int32_t* labels, int rows, int classes, float* loss, float* factor)
{
    __shared__ float sums[256];
    __shared__ int counts[256];
    const long long base = (long long)blockIdx.x * rows;
    float sum = 0.f;
    int count = 0;
#pragma unroll 4
    for (int t = threadIdx.x; t < rows; t += 256) {
        sum += row_loss[base + t];
        count += (unsigned)labels[base + t] < (unsigned)classes;
    }
    mean_of_rows<256>(sum, count, sums, counts, loss + blockIdx.x, factor + blockIdx.x);
}

// Few rows: G of the whole vocabulary from its logits, 64 columns a workgroup, its W waves taking the rows in turn, and db.  32-bit G takes the
// logits' place.  Bound by memory and, in small cases, by the rounds of eight rows: 8 x 200 rows x 4099 classes fp32 16.5 us = 3.2 TB/s (four
// waves 17.2), 128 x 10007 bf16 5.3 us (7.5).
template <typename T, int W>
__global__ __launch_bounds__(W * 64) void gradient_columns_kernel(const float* z, const int32_t* labels, const float2* norm, int rows, int classes, int ld,
                                                               T* g, const float* factor, float* db, long long db_rep)
{
    constexpr int U = 8;                                       // rows at a time: their loads before the first store, which may be theirs
    __shared__ float sums[W][64];
    const int wave = threadIdx.x >> 6, c = blockIdx.x * 64 + (threadIdx.x & 63), k = blockIdx.y;
    const long long first = (long long)k * rows;
    float sum = 0.f;
    for (int t0 = wave; t0 < rows; t0 += W * U) {
        float v[U];
        float2 l[U];
        int y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long t = first + min(t0 + W * u, rows - 1);
            v[u] = z[t * ld + c];
            l[u] = norm[t];
            y[u] = labels[t];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t0 + W * u >= rows) break;
            const bool live = (unsigned)y[u] < (unsigned)classes;
            const float p = live && c < classes ? exp_down(v[u] - l[u].x) * (1.f / l[u].y) - (c == y[u] ? 1.f : 0.f) : 0.f;
            sum += p;
            g[(first + t0 + W * u) * ld + c] = (T)p;
        }
    }
    if (!db) return;
    sums[wave][threadIdx.x & 63] = sum;
    __syncthreads();
    if (wave != 0 || c >= classes) return;
#pragma unroll
    for (int w = 1; w < W; ++w) sum += sums[w][threadIdx.x];
    db[k * db_rep + c] = sum * factor[k];
}

// G of a piece, unscaled, and its column sums over a wave's rows (EXACT: as above).  With the product 10 to 15 % slower than the statistics (2.04 ms and
// 205 us for the sizes there): G is written.
template <bool EXACT> struct Softmax {
    const float* bias;
    long long bias_rep;
    const int32_t* labels;
    const float2* norm;            // a row's largest logit and the sum of the exp of the distances to it
    float* sums;                   // [replicas][row blocks][ld] or null
    int rows, c0, classes, ld, blocks;          // the piece holds the classes from c0; ld: its columns, rounded up
    // of the wave's block i of 32 rows; zero in rows that take no part and beyond the classes
    template <int TM, int TN> __device__ __forceinline__ void block(const Tile<TM, TN>& t, int i, float (&v)[TN][16]) const
    {
        const int m = t.m0 + 32 * i + (t.lane & 31), n0 = c0 + t.n0;
        const int y = m < rows ? labels[(long long)t.rep * rows + m] : -1;
        const bool live = (unsigned)y < (unsigned)classes;
        const float2 l = live ? norm[(long long)t.rep * rows + m] : float2{0.f, 1.f};
        logits_of(t, i, n0, classes, bias ? bias + t.rep * bias_rep : nullptr, v);
        if (EXACT || bias || !folds(l.x)) {
            const float inv = 1.f / l.y;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) v[j][e] = live ? exp_down(v[j][e] - l.x) * inv : 0.f;
        } else {
            const float shift = -l.x * kLog2e - __builtin_amdgcn_logf(l.y);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) v[j][e] = live ? __builtin_amdgcn_exp2f(__builtin_fmaf(v[j][e], kLog2e, shift)) : 0.f;
        }
        at_label<TN>(t.lane, n0, live ? y : -1, [&](int j, int e) { v[j][e] -= 1.f; });
    }
    template <int TM, int TN> __device__ __forceinline__ void store_sums(const Tile<TM, TN>& t, const float (&column)[TN][16]) const
    {
        float* out = sums + ((long long)t.rep * blocks + t.m0 / (32 * TM)) * ld;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float v = sum_over<32>(column[j][e]);
                const int n = t.n0 + 32 * j + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4;
                if ((t.lane & 31) == 0 && n < ld) out[n] = v;
            }
    }
};
// into [replicas][rows][ld] of the operands' type, for the general product
template <bool EXACT, typename T> struct Gradient {
    static constexpr bool kLaneM = true, kStaged = false, kSums = false;
    Softmax<EXACT> soft;
    T* g;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t) const
    {
        float column[TN][16] = {};
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = t.m0 + 32 * i + (t.lane & 31);
            float v[TN][16];
            soft.block(t, i, v);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = t.n0 + 32 * j + 8 * q + 4 * (t.lane >> 5);
#pragma unroll
                    for (int e = 0; e < 4; ++e) column[j][4 * q + e] += v[j][4 * q + e];
                    if (m >= soft.rows || n >= soft.ld) continue;
                    T* out = g + ((long long)t.rep * soft.rows + m) * soft.ld + n;
                    if (sizeof(T) == 4) *(f4*)out = f4{v[j][4 * q], v[j][4 * q + 1], v[j][4 * q + 2], v[j][4 * q + 3]};
                    else *(u2*)out = u2{to_bf16x2(v[j][4 * q], v[j][4 * q + 1]), to_bf16x2(v[j][4 * q + 2], v[j][4 * q + 3])};
                }
        }
        if (soft.sums) soft.store_sums(t, column);
    }
};
// into planes [PL][replicas][rows][ld] for the direct product: bf16, or two fp16 parts (|G| <= 1)
template <int PL> struct GradientRows {
    static constexpr bool kLaneM = true, kStaged = true, kSums = false;
    Softmax<PL == 2> soft;
    __bf16* g;
    long long plane;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t, char* lds) const
    {
        float column[TN][16] = {};
        const RowStage<TN> stage{lds + t.wave * RowStage<TN>::kBytes};
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            float v[TN][16];
            soft.block(t, i, v);
            if (soft.sums) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) column[j][e] += v[j][e];
            }
            u2 part[PL][TN][4];
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (PL == 2) split2(f4{v[j][4 * q], v[j][4 * q + 1], v[j][4 * q + 2], v[j][4 * q + 3]}, up_scale(kOneBits), part[0][j][q], part[PL - 1][j][q]);
                    else part[0][j][q] = u2{to_bf16x2(v[j][4 * q], v[j][4 * q + 1]), to_bf16x2(v[j][4 * q + 2], v[j][4 * q + 3])};
                }
#pragma unroll
            for (int s = 0; s < PL; ++s) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) stage.put(t.lane, j, q, part[s][j][q]);
                stage.take(t.lane, [&](int r, int c, const u4& w) {
                    const int m = t.m0 + 32 * i + r, n = t.n0 + c;
                    if (m < soft.rows && n < soft.ld) *(u4*)(g + s * plane + ((long long)t.rep * soft.rows + m) * soft.ld + n) = w;
                });
            }
        }
        if (soft.sums) soft.store_sums(t, column);
    }
};

// The whole vocabulary in one piece: G from its logits, bf16 or two fp16 parts, and its column sums over `depth` rows, 256 columns a workgroup,
// every fourth row a wave.  Bound by memory: 2 x 1000 x 20011 fp32 58 us = 5.5 TB/s, 4 x 512 x 32000 bf16 68 us = 5.8.
template <int PL> __global__ __launch_bounds__(256) void gradient_planes_kernel(const float* z, const int32_t* labels, const float2* norm, int rows, int classes, int ld,
                                                              int depth, __bf16* g, long long plane, float* sums)
{
    constexpr int U = 4;
    __shared__ f4 part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (blockIdx.x * 64 + lane) * 4, k = blockIdx.z;
    const int first = blockIdx.y * depth, last = min(rows, first + depth);
    const bool in = c < ld;                                    // whole chunks: ld is a multiple of 128
    const long long line = (long long)k * rows;
    f4 sum{0.f, 0.f, 0.f, 0.f};
    for (int t0 = first + wave; t0 < last; t0 += 4 * U) {
        f4 v[U];
        float2 l[U];
        int y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long t = line + min(t0 + 4 * u, last - 1);
            v[u] = *(const f4*)(z + t * ld + (in ? c : 0));
            l[u] = norm[t];
            y[u] = labels[t];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t0 + 4 * u >= last || !in) break;
            const bool live = (unsigned)y[u] < (unsigned)classes;
            const float inv = 1.f / l[u].y;
            f4 p;
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = live && c + e < classes ? exp_down(v[u][e] - l[u].x) * inv - (c + e == y[u] ? 1.f : 0.f) : 0.f;
            sum += p;
            u2 high, low;
            if (PL == 2) split2(p, up_scale(kOneBits), high, low);
            else high = u2{to_bf16x2(p[0], p[1]), to_bf16x2(p[2], p[3])};
            const long long at = (line + t0 + 4 * u) * ld + c;
            *(u2*)(g + at) = high;
            if (PL == 2) *(u2*)(g + plane + at) = low;
        }
    }
    if (!sums) return;
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && in) *(f4*)(sums + ((long long)k * gridDim.y + blockIdx.y) * ld + c) = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

// db of a piece: the row blocks' sums in ascending order (20011 classes: 5.4 us, a launch)
__global__ __launch_bounds__(256) void bias_grad_kernel(const float* sums, int blocks, int ld, int c0, int cols, const float* factor, float* db, long long rep)
{
    const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.y;
    if (c >= cols) return;
    float v = 0.f;
    for (int b = 0; b < blocks; ++b) v += sums[((long long)k * blocks + b) * ld + c];
    db[k * rep + c0 + c] = v * factor[k];
}

// Which kernels, the piece of the vocabulary and the working memory, from the sizes alone.
//   few rows   the products through registers read W as it is, 32, 64 or 128 x 128 tiles, the logits' contraction in shares where there are
//              few of them
//   more       products straight from memory to LDS: twice to three times the rate, but x (unlabelled rows as zeros) and a W of 32-bit or
//              unaligned values are laid out first, there are more launches, and few tiles leave most of the chip idle
struct Plan {
    bool direct, small, keep;      // small: 32 rows a tile, not 64; keep: the logits of the one piece there is stay for its G
    int bm, bn, wave_m, parts, z_splits, z_len, piece, pieces, blocks, splits, split_len, w_tile, w_splits, w_len, ldx, planes;
    size_t norm, z_label, row_loss, factor, part, g, z, sums, share, w_share, x, w, top, total;
};
// of G, and of a laid-out piece of W: a 32-bit W of more than one piece is laid out again for the gradient (16 x 699 x 576 x 9056: 2.36 ms
// with 256 MiB, 2.10 with 512 and 1024; bf16 the same with each)
constexpr long long kPieceBytes = 512ll << 20;

int up_to(long long v, int unit) { return (int)((v + unit - 1) / unit * unit); }
// tiles 128 wide in this direction, not 256: they are 15 to 20 % slower for the work they hold (2 x 4096 x 2048 x 65536 bf16: dx 2.14 ms
// against 1.87, dW 2.13 against 1.86), and 256 wide ones hold up to twice the work
bool narrow(int v) { return 1.18 * up_to(v, 128) < up_to(v, 256); }

// Rows up to which W is read as it is: more where W is small, and where its features are many for its tiles.  Loss and gradients through
// registers / laid out, us (the rule's own bound in brackets):
//   bf16             4 x 512 x 32000 (41 rows), 32 rows 107 / 128, 64 rows 130 / 136, 96 rows 155 / 139; 2048 x 20000 (78), 48 rows 84 / 79, 128 rows
//                    111 / 92; 4096 x 10008 (172), 128 rows 106 / 107, 192 rows 143 / 117; 2048 x 5000 (224), 192 rows 67 / 68, 256 rows 77 / 71
//   bf16, unaligned  4 x 512 x 32001 (138), 128 rows 176 / 197, 160 rows 293 / 236; 2048 x 20011 (174), 128 rows 115 / 125, 192 rows 153 / 147;
//                    8 x 200 x 4099 (221), 256 rows 80 / 86, 320 rows 96 / 86
//   fp32             4 x 512 x 32000 (215), 192 rows 597 / 593, 256 rows 695 / 646; 2048 x 20011 (234), 192 rows 350 / 391, 256 rows 441 / 413;
//                    12 x 520 x 8739 (218), 192 rows 588 / 594, 256 rows 668 / 667; 8 x 200 x 4099 (353), 320 rows 161 / 169, 384 rows 180 / 177
// Sizes alone decide, since the working memory is asked for before a W is seen: bf16 classes that are no multiple of eight stand for a W that
// has to be copied, and a W inside rows of an odd stride is copied all the same.
double few_rows(int n, int features, int classes, int bf16)
{
    const double values = (double)n * features * classes, deep = std::min(125., features / ((double)n * classes / 256));
    if (!bf16) return 200 + std::min(165., 1.0e9 / values) + 0.4 * deep;
    return (classes % 8 ? 128 + std::min(100., 0.6e9 / values) : 30 + std::min(200., 0.7e9 / values)) + 1.2 * deep;
}

// Into how many shares the logits' contraction over few rows is cut.  A workgroup, of 128 classes, takes 12 ns a feature (bf16 W, 32 rows; 24:
// 64 rows) or 35 (fp32; 43), three of them share a compute unit, and together they read W at 5 TB/s at best; shares cost a launch and
// their bytes.  One row, 4096 x 10007 fp32: one share 142 us, eight 42; 2048 x 5000: 75 and 21; 512 x 32000, two: 26 and 24, and one is taken.
int logit_shares(const Plan& p, int n, int rows, int features, int classes, int bf16)
{
    const double groups = (double)n * p.parts * ((rows + p.bm - 1) / p.bm), feature = (bf16 ? (p.small ? 12 : 24) : p.small ? 35 : 43) * 1e-9;
    const double read = (double)n * features * classes * (bf16 ? 2 : 4) / 5e12;
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 32 && (s == 1 || features / s >= 128); ++s) {
        const double cost = std::max(std::ceil(groups * s / 768) * features / s * feature, read) + (s > 1 ? 4e-6 + (double)n * rows * p.piece * 4 * (2 * s + 1) / 4e12 : 0);
        if (s == 1 || cost < (best == 1 ? 0.9 : 1) * least) { best = s; least = cost; }
    }
    return best;
}

Plan plan_of(int n, int rows, int features, int classes, int bf16, bool grad)
{
    Plan p{};
    p.direct = rows > few_rows(n, features, classes, bf16) || (rows && std::min(features, classes) < 8);       // fewer values a row than a chunk: laid out
    p.small = rows <= 32;
    // 128 rows a tile where they hold no more than 64 do (16 x 256 x 10007 fp32, 96 rows 263 us against 290, 132 rows 419 against 410)
    p.bm = p.small ? 32 : rows <= 64 || up_to(rows, 128) > up_to(rows, 64) ? 64 : 128;
    p.bn = 128;
    // smaller tiles where larger ones would leave half of the chip without one (statistics of 200 x 1024 x 10000 bf16: 14.7 us against 29.4; 500 x 512 x
    // 8000 fp32 28 against 42)
    if (p.direct) {
        auto tiles = [&](int m, int n_) { return (long long)n * ((rows + m - 1) / m) * ((classes + n_ - 1) / n_); };
        p.bm = narrow(rows) || tiles(256, 256) < 128 ? 128 : 256;
        p.bn = p.bm == 128 && tiles(128, 256) < 128 ? 128 : 256;
    }
    const int bn = p.bn;
    p.wave_m = p.direct || p.bm == 128 ? p.bm / 2 : 32;
    p.planes = p.direct && !bf16 ? 2 : 1;
    p.parts = up_to(classes, bn) / bn;
    p.blocks = up_to(rows, p.bm) / p.wave_m;
    const long long lines = (long long)n * rows, es = p.direct ? (bf16 ? 2 : 4) : bf16 ? 6 : 4;      // of G and, few rows, the logits
    long long most = grad ? kPieceBytes / std::max<long long>(1, lines * es) : up_to(classes, bn);
    if (p.direct) most = std::min(most, kPieceBytes / ((long long)n * features * 2 * p.planes));
    most = std::max<long long>(1024, most / bn * bn);
    p.pieces = (int)((classes + most - 1) / most);
    p.piece = up_to((classes + p.pieces - 1) / p.pieces, bn);
    // through registers a piece has eight columns at least, so that no load begins before a row or ends behind it (tile_product.h)
    while (!p.direct && classes > p.piece && (classes - 1) % p.piece < 7) p.piece += bn;
    p.pieces = (classes + p.piece - 1) / p.piece;
    // z as 32-bit floats costs its bytes, in the statistics' kernel and in gradient_planes_kernel; forming it again costs the product.
    // fp32, three products: 2 x 1000 x 777 x 20011 in all 1027 us against 1191, 4 x 2656 x 64 x 2036 171 against 174.  bf16, 4 x 512 rows x 32000: 512
    // features 434 against 416, 1024 656 against 711, 2048 1080 against 1262.
    p.keep = p.direct && grad && p.pieces == 1 && (!bf16 || features >= 768) && lines * p.piece * (es + 4) <= kPieceBytes;
    p.ldx = up_to(features, 8);
    const int bd = p.direct && !narrow(features) ? 256 : 128;              // columns of dx a tile
    const long long tiles = (long long)n * ((rows + p.bm - 1) / p.bm) * ((features + bd - 1) / bd);
    const int products = bf16 ? 1 : 3;
    p.splits = p.direct ? best_shares(tiles, p.piece / kSlab * products, (double)lines * p.ldx * 4)
                        : (int)std::max<long long>(1, std::min<long long>(512 / std::max<long long>(1, tiles), p.piece / 128));
    p.split_len = up_to((p.piece + p.splits - 1) / p.splits, 128);
    p.splits = (p.piece + p.split_len - 1) / p.split_len;
    // dW of a piece: few tiles are made smaller (400 x 512 x 8000 bf16 9 us against 16, 500 rows fp32 25 against 53); with more rows than that pays
    // for the rows are cut in shares
    const long long dw_tiles = (long long)n * ((features + bd - 1) / bd) * (p.piece / 256);
    p.w_tile = dw_tiles < 128 && rows <= 512 ? 128 : 256;
    p.w_splits = p.direct && p.w_tile == 256 ? best_shares(dw_tiles, (rows + kSlab - 1) / kSlab * products, (double)n * features * p.piece * 4) : 1;
    p.w_len = up_to((rows + p.w_splits - 1) / p.w_splits, 64);
    if (rows) p.w_splits = (rows + p.w_len - 1) / p.w_len;
    p.z_splits = !p.direct && p.pieces == 1 ? logit_shares(p, n, rows, features, classes, bf16) : 1;
    p.z_len = up_to((features + p.z_splits - 1) / p.z_splits, 128);
    p.z_splits = (features + p.z_len - 1) / p.z_len;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    p.norm = take((size_t)lines * 8);
    p.z_label = take((size_t)lines * 4);
    p.row_loss = take((size_t)lines * 4);
    p.factor = take((size_t)n * 4);
    p.part = take((size_t)lines * p.parts * 8);
    if (p.direct) {
        p.x = take((size_t)lines * p.ldx * 2 * p.planes);
        p.w = take((size_t)n * features * p.piece * 2 * p.planes);
        p.top = take((size_t)n * 8);
    }
    if (p.keep) p.z = take((size_t)lines * p.piece * 4);
    if (!p.direct && (p.z_splits > 1 || grad) && (bf16 || !grad)) p.z = take((size_t)lines * p.piece * 4 * p.z_splits);
    if (grad) {
        p.g = take((size_t)lines * p.piece * (p.direct ? es : bf16 ? 2 : 4 * p.z_splits));
        if (!p.direct && !bf16) p.z = p.g;                // 32-bit G takes the logits' place
        p.sums = take((size_t)n * p.blocks * p.piece * 4);
        p.share = take((size_t)p.splits * lines * p.ldx * 4);
        if (p.w_splits > 1) p.w_share = take((size_t)p.w_splits * n * features * p.piece * 4);
    }
    p.total = at;
    return p;
}

// the pointers into the working memory
struct Work {
    float *z_label, *factor, *row_loss, *z, *sums, *share, *w_share;
    float2 *norm, *part;
    char* g;
    __bf16 *x, *w;
    unsigned* top;                 // [2][replicas]: of x and of W
    Work(const LossArgs& a, const Plan& p)
    {
        char* at = (char*)a.work;
        norm = (float2*)(at + p.norm); z_label = (float*)(at + p.z_label); factor = (float*)(at + p.factor);
        row_loss = a.row_loss ? a.row_loss : (float*)(at + p.row_loss);
        sums = (float*)(at + p.sums); share = (float*)(at + p.share); w_share = (float*)(at + p.w_share); part = (float2*)(at + p.part);
        g = at + p.g; z = (float*)(at + p.z); x = (__bf16*)(at + p.x); w = (__bf16*)(at + p.w); top = (unsigned*)(at + p.top);
    }
};

hipError_t join_rows(const LossArgs& a, const Plan& p, const Work& w, hipStream_t s)
{
    int per = 256;                                             // rows a workgroup
    while (per > 4 && per / 2 >= a.rows) per /= 2;
    while (per > 32 && p.parts >= 2048 / per) per /= 2;
    int all = 4;                                               // one workgroup of 1024 for a replica's rows, sixteen pairs a thread at most: 4.6 us less
    while (all < a.rows) all *= 2;
    const bool large = a.rows > per && all <= 1024 && (long long)all * p.parts <= 16384, alone = large || a.rows <= per;
    if (a.rows) {
        if (large)
            row_loss_kernel<1024><<<dim3(1, (unsigned)a.n), 1024, 0, s>>>(w.part, w.z_label, a.labels, a.rows, a.classes, p.parts, 1024 / all, w.norm,
                                                                          w.row_loss, a.loss, w.factor);
        else
            row_loss_kernel<256><<<dim3((unsigned)((a.rows + per - 1) / per), (unsigned)a.n), 256, 0, s>>>(
                w.part, w.z_label, a.labels, a.rows, a.classes, p.parts, 256 / per, w.norm, w.row_loss, alone ? a.loss : nullptr, w.factor);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || alone) return e;
    }
    mean_loss_kernel<<<(unsigned)a.n, 256, 0, s>>>(w.row_loss, a.labels, a.rows, a.classes, a.loss, w.factor);
    return hipGetLastError();
}
hipError_t bias_grad(const LossArgs& a, const Plan& p, const Work& w, int ld, int c0, int cols, hipStream_t s)
{
    if (!a.db.p) return hipSuccess;
    bias_grad_kernel<<<dim3((unsigned)((cols + 255) / 256), (unsigned)a.n), 256, 0, s>>>(w.sums, a.rows ? p.blocks : 0, ld, c0, cols, w.factor,
                                                                                          (float*)a.db.p, a.db.rep);
    return hipGetLastError();
}
template <typename T> hipError_t input_grad(const LossArgs& a, const Plan& p, const Work& w, hipStream_t s)
{
    if (!a.dx.p || !a.rows) return hipSuccess;
    return join_shares<T>(w.share, p.splits, a.n, a.rows, a.features, p.ldx, Labelled{a.labels, a.classes}, w.factor, a.dx, nullptr, 0, s);
}

// few rows: everything through registers.  Where one piece holds the whole vocabulary its logits stay in it for the gradient.
template <typename T, int BM, int WM, int WN> hipError_t run_general(const LossArgs& a, const Plan& p, hipStream_t s)
{
    constexpr bool exact = sizeof(T) == 4;
    const Work k(a, p);
    const bool once = a.grad && p.pieces == 1;
    hipError_t e = hipSuccess;
    const Source<T> x = source<T>(a.x, a.rows, a.features);
    const float* bias = (const float*)a.bias.p;
    if (a.rows && p.z_splits > 1) {
        const StoreShare<> store{k.z, a.rows, a.classes, p.piece, a.rows, a.n, false, false};
        e = launch_product<BM, 128, WM, WN, true, false>(x, source<T>(a.w, a.features, a.classes), a.n, a.rows, a.classes, a.features, p.z_splits, p.z_len, store, s);
        if (e == hipSuccess) e = launch_join_logits(a, k.z, p.z_splits, p.piece, k.part, k.z_label, s);
    } else if (a.rows) {
        const Statistics<exact, BM, 128, WN> stats{bias, a.bias.rep, a.labels, k.part, k.z_label, once ? k.z : nullptr, a.rows, 0, a.classes, p.parts, p.piece};
        e = launch_product<BM, 128, WM, WN, true, false>(x, source<T>(a.w, a.features, a.classes), a.n, a.rows, a.classes, a.features, 1, a.features, stats, s);
    }
    if (e != hipSuccess) return e;
    if ((e = join_rows(a, p, k, s)) != hipSuccess || !a.grad) return e;
    const Labelled live{a.labels, a.classes};
    for (int i = 0; i < p.pieces; ++i) {
        const int c0 = i * p.piece, cols = std::min(p.piece, a.classes - c0), ld = up_to(cols, 128);
        const Source<T> w = source<T>(Rows{(T*)a.w.p + c0, a.w.rep, a.w.row}, a.features, cols);
        const Source<T> g = source<T>(Rows{k.g, (long long)a.rows * ld, ld}, a.rows, ld);            // zero beyond cols
        if (once) {
            const dim3 grid((unsigned)(ld / 64), (unsigned)a.n);
            if (a.rows <= 64) gradient_columns_kernel<T, 4><<<grid, 256, 0, s>>>(k.z, a.labels, k.norm, a.rows, a.classes, ld, (T*)k.g, k.factor, (float*)a.db.p, a.db.rep);
            else gradient_columns_kernel<T, 16><<<grid, 1024, 0, s>>>(k.z, a.labels, k.norm, a.rows, a.classes, ld, (T*)k.g, k.factor, (float*)a.db.p, a.db.rep);
            e = hipGetLastError();
        } else if (a.rows) {
            const Softmax<exact> soft{bias, a.bias.rep, a.labels, k.norm, a.db.p ? k.sums : nullptr, a.rows, c0, a.classes, ld, p.blocks};
            e = launch_product<BM, 128, WM, WN, true, false>(x, w, a.n, a.rows, cols, a.features, 1, a.features, Gradient<exact, T>{soft, (T*)k.g}, s);
            if (e == hipSuccess) e = bias_grad(a, p, k, ld, c0, cols, s);
        }
        if (e != hipSuccess) return e;
        if (a.dx.p && a.rows) {
            const StoreShare<> store{k.share, a.rows, a.features, p.ldx, a.rows, a.n, i > 0, false};
            e = launch_product<BM, 128, WM, WN, true, true>(g, w, a.n, a.rows, a.features, cols, p.splits, p.split_len, store, s);
            if (e != hipSuccess) return e;
        }
        if (a.dw.p && once && a.rows && a.rows <= kFewWeights && a.classes >= 4) {
            if ((e = launch_few_weights<T>(a, (const T*)k.g, ld, k.factor, s)) != hipSuccess) return e;
        } else if (a.dw.p) {
            const StoreTile<T> store{(T*)a.dw.p + c0, a.dw.rep, a.dw.row, k.factor, a.features, cols, nullptr, 0};
            // 128 x 128 tiles where they give every compute unit four (16 x 256 x 10007 fp32, 96 rows: 246 us in all against 257), else 64 x 128 (2 x 1024 x
            // 4099: 92 against 94)
            const Source<T, true> xt = source<T, true>(a.x, a.rows, a.features, live);
            if ((long long)a.n * ((a.features + 127) / 128) * ((cols + 127) / 128) >= 1024)
                e = launch_product<128, 128, 2, 4, false, false>(xt, g, a.n, a.features, cols, a.rows, 1, std::max(1, a.rows), store, s);
            else
                e = launch_product<64, 128, 2, 4, false, false>(xt, g, a.n, a.features, cols, a.rows, 1, std::max(1, a.rows), store, s);
            if (e != hipSuccess) return e;
        }
    }
    return input_grad<T>(a, p, k, s);
}

template <typename T, int PL, class Store>
hipError_t weight_grad(const Plane3& x, const Plane3& g, const LossArgs& a, int cols, const Plan& p, const Store& store, hipStream_t s)
{
    if constexpr (!std::is_same_v<Store, StoreShare<>>)        // (small tiles take no shares)
        if (p.w_tile == 128) return launch_direct<PL, PL, 128, 128, 2, 4, false, false>(x, g, a.n, a.features, cols, a.rows, p.w_splits, p.w_len, store, s);
    if (narrow(a.features)) return launch_direct<PL, PL, 128, 256, 2, 4, false, false>(x, g, a.n, a.features, cols, a.rows, p.w_splits, p.w_len, store, s);
    return launch_direct<PL, PL, 256, 256, 2, 4, false, false>(x, g, a.n, a.features, cols, a.rows, p.w_splits, p.w_len, store, s);
}

// more rows: operands straight from memory to LDS
template <typename T, int BM, int BN, int WN> hipError_t run_direct(const LossArgs& a, const Plan& p, hipStream_t s)
{
    constexpr int PL = sizeof(T) == 4 ? 2 : 1;
    const Work k(a, p);
    const float* bias = (const float*)a.bias.p;
    const Labelled live{a.labels, a.classes};
    hipError_t e = hipSuccess;
    const unsigned *top_x = nullptr, *top_w = nullptr;
    if (PL == 2) {
        top_x = k.top; top_w = k.top + a.n;
        for (int i = 0; i < 2 * a.n && e == hipSuccess; i += 1024) { clear_kernel<<<1, 1024, 0, s>>>(k.top + i, std::min(1024, 2 * a.n - i)); e = hipGetLastError(); }
        if (e == hipSuccess) e = find_largest(a.n, Magnitudes{(const float*)a.x.p, a.x.rep, a.x.row, a.rows, a.features, live, k.top},
                                              Magnitudes{(const float*)a.w.p, a.w.rep, a.w.row, a.features, a.classes, {nullptr, 0}, k.top + a.n}, s);
    }
    if (e == hipSuccess) e = lay_out<T, PL>(a.n, a.rows, a.features, p.ldx, a.x, live, top_x, k.x, s);
    if (e != hipSuccess) return e;
    const Plane3 x{k.x, (long long)a.rows * p.ldx, (long long)a.n * a.rows * p.ldx, p.ldx, a.rows, p.ldx, top_x};
    // W as it is, or laid out a piece at a time
    const bool as_is = PL == 1 && is_plane(a.w, a.classes);
    auto weights = [&](int c0, int cols, bool there, Plane3& w) -> hipError_t {
        if (as_is) { w = Plane3{(const __bf16*)a.w.p + c0, a.w.rep, 0, (int)a.w.row, a.features, cols, nullptr}; return hipSuccess; }
        const int ld = up_to(cols, 8);
        w = Plane3{k.w, (long long)a.features * ld, (long long)a.n * a.features * ld, ld, a.features, ld, top_w};
        if (there) return hipSuccess;
        return lay_out<T, PL>(a.n, a.features, cols, ld, Rows{(T*)a.w.p + c0, a.w.rep, a.w.row}, Labelled{nullptr, 0}, top_w, k.w, s);
    };
    Plane3 w;
    const int step = as_is ? a.classes : p.piece;
    for (int c0 = 0; c0 < a.classes; c0 += step) {
        const int cols = std::min(step, a.classes - c0);
        if ((e = weights(c0, cols, false, w)) != hipSuccess) return e;
        const Statistics<PL == 2, BM, BN, WN> stats{bias, a.bias.rep, a.labels, k.part, k.z_label, p.keep ? k.z : nullptr, a.rows, c0, a.classes, p.parts, p.piece};
        e = launch_direct<PL, PL, BM, BN, 2, WN, true, false>(x, w, a.n, a.rows, cols, a.features, 1, a.features, stats, s);
        if (e != hipSuccess) return e;
    }
    if ((e = join_rows(a, p, k, s)) != hipSuccess || !a.grad) return e;
    for (int i = 0; i < p.pieces; ++i) {
        const int c0 = i * p.piece, cols = std::min(p.piece, a.classes - c0), ld = up_to(cols, BN);
        if ((e = weights(c0, cols, p.pieces == 1, w)) != hipSuccess) return e;
        const Plane3 g{(const __bf16*)k.g, (long long)a.rows * ld, (long long)a.n * a.rows * ld, ld, a.rows, ld, nullptr};
        const Softmax<PL == 2> soft{bias, a.bias.rep, a.labels, k.norm, a.db.p ? k.sums : nullptr, a.rows, c0, a.classes, ld, p.blocks};
        if (p.keep) {
            gradient_planes_kernel<PL><<<dim3((unsigned)((ld + 255) / 256), (unsigned)p.blocks, (unsigned)a.n), 256, 0, s>>>(
                k.z, a.labels, k.norm, a.rows, a.classes, ld, p.wave_m, (__bf16*)k.g, g.plane, soft.sums);
            e = hipGetLastError();
        } else e = launch_direct<PL, PL, BM, BN, 2, WN, true, false>(x, w, a.n, a.rows, cols, a.features, 1, a.features, GradientRows<PL>{soft, (__bf16*)k.g, g.plane}, s);
        if (e != hipSuccess) return e;
        if (a.dx.p) {
            const StoreShare<> store{k.share, a.rows, a.features, p.ldx, a.rows, a.n, i > 0, false};
            if (narrow(a.features)) e = launch_direct<PL, PL, BM, 128, 4, 2, true, true>(g, w, a.n, a.rows, a.features, w.cols, p.splits, p.split_len, store, s);
            else e = launch_direct<PL, PL, BM, 256, 2, 4, true, true>(g, w, a.n, a.rows, a.features, w.cols, p.splits, p.split_len, store, s);
            if (e != hipSuccess) return e;
        }
        if (a.dw.p) {
            const Rows out{(T*)a.dw.p + c0, a.dw.rep, a.dw.row};
            if (p.w_splits > 1) {
                e = weight_grad<T, PL>(x, g, a, cols, p, StoreShare<>{k.w_share, a.features, cols, ld, a.features, a.n, false, false}, s);
                if (e == hipSuccess) e = join_shares<T>(k.w_share, p.w_splits, a.n, a.features, cols, ld, Labelled{nullptr, 0}, k.factor, out, nullptr, 0, s);
            } else if constexpr (PL == 1) e = weight_grad<T, PL>(x, g, a, cols, p, StoreRows{(__bf16*)out.p, out.rep, out.row, k.factor, a.features, cols}, s);
            else e = weight_grad<T, PL>(x, g, a, cols, p, StoreTile<float>{(float*)out.p, out.rep, out.row, k.factor, a.features, cols, nullptr, 0}, s);
            if (e != hipSuccess) return e;
        }
        if ((e = bias_grad(a, p, k, ld, c0, cols, s)) != hipSuccess) return e;
    }
    return input_grad<T>(a, p, k, s);
}

}  // namespace

size_t loss_work_bytes(int n, int rows, int features, int classes, int bf16, bool grad)
{
    const size_t forward = plan_of(n, rows, features, classes, bf16, false).total;         // a workspace for the gradient serves the loss alone too
    return grad ? std::max(forward, plan_of(n, rows, features, classes, bf16, true).total) : forward;
}

hipError_t launch_loss(const LossArgs& a, hipStream_t s)
{
    const Plan p = plan_of(a.n, a.rows, a.features, a.classes, a.bf16, a.grad);
    if (p.direct) {
        if (a.bf16) return p.bm == 256 ? run_direct<__bf16, 256, 256, 4>(a, p, s) : p.bn == 256 ? run_direct<__bf16, 128, 256, 4>(a, p, s) : run_direct<__bf16, 128, 128, 4>(a, p, s);
        return p.bm == 256 ? run_direct<float, 256, 256, 4>(a, p, s) : p.bn == 256 ? run_direct<float, 128, 256, 4>(a, p, s) : run_direct<float, 128, 128, 4>(a, p, s);
    }
    if (p.bm == 128) return a.bf16 ? run_general<__bf16, 128, 2, 4>(a, p, s) : run_general<float, 128, 2, 4>(a, p, s);
    if (a.bf16) return p.small ? run_general<__bf16, 32, 1, 4>(a, p, s) : run_general<__bf16, 64, 2, 4>(a, p, s);
    return p.small ? run_general<float, 32, 1, 4>(a, p, s) : run_general<float, 64, 2, 4>(a, p, s);
}

}  // namespace head
}  // namespace hadfl
