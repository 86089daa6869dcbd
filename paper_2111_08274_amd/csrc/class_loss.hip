// Softmax cross entropy of a last dense layer over many classes, and its gradient, in pieces of the vocabulary.
//   1. logits' statistics: z = x W + b a tile at a time; a tile leaves, per row, its largest logit and the sum of exp of the
//      distances to it, and the label's logit where the tile holds it.  Nothing of z is stored.
//   2. per row: the tiles' pairs joined, lse = max + log(sum); row losses, their mean and 1 / (labelled rows).
//   3. for every piece of the vocabulary: z again, G = exp(z - lse) - onehot into a buffer of [rows][piece], then
//      dx += G W^T (shares of the contraction side by side, added in a fixed order) and dW = x^T G.
// A row without a label has G = 0 and its x is read as zeros.
#include "tile_product.h"

namespace hadfl {
namespace head {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLog2eLow = 1.92596299112661746887e-8f, kLn2 = 0.693147180559945309417f;

// exp of a number that is not positive.  EXACT: the product with log2(e) in two parts, else its rounding error, |t| * 2^-24,
// would show in a 32-bit gradient
template <bool EXACT> __device__ __forceinline__ float exp_down(float t)
{
    const float y = t * kLog2e;
    const float p = __builtin_amdgcn_exp2f(y);
    if (!EXACT || !(y > -126.f)) return p;
    const float rest = __builtin_fmaf(t, kLog2e, -y) + t * kLog2eLow;
    return __builtin_fmaf(p, rest * kLn2, p);
}

// the statistics of a wave's columns
template <bool EXACT> struct Statistics {
    static constexpr bool kLaneM = true;
    const float* bias;
    long long bias_rep;
    const int32_t* labels;
    float2* part;                  // [replicas][parts][rows]
    float* z_label;                // [replicas][rows]
    int rows, classes, parts;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t) const
    {
        const float* b = bias ? bias + t.rep * bias_rep : nullptr;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = t.m0 + 32 * i + (t.lane & 31);
            const int y = m < rows ? labels[(long long)t.rep * rows + m] : -1;
            float z[TN][16], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int n = t.n0 + 32 * j + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4;
                    z[j][e] = n < classes ? t.acc[i][j][e] + (b ? b[n] : 0.f) : -INFINITY;
                    top = z[j][e] > top || z[j][e] != z[j][e] ? z[j][e] : top;
                    if (n == y && n < classes) z_label[(long long)t.rep * rows + m] = z[j][e];
                }
            const float other = __shfl_xor(top, 32);
            top = other > top || other != other ? other : top;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += top == -INFINITY ? 0.f : exp_down<EXACT>(z[j][e] - top);
            sum += __shfl_xor(sum, 32);
            if (t.lane < 32 && m < rows) part[((long long)t.rep * parts + t.n0 / (32 * TN)) * rows + m] = float2{top, sum};
        }
    }
};

// the pairs of a row's tiles joined: `shares` threads a row, in ascending order of the tiles within a share and of the shares
__global__ __launch_bounds__(256) void row_loss_kernel(const float2* part, const float* z_label, const int32_t* labels, int rows, int classes,
                                                       int parts, int shares, float* lse, float* row_loss)
{
    __shared__ float2 got[256];
    const int per = 256 / shares, r = threadIdx.x % per, share = threadIdx.x / per, k = blockIdx.y, t = blockIdx.x * per + r;
    const float2* src = part + (long long)k * parts * rows + t;
    float top = -INFINITY, sum = 0.f;
    if (t < rows)
        for (int p = share; p < parts; p += shares) {
            const float2 v = src[(long long)p * rows];
            const float m = v.x > top || v.x != v.x ? v.x : top;
            if (m != -INFINITY) { sum = sum * expf(top - m) + v.y * expf(v.x - m); top = m; }
        }
    got[threadIdx.x] = float2{top, sum};
    __syncthreads();
    if (share || t >= rows) return;
    for (int q = 1; q < shares; ++q) {
        const float2 v = got[q * per + r];
        const float m = v.x > top || v.x != v.x ? v.x : top;
        if (m != -INFINITY) { sum = sum * expf(top - m) + v.y * expf(v.x - m); top = m; }
    }
    const long long at = (long long)k * rows + t;
    const float l = top + logf(sum);
    lse[at] = l;
    row_loss[at] = (unsigned)labels[at] < (unsigned)classes ? l - z_label[at] : 0.f;
}

// a replica's mean loss and the factor 1 / (labelled rows), 0 without any
__global__ __launch_bounds__(256) void mean_loss_kernel(const float* row_loss, const int32_t* labels, int rows, int classes, float* loss, float* factor)
{
    __shared__ float sums[256];
    __shared__ int counts[256];
    const long long base = (long long)blockIdx.x * rows;
    float sum = 0.f;
    int count = 0;
    for (int t = threadIdx.x; t < rows; t += 256) {
        sum += row_loss[base + t];
        count += (unsigned)labels[base + t] < (unsigned)classes;
    }
    sums[threadIdx.x] = sum;
    counts[threadIdx.x] = count;
    for (int d = 128; d > 0; d /= 2) {
        __syncthreads();
        if (threadIdx.x < d) { sums[threadIdx.x] += sums[threadIdx.x + d]; counts[threadIdx.x] += counts[threadIdx.x + d]; }
    }
    if (threadIdx.x == 0) {
        factor[blockIdx.x] = counts[0] ? 1.f / (float)counts[0] : 0.f;
        loss[blockIdx.x] = counts[0] ? sums[0] / (float)counts[0] : 0.f;
    }
}

// G of a piece, unscaled, and its column sums over a wave's rows
template <bool EXACT, typename T> struct Gradient {
    static constexpr bool kLaneM = true;
    const float* bias;
    long long bias_rep;
    const int32_t* labels;
    const float* lse;
    T* g;                          // [replicas][rows][ld], all ld columns are written
    float* sums;                   // [replicas][row blocks][ld] or null
    int rows, c0, classes, ld, blocks;          // the piece holds the classes from c0
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t) const
    {
        const float* b = bias ? bias + t.rep * bias_rep : nullptr;
        float column[TN][16] = {};
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = t.m0 + 32 * i + (t.lane & 31);
            const int y = m < rows ? labels[(long long)t.rep * rows + m] : -1;
            const bool live = (unsigned)y < (unsigned)classes;
            const float l = live ? lse[(long long)t.rep * rows + m] : 0.f;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = t.n0 + 32 * j + 8 * q + 4 * (t.lane >> 5);
                    if (n >= ld) continue;
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = c0 + n + e;
                        v[e] = live && c < classes ? exp_down<EXACT>(t.acc[i][j][4 * q + e] + (b ? b[c] : 0.f) - l) - (c == y ? 1.f : 0.f) : 0.f;
                        column[j][4 * q + e] += v[e];
                    }
                    if (m >= rows) continue;
                    T* out = g + ((long long)t.rep * rows + m) * ld + n;
                    if (sizeof(T) == 4) *(f4*)out = f4{v[0], v[1], v[2], v[3]};
                    else *(u2*)out = u2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
                }
        }
        if (!sums) return;
        float* out = sums + ((long long)t.rep * blocks + t.m0 / (32 * TM)) * ld;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float v = column[j][e];
#pragma unroll
                for (int d = 1; d < 32; d *= 2) v += __shfl_xor(v, d);
                const int n = t.n0 + 32 * j + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4;
                if ((t.lane & 31) == 0 && n < ld) out[n] = v;
            }
    }
};

// db of a piece: the row blocks' sums in ascending order
__global__ __launch_bounds__(256) void bias_grad_kernel(const float* sums, int blocks, int ld, int c0, int cols, const float* factor, float* db, long long rep)
{
    const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.y;
    if (c >= cols) return;
    float v = 0.f;
    for (int b = 0; b < blocks; ++b) v += sums[((long long)k * blocks + b) * ld + c];
    db[k * rep + c0 + c] = v * factor[k];
}

// dx: the shares of the contraction in ascending order; zero for a row without a label
template <typename T>
__global__ __launch_bounds__(256) void input_grad_kernel(const float* share, int splits, int replicas, int rows, int cols, int ld, Labelled live,
                                                         const float* factor, T* dx, long long rep, long long row)
{
    const int k = blockIdx.z, t = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x;
    if (c >= cols) return;
    const long long at = ((long long)k * rows + t) * ld + c, step = (long long)replicas * rows * ld;
    float v = 0.f;
    for (int s = 0; s < splits; ++s) v += share[s * step + at];
    live.labels += (long long)k * rows;
    dx[k * rep + t * row + c] = (T)(live.at(t) ? v * factor[k] : 0.f);
}

struct Plan {
    bool small;                    // 32 x 128 tiles instead of 128 x 128
    int parts, piece, pieces, blocks, splits, split_len, ldx;
    size_t lse, z_label, row_loss, factor, part, g, sums, share, total;
};
constexpr long long kPieceBytes = 256ll << 20;

int up_to(long long v, int unit) { return (int)((v + unit - 1) / unit * unit); }

Plan plan_of(int n, int rows, int features, int classes, int bf16, bool grad)
{
    Plan p{};
    p.small = rows <= 32;
    const int bm = p.small ? 32 : 128, wave_n = p.small ? 32 : 64, wave_m = p.small ? 32 : 64;
    p.parts = up_to(classes, 128) / wave_n;
    p.blocks = up_to(rows, bm) / wave_m;
    const long long lines = (long long)n * rows, es = bf16 ? 2 : 4;
    const long long most = std::max<long long>(1024, kPieceBytes / std::max<long long>(1, lines * es) / 128 * 128);
    p.pieces = (int)((classes + most - 1) / most);
    p.piece = up_to((classes + p.pieces - 1) / p.pieces, 128);
    p.pieces = (classes + p.piece - 1) / p.piece;
    p.ldx = up_to(features, 4);
    const long long tiles = (long long)n * ((rows + bm - 1) / bm) * ((features + 127) / 128);
    p.splits = (int)std::max<long long>(1, std::min<long long>(512 / std::max<long long>(1, tiles), p.piece / 512));
    p.split_len = up_to((p.piece + p.splits - 1) / p.splits, 128);
    p.splits = (p.piece + p.split_len - 1) / p.split_len;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    p.lse = take((size_t)lines * 4);
    p.z_label = take((size_t)lines * 4);
    p.row_loss = take((size_t)lines * 4);
    p.factor = take((size_t)n * 4);
    p.part = take((size_t)lines * p.parts * 8);
    if (grad) {
        p.g = take((size_t)lines * p.piece * es);
        p.sums = take((size_t)n * p.blocks * p.piece * 4);
        p.share = take((size_t)p.splits * lines * p.ldx * 4);
    }
    p.total = at;
    return p;
}

template <class S> S source(const Rows& r, int rows, int cols, bool vec, Labelled live = {nullptr, 0})
{
    typedef decltype(S::p) P;
    return S{(P)r.p, r.rep, r.row, rows, cols, vec, live};
}

template <class S, typename T, int BM, int BN, int WM, int WN> hipError_t run(const LossArgs& a, const Plan& p, hipStream_t s)
{
    constexpr bool exact = sizeof(T) == 4;
    char* work = (char*)a.work;
    float *lse = (float*)(work + p.lse), *z_label = (float*)(work + p.z_label), *factor = (float*)(work + p.factor);
    float* row_loss = a.row_loss ? a.row_loss : (float*)(work + p.row_loss);
    float2* part = (float2*)(work + p.part);
    hipError_t e = hipSuccess;
    const S x = source<S>(a.x, a.rows, a.features, chunked(a.x, a.bf16, a.features));
    const S w = source<S>(a.w, a.features, a.classes, chunked(a.w, a.bf16, a.classes));
    const float* bias = (const float*)a.bias.p;
    if (a.rows) {
        const Statistics<exact> stats{bias, a.bias.rep, a.labels, part, z_label, a.rows, a.classes, p.parts};
        e = launch_product<BM, BN, WM, WN, true, false>(x, w, a.n, a.rows, a.classes, a.features, 1, a.features, stats, s);
        if (e != hipSuccess) return e;
        int per = 256;
        while (per > 4 && per / 2 >= a.rows) per /= 2;
        while (per > 32 && p.parts >= 512 / per) per /= 2;
        const int shares = 256 / per;
        row_loss_kernel<<<dim3((unsigned)((a.rows + per - 1) / per), (unsigned)a.n), 256, 0, s>>>(part, z_label, a.labels, a.rows, a.classes, p.parts,
                                                                                               shares, lse, row_loss);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    mean_loss_kernel<<<(unsigned)a.n, 256, 0, s>>>(row_loss, a.labels, a.rows, a.classes, a.loss, factor);
    if ((e = hipGetLastError()) != hipSuccess || !a.grad) return e;
    T* g = (T*)(work + p.g);
    float *sums = (float*)(work + p.sums), *share = (float*)(work + p.share);
    const Labelled live{a.labels, a.classes};
    for (int i = 0; i < p.pieces; ++i) {
        const int c0 = i * p.piece, cols = std::min(p.piece, a.classes - c0), ld = up_to(cols, 128);
        Rows wr = a.w;
        wr.p = (T*)a.w.p + c0;
        const S wp = source<S>(wr, a.features, cols, chunked(wr, a.bf16, cols));
        const Rows gr{g, (long long)a.rows * ld, ld};
        const S gs = source<S>(gr, a.rows, ld, true);          // zero beyond cols
        if (a.rows) {
            const Gradient<exact, T> grad{bias, a.bias.rep, a.labels, lse, g, a.db.p ? sums : nullptr, a.rows, c0, a.classes, ld, p.blocks};
            e = launch_product<BM, BN, WM, WN, true, false>(x, wp, a.n, a.rows, cols, a.features, 1, a.features, grad, s);
            if (e != hipSuccess) return e;
        }
        if (a.dx.p && a.rows) {
            const StoreShare store{share, a.rows, a.features, p.ldx, a.n, i > 0};
            e = launch_product<BM, BN, WM, WN, true, true>(gs, wp, a.n, a.rows, a.features, cols, p.splits, p.split_len, store, s);
            if (e != hipSuccess) return e;
        }
        if (a.dw.p) {
            const StoreTile<T> store{(T*)a.dw.p + c0, a.dw.rep, a.dw.row, factor, a.features, cols};
            const S xl = source<S>(a.x, a.rows, a.features, x.vec, live);
            e = launch_product<128, 128, 2, 2, false, false>(xl, gs, a.n, a.features, cols, a.rows, 1, std::max(1, a.rows), store, s);
            if (e != hipSuccess) return e;
        }
        if (a.db.p) {
            bias_grad_kernel<<<dim3((unsigned)((cols + 255) / 256), (unsigned)a.n), 256, 0, s>>>(sums, a.rows ? p.blocks : 0, ld, c0, cols, factor,
                                                                                                  (float*)a.db.p, a.db.rep);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    if (a.dx.p && a.rows) {
        input_grad_kernel<T><<<dim3((unsigned)a.rows, (unsigned)((a.features + 255) / 256), (unsigned)a.n), 256, 0, s>>>(
            share, p.splits, a.n, a.rows, a.features, p.ldx, live, factor, (T*)a.dx.p, a.dx.rep, a.dx.row);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t loss_work_bytes(int n, int rows, int features, int classes, int bf16, bool grad)
{
    return plan_of(n, rows, features, classes, bf16, grad).total;
}

hipError_t launch_loss(const LossArgs& a, hipStream_t s)
{
    const Plan p = plan_of(a.n, a.rows, a.features, a.classes, a.bf16, a.grad);
    if (a.bf16) return p.small ? run<SourceBf16, __bf16, 32, 128, 1, 4>(a, p, s) : run<SourceBf16, __bf16, 128, 128, 2, 2>(a, p, s);
    return p.small ? run<SourceF32, float, 32, 128, 1, 4>(a, p, s) : run<SourceF32, float, 128, 128, 2, 2>(a, p, s);
}

}  // namespace head
}  // namespace hadfl
