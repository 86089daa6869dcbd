// The loss over a large vocabulary for few rows (a token, a small batch), where what counts is to stream W and dW.
//   logits   where W has many features for its classes it is contracted in shares (one workgroup a column of tiles would walk down all of
//            its features: 4096 x 10007 fp32, one row, 142 us against 42); the shares are added here
//   dW       up to eight rows by plain multiply-adds in 32 bits: a lane holds G of its classes for all rows and writes one feature after
//            another, whole lines at a time, with no operand brought into a matrix instruction's layout
#include "head.h"

namespace hadfl {
namespace head {

using namespace tiles;

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
typedef unsigned int u2any __attribute__((ext_vector_type(2), aligned(2)));

// four consecutive values as they are in memory
template <typename T> struct Four;
template <> struct Four<float> {
    u4 v;
    __device__ __forceinline__ void load(const float* p) { v = *(const u4any*)p; }
    __device__ __forceinline__ f4 get() const { return __builtin_bit_cast(f4, v); }
    static __device__ __forceinline__ void store(float* p, const f4& w) { *(u4any*)p = __builtin_bit_cast(u4, w); }
};
template <> struct Four<__bf16> {
    u2 v;
    __device__ __forceinline__ void load(const __bf16* p) { v = *(const u2any*)p; }
    __device__ __forceinline__ f4 get() const
    {
        return __builtin_bit_cast(f4, (u4{v[0] << 16, v[0] & 0xffff0000u, v[1] << 16, v[1] & 0xffff0000u}));
    }
    static __device__ __forceinline__ void store(__bf16* p, const f4& w) { *(u2any*)p = u2{to_bf16x2(w[0], w[1]), to_bf16x2(w[2], w[3])}; }
};

// Logits from the shares of their contraction, [splits][replicas][rows][ld], 128 classes a workgroup, with the bias, into [replicas][rows][ld]
// (the first share's place), and their statistics.  Eight rows a workgroup: 128 rows x 10007 classes in eight shares 8.9 us, latency.
__global__ __launch_bounds__(256) void join_logits_kernel(const float* share, int splits, long long step, const float* bias, long long bias_rep,
                                                          const int32_t* labels, int rows, int classes, int ld, int tiles, float2* part, float* z_label, float* z)
{
    __shared__ float tops[4][4], sums[4][4];
    const int tile = blockIdx.x, k = blockIdx.y, tid = threadIdx.x, lane = tid & 63, pair = tid >> 7, c = tile * 128 + (tid & 127);
    const float b = bias && c < classes ? bias[k * bias_rep + c] : 0.f;
    const int m0 = blockIdx.z * 8;                             // eight rows a workgroup, four a half of it
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const long long at = ((long long)k * rows + min(m0 + 2 * u + pair, rows - 1)) * ld + c;
        v[u] = 0.f;
#pragma unroll 4
        for (int s = 0; s < splits; ++s) v[u] += share[s * step + at];
        v[u] = c < classes ? v[u] + b : -INFINITY;
        const float top = max_over<64>(v[u]);
        if (lane == 0) tops[tid >> 6][u] = top;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const float top = __builtin_fmaxf(tops[2 * pair][u], tops[2 * pair + 1][u]), base = top == -INFINITY ? 0.f : top;
        const float sum = sum_over<64>(__builtin_amdgcn_exp2f((v[u] - base) * kLog2e));
        if (lane == 0) sums[tid >> 6][u] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int m = m0 + 2 * u + pair;
        if (m >= rows) continue;
        const long long line = (long long)k * rows + m;
        z[line * ld + c] = v[u];
        if (c < classes && labels[line] == c) z_label[line] = v[u];
        if ((tid & 127) == 0)
            part[((long long)k * tiles + tile) * rows + m] =
                float2{__builtin_fmaxf(tops[2 * pair][u], tops[2 * pair + 1][u]), sums[2 * pair][u] + sums[2 * pair + 1][u]};
    }
}

// dW of 256 classes and kDepth features a workgroup: a lane holds G of four classes and all rows, and writes the classes' values of one feature
// after another; x, transposed, from LDS, the same address for a wave.  Bound by the stores: 4 x 512 x 32000 fp32, 8 rows, 54 us = 4.8 TB/s (the
// product on the matrix cores 67), bf16 27 us (34); at 16 rows the multiply-adds take as long as the stores, and the product is no slower.
constexpr int kDepth = 32, TR = kFewWeights;
template <typename T>
__global__ __launch_bounds__(256) void few_weights_kernel(const T* x, long long x_rep, long long x_row, const int32_t* labels, const T* g, int ld, int rows,
                                                          int features, int classes, int tiles, int blocks, int total, const float* factor, T* dw,
                                                          long long dw_rep, long long dw_row)
{
    constexpr int P = TR + 4;
    __shared__ __attribute__((aligned(16))) float xs[kDepth][P];
    const unsigned item = blockIdx.y * gridDim.x + logical_block();
    if (item >= (unsigned)total) return;
    const int block = item % blocks, tile = item / blocks % tiles, k = item / blocks / tiles;
    const int tid = threadIdx.x, c = tile * 256 + (tid & 63) * 4, d0 = block * kDepth, count = min(kDepth, features - d0);
    Four<T> four[TR];
#pragma unroll
    for (int t = 0; t < TR; ++t) four[t].load(g + ((long long)k * rows + min(t, rows - 1)) * ld + min(c, ld - 4));
    for (int i = tid; i < kDepth * TR; i += 256) {
        const int t = i / kDepth, d = i % kDepth;
        const bool live = t < rows && (unsigned)labels[(long long)k * rows + min(t, rows - 1)] < (unsigned)classes;
        xs[d][t] = live && d < count ? up(x[k * x_rep + t * x_row + d0 + d]) : 0.f;
    }
    __syncthreads();
    if (c >= classes) return;
    f4 gv[TR];
#pragma unroll
    for (int t = 0; t < TR; ++t) gv[t] = t < rows ? four[t].get() : f4{0.f, 0.f, 0.f, 0.f};
    const float f = factor[k];
    T* out = dw + k * dw_rep + (long long)d0 * dw_row + c;
    for (int d = tid >> 6; d < count; d += 4) {
        f4 v = {};
#pragma unroll
        for (int q = 0; q < TR / 4; ++q) {
            const f4 xv = *(const f4*)&xs[d][4 * q];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(xv[j], gv[4 * q + j][e], v[e]);
        }
        v *= f;
        T* to = out + d * dw_row;
        if (c + 4 <= classes) Four<T>::store(to, v);
        else for (int e = 0; e < 4; ++e) if (c + e < classes) to[e] = (T)v[e];
    }
}

}  // namespace

template <typename T> hipError_t launch_few_weights(const LossArgs& a, const T* g, int ld, const float* factor, hipStream_t s)
{
    const int tiles = (a.classes + 255) / 256, blocks = (a.features + kDepth - 1) / kDepth;
    const long long total = (long long)a.n * tiles * blocks;
    if (total > 0x7fffff00ll) return hipErrorInvalidValue;
    few_weights_kernel<T><<<line_grid(die_grid(total), 256), 256, 0, s>>>((const T*)a.x.p, a.x.rep, a.x.row, a.labels, g, ld, a.rows, a.features, a.classes, tiles, blocks,
                                                          (int)total, factor, (T*)a.dw.p, a.dw.rep, a.dw.row);
    return hipGetLastError();
}
hipError_t launch_join_logits(const LossArgs& a, float* share, int splits, int ld, float2* part, float* z_label, hipStream_t s)
{
    const int tiles = (a.classes + 127) / 128;
    join_logits_kernel<<<dim3((unsigned)tiles, (unsigned)a.n, (unsigned)((a.rows + 7) / 8)), 256, 0, s>>>(
        share, splits, (long long)a.n * a.rows * ld, (const float*)a.bias.p, a.bias.rep, a.labels, a.rows, a.classes, ld, tiles, part, z_label, share);
    return hipGetLastError();
}
template hipError_t launch_few_weights<float>(const LossArgs&, const float*, int, const float*, hipStream_t);
template hipError_t launch_few_weights<__bf16>(const LossArgs&, const __bf16*, int, const float*, hipStream_t);

}  // namespace head
}  // namespace hadfl
