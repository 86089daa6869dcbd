// Parameter gradients of a dense layer whose input was kept in 8 bits: dW = x^T dy with x read straight from the checkpoint,
// db = sum_t dy.  q * 2^e is exact in bf16, so a bf16 dy needs one product and a 32-bit dy, in three bf16 planes, three.
#include "tile_product.h"

namespace hadfl {
namespace head {

namespace {

// column sums of a share of the rows, a thread per column
template <typename T>
__global__ __launch_bounds__(256) void column_sums_kernel(const T* x, long long rep, long long row, int rows, int cols, int per, float* part)
{
    const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.z;
    if (c >= cols) return;
    const int t0 = blockIdx.y * per, t1 = min(rows, t0 + per);
    const T* src = x + k * rep + c;
    float v = 0.f;
#pragma unroll 8
    for (int t = t0; t < t1; ++t) v += up(src[t * row]);
    part[((long long)k * gridDim.y + blockIdx.y) * cols + c] = v;
}
// and the shares in ascending order
__global__ __launch_bounds__(256) void add_shares_kernel(const float* part, int shares, int cols, float* out, long long rep)
{
    const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.y;
    if (c >= cols) return;
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < shares; ++s) v += part[((long long)k * shares + s) * cols + c];
    out[k * rep + c] = v;
}

int shares_of(int n, int rows, int cols)
{
    const int most = std::max(1, 2048 / (n * ((cols + 255) / 256)));
    return std::max(1, std::min(most, (rows + 31) / 32));
}

}  // namespace

size_t dense_work_bytes(int n, int rows, int, int out, int)
{
    return align256((size_t)n * shares_of(n, rows, out) * out * sizeof(float));
}

template <typename T> static hipError_t run(const DenseArgs& a, hipStream_t s)
{
    hipError_t e;
    if (a.db.p) {
        const int shares = shares_of(a.n, a.rows, a.out), per = (a.rows + shares - 1) / shares;
        float* part = (float*)a.work;
        column_sums_kernel<T><<<dim3((unsigned)((a.out + 255) / 256), (unsigned)shares, (unsigned)a.n), 256, 0, s>>>(
            (const T*)a.dy.p, a.dy.rep, a.dy.row, a.rows, a.out, per, part);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        add_shares_kernel<<<dim3((unsigned)((a.out + 255) / 256), (unsigned)a.n), 256, 0, s>>>(part, shares, a.out, (float*)a.db.p, a.db.rep);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const SourcePacked x{a.x, a.rows, a.in};
    const Source<T> dy = source<T>(a.dy, a.rows, a.out);
    const StoreTile<float> store{(float*)a.dw.p, a.dw.rep, a.dw.row, nullptr, a.in, a.out};
    return launch_product<128, 128, 2, 2, false, false>(x, dy, a.n, a.in, a.out, a.rows, 1, std::max(1, a.rows), store, s);
}

hipError_t launch_dense_grad(const DenseArgs& a, hipStream_t s)
{
    return a.bf16 ? run<__bf16>(a, s) : run<float>(a, s);
}

}  // namespace head
}  // namespace hadfl
