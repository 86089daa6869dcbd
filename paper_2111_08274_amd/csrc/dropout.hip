// Dropout with an optional residual: y = r + x D, D = scale where the value stays and 0 elsewhere, a dropped value whatever it holds.  The
// mask is drawn again wherever it is needed, from the counter of the value's place: the gradient is the same call on dy.  A chunk of eight values a
// thread takes one Philox; sixteen bits a value, so that the twenty wide multiplications hide behind the chunk's bytes.  Bound by memory: 16 x 2048 x
// 4096 bf16 onto a residual, and its gradient, 1.34 GB in 269 us = 5.0 TB/s (a copy reaches 4.7).
#include "layer.h"

namespace hadfl {
namespace layer {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, long long xrep, long long xrow, const T* res, long long rrep, long long rrow, T* y,
                                                      long long yrep, long long yrow, int rows, int cols, int chunks, long long total, Draws d)
{
    const long long at = head::line_block() * 256 + threadIdx.x;    // (replica, row, chunk of eight)
    if (at >= total) return;
    const long long line = at / chunks;
    const int c = (int)(at - line * chunks) * 8, k = (int)(line / rows), t = (int)(line - (long long)k * rows);
    Chunk<T> in, add;
    in.load(x + k * xrep + t * xrow + c, cols - c);
    if (res) add.load(res + k * rrep + t * rrow + c, cols - c);
    float v[8], r[8];
    in.get(v);
    if (d.limit) kept8(d, call_of(d), k, t, c, [&](int e, bool kept) { v[e] = kept ? v[e] * d.scale : 0.f; });
    if (res) {
        add.get(r);
        each8([&](int e) { v[e] += r[e]; });
    }
    head::store_chunk(y + k * yrep + t * yrow + c, cols - c, v);
}

template <typename T> hipError_t run(int n, int rows, int cols, const Rows& x, const Rows& r, const Rows& y, const Draws& d, hipStream_t s)
{
    const int chunks = (cols + 7) / 8;
    const long long total = (long long)n * rows * chunks;
    if (total == 0) return hipSuccess;
    dropout_kernel<T><<<head::line_grid((total + 255) / 256, 256), 256, 0, s>>>((const T*)x.p, x.rep, x.row, (const T*)r.p, r.rep, r.row, (T*)y.p, y.rep, y.row,
                                                                                rows, cols, chunks, total, d);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int n, int rows, int cols, int bf16, const Rows& x, const Rows& residual, const Rows& y, const Draws& d, hipStream_t s)
{
    return bf16 ? run<__bf16>(n, rows, cols, x, residual, y, d, s) : run<float>(n, rows, cols, x, residual, y, d, s);
}

}  // namespace layer
}  // namespace hadfl
