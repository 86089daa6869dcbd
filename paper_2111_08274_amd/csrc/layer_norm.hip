// Layer norm of rows, forward and backward, grouped over replicas.
//   forward   mean, then the mean of the squared distances from it (two passes over registers: no cancellation), y
//   backward  with xh = (x - mean) * rstd and g = dy * gamma: two means over the row, mean(g) and mean(g * xh), give dx; the
//             parameter sums dgamma = sum_t dy * xh, dbeta = sum_t dy stay in registers while a thread walks down its
//             rows (a thread keeps its columns), and one partial per workgroup is added up by a second, small launch in
//             ascending order: no atomics, the same bits every time.
// Memory bound: a row is read once into registers (NL lanes, 8 * CH values a lane), both passes run there, and the next row is
// loaded meanwhile.  16 x 4096 x 512 bf16: forward 26 us = 5.2 TB/s, backward 39.5 us = 5.1, the sums' launch 4.6; 4 x 4096 x 4096: 46 us = 5.8 and,
// from the 8-bit checkpoint, 73 us = 4.6; fp32 100 us = 5.4 and 120 us = 5.0.  Few rows are latency: one row of 512 2.1 us.
#include "head.h"

namespace hadfl {
namespace head {

namespace {

// first column of chunk i of a lane
template <int NL> __device__ __forceinline__ int column(int lane, int i) { return (i * NL + lane) * 8; }

// a lane's chunks of a row, as they are in memory: the next row is on its way while one is worked on
template <typename T, int NL, int CH> struct RowOf {
    Chunk<T> chunk[CH];
    __device__ __forceinline__ void load(const T* row, int lane, int cols)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) chunk[i].load(row + column<NL>(lane, i), cols - column<NL>(lane, i));
    }
    __device__ __forceinline__ void get(float (&v)[CH][8]) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) chunk[i].get(v[i]);
    }
};
// the same from an 8-bit checkpoint, whose surplus columns are zero
template <int NL, int CH> struct KeptOf {
    tiles::u2 q[CH];
    unsigned e[CH];
    __device__ __forceinline__ void load(const Packed& kept, long long line, int lane)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = column<NL>(lane, i);
            q[i] = tiles::u2{0, 0};
            e[i] = 1;
            if (c >= kept.cols) continue;
            q[i] = *(const tiles::u2*)(kept.q + line * kept.cols + c);
            e[i] = kept.e[line * (kept.cols / kGroup) + c / kGroup];
        }
    }
    __device__ __forceinline__ void get(float (&v)[CH][8]) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = (float)(int)(int8_t)(q[i][j / 4] >> (8 * (j % 4))) * group_unit(e[i]);
    }
};
// gamma, beta: in memory as any row of floats
template <int NL, int CH>
__device__ __forceinline__ void load_param(const float* p, int lane, int cols, float (&v)[CH][8])
{
    RowOf<float, NL, CH> r;
    r.load(p, lane, cols);
    r.get(v);
}
template <typename T, int NL, int CH>
__device__ __forceinline__ void store_row(T* row, int lane, int cols, const float (&v)[CH][8])
{
#pragma unroll
    for (int i = 0; i < CH; ++i) store_chunk(row + column<NL>(lane, i), cols - column<NL>(lane, i), v[i]);
}

// sums over the NL lanes of a row, to all of them; NL = 256: the whole workgroup, through LDS in two slots used in turn, so that one barrier
// a sum is enough
template <int NL> struct RowSum {
    float (*slot)[4][2];
    int turn = 0;
    __device__ __forceinline__ void add(float& a, float& b)
    {
        constexpr int W = NL < 64 ? NL : 64;
        a = sum_over<W>(a);
        b = sum_over<W>(b);
        if (NL == 256) {
            const int w = threadIdx.x / 64;
            if ((threadIdx.x & 63) == 0) { slot[turn][w][0] = a; slot[turn][w][1] = b; }
            __syncthreads();
            a = (slot[turn][0][0] + slot[turn][1][0]) + (slot[turn][2][0] + slot[turn][3][0]);
            b = (slot[turn][0][1] + slot[turn][1][1]) + (slot[turn][2][1] + slot[turn][3][1]);
            turn ^= 1;
        }
    }
    __device__ __forceinline__ void add(float& a)
    {
        float none = 0.f;
        if (NL == 256) add(a, none);
        else a = sum_over<NL < 64 ? NL : 64>(a);
    }
};

template <typename T, int NL, int CH>
__global__ __launch_bounds__(256) void norm_forward_kernel(NormArgs a)
{
    constexpr int RPB = 256 / NL;                              // rows a workgroup works on at once
    __shared__ float slot[2][4][2];
    const int lane = threadIdx.x % NL, k = blockIdx.y, step = gridDim.x * RPB;
    const T* x = (const T*)a.x.p + k * a.x.rep;
    RowOf<T, NL, CH> next;
    int t = blockIdx.x * RPB + threadIdx.x / NL;
    if (t < a.rows) next.load(x + t * a.x.row, lane, a.cols);
    float g[CH][8], b[CH][8];
    load_param<NL, CH>((const float*)a.gamma.p + k * a.gamma.rep, lane, a.cols, g);
    load_param<NL, CH>((const float*)a.beta.p + k * a.beta.rep, lane, a.cols, b);
    RowSum<NL> sum{slot};
    const float inv = 1.f / (float)a.cols;
    for (; t < a.rows; t += step) {
        float v[CH][8], m = 0.f, q = 0.f;
        next.get(v);
        if (t + step < a.rows) next.load(x + (t + step) * a.x.row, lane, a.cols);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m += v[i][e];
        sum.add(m);
        m *= inv;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] = column<NL>(lane, i) + e < a.cols ? v[i][e] - m : 0.f;
                q += v[i][e] * v[i][e];
            }
        sum.add(q);
        const float r = 1.f / __builtin_sqrtf(q * inv + a.eps);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * r * g[i][e] + b[i][e];
        store_row<T, NL, CH>((T*)a.y.p + k * a.y.rep + t * a.y.row, lane, a.cols, v);
        if (lane == 0 && a.mean) { a.mean[(long long)k * a.rows + t] = m; a.rstd[(long long)k * a.rows + t] = r; }
    }
}

template <typename T, bool KEPT, int NL, int CH>
__global__ __launch_bounds__(256) void norm_backward_kernel(NormArgs a, float* partial)
{
    constexpr int RPB = 256 / NL;
    __shared__ float slot[2][4][2];
    __shared__ float parts[NL == 256 ? 1 : 256][17];           // 17: the sums below read a column of it
    const int lane = threadIdx.x % NL, k = blockIdx.y, step = gridDim.x * RPB;
    const T *x = (const T*)a.x.p + k * a.x.rep, *dy = (const T*)a.dy.p + k * a.dy.rep;
    const long long lines = (long long)k * a.rows;
    RowOf<T, NL, CH> next_d, next_x;
    KeptOf<NL, CH> next_k;
    float next_m = 0.f, next_r = 0.f;
    auto fetch = [&](int t) {
        next_d.load(dy + t * a.dy.row, lane, a.cols);
        if (KEPT) next_k.load(a.kept, lines + t, lane);
        else next_x.load(x + t * a.x.row, lane, a.cols);
        next_m = a.mean[lines + t];
        next_r = a.rstd[lines + t];
    };
    int t = blockIdx.x * RPB + threadIdx.x / NL;
    if (t < a.rows) fetch(t);
    float g[CH][8], sg[CH][8] = {}, sb[CH][8] = {};
    load_param<NL, CH>((const float*)a.gamma.p + k * a.gamma.rep, lane, a.cols, g);
    RowSum<NL> sum{slot};
    const float inv = 1.f / (float)a.cols;
    for (; t < a.rows; t += step) {
        float v[CH][8], d[CH][8], m1 = 0.f, m2 = 0.f;
        const float m = next_m, r = next_r;
        next_d.get(d);
        if (KEPT) next_k.get(v);
        else next_x.get(v);
        if (t + step < a.rows) fetch(t + step);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = column<NL>(lane, i) + e < a.cols ? (v[i][e] - m) * r : 0.f;
                v[i][e] = xh;
                sg[i][e] += d[i][e] * xh;
                sb[i][e] += d[i][e];
                d[i][e] *= g[i][e];
                m1 += d[i][e];
                m2 += d[i][e] * xh;
            }
        sum.add(m1, m2);
        m1 *= inv;
        m2 *= inv;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) d[i][e] = r * (d[i][e] - m1 - v[i][e] * m2);
        store_row<T, NL, CH>((T*)a.dx.p + k * a.dx.rep + t * a.dx.row, lane, a.cols, d);
    }
    // the workgroup's sums: to its partial, or straight to the result where it is the replica's only one
    float* og = partial ? partial + ((long long)k * gridDim.x + blockIdx.x) * 2 * a.cols : (float*)a.dgamma.p + k * a.dgamma.rep;
    float* ob = partial ? og + a.cols : (float*)a.dbeta.p + k * a.dbeta.rep;
    if (RPB == 1) {
        store_row<float, NL, CH>(og, lane, a.cols, sg);
        store_row<float, NL, CH>(ob, lane, a.cols, sb);
        return;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {                             // of the rows side by side, in ascending order
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) { parts[threadIdx.x][e] = sg[i][e]; parts[threadIdx.x][8 + e] = sb[i][e]; }
        __syncthreads();
        for (int w = threadIdx.x; w < NL * 16; w += 256) {
            const int l = w / 16, e = w % 16, c = column<NL>(l, i) + (e & 7);
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < RPB; ++j) s += parts[j * NL + l][e];
            if (c < a.cols) (e < 8 ? og : ob)[c] = s;
        }
    }
}

// Rows longer than the registers of a workgroup hold: the row is read again for every pass, an element a lane and load, from the caches.  A fallback,
// at half the rate of the kernels above and less where there are few rows for the compute units: 2 x 4096 x 8200 bf16 forward 136 us = 2.0 TB/s, backward
// 168 (8192 columns: 43 and 69), fp32 209 and 262 (98 and 116); 1024 x 65536 bf16 224 and 235.
template <typename T>
__global__ __launch_bounds__(256) void norm_forward_long_kernel(NormArgs a)
{
    __shared__ float slot[2][4][2];
    const int k = blockIdx.y, t = blockIdx.x;
    const T* x = (const T*)a.x.p + k * a.x.rep + t * a.x.row;
    T* y = (T*)a.y.p + k * a.y.rep + t * a.y.row;
    const float *g = (const float*)a.gamma.p + k * a.gamma.rep, *b = (const float*)a.beta.p + k * a.beta.rep;
    RowSum<256> sum{slot};
    const float inv = 1.f / (float)a.cols;
    float m = 0.f, q = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) m += up(x[c]);
    sum.add(m);
    m *= inv;
    for (int c = threadIdx.x; c < a.cols; c += 256) { const float v = up(x[c]) - m; q += v * v; }
    sum.add(q);
    const float r = 1.f / __builtin_sqrtf(q * inv + a.eps);
    for (int c = threadIdx.x; c < a.cols; c += 256) y[c] = (T)((up(x[c]) - m) * r * g[c] + b[c]);
    if (threadIdx.x == 0 && a.mean) { a.mean[(long long)k * a.rows + t] = m; a.rstd[(long long)k * a.rows + t] = r; }
}

template <typename T, bool KEPT>
__device__ __forceinline__ float centred(const NormArgs& a, int k, int t, int c, float m, float r)
{
    const long long line = (long long)k * a.rows + t;
    const float x = KEPT ? (float)(int)a.kept.q[line * a.kept.cols + c] * group_unit(a.kept.e[line * (a.kept.cols / kGroup) + c / kGroup])
                         : up(((const T*)a.x.p)[k * a.x.rep + t * a.x.row + c]);
    return (x - m) * r;
}
template <typename T, bool KEPT>
__global__ __launch_bounds__(256) void norm_backward_long_kernel(NormArgs a)
{
    __shared__ float slot[2][4][2];
    const int k = blockIdx.y, t = blockIdx.x;
    const T* dy = (const T*)a.dy.p + k * a.dy.rep + t * a.dy.row;
    T* dx = (T*)a.dx.p + k * a.dx.rep + t * a.dx.row;
    const float* g = (const float*)a.gamma.p + k * a.gamma.rep;
    const float m = a.mean[(long long)k * a.rows + t], r = a.rstd[(long long)k * a.rows + t];
    RowSum<256> sum{slot};
    const float inv = 1.f / (float)a.cols;
    float m1 = 0.f, m2 = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) {
        const float d = up(dy[c]) * g[c];
        m1 += d;
        m2 += d * centred<T, KEPT>(a, k, t, c, m, r);
    }
    sum.add(m1, m2);
    m1 *= inv;
    m2 *= inv;
    for (int c = threadIdx.x; c < a.cols; c += 256)
        dx[c] = (T)(r * (up(dy[c]) * g[c] - m1 - centred<T, KEPT>(a, k, t, c, m, r) * m2));
}
// their parameter sums: a thread per column, a workgroup per column block and share of the rows; runs before the kernel above,
// whose dx may be dy
template <typename T, bool KEPT>
__global__ __launch_bounds__(256) void norm_columns_long_kernel(NormArgs a, float* partial)
{
    const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.z;
    if (c >= a.cols) return;
    float sg = 0.f, sb = 0.f;
    for (int t = blockIdx.y; t < a.rows; t += gridDim.y) {
        const float d = up(((const T*)a.dy.p)[k * a.dy.rep + t * a.dy.row + c]);
        sg += d * centred<T, KEPT>(a, k, t, c, a.mean[(long long)k * a.rows + t], a.rstd[(long long)k * a.rows + t]);
        sb += d;
    }
    float* out = partial + ((long long)k * gridDim.y + blockIdx.y) * 2 * a.cols;
    out[c] = sg;
    out[a.cols + c] = sb;
}

// dgamma, dbeta: the partials of a replica, S shares of them side by side, each in ascending order
template <int S> __global__ __launch_bounds__(256) void norm_sums_kernel(const float* partial, int parts, int cols, Rows dgamma, Rows dbeta)
{
    constexpr int C = 256 / S;
    __shared__ float share[S][C];
    const int k = blockIdx.y, c = blockIdx.x * C + threadIdx.x % C, w = threadIdx.x / C;         // of both vectors, end to end
    const float* src = partial + (long long)k * parts * 2 * cols + c;
    float v = 0.f;
    if (c < 2 * cols) {
#pragma unroll 8
        for (int p = w; p < parts; p += S) v += src[(long long)p * 2 * cols];
    }
    share[w][threadIdx.x % C] = v;
    __syncthreads();
    if (w || c >= 2 * cols) return;
    v = 0.f;
#pragma unroll
    for (int j = 0; j < S; ++j) v += share[j][threadIdx.x];
    if (c < cols) ((float*)dgamma.p)[k * dgamma.rep + c] = v;
    else ((float*)dbeta.p)[k * dbeta.rep + c - cols] = v;
}

constexpr int kLongest = 8192;     // columns that a workgroup keeps in registers

// Lanes of a row.  A wave per row needs no barrier; the backward pass, which holds seven rows' worth of registers, is faster with a workgroup
// per row from 1024 columns on (4 x 4096 x 2048 bf16: 41 us against 52), the forward pass from 1536 (4 x 4096 x 1536 bf16: 17.5 against 25.7 the
// other way).
int lanes_of(int cols, bool backward) { return cols <= 128 ? 16 : cols <= (backward ? 1024 : 1536) ? 64 : 256; }
int chunks_of(int cols, int lanes) { return (cols + lanes * 8 - 1) / (lanes * 8); }

// Workgroups per replica of the backward pass: four for every compute unit, two where their partials are long (2 x 4096 x 8192 bf16: 86 us
// against 100; 4 x 4096 x 1536: 34 against 48 the other way), but fewer where a thread would not have four rows to add up, and then at
// least one for every compute unit.
int groups_of(int n, int rows, int cols)
{
    if (cols > kLongest) return std::max(1, std::min((rows + 15) / 16, std::max(1, 4096 / (n * ((cols + 255) / 256)))));
    const int rpb = 256 / lanes_of(cols, true), all = (rows + rpb - 1) / rpb;
    return std::max(1, std::min(all, std::max(256 / n, std::min((cols > 2048 ? 512 : 1024) / n, all / 4))));
}

template <typename T> hipError_t forward(const NormArgs& a, hipStream_t s)
{
    const int lanes = lanes_of(a.cols, false), rpb = 256 / lanes;
    const dim3 grid((unsigned)std::max(1, std::min((a.rows + rpb - 1) / rpb, std::max(1, 2048 / a.n))), (unsigned)a.n);
#define HADFL_CASE(NL, CH) case NL * 8 + CH: norm_forward_kernel<T, NL, CH><<<grid, 256, 0, s>>>(a); break;
    switch (lanes * 8 + chunks_of(a.cols, lanes)) {
        HADFL_CASE(16, 1) HADFL_CASE(64, 1) HADFL_CASE(64, 2) HADFL_CASE(64, 3) HADFL_CASE(256, 1) HADFL_CASE(256, 2) HADFL_CASE(256, 3) HADFL_CASE(256, 4)
        default: return hipErrorInvalidValue;
    }
#undef HADFL_CASE
    return hipGetLastError();
}
template <typename T, bool KEPT> hipError_t backward(const NormArgs& a, float* partial, int groups, hipStream_t s)
{
    const dim3 grid((unsigned)groups, (unsigned)a.n);
#define HADFL_CASE(NL, CH) case NL * 8 + CH: norm_backward_kernel<T, KEPT, NL, CH><<<grid, 256, 0, s>>>(a, partial); break;
    const int lanes = lanes_of(a.cols, true);
    switch (lanes * 8 + chunks_of(a.cols, lanes)) {
        HADFL_CASE(16, 1) HADFL_CASE(64, 1) HADFL_CASE(64, 2) HADFL_CASE(256, 1) HADFL_CASE(256, 2) HADFL_CASE(256, 3) HADFL_CASE(256, 4)
        default: return hipErrorInvalidValue;
    }
#undef HADFL_CASE
    return hipGetLastError();
}
template <typename T, bool KEPT> hipError_t backward_any(const NormArgs& a, hipStream_t s)
{
    const int groups = groups_of(a.n, a.rows, a.cols);
    float* partial = a.work;
    hipError_t e;
    if (a.cols > kLongest) {
        norm_columns_long_kernel<T, KEPT><<<dim3((unsigned)((a.cols + 255) / 256), (unsigned)groups, (unsigned)a.n), 256, 0, s>>>(a, partial);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (a.rows) norm_backward_long_kernel<T, KEPT><<<dim3((unsigned)a.rows, (unsigned)a.n), 256, 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    } else {
        if (groups == 1) partial = nullptr;
        e = backward<T, KEPT>(a, partial, groups, s);
        if (e != hipSuccess || groups == 1) return e;
    }
    // whole lines of 32 columns, or half lines and twice the workgroups where those would not fill the chip (1 x 4096 x 768: 14 us for the
    // backward pass against 21)
    if ((long long)a.n * 2 * a.cols >= 256 * 32)
        norm_sums_kernel<8><<<dim3((unsigned)((2 * a.cols + 31) / 32), (unsigned)a.n), 256, 0, s>>>(partial, groups, a.cols, a.dgamma, a.dbeta);
    else
        norm_sums_kernel<16><<<dim3((unsigned)((2 * a.cols + 15) / 16), (unsigned)a.n), 256, 0, s>>>(partial, groups, a.cols, a.dgamma, a.dbeta);
    return hipGetLastError();
}

}  // namespace

size_t norm_work_bytes(int n, int rows, int cols)
{
    return align256((size_t)n * groups_of(n, rows, cols) * 2 * cols * sizeof(float));
}

hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    if (a.cols > kLongest) {
        const dim3 grid((unsigned)a.rows, (unsigned)a.n);
        if (a.bf16) norm_forward_long_kernel<__bf16><<<grid, 256, 0, s>>>(a);
        else norm_forward_long_kernel<float><<<grid, 256, 0, s>>>(a);
        return hipGetLastError();
    }
    return a.bf16 ? forward<__bf16>(a, s) : forward<float>(a, s);
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s)
{
    if (a.bf16) return a.kept.q ? backward_any<__bf16, true>(a, s) : backward_any<__bf16, false>(a, s);
    return a.kept.q ? backward_any<float, true>(a, s) : backward_any<float, false>(a, s);
}

}  // namespace head
}  // namespace hadfl
