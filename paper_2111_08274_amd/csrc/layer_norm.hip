// Layer norm of rows, forward and backward, grouped over replicas.
//   forward   mean, then the mean of the squared distances from it (two passes over registers: no cancellation), y
//   backward  with xh = (x - mean) * rstd and g = dy * gamma: two means over the row, mean(g) and mean(g * xh), give dx; the
//             parameter sums dgamma = sum_t dy * xh, dbeta = sum_t dy stay in registers while a thread walks down its
//             rows (a thread keeps its columns), and one partial per workgroup is added up by a second, small launch in
//             ascending order: no atomics, the same bits every time.
// Memory bound: a row is read once into registers (NL lanes, 8 * CH values a lane), both passes run there.
#include "head.h"

namespace hadfl {
namespace head {

namespace {

// lanes per row and chunks of eight values a lane; VEC: chunks of consecutive values from 16-byte aligned rows, else lane i
// holds the columns i, i + NL, ... (unaligned rows in whole cache lines all the same)
template <int NL, bool VEC> __device__ __forceinline__ int column(int lane, int i, int e)
{
    return VEC ? (i * NL + lane) * 8 + e : (i * 8 + e) * NL + lane;
}

template <typename T, int NL, int CH, bool VEC>
__device__ __forceinline__ void load_row(const T* row, int lane, int cols, float (&v)[CH][8])
{
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (VEC) {
            if (column<NL, VEC>(lane, i, 0) < cols) load8(row + column<NL, VEC>(lane, i, 0), v[i]);
            else for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) { const int c = column<NL, VEC>(lane, i, e); v[i][e] = c < cols ? up(row[c]) : 0.f; }
        }
    }
}
template <int NL, int CH, bool VEC>
__device__ __forceinline__ void load_kept(const Packed& kept, long long line, int lane, int cols, float (&v)[CH][8])
{
    const int8_t* q = kept.q + line * kept.cols;
    const uint8_t* exps = kept.e + line * (kept.cols / kGroup);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (VEC) {
            const int c = column<NL, VEC>(lane, i, 0);
            if (c < cols) {
                const tiles::u2 w = *(const tiles::u2*)(q + c);
                const float unit = group_unit(exps[c / kGroup]);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = (float)(int)(int8_t)(w[e / 4] >> (8 * (e % 4))) * unit;
            } else for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = column<NL, VEC>(lane, i, e);
                v[i][e] = c < cols ? (float)(int)q[c] * group_unit(exps[c / kGroup]) : 0.f;
            }
        }
    }
}
template <typename T, int NL, int CH, bool VEC>
__device__ __forceinline__ void store_row(T* row, int lane, int cols, const float (&v)[CH][8])
{
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (VEC) {
            if (column<NL, VEC>(lane, i, 0) < cols) store8(row + column<NL, VEC>(lane, i, 0), v[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) { const int c = column<NL, VEC>(lane, i, e); if (c < cols) row[c] = (T)v[i][e]; }
        }
    }
}
// parameter vectors have no alignment of their own: gamma may start anywhere in a parameter row
template <int NL, int CH, bool VEC>
__device__ __forceinline__ void load_param(const float* p, int lane, int cols, float (&v)[CH][8])
{
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) { const int c = column<NL, VEC>(lane, i, e); v[i][e] = c < cols ? p[c] : 0.f; }
}

// sums of two values over the NL lanes of a row, to all of them; NL = 256: the whole workgroup, through LDS in two slots used
// in turn, so that one barrier a sum is enough
template <int NL> struct RowSum {
    float (*slot)[4][2];
    int turn = 0;
    __device__ __forceinline__ void add(float& a, float& b)
    {
#pragma unroll
        for (int d = 1; d < (NL < 64 ? NL : 64); d *= 2) { a += __shfl_xor(a, d); b += __shfl_xor(b, d); }
        if (NL == 256) {
            const int w = threadIdx.x / 64;
            if ((threadIdx.x & 63) == 0) { slot[turn][w][0] = a; slot[turn][w][1] = b; }
            __syncthreads();
            a = (slot[turn][0][0] + slot[turn][1][0]) + (slot[turn][2][0] + slot[turn][3][0]);
            b = (slot[turn][0][1] + slot[turn][1][1]) + (slot[turn][2][1] + slot[turn][3][1]);
            turn ^= 1;
        }
    }
};

template <typename T, int NL, int CH, bool VEC>
__global__ __launch_bounds__(256) void norm_forward_kernel(NormArgs a)
{
    constexpr int RPB = 256 / NL;                              // rows a workgroup works on at once
    __shared__ float slot[2][4][2];
    const int lane = threadIdx.x % NL, k = blockIdx.y, step = gridDim.x * RPB;
    float g[CH][8], b[CH][8];
    load_param<NL, CH, VEC>((const float*)a.gamma.p + k * a.gamma.rep, lane, a.cols, g);
    load_param<NL, CH, VEC>((const float*)a.beta.p + k * a.beta.rep, lane, a.cols, b);
    RowSum<NL> sum{slot};
    const float inv = 1.f / (float)a.cols;
    for (int t = blockIdx.x * RPB + threadIdx.x / NL; t < a.rows; t += step) {
        float v[CH][8], m = 0.f, q = 0.f, none = 0.f;
        load_row<T, NL, CH, VEC>((const T*)a.x.p + k * a.x.rep + t * a.x.row, lane, a.cols, v);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m += v[i][e];
        sum.add(m, none);
        m *= inv;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] = column<NL, VEC>(lane, i, e) < a.cols ? v[i][e] - m : 0.f;
                q += v[i][e] * v[i][e];
            }
        sum.add(q, none);
        const float r = 1.f / __builtin_sqrtf(q * inv + a.eps);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * r * g[i][e] + b[i][e];
        store_row<T, NL, CH, VEC>((T*)a.y.p + k * a.y.rep + t * a.y.row, lane, a.cols, v);
        if (lane == 0 && a.mean) { a.mean[(long long)k * a.rows + t] = m; a.rstd[(long long)k * a.rows + t] = r; }
    }
}

template <typename T, bool KEPT, int NL, int CH, bool VEC>
__global__ __launch_bounds__(256) void norm_backward_kernel(NormArgs a, float* partial)
{
    constexpr int RPB = 256 / NL;
    __shared__ float slot[2][4][2];
    __shared__ float parts[NL == 256 ? 1 : 256][17];           // 17: the sums below read a column of it
    const int lane = threadIdx.x % NL, k = blockIdx.y, step = gridDim.x * RPB;
    float g[CH][8], sg[CH][8] = {}, sb[CH][8] = {};
    load_param<NL, CH, VEC>((const float*)a.gamma.p + k * a.gamma.rep, lane, a.cols, g);
    RowSum<NL> sum{slot};
    const float inv = 1.f / (float)a.cols;
    for (int t = blockIdx.x * RPB + threadIdx.x / NL; t < a.rows; t += step) {
        const long long line = (long long)k * a.rows + t;
        float v[CH][8], d[CH][8], m1 = 0.f, m2 = 0.f;
        load_row<T, NL, CH, VEC>((const T*)a.dy.p + k * a.dy.rep + t * a.dy.row, lane, a.cols, d);
        if (KEPT) load_kept<NL, CH, VEC>(a.kept, line, lane, a.cols, v);
        else load_row<T, NL, CH, VEC>((const T*)a.x.p + k * a.x.rep + t * a.x.row, lane, a.cols, v);
        const float m = a.mean[line], r = a.rstd[line];
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = column<NL, VEC>(lane, i, e) < a.cols ? (v[i][e] - m) * r : 0.f;
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
        store_row<T, NL, CH, VEC>((T*)a.dx.p + k * a.dx.rep + t * a.dx.row, lane, a.cols, d);
    }
    // the workgroup's sums: to its partial, or straight to the result where it is the replica's only one
    float* og = partial ? partial + ((long long)k * gridDim.x + blockIdx.x) * 2 * a.cols : (float*)a.dgamma.p + k * a.dgamma.rep;
    float* ob = partial ? og + a.cols : (float*)a.dbeta.p + k * a.dbeta.rep;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (RPB > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) { parts[threadIdx.x][e] = sg[i][e]; parts[threadIdx.x][8 + e] = sb[i][e]; }
            __syncthreads();
        }
        // sixteen sums a lane of the row: spread over all threads
        for (int w = threadIdx.x; w < NL * 16; w += 256) {
            const int l = RPB > 1 ? w / 16 : lane;
            if (RPB > 1) {
                const int e = w % 16, c = column<NL, VEC>(l, i, e & 7);
                float v = 0.f;
#pragma unroll
                for (int j = 0; j < RPB; ++j) v += parts[j * NL + l][e];
                if (c < a.cols) (e < 8 ? og : ob)[c] = v;
            }
        }
        if (RPB == 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = column<NL, VEC>(lane, i, e);
                if (c < a.cols) { og[c] = sg[i][e]; ob[c] = sb[i][e]; }
            }
        }
    }
}

// rows longer than the registers of a workgroup hold: the row is read again for every pass
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
    float m = 0.f, q = 0.f, none = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) m += up(x[c]);
    sum.add(m, none);
    m *= inv;
    for (int c = threadIdx.x; c < a.cols; c += 256) { const float v = up(x[c]) - m; q += v * v; }
    sum.add(q, none);
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

// dgamma, dbeta: the partials of a replica in ascending order, eight shares of them side by side
__global__ __launch_bounds__(256) void norm_sums_kernel(const float* partial, int parts, int cols, Rows dgamma, Rows dbeta)
{
    __shared__ float share[8][32];
    const int k = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x % 32, w = threadIdx.x / 32;      // of both vectors, end to end
    const float* src = partial + (long long)k * parts * 2 * cols + c;
    float v = 0.f;
    if (c < 2 * cols) {
#pragma unroll 8
        for (int p = w; p < parts; p += 8) v += src[(long long)p * 2 * cols];
    }
    share[w][threadIdx.x % 32] = v;
    __syncthreads();
    if (w || c >= 2 * cols) return;
    v = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) v += share[j][threadIdx.x];
    if (c < cols) ((float*)dgamma.p)[k * dgamma.rep + c] = v;
    else ((float*)dbeta.p)[k * dbeta.rep + c - cols] = v;
}

constexpr int kLongest = 8192;     // columns that a workgroup keeps in registers

int lanes_of(int cols) { return cols <= 128 ? 16 : cols <= 2048 ? 64 : 256; }
int chunks_of(int cols) { const int per = lanes_of(cols) * 8; return (cols + per - 1) / per; }

// workgroups per replica: enough to fill the chip four deep, each with whole rows
int groups_of(int n, int rows, int cols)
{
    if (cols > kLongest) return std::max(1, std::min((rows + 15) / 16, std::max(1, 4096 / (n * ((cols + 255) / 256)))));
    const int rpb = 256 / lanes_of(cols);
    return std::max(1, std::min((rows + rpb - 1) / rpb, std::max(1, 1024 / n)));
}

template <typename T, bool VEC> hipError_t forward(const NormArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)groups_of(a.n, a.rows, a.cols), (unsigned)a.n);
#define HADFL_CASE(NL, CH) case NL * 8 + CH: norm_forward_kernel<T, NL, CH, VEC><<<grid, 256, 0, s>>>(a); break;
    switch (lanes_of(a.cols) * 8 + chunks_of(a.cols)) {
        HADFL_CASE(16, 1) HADFL_CASE(64, 1) HADFL_CASE(64, 2) HADFL_CASE(64, 3) HADFL_CASE(64, 4)
        HADFL_CASE(256, 2) HADFL_CASE(256, 3) HADFL_CASE(256, 4)
        default: return hipErrorInvalidValue;
    }
#undef HADFL_CASE
    return hipGetLastError();
}
template <typename T, bool KEPT, bool VEC> hipError_t backward(const NormArgs& a, float* partial, int groups, hipStream_t s)
{
    const dim3 grid((unsigned)groups, (unsigned)a.n);
#define HADFL_CASE(NL, CH) case NL * 8 + CH: norm_backward_kernel<T, KEPT, NL, CH, VEC><<<grid, 256, 0, s>>>(a, partial); break;
    switch (lanes_of(a.cols) * 8 + chunks_of(a.cols)) {
        HADFL_CASE(16, 1) HADFL_CASE(64, 1) HADFL_CASE(64, 2) HADFL_CASE(64, 3) HADFL_CASE(64, 4)
        HADFL_CASE(256, 2) HADFL_CASE(256, 3) HADFL_CASE(256, 4)
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
        const bool vec = chunked(a.dy, a.bf16, a.cols) && chunked(a.dx, a.bf16, a.cols) && (KEPT || chunked(a.x, a.bf16, a.cols));
        if (groups == 1) partial = nullptr;
        e = vec ? backward<T, KEPT, true>(a, partial, groups, s) : backward<T, KEPT, false>(a, partial, groups, s);
        if (e != hipSuccess || groups == 1) return e;
    }
    norm_sums_kernel<<<dim3((unsigned)((2 * a.cols + 31) / 32), (unsigned)a.n), 256, 0, s>>>(partial, groups, a.cols, a.dgamma, a.dbeta);
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
    const bool vec = chunked(a.x, a.bf16, a.cols) && chunked(a.y, a.bf16, a.cols);
    if (a.bf16) return vec ? forward<__bf16, true>(a, s) : forward<__bf16, false>(a, s);
    return vec ? forward<float, true>(a, s) : forward<float, false>(a, s);
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s)
{
    if (a.bf16) return a.kept.q ? backward_any<__bf16, true>(a, s) : backward_any<__bf16, false>(a, s);
    return a.kept.q ? backward_any<float, true>(a, s) : backward_any<float, false>(a, s);
}

}  // namespace head
}  // namespace hadfl
