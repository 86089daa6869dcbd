// Operators of a language model's head (layer norm, 8-bit checkpoints, loss over a large vocabulary): launch wrappers and
// the pieces that their kernels share.
#pragma once
#include "hadfl_internal.h"
#include "mfma_tiles.h"

namespace hadfl {
namespace head {

struct Rows {                      // hadfl_rows, typed by the kernel that takes it
    void* p;
    long long rep, row;
};
inline Rows rows_of(const hadfl_rows* r) { return r ? Rows{r->data, r->replica_stride, r->row_stride} : Rows{nullptr, 0, 0}; }
// every row starts on 16 bytes and holds whole chunks of eight values
inline bool chunked(const Rows& r, int bf16, long long cols)
{
    const long long unit = bf16 ? 8 : 4;
    return ((uintptr_t)r.p & 15) == 0 && r.rep % unit == 0 && r.row % unit == 0 && cols % 8 == 0;
}

constexpr int kGroup = 32;         // values of a row that share an exponent
inline long long packed_cols(long long cols) { return (cols + kGroup - 1) / kGroup * kGroup; }
inline size_t align256(size_t n) { return (n + 255) / 256 * 256; }
struct Packed {                    // an 8-bit checkpoint: int8 [rows][cols rounded up], then exponents + 127
    const int8_t* q;
    const uint8_t* e;
    long long cols;                // rounded up
};
inline Packed packed_of(const void* p, long long rows, long long cols)
{
    const long long f = packed_cols(cols);
    return Packed{(const int8_t*)p, (const uint8_t*)p + align256((size_t)(rows * f)), f};
}
inline size_t packed_bytes(long long rows, long long cols)
{
    const long long f = packed_cols(cols);
    return align256((size_t)(rows * f)) + align256((size_t)(rows * (f / kGroup)));
}

// ---- layer norm ---------------------------------------------------------------------------------------------------
struct NormArgs {
    int n, rows, cols, bf16;
    float eps;
    Rows x, gamma, beta, y, dy, dx, dgamma, dbeta;
    float *mean, *rstd, *work;
    Packed kept;                   // q null: x from its tensor
};
size_t norm_work_bytes(int n, int rows, int cols);
hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s);

// ---- 8-bit checkpoints --------------------------------------------------------------------------------------------
hipError_t launch_pack(int n, int rows, int cols, int bf16, const Rows& x, void* packed, hipStream_t s);
hipError_t launch_unpack(int n, int rows, int cols, int bf16, const void* packed, const Rows& out, hipStream_t s);

// ---- dense layer: parameter gradients from a checkpoint ----------------------------------------------------------
struct DenseArgs {
    int n, rows, in, out, bf16;
    Packed x;
    Rows dy, dw, db;
    void* work;
};
size_t dense_work_bytes(int n, int rows, int in, int out, int bf16);
hipError_t launch_dense_grad(const DenseArgs& a, hipStream_t s);

// ---- loss over a large vocabulary ---------------------------------------------------------------------------------
struct LossArgs {
    int n, rows, features, classes, bf16;
    Rows x, w, bias, dx, dw, db;
    const int32_t* labels;
    float *loss, *row_loss;
    bool grad;
    void* work;
};
size_t loss_work_bytes(int n, int rows, int features, int classes, int bf16, bool grad);
hipError_t launch_loss(const LossArgs& a, hipStream_t s);

// ---- device pieces ------------------------------------------------------------------------------------------------
__device__ __forceinline__ float up(__bf16 v) { return (float)v; }
__device__ __forceinline__ float up(float v) { return v; }

// eight consecutive values from an address of 16 bytes' alignment
__device__ __forceinline__ void load8(const float* p, float* v)
{
    const tiles::f4 a = *(const tiles::f4*)p, b = *(const tiles::f4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
}
__device__ __forceinline__ void load8(const __bf16* p, float* v)
{
    const tiles::u4 a = *(const tiles::u4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __builtin_bit_cast(float, a[e] << 16);
        v[2 * e + 1] = __builtin_bit_cast(float, a[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store8(float* p, const float* v)
{
    *(tiles::f4*)p = tiles::f4{v[0], v[1], v[2], v[3]};
    *(tiles::f4*)(p + 4) = tiles::f4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(__bf16* p, const float* v)
{
    *(tiles::u4*)p = tiles::u4{tiles::to_bf16x2(v[0], v[1]), tiles::to_bf16x2(v[2], v[3]), tiles::to_bf16x2(v[4], v[5]),
                               tiles::to_bf16x2(v[6], v[7])};
}
// 2^e of a group from its stored byte; 255 gives infinity, whose product with the group's zeros is the NaN it stands for
__device__ __forceinline__ float group_unit(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

}  // namespace head
}  // namespace hadfl
