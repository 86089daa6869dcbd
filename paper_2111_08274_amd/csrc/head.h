// Operators of a language model's head (layer norm, 8-bit checkpoints, loss over a large vocabulary): launch wrappers and
// the pieces that their kernels share.
#pragma once
#include <algorithm>

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

// A line of workgroups as a grid whose rows have fewer than 2^32 threads, which is what one dimension of a launch may have, and whole turns of the
// chip's eight dies.
inline dim3 line_grid(long long blocks, int threads)
{
    const long long row = std::min(blocks, 0xffffffffll / threads / tiles::kDies * tiles::kDies);
    return dim3((unsigned)row, (unsigned)((blocks + row - 1) / row));
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
// few rows: logits [replicas][rows][ld], ld a multiple of 128, from the shares of their contraction (into the first one's place), their
// statistics per 128 classes (part [replicas][tiles][rows]: the largest logit and the sum of exp of the distances to it), the labels' logits
hipError_t launch_join_logits(const LossArgs& a, float* share, int splits, int ld, float2* part, float* z_label, hipStream_t s);
// dW from G [replicas][rows][ld], at most kFewWeights rows, at least four classes
constexpr int kFewWeights = 8;
template <typename T> hipError_t launch_few_weights(const LossArgs& a, const T* g, int ld, const float* factor, hipStream_t s);

// ---- device pieces ------------------------------------------------------------------------------------------------
// this workgroup's place in the line of line_grid()
__device__ __forceinline__ long long line_block() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }
__device__ __forceinline__ float up(__bf16 v) { return (float)v; }
__device__ __forceinline__ float up(float v) { return v; }
// Eight consecutive values of a row, as they are in memory.  Vector accesses need no alignment of their own on this chip (a chunk
// across a line's end is two accesses), so rows of any stride are read 16 bytes a lane; only a row's last chunk may hold fewer values.
typedef unsigned int u4any __attribute__((ext_vector_type(4), aligned(2)));
// said to be in global memory: a pointer chosen between two would else be loaded through the path that also serves LDS, whose loads are
// only waited for all together
__device__ __forceinline__ tiles::u4 load16(const void* p) { return *(const __attribute__((address_space(1))) u4any*)(unsigned long long)p; }
template <typename T> struct Chunk;
// keeps a short chunk's eight comparisons where they are used: hoisted out of a loop over rows they would fill the scalar registers
__device__ __forceinline__ int here(int left) { asm volatile("" : "+v"(left)); return left; }
template <> struct Chunk<float> {
    tiles::u4 a, b;
    __device__ __forceinline__ void load(const float* p, int left)
    {
        if (left >= 8) { a = load16(p); b = load16(p + 4); return; }
        a = b = tiles::u4{0, 0, 0, 0};
        const unsigned* w = (const unsigned*)p;
        left = here(left);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) { if (e < 4) a[e] = w[e]; else b[e - 4] = w[e]; }
    }
    __device__ __forceinline__ void get(float* v) const
    {
        const tiles::f4 low = __builtin_bit_cast(tiles::f4, a), high = __builtin_bit_cast(tiles::f4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = low[e]; v[4 + e] = high[e]; }
    }
};
template <> struct Chunk<__bf16> {
    tiles::u4 a;
    __device__ __forceinline__ void load(const __bf16* p, int left)
    {
        if (left >= 8) { a = load16(p); return; }
        a = tiles::u4{0, 0, 0, 0};
        const unsigned short* w = (const unsigned short*)p;
        left = here(left);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) a[e / 2] |= (unsigned)w[e] << (16 * (e % 2));
    }
    __device__ __forceinline__ void get(float* v) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __builtin_bit_cast(float, a[e] << 16);
            v[2 * e + 1] = __builtin_bit_cast(float, a[e] & 0xffff0000u);
        }
    }
};
__device__ __forceinline__ void store_chunk(float* p, int left, const float* v)
{
    if (left >= 8) {
        *(u4any*)p = __builtin_bit_cast(tiles::u4, (tiles::f4{v[0], v[1], v[2], v[3]}));
        *(u4any*)(p + 4) = __builtin_bit_cast(tiles::u4, (tiles::f4{v[4], v[5], v[6], v[7]}));
        return;
    }
    left = here(left);
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < left) p[e] = v[e];
}
__device__ __forceinline__ void store_chunk(__bf16* p, int left, const float* v)
{
    if (left >= 8) {
        *(u4any*)p = tiles::u4{tiles::to_bf16x2(v[0], v[1]), tiles::to_bf16x2(v[2], v[3]), tiles::to_bf16x2(v[4], v[5]), tiles::to_bf16x2(v[6], v[7])};
        return;
    }
    left = here(left);
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < left) p[e] = (__bf16)v[e];
}
// The value of another lane, such that after the steps 1, 2, 4, ... N / 2 of  v = f(v, other<step>(v))  all lanes of a group of N hold f over
// the group: within 16 lanes by moves that the arithmetic instruction does on the way (a mirror in place of an exchange: both halves hold their
// own total by then), beyond by the exchange of lane rows; neither takes the way through LDS that a general shuffle does.
template <int STEP> __device__ __forceinline__ float other(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    if constexpr (STEP == 16) {
        const auto w = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return __builtin_bit_cast(float, (threadIdx.x & 16) ? w[0] : w[1]);
    } else if constexpr (STEP == 32) {
        const auto w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return __builtin_bit_cast(float, (threadIdx.x & 32) ? w[0] : w[1]);
    } else {
        constexpr int kMove = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;     // quads 1032, 2301, mirrors of 8 and 16 lanes
        return __builtin_bit_cast(float, (unsigned)__builtin_amdgcn_update_dpp(0, (int)u, kMove, 0xf, 0xf, true));
    }
}
template <int N> __device__ __forceinline__ float sum_over(float v)
{
    if constexpr (N > 1) v += other<1>(v);
    if constexpr (N > 2) v += other<2>(v);
    if constexpr (N > 4) v += other<4>(v);
    if constexpr (N > 8) v += other<8>(v);
    if constexpr (N > 16) v += other<16>(v);
    if constexpr (N > 32) v += other<32>(v);
    return v;
}
template <int N> __device__ __forceinline__ float max_over(float v)
{
    if constexpr (N > 1) v = __builtin_fmaxf(v, other<1>(v));
    if constexpr (N > 2) v = __builtin_fmaxf(v, other<2>(v));
    if constexpr (N > 4) v = __builtin_fmaxf(v, other<4>(v));
    if constexpr (N > 8) v = __builtin_fmaxf(v, other<8>(v));
    if constexpr (N > 16) v = __builtin_fmaxf(v, other<16>(v));
    if constexpr (N > 32) v = __builtin_fmaxf(v, other<32>(v));
    return v;
}
// 2^e of a group from its stored byte; 255 gives infinity, whose product with the group's zeros is the NaN it stands for
__device__ __forceinline__ float group_unit(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

}  // namespace head
}  // namespace hadfl
