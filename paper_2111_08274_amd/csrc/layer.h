// Operators of a next-word model's layers and answers (dense layer with its epilogue, dropout, log probabilities of tokens):
// launch wrappers and the pieces that their kernels share.
#pragma once
#include "head.h"
#include "philox.h"

namespace hadfl {
namespace layer {

using head::Chunk;
using head::Packed;
using head::Rows;
using head::rows_of;

// ---- dropout --------------------------------------------------------------------------------------------------------
// What decides which values stay: a value of row r, column j of replica k has the 16 bits j % 8 of Philox at the counter
// (r, j / 8 + 2^16 k, call) and is kept if they are at least `limit`, 65536 times the probability, rounded.  One Philox serves
// eight values; `scale` is one over the share that stays.
struct Draws {
    uint32_t k0, k1;
    unsigned long long call;
    const unsigned long long* counter;                         // on the device, added to call, or null
    unsigned limit;                                            // 0: everything stays
    float scale;
};
inline unsigned drop_limit(float p) { return std::min(65535u, (unsigned)(65536.0 * (double)p + 0.5)); }
inline Draws draws_of(const hadfl_draw* d, float p)
{
    const unsigned limit = drop_limit(p);
    if (!d) return Draws{0, 0, 0, nullptr, limit, 1.f};
    return Draws{(uint32_t)d->seed, (uint32_t)(d->seed >> 32), d->call, (const unsigned long long*)d->counter, limit, 65536.f / (float)(65536u - limit)};
}

// ---- entry points' arguments ------------------------------------------------------------------------------------------
enum Activation { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };
struct LayerArgs {
    int n, rows, in, out, bf16, act;
    Rows x, w, bias, residual, pre, y, dy, dx, dw, db;
    Packed packed;                                             // q null: x from its tensor
    Draws draws;
    void* work;
};
size_t layer_work_bytes(int n, int rows, int in, int out, int bf16, int act, float drop, bool grad);
hipError_t launch_layer_forward(const LayerArgs& a, hipStream_t s);
hipError_t launch_layer_backward(const LayerArgs& a, hipStream_t s);

hipError_t launch_dropout(int n, int rows, int cols, int bf16, const Rows& x, const Rows& residual, const Rows& y, const Draws& d, hipStream_t s);

struct ScoreArgs {
    int n, rows, classes, n_tokens, n_top, bf16;
    Rows logits, dlogits;
    const int32_t* tokens;
    float *logp, *entropy, *stats, *top_logp;
    int32_t* top;
    const float *dlogp, *dentropy;
    void* work;
};
size_t score_work_bytes(int n, int rows, int classes, int n_top, int bf16);
hipError_t launch_scores_forward(const ScoreArgs& a, hipStream_t s);
hipError_t launch_scores_backward(const ScoreArgs& a, hipStream_t s);

// ---- device pieces ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned long long call_of(const Draws& d) { return d.call + (d.counter ? *d.counter : 0ull); }
// which of the eight values from column c (a multiple of eight) stay: f(i, kept)
template <class F> __device__ __forceinline__ void kept8(const Draws& d, unsigned long long call, int k, int r, int c, F&& f)
{
    const U4 o = philox4x32_10(U4{(uint32_t)r, (uint32_t)(c >> 3) + ((uint32_t)k << 16), (uint32_t)call, (uint32_t)(call >> 32)}, d.k0, d.k1);
    const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f(i, (i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu) >= d.limit);
}

// gelu(z) = z s(2u), u = sqrt(2 / pi) (z + 0.044715 z^3), which is z (1 + tanh u) / 2; silu(z) = z s(z); s(t) = 1 / (1 + e^-t).
// The exponent overflows to the limit of either side.
constexpr float kGeluA = 1.5957691216057308f, kGeluB = 0.044715f, kLog2 = 1.44269504088896340736f;
__device__ __forceinline__ float sigmoid(float t) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2 * t)); }
__device__ __forceinline__ float activate(float z, int act)
{
    if (act == kRelu) return z < 0.f ? 0.f : z;                // a NaN stays
    if (act == kGelu) return z * sigmoid(kGeluA * z * __builtin_fmaf(kGeluB * z, z, 1.f));
    if (act == kSilu) return z * sigmoid(z);
    return z;
}
// What ReLU passes on of v: nothing where it is off, whatever v holds.
__device__ __forceinline__ float relu_slope(float v, float z) { return z > 0.f ? v : z == z ? 0.f : z; }
// The curved activations' derivative: with E = e^-t, s = 1 / (1 + E) and 1 - s = E s, which loses nothing where s is almost one.  Where E would leave the
// floats they are straight.
__device__ __forceinline__ float slope(float z, int act)
{
    const float most = act == kSilu ? 80.f : 10.f;
    z = z > most ? most : z < -most ? -most : z;
    const float t = act == kSilu ? z : kGeluA * z * __builtin_fmaf(kGeluB * z, z, 1.f), along = act == kSilu ? z : kGeluA * z * __builtin_fmaf(3.f * kGeluB * z, z, 1.f);
    const float e = __builtin_amdgcn_exp2f(-kLog2 * t), s = __builtin_amdgcn_rcpf(1.f + e);
    return s * __builtin_fmaf(along, e * s, 1.f);
}
template <class F> __device__ __forceinline__ void each8(F&& f)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) f(e);
}
__device__ __forceinline__ void activate8(float (&v)[8], int act)
{
    if (act == kRelu) each8([&](int e) { v[e] = activate(v[e], kRelu); });
    else if (act == kGelu) each8([&](int e) { v[e] = activate(v[e], kGelu); });
    else if (act == kSilu) each8([&](int e) { v[e] = activate(v[e], kSilu); });
}

}  // namespace layer
}  // namespace hadfl
