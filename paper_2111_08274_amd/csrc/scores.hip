// What a row of logits says: log probabilities of given tokens, entropy, the n_top largest; and the gradient of the first two.
// With m = max z, S = sum exp(z - m), E = sum (z - m) exp(z - m):  log p_j = (z_j - m) - log S,  H = log S - E / S.
//   forward    a workgroup holds its piece of a row in registers: every logit is read once, m is known before the first exp.  A row of
//              more pieces than one is joined by a second launch.
//   gradient   dz_j = sum_i g_i [t_i = j] - p_j (sum_i g_i + dH (log p_j + H)), from the statistics that the forward pass left
// Both are bound by memory: 2 x 4096 rows of 65536 bf16 with five alternatives 229 us = 4.7 TB/s, the gradient of 4 x 1000 rows of 32000 97 us = 5.3.
// The alternatives cost little beside it: a wave's n_top-th largest of its lanes' largest values bounds those of the whole piece from below, the few
// values that reach the best such bound are listed and each is ranked against the list.  Where more tie than the list holds, the piece is read again,
// n_top times.
#include "layer.h"

namespace hadfl {
namespace layer {

using namespace head;

namespace {

constexpr int kList = 512;         // candidates that a workgroup ranks at once
constexpr int kPieces = 64;        // that a wave joins

__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(t * kLog2); }
// orders as the logits do, zeros of either sign alike, a NaN above all but below what stands before the first place
constexpr unsigned kNan = 0xfffffffeu;
__device__ __forceinline__ unsigned key_of(float z)
{
    if (z != z) return kNan;
    const unsigned u = __builtin_bit_cast(unsigned, z + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(unsigned key)
{
    if (key == kNan) return __builtin_bit_cast(float, 0x7fc00000u);
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// of equal logits the first is the larger
__device__ __forceinline__ unsigned long long place(unsigned key, int index) { return (unsigned long long)key << 32 | (unsigned)~index; }
__device__ __forceinline__ int index_of(unsigned long long p) { return ~(int)(unsigned)p; }

template <int N> __device__ __forceinline__ unsigned long long most_over(unsigned long long v)
{
#pragma unroll
    for (int d = 1; d < N; d *= 2) {
        const unsigned long long w = (unsigned long long)(unsigned)__shfl_xor((int)(v >> 32), d) << 32 | (unsigned)__shfl_xor((int)(unsigned)v, d);
        v = w > v ? w : v;
    }
    return v;
}

// a chunk of fewer than eight values, or none
__device__ __forceinline__ void load_or_out(Chunk<float>& v, const float* p, int left)
{
    v.a = v.b = tiles::u4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u};
    left = here(left);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) { if (e < 4) v.a[e] = ((const unsigned*)p)[e]; else v.b[e - 4] = ((const unsigned*)p)[e]; }
}
__device__ __forceinline__ void load_or_out(Chunk<__bf16>& v, const __bf16* p, int left)
{
    v.a = tiles::u4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
    left = here(left);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) v.a[e / 2] = e % 2 ? (v.a[e / 2] & 0xffffu) | (unsigned)((const unsigned short*)p)[e] << 16 : (v.a[e / 2] & 0xffff0000u) | ((const unsigned short*)p)[e];
}

struct Sums { float top, s, e; };  // m, S, E; m = -inf: nothing yet, S = 0 or NaN
__device__ __forceinline__ void join(Sums& a, const Sums& b)
{
    const float top = fmaxf(a.top, b.top);
    auto at = [&](const Sums& v) -> Sums {
        if (v.top == -INFINITY) return Sums{top, v.s, 0.f};
        const float d = v.top - top, f = exp_of(d);
        return Sums{top, v.s * f, f == 0.f ? 0.f : (v.e + d * v.s) * f};
    };
    const Sums x = at(a), y = at(b);
    a = Sums{top, x.s + y.s, x.e + y.e};
}
// m, log S and H of a whole row; a row of -inf alone: -inf, 0, 0
struct Row { float top, log_s, entropy; };
__device__ __forceinline__ Row row_of(const Sums& v)
{
    if (v.top == -INFINITY && v.s == 0.f) return Row{-INFINITY, 0.f, 0.f};
    const float l = logf(v.s), h = l - v.e / v.s;
    return Row{v.top, l, h < 0.f ? 0.f : h};                   // a NaN stays
}
__device__ __forceinline__ float log_p(float z, const Row& r) { return r.top == -INFINITY && r.log_s == 0.f ? (z == z ? -INFINITY : z) : (z - r.top) - r.log_s; }

// what a finished row leaves
struct Out {
    const int32_t* tokens;
    float *logp, *entropy, *stats, *top_logp;
    int32_t* top;
    int n_tokens, n_top, classes;
};
template <typename T> __device__ __forceinline__ void finish_row(const Out& o, const T* z, long long line, const Row& r, int tid, int nt)
{
    for (int i = tid; i < o.n_tokens; i += nt) {
        const int t = o.tokens[line * o.n_tokens + i];
        o.logp[line * o.n_tokens + i] = (unsigned)t < (unsigned)o.classes ? log_p(up(z[t]), r) : 0.f;
    }
    if (tid) return;
    if (o.entropy) o.entropy[line] = r.entropy;
    if (o.stats) { o.stats[line * 3] = r.top; o.stats[line * 3 + 1] = r.log_s; o.stats[line * 3 + 2] = r.entropy; }
}
__device__ __forceinline__ void finish_top(const Out& o, long long line, const Row& r, int rank, unsigned long long p)
{
    o.top[line * o.n_top + rank] = index_of(p);
    o.top_logp[line * o.n_top + rank] = log_p(logit_of((unsigned)(p >> 32)), r);
}

// A piece of a row: `size` classes from `size * piece`, U chunks of eight a thread.  part, best: where its sums and its largest go if the row has
// more pieces.
template <typename T, int NT, int U>
__global__ __launch_bounds__(NT) void scores_kernel(const T* logits, long long rep, long long row, int rows, int pieces, int size, long long total, Out o,
                                                    Sums* part, unsigned long long* best)
{
    constexpr int W = NT / 64;
    __shared__ float tops[W], limits[W], sums[W], weighted[W];
    __shared__ unsigned long long list[kList], firsts[W];
    __shared__ int count;
    const long long at = line_block();
    if (at >= total) return;
    const long long line = at / pieces;
    const int piece = (int)(at - line * pieces), k = (int)(line / rows), t = (int)(line - (long long)k * rows);
    const int tid = threadIdx.x, wave = tid / 64, begin = piece * size, n = min(size, o.classes - begin);
    const T* z = logits + k * rep + t * row;
    Chunk<T> v[U];                                             // what lies outside counts as -inf
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (u * NT + tid) * 8;
        if (c + 8 <= n) v[u].load(z + begin + c, 8);
        else load_or_out(v[u], z + begin + c, n - c);
    }
    float most[U], mine = -INFINITY;                           // NaNs show in the sum
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float x[8];
        v[u].get(x);
        most[u] = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) most[u] = __builtin_fmaxf(most[u], x[e]);
        mine = __builtin_fmaxf(mine, most[u]);
    }
    const float top_wave = max_over<64>(mine);
    if (tid == 0) count = 0;
    if (o.n_top) {
        // at least n_top of this wave's values are not below the n_top-th largest of its lanes' largest
        float left = mine, limit = -INFINITY;
        for (int i = 0; i < o.n_top; ++i) {
            limit = max_over<64>(left);
            const unsigned long long who = __ballot(left == limit);
            if ((tid & 63) == __ffsll((long long)who) - 1) left = -INFINITY;
        }
        if ((tid & 63) == 0) limits[wave] = limit;
    }
    if ((tid & 63) == 0) tops[wave] = top_wave;
    __syncthreads();
    float top = tops[0];
#pragma unroll
    for (int w = 1; w < W; ++w) top = __builtin_fmaxf(top, tops[w]);
    const float base = top == -INFINITY ? 0.f : top;
    float s = 0.f, e = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float x[8];
        v[u].get(x);
        each8([&](int i) {
            const float d = x[i] - base, p = exp_of(d);
            s += p;
            e = __builtin_fmaf(__builtin_fmaxf(d, -1e30f), p, e);         // -inf has no weight
        });
    }
    const bool nans = s != s;
    s = sum_over<64>(s);
    e = sum_over<64>(e);
    if ((tid & 63) == 0) { sums[wave] = s; weighted[wave] = e; }
    if (o.n_top) {
        float limit = limits[0];
#pragma unroll
        for (int w = 1; w < W; ++w) limit = __builtin_fmaxf(limit, limits[w]);
        // few chunks hold any: which of their values is noted in bits, the values themselves are read again
        unsigned bits[(U + 3) / 4] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (most[u] < limit && !nans) continue;
            float x[8];
            v[u].get(x);
            each8([&](int i) { bits[u / 4] |= x[i] < limit ? 0u : 1u << (8 * (u % 4) + i); });
        }
#pragma unroll
        for (int w = 0; w < (U + 3) / 4; ++w)
            while (bits[w]) {
                const int bit = __builtin_ctz(bits[w]), i = ((4 * w + bit / 8) * NT + tid) * 8 + bit % 8;
                bits[w] &= bits[w] - 1;
                if (i >= n) continue;
                const int q = atomicAdd(&count, 1);
                if (q < kList) list[q] = place(key_of(up(z[begin + i])), begin + i);
            }
    }
    __syncthreads();
    Sums all{top, sums[0], weighted[0]};
#pragma unroll
    for (int w = 1; w < W; ++w) { all.s += sums[w]; all.e += weighted[w]; }
    const Row r = row_of(all);
    auto give = [&](int rank, unsigned long long p) {
        if (pieces > 1) best[at * o.n_top + rank] = p;
        else finish_top(o, line, r, rank, p);
    };
    if (pieces > 1) { if (tid == 0) part[at] = all; }
    else finish_row(o, z, line, r, tid, NT);
    if (!o.n_top) return;
    const int have = count;
    if (have <= kList) {
        for (int i = tid; i < have; i += NT) {
            const unsigned long long p = list[i];
            int rank = 0;
            for (int j = 0; j < have; ++j) rank += list[j] > p;
            if (rank < o.n_top) give(rank, p);
        }
        return;
    }
    // too many that tie, or a row of masks: the largest below the last one, n_top times
    unsigned long long last = ~0ull;
    for (int i = 0; i < o.n_top; ++i) {
        unsigned long long p = 0;
#pragma unroll 4
        for (int j = tid; j < n; j += NT) {
            const unsigned long long q = place(key_of(up(z[begin + j])), begin + j);
            p = q < last && q > p ? q : p;
        }
        p = most_over<64>(p);
        if ((tid & 63) == 0) firsts[wave] = p;
        __syncthreads();
        p = firsts[0];
#pragma unroll
        for (int w = 1; w < W; ++w) p = firsts[w] > p ? firsts[w] : p;
        __syncthreads();
        if (tid == 0) give(i, p);
        last = p;
    }
}

// Rows of several pieces: a wave a row, a lane a piece.
template <typename T>
__global__ __launch_bounds__(256) void join_scores_kernel(const T* logits, long long rep, long long row, int rows, int pieces, long long lines, Out o,
                                                          const Sums* part, const unsigned long long* best)
{
    const long long line = line_block() * 4 + threadIdx.x / 64;
    if (line >= lines) return;
    const int lane = threadIdx.x & 63, k = (int)(line / rows), t = (int)(line - (long long)k * rows);
    Sums v = lane < pieces ? part[line * pieces + lane] : Sums{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        // in the order of the pieces on both sides, so that all lanes hold the same
        const Sums w{__shfl_xor(v.top, d), __shfl_xor(v.s, d), __shfl_xor(v.e, d)};
        Sums a = lane & d ? w : v;
        join(a, lane & d ? v : w);
        v = a;
    }
    const Row r = row_of(v);
    finish_row(o, logits + k * rep + t * row, line, r, lane, 64);
    int next = 0;
    const unsigned long long* mine = best + (line * pieces + lane) * o.n_top;
    unsigned long long head = o.n_top && lane < pieces ? mine[0] : 0;
    for (int i = 0; i < o.n_top; ++i) {
        const unsigned long long p = most_over<64>(head);
        if (lane == 0) finish_top(o, line, r, i, p);
        if (head == p) head = ++next < o.n_top ? mine[next] : 0;
    }
}

// Eight columns a lane, U chunks; a token's column is written once more, whole, by the lane that has the token: its logit is read before any
// store, since the gradient may take the logits' place.
template <typename T, int U>
__global__ __launch_bounds__(256) void scores_grad_kernel(const T* logits, long long rep, long long row, int rows, int classes, int blocks, long long total,
                                                          const int32_t* tokens, int n_tokens, const float* stats, const float* dlogp, const float* dentropy,
                                                          T* dz, long long drep, long long drow)
{
    const long long at = line_block();
    if (at >= total) return;
    const long long line = at / blocks;
    const int begin = (int)(at - line * blocks) * U * 2048, end = min(classes, begin + U * 2048), k = (int)(line / rows), t = (int)(line - (long long)k * rows);
    const int tid = threadIdx.x;
    const T* z = logits + k * rep + t * row;
    T* out = dz + k * drep + t * drow;
    const float top = stats[line * 3], log_s = stats[line * 3 + 1], entropy = stats[line * 3 + 2], dh = dentropy ? dentropy[line] : 0.f;
    const bool empty = top == -INFINITY && log_s == 0.f;
    const float base = top == -INFINITY ? 0.f : top;
    Chunk<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = begin + (u * 256 + tid) * 8;
        v[u].load(z + (c < end ? c : 0), c < end ? end - c : 0);
    }
    const int32_t* given = tokens + line * n_tokens;
    const float* g = dlogp + line * n_tokens;
    float all = 0.f;
    for (int i = 0; i < n_tokens; ++i)
        if ((unsigned)given[i] < (unsigned)classes) all += g[i];
    auto part = [&](float x) {
        const float d = x - base - log_s, p = exp_of(d);
        return p == 0.f ? 0.f : -p * (all + dh * (d + entropy));
    };
    const int mine = tid < n_tokens ? given[tid] : -1;
    const bool fix = mine >= begin && mine < end && !empty;
    const float x = fix ? up(z[mine]) : 0.f;
    if (n_tokens) __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = begin + (u * 256 + tid) * 8;
        if (c >= end) continue;
        float w[8];
        v[u].get(w);
        each8([&](int e) { w[e] = part(w[e]); });
        store_chunk(out + c, end - c, w);
    }
    if (!n_tokens) return;
    __syncthreads();
    if (!fix) return;
    float sum = part(x);
    for (int i = 0; i < n_tokens; ++i)
        if (given[i] == mine) sum += g[i];
    out[mine] = (T)sum;
}

// Threads, chunks a thread and pieces of a row.  256 threads: workgroups at different stages share a compute unit, so loads and exponentials overlap
// (8192 rows of 65536 bf16, five alternatives: 228 us = 4.7 TB/s, what a copy reaches, with 512 threads 287, with 1024 329).  Few logits: one
// launch is less than a second one's 3 us, 1024 threads for rows that they hold whole, and where rows would have
// more pieces than a wave has lanes (256 / 1024 threads: 1 x 32000 19.0 / 15.6, 1024 x 32000 27.1 /
// 26.0, 512 x 60000 26.8 / 26.1, 1024 x 60000 38.7 / 45.7; fp32 1024 x 32000 31.8 / 31.0).
// A row of more pieces than one has at least 4096 classes a piece and loses at most seven of them to each piece's rounding: the last one still
// holds as many as there are alternatives, so that every piece gives n_top of them.
struct Plan { int nt, u, pieces, size; };
Plan plan_of(long long lines, int classes, int bf16)
{
    const int most = bf16 ? 8 : 4;                             // chunks a thread holds in 32 registers
    Plan p{};
    p.nt = (classes > 2048 * most && classes <= 8192 * most && (double)lines * classes <= 33e6) || classes > kPieces * 2048 * most ? 1024 : 256;
    p.pieces = (classes + p.nt * 8 * most - 1) / (p.nt * 8 * most);
    p.size = ((classes + p.pieces - 1) / p.pieces + 7) / 8 * 8;
    p.pieces = (classes + p.size - 1) / p.size;
    p.u = most;
    while (p.u > most / (p.nt == 256 ? 4 : 2) && p.nt * 8 * (p.u / 2) >= p.size) p.u /= 2;
    return p;
}
size_t part_bytes(const Plan& p, long long lines) { return p.pieces > 1 ? align256((size_t)lines * p.pieces * sizeof(Sums)) : 0; }

template <typename T> hipError_t forward(const ScoreArgs& a, hipStream_t s)
{
    constexpr int M = sizeof(T) == 2 ? 8 : 4;
    const long long lines = (long long)a.n * a.rows;
    if (lines == 0) return hipSuccess;
    const Plan p = plan_of(lines, a.classes, a.bf16);
    Sums* part = (Sums*)a.work;
    unsigned long long* best = (unsigned long long*)((char*)a.work + part_bytes(p, lines));
    const Out o{a.tokens, a.logp, a.entropy, a.stats, a.top_logp, a.top, a.n_tokens, a.n_top, a.classes};
    auto* kernel = p.nt == 256 ? (p.u == M ? scores_kernel<T, 256, M> : p.u == M / 2 ? scores_kernel<T, 256, M / 2> : scores_kernel<T, 256, M / 4>)
                               : (p.u == M ? scores_kernel<T, 1024, M> : scores_kernel<T, 1024, M / 2>);
    const long long total = lines * p.pieces;
    kernel<<<line_grid(total, p.nt), p.nt, 0, s>>>((const T*)a.logits.p, a.logits.rep, a.logits.row, a.rows, p.pieces, p.size, total, o, part, best);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.pieces == 1) return e;
    join_scores_kernel<T><<<line_grid((lines + 3) / 4, 256), 256, 0, s>>>((const T*)a.logits.p, a.logits.rep, a.logits.row, a.rows, p.pieces, lines, o, part, best);
    return hipGetLastError();
}

template <typename T> hipError_t backward(const ScoreArgs& a, hipStream_t s)
{
    constexpr int U = sizeof(T) == 2 ? 4 : 2;
    const int blocks = (a.classes + U * 2048 - 1) / (U * 2048);
    const long long total = (long long)a.n * a.rows * blocks;
    if (total == 0) return hipSuccess;
    scores_grad_kernel<T, U><<<line_grid(total, 256), 256, 0, s>>>((const T*)a.logits.p, a.logits.rep, a.logits.row, a.rows, a.classes, blocks, total, a.tokens,
                                                                   a.n_tokens, a.stats, a.dlogp, a.dentropy, (T*)a.dlogits.p, a.dlogits.rep, a.dlogits.row);
    return hipGetLastError();
}

}  // namespace

size_t score_work_bytes(int n, int rows, int classes, int n_top, int bf16)
{
    const long long lines = (long long)n * rows;
    const Plan p = plan_of(lines, classes, bf16);
    return p.pieces > 1 ? part_bytes(p, lines) + align256((size_t)lines * p.pieces * n_top * 8) : 0;
}
hipError_t launch_scores_forward(const ScoreArgs& a, hipStream_t s) { return a.bf16 ? forward<__bf16>(a, s) : forward<float>(a, s); }
hipError_t launch_scores_backward(const ScoreArgs& a, hipStream_t s) { return a.bf16 ? backward<__bf16>(a, s) : backward<float>(a, s); }

}  // namespace layer
}  // namespace hadfl
