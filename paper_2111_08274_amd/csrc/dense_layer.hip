// A dense layer and its gradient, grouped over replicas: y = r + D(a(x W + b)), a an activation, D dropout, r a residual.
//   forward    one product whose epilogue does the rest on 32-bit sums, eight columns of a row at a time; pre = x W + b is left for the
//              gradient where that is asked for
//   gradient   dz = D'(dy) a'(pre) and its column sums db in one pass over dy, then dx = dz W^T and dW = x^T dz
// bf16: a dz that is no bf16 value (a curved activation, a dropout's scale) enters the two products as two bf16 parts, off by 2^-15 of a value at
// most (from 2^-111 on, where the second part is a normal number); db is summed before that.  fp32: operands enter as three bf16 parts, six products.
#include "direct_product.h"
#include "layer.h"

namespace hadfl {
namespace layer {

using namespace head;

namespace {

// ---- epilogue -----------------------------------------------------------------------------------------------------------
// 32-bit sums to what the layer returns, eight columns of a row at a time; a null pointer leaves its part out.
template <typename T> struct Finish {
    const float* bias;
    long long bias_rep;
    Rows residual, pre, y;
    int rows, cols, act;
    Draws draws;
    // A lane's eight columns from n, in rows m, m + step, ...: what stays the same from row to row, and where its tensors stand.
    struct Columns {
        const T* residual;
        T *pre, *y;
        long long residual_step, pre_step, y_step;
        unsigned long long call;
        float bias[8];
        int k, m, n, step;
    };
    __device__ __forceinline__ Columns columns(int k, int m, int n, int step) const
    {
        Columns c{};
        if (residual.p) c.residual = (const T*)residual.p + k * residual.rep + m * residual.row + n;
        if (pre.p) c.pre = (T*)pre.p + k * pre.rep + m * pre.row + n;
        c.y = (T*)y.p + k * y.rep + m * y.row + n;
        c.residual_step = step * residual.row; c.pre_step = step * pre.row; c.y_step = step * y.row;
        if (bias && n < cols) {
            Chunk<float> b;
            b.load(bias + k * bias_rep + n, cols - n);
            b.get(c.bias);
        }
        c.call = draws.limit ? call_of(draws) : 0ull;
        c.k = k; c.m = m; c.n = n; c.step = step;
        return c;
    }
    // the residual of the row `ahead` steps on
    __device__ __forceinline__ void fetch(const Columns& c, int ahead, Chunk<T>& add) const
    {
        if (residual.p && c.m + ahead * c.step < rows && c.n < cols) add.load(c.residual + ahead * c.residual_step, cols - c.n);
    }
    __device__ __forceinline__ void row(Columns& c, const Chunk<T>& add, float (&v)[8]) const
    {
        if (c.m < rows && c.n < cols) {
            const int left = cols - c.n;
            if (bias) each8([&](int e) { v[e] += c.bias[e]; });
            if (pre.p) store_chunk(c.pre, left, v);
            activate8(v, act);
            if (draws.limit) kept8(draws, c.call, c.k, c.m, c.n, [&](int e, bool kept) { v[e] = kept ? v[e] * draws.scale : 0.f; });
            if (residual.p) {
                float w[8];
                add.get(w);
                each8([&](int e) { v[e] += w[e]; });
            }
            store_chunk(c.y, left, v);
        }
        c.m += c.step;
        c.residual += c.residual_step; c.pre += c.pre_step; c.y += c.y_step;
    }
};
// only the store, rounded
template <typename T> Finish<T> store_only(const Rows& y, int rows, int cols)
{
    return Finish<T>{nullptr, 0, {}, {}, y, rows, cols, kNone, Draws{0, 0, 0, nullptr, 0, 1.f}};
}

// A wave's blocks of 32 rows through LDS, as floats: a lane holds four consecutive columns of a row, Finish takes eight, the same ones in every block.
// The blocks go through one loop: unrolled, a 256 x 256 tile's epilogue was 96 KiB of code, more than the instruction cache holds.  The residual of
// a block is on its way while the one before is finished.
template <typename T> struct FinishTile {
    static constexpr bool kLaneM = true, kStaged = true, kSums = false;
    template <int TN> static constexpr int pitch() { return TN * 128 + 16; }
    template <int TN> static constexpr int bytes() { return 32 * pitch<TN>(); }
    Finish<T> finish;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t, char* lds) const
    {
        constexpr int kPitch = pitch<TN>(), kAcross = TN * 4, kDown = 64 / kAcross, kRows = 32 / kDown;
        char* p = lds + t.wave * bytes<TN>();
        const int r = t.lane / kAcross, c = t.lane % kAcross * 8;
        auto columns = finish.columns(t.rep, t.m0 + r, t.n0 + c, kDown);
        Chunk<T> next[kRows] = {};
#pragma unroll
        for (int u = 0; u < kRows; ++u) finish.fetch(columns, u, next[u]);
#pragma unroll 1
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int b = 0; b < TM; ++b) {
                if (b != i) continue;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *(f4*)(p + (t.lane & 31) * kPitch + (32 * j + 8 * q + 4 * (t.lane >> 5)) * 4) =
                            f4{t.acc[b][j][4 * q], t.acc[b][j][4 * q + 1], t.acc[b][j][4 * q + 2], t.acc[b][j][4 * q + 3]};
            }
            Chunk<T> now[kRows];
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                now[u] = next[u];
                if (i + 1 < TM) finish.fetch(columns, kRows + u, next[u]);
            }
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const char* at = p + (r + u * kDown) * kPitch + c * 4;
                const f4 low = *(const f4*)at, high = *(const f4*)(at + 16);
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[e] = low[e]; v[4 + e] = high[e]; }
                finish.row(columns, now[u], v);
            }
        }
    }
};

// ---- products -------------------------------------------------------------------------------------------------------------
template <class SA, bool A_ALONG, class SB, bool B_ALONG, int BM, int BN, int WM, int WN, int KS, int NBUF, int AHEAD, class Epi>
__global__ __launch_bounds__(WM * WN * 64) void layer_product_kernel(SA a, SB b, int K, int tiles_m, int tiles_n, int splits, int split_len, int total, Epi epi)
{
    product_tile<SA, A_ALONG, SB, B_ALONG, BM, BN, WM, WN, KS, NBUF, AHEAD>(a, b, K, tiles_m, tiles_n, splits, split_len, total, epi);
}
// f(a, b) for the planes of A and B whose products are kept, the small ones first: of three bf16 parts each what is left out is below 2^-24 of the product
template <int PA, int PB, class F> __device__ __forceinline__ void each_pair(F&& f)
{
    constexpr int most = PA + PB - 2 < 2 ? PA + PB - 2 : 2;
#pragma unroll
    for (int sum = most; sum >= 0; --sum)
#pragma unroll
        for (int a = PA - 1; a >= 0; --a)
            if (a <= sum && sum - a < PB) f(a, sum - a);
}

// dz as slope_kernel leaves it in two parts: planes of bf16, rows of whole chunks
struct TwoParts {
    static constexpr int kPlanes = 2;
    struct Raw { Chunk<__bf16> high, low; bool in; };
    const __bf16* p;
    long long rep, row;
    int rows, cols;
    long long plane;
    __device__ __forceinline__ void bind(int k) { p += k * rep; }
    __device__ __forceinline__ Raw load(int r, int c) const
    {
        Raw v;
        v.in = r < rows && c < cols;
        const __bf16* at = p + (v.in ? r * row + c : 0ll);
        v.high.load(at, 8);
        v.low.load(at + plane, 8);
        return v;
    }
    __device__ __forceinline__ bool has_tail(int, int) const { return false; }
    __device__ __forceinline__ void planes(const Raw& v, int, bool, u4 (&out)[2]) const
    {
        out[0] = v.in ? v.high.a : u4{0, 0, 0, 0};
        out[1] = v.in ? v.low.a : u4{0, 0, 0, 0};
    }
};

// Operands in planes of bf16, straight from memory to LDS (direct_product.h: Loader): one plane each in slabs of 64 k, or two parts against one plane, or
// three parts of 32-bit values each in slabs of 32, all planes of a slab together.  A wave reads the operands of a step of 16 k while it multiplies the step before, across slabs too: the
// barrier that frees a slab's image and says that the next one has arrived lies before the slab's last step, whose operands are in registers by then, so
// that the matrix cores have work while the first operands of the next slab are read.  4 x 8192 rows x 4096 x 4096 bf16 with bias and dropout onto a
// residual: 1001 us = 1098 TFLOP/s, the matrix cores busy 57 to 58 % of the time; the product alone 944.  The library's product 858, 70 % busy, at no
// higher clock (both 1.4 to 1.8 GHz over twelve launches in a row).  Two parts against one plane: dx of 16 x 1024 x 512 x 2048 71 us, dW 63 (of one part
// 44 and 40): an operand read for two products, the matrix cores busy 45 and 55 % of the time.
template <bool A_ALONG, bool B_ALONG, int PA, int PB, int BM, int BN, int WM, int WN, class Epi>
__global__ __launch_bounds__(WM * WN * 64) void layer_planes_kernel(Plane3 a, Plane3 b, int K, int tiles_m, int tiles_n, int splits, int split_len, int total, Epi epi)
{
    constexpr int NT = WM * WN * 64, TM = BM / WM / 32, TN = BN / WN / 32, KS = PA + PB == 2 ? kSlab : kSlab / 2, kSteps = KS / 16;
    typedef Loader<A_ALONG, BM, NT, KS> LA;
    typedef Loader<B_ALONG, BN, NT, KS> LB;
    constexpr int kImage = PA * LA::kBytes + PB * LB::kBytes, IMAGES = kImage > 49152 ? 2 : kImage > 32768 ? 3 : 4, kLoads = PA * LA::kLoads + PB * LB::kLoads;
    __shared__ __attribute__((aligned(16))) char images[IMAGES * kImage];
    if constexpr (Epi::kStaged) static_assert(WM * WN * Epi::template bytes<TN>() <= IMAGES * kImage, "the epilogue's blocks lie in the images");

    const unsigned item = blockIdx.y * gridDim.x + logical_block();
    if (item >= (unsigned)total) return;
    const int per = tiles_m * tiles_n, r = item / per;
    int tm_i, tn_i;
    place_tile(item - r * per, tiles_m, tiles_n, tm_i, tn_i);
    Tile<TM, TN> t;
    t.split = r % splits;
    t.rep = r / splits;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    t.lane = tid & 63;
    t.wave = wave;
    const int bm = t.bm = tm_i * BM, bn = t.bn = tn_i * BN, wm = (wave % WM) * TM * 32, wn = (wave / WM) * TN * 32;
    t.m0 = bm + wm;
    t.n0 = bn + wn;
    const __bf16 *pa = a.p + t.rep * a.rep, *pb = b.p + t.rep * b.rep;
    const int k_begin = t.split * split_len, k_end = min(K, k_begin + split_len), slabs = k_begin < k_end ? (k_end - k_begin + KS - 1) / KS : 0;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) t.acc[i][j] = f16{};
    LA la;
    LB lb;
    la.init(tid, a.ld);
    lb.init(tid, b.ld);

    auto issue = [&](int slab, char* image) {
#pragma unroll
        for (int s = 0; s < PA; ++s) la.issue(a, pa + s * a.plane, bm, k_begin + slab * KS, wave, image + s * LA::kBytes);
#pragma unroll
        for (int s = 0; s < PB; ++s) lb.issue(b, pb + s * b.plane, bn, k_begin + slab * KS, wave, image + PA * LA::kBytes + s * LB::kBytes);
    };
    bf16x8 fa[2][PA][TM], fb[2][PB][TN];
    auto read = [&](const char* image, int step, int to) {
#pragma unroll
        for (int s = 0; s < (PA > PB ? PA : PB); ++s) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
                if (s < PA) fa[to][s][i] = LA::read(image + s * LA::kBytes, wm + 32 * i, step, t.lane);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                if (s < PB) fb[to][s][j] = LB::read(image + PA * LA::kBytes + s * LB::kBytes, wn + 32 * j, step, t.lane);
        }
    };
    auto multiply = [&](int from) {
        each_pair<PA, PB>([&](int p, int q) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const bf16x8 &x = fa[from][p][i], &y = fb[from][q][j];
                    t.acc[i][j] = Epi::kLaneM ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, x, t.acc[i][j], 0, 0, 0)
                                              : __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, t.acc[i][j], 0, 0, 0);
                }
        });
    };
    // Slab i + 1 is there when at most the loads of the IMAGES - 2 slabs after it are outstanding (they finish in order).
    auto turn = [&](int i, char* image, char* next) {
        if (i >= slabs) return;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s + 1 < kSteps) read(image, s + 1, (s + 1) % 2);
            else if (i + 1 < slabs) {
                if (IMAGES > 2 && i + IMAGES - 1 < slabs) slab_barrier<(IMAGES - 2) * kLoads>();
                else slab_barrier<0>();
                if (i + IMAGES < slabs) issue(i + IMAGES, image);
                read(next, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(s % 2);
        }
    };
    static_assert(kSteps % 2 == 0, "a slab ends where the next one's first operands go");
#pragma unroll
    for (int i = 0; i < IMAGES; ++i)
        if (i < slabs) issue(i, images + i * kImage);
    if (slabs >= IMAGES) slab_barrier<(IMAGES - 1) * kLoads>();
    else slab_barrier<0>();
    if (slabs) read(images, 0, 0);
    for (int i = 0; i < slabs; i += IMAGES) {
#pragma unroll
        for (int u = 0; u < IMAGES; ++u) turn(i + u, images + u * kImage, images + (u + 1) % IMAGES * kImage);
    }
    if constexpr (Epi::kStaged) {
        __syncthreads();                                       // the images are free
        epi(t, images);
    } else epi(t);
}

// Few rows of a short contraction, whose time is latency: a workgroup takes 32 rows x 32 TN columns and its NW waves a share of the contraction each, in
// slabs of 32 k that a wave stages for itself (no barrier), two in flight.  The shares are added from LDS in ascending order and finished there: one
// launch.  One row of 512 x 2048 bf16 5.0 us in a graph (shares by workgroups and a second launch 7.3), 4 x 32 rows of 512 x 128 fp32 6.4 (8.0), of 784 x 128 8.8.
template <class SA, class SB, bool B_ALONG, int TN, int NW, typename T>
__global__ __launch_bounds__(NW * 64) void layer_few_kernel(SA a, SB b, int K, int tiles_m, int tiles_n, int total, Finish<T> finish)
{
    constexpr int PA = SA::kPlanes, PB = SB::kPlanes, KS = 32, AHEAD = 2;
    typedef Image<true, 32, KS> IA;
    typedef Image<B_ALONG, 32 * TN, KS> IB;
    constexpr int NA = IA::kChunks / 64, NB = IB::kChunks / 64;
    constexpr unsigned kWave = PA * IA::kPlane + PB * IB::kPlane, kPitch = TN * 128 + 16, kSums = NW * 32 * kPitch;
    __shared__ __attribute__((aligned(16))) char smem[NW * kWave > kSums ? NW * kWave : kSums];

    const unsigned item = blockIdx.y * gridDim.x + logical_block();
    if (item >= (unsigned)total) return;
    const int at_m = item % tiles_m, rest = item / tiles_m, m0 = at_m * 32, n0 = rest % tiles_n * 32 * TN, rep = rest / tiles_n;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    a.bind(rep);
    b.bind(rep);
    const int slabs = (K + KS - 1) / KS, per = (slabs + NW - 1) / NW, k_begin = min(wave * per * KS, K), k_end = min(K, k_begin + per * KS);
    char* image = smem + wave * kWave;
    f16 acc[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[j] = f16{};
    typename SA::Raw ra[AHEAD][NA];
    typename SB::Raw rb[AHEAD][NB];
    auto fetch = [&](int k0, int slot) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int id = lane + i * 64, r = id / IB::kAcross, c = id % IB::kAcross * 8;
            rb[slot][i] = B_ALONG ? b.load(n0 + r, k0 + c) : b.load(k0 + r, n0 + c);
        }
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int id = lane + i * 64;
            ra[slot][i] = a.load(m0 + id / IA::kAcross, k0 + id % IA::kAcross * 8);
        }
    };
    auto slab = [&](int k0, int slot) {
        const bool tail_a = a.has_tail(k0, k0 + KS), tail_b = B_ALONG ? b.has_tail(k0, k0 + KS) : b.has_tail(n0, n0 + 32 * TN);
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int id = lane + i * 64, r = id / IA::kAcross, c = id % IA::kAcross;
            u4 p[PA];
            a.planes(ra[slot][i], k0 + c * 8, tail_a, p);
#pragma unroll
            for (int s = 0; s < PA; ++s) *(u4*)(image + s * IA::kPlane + r * IA::kPitch + c * 16) = p[s];
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int id = lane + i * 64, r = id / IB::kAcross, c = id % IB::kAcross;
            u4 p[PB];
            b.planes(rb[slot][i], (B_ALONG ? k0 : n0) + c * 8, tail_b, p);
#pragma unroll
            for (int s = 0; s < PB; ++s) *(u4*)(image + PA * IA::kPlane + s * IB::kPlane + r * IB::kPitch + c * 16) = p[s];
        }
        if (k0 + AHEAD * KS < k_end) fetch(k0 + AHEAD * KS, slot);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");        // this wave's stores before its reads: LDS keeps their order
#pragma unroll
        for (int ks = 0; ks < KS / 16; ++ks) {
            bf16x8 fa[PA], fb[TN][PB];
#pragma unroll
            for (int s = 0; s < PA; ++s) fa[s] = IA::read(image + s * IA::kPlane, 0, ks, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int s = 0; s < PB; ++s) fb[j][s] = IB::read(image + PA * IA::kPlane + s * IB::kPlane, 32 * j, ks, lane);
            each_pair<PA, PB>([&](int p, int q) {
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j][q], fa[p], acc[j], 0, 0, 0);
            });
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (k_begin + i * KS < k_end) fetch(k_begin + i * KS, i);
    for (int k0 = k_begin; k0 < k_end; k0 += AHEAD * KS) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (k0 + u * KS < k_end) slab(k0 + u * KS, u);
    }
    __syncthreads();                                           // the images are free
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(f4*)(smem + (wave * 32 + (lane & 31)) * kPitch + (32 * j + 8 * q + 4 * (lane >> 5)) * 4) = f4{acc[j][4 * q], acc[j][4 * q + 1], acc[j][4 * q + 2], acc[j][4 * q + 3]};
    __syncthreads();
    for (int id = threadIdx.x; id < 128 * TN; id += NW * 64) {
        const int r = id / (4 * TN), c = id % (4 * TN) * 8;
        auto columns = finish.columns(rep, m0 + r, n0 + c, 0);
        Chunk<T> add = {};
        finish.fetch(columns, 0, add);
        f4 low{}, high{};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const char* at = smem + (w * 32 + r) * kPitch + c * 4;
            low += *(const f4*)at;
            high += *(const f4*)(at + 16);
        }
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = low[e]; v[4 + e] = high[e]; }
        finish.row(columns, add, v);
    }
}

// The shares of a contraction, [splits][replicas][rows][ld] floats, added in ascending order and finished.
template <typename T>
__global__ __launch_bounds__(256) void finish_shares_kernel(const float* share, int splits, long long step, int ld, long long total, Finish<T> finish)
{
    const long long at = line_block() * 256 + threadIdx.x;
    if (at >= total) return;
    const float* src = share + at * 8;
    f4 a = {}, b = {};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) { a += *(const f4*)(src + s * step); b += *(const f4*)(src + s * step + 4); }
    const int chunks = ld / 8;
    const long long line = at / chunks;
    const int c = (int)(at - line * chunks) * 8, k = (int)(line / finish.rows), t = (int)(line - (long long)k * finish.rows);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    auto columns = finish.columns(k, t, c, 0);
    Chunk<T> add = {};
    finish.fetch(columns, 0, add);
    finish.row(columns, add, v);
}

int up_to(long long v, int unit) { return (int)((v + unit - 1) / unit * unit); }

// A product's tiles and into how many shares its contraction is cut.
struct Shape {
    bool planes;                   // operands straight from memory to LDS
    int bm, bn, splits, len;
    bool few;                      // at most 32 rows, the shares within a workgroup
};
size_t share_bytes(const Shape& p, int n, int M, int N) { return p.splits > 1 ? align256((size_t)p.splits * n * M * up_to(N, 8) * 4) : 0; }

Shape cut(Shape p, int K, int splits, int unit)
{
    p.len = std::max(unit, up_to((K + splits - 1) / splits, unit));
    p.splits = std::max(1, (K + p.len - 1) / p.len);
    return p;
}
// Tiles that there are, with what they cost in nanoseconds a k of a contraction: of a workgroup alone on its compute unit, and of each of several there
// (`most` fit), measured over 64 to 8192 rows, 200 to 4096 inputs and outputs; and in microseconds what a tile costs beside.  two: one operand of bf16 in
// two parts, for which what is not there never was the best by more than 4 % over 38 products of 24 to 8192 rows (tiles chosen: within 3 % of the best, but
// dx of 128 x 512 x 2048, 7 %).
struct Choice {
    bool planes;
    int bm, bn, most;
    struct { double alone, shared; } f32, bf16, two;           // zero: not there
    double tile;
};
constexpr Choice kChoices[] = {{false, 32, 128, 3, {23, 15}, {6.3, 5}, {7.5, 5.5}, 3}, {false, 64, 64, 4, {25, 15.5}, {8.8, 4.9}, {12, 6}, 3},
                               {false, 64, 128, 2, {33, 28}, {7.5, 7.3}, {0, 0}, 3}, {false, 128, 128, 2, {44, 46}, {10, 11}, {0, 0}, 4},
                               {true, 128, 128, 1, {0, 0}, {6, 9.6}, {16.5, 16.5}, 4}, {true, 128, 256, 1, {73, 73}, {11.5, 16}, {27, 27}, 5},
                               {true, 256, 256, 1, {0, 0}, {21, 28}, {50, 50}, 8}};
struct Chosen { Shape shape; double cost; };
// Whether a product goes to layer_few_kernel: a workgroup for every compute unit at most, and no more than four slabs a wave.  us in graphs, other way /
// this: one row bf16 of 512 x 8192 7.4 / 5.1, 1024 x 8192 7.2 / 6.5, 2048 x 2048 7.4 / 9.0; four of 512 x 2048 7.4 / 5.1, of 512 x 8192 (512 workgroups)
// 8.0 / 8.5; fp32 512 x 8192 9.1 / 6.7, 1024 x 2048 8.3 / 9.6 (but a launch less), 2048 x 2048 10.7 / 15.3.
constexpr int few_columns(bool bf16) { return bf16 ? 64 : 32; }       // fp32: what three planes of eight waves leave room for
bool is_few(int n, int M, int N, int K, int bf16)
{
    const int columns = few_columns(bf16);
    return M <= 64 && K <= 1024 && (long long)n * ((M + 31) / 32) * ((N + columns - 1) / columns) <= 256;
}
// The cheapest tiles and shares by that, with operands in planes or through registers.  A share is written and read at 5 TB/s, and joining them is one
// more launch, 4 us.  us, planes / registers, the best tiles of each: fp32 y of 8192 x 4096 x 4096 1323 / 1493, 4096 x 1024 x 4096 183 / 196, 16 x 1024 x
// 512 x 2048 221 / 200, 2 x 1001 x 777 x 1111 52 / 44; bf16 dx and dW of 8192 x 4096 x 4096 504 / 801, 16 x 1024 x 512 x 2048 129 / 145, 2 x 1001 x 777 x
// 1111 49 / 42.  Of 56 layers and pairs of dx and dW of 100 to 8192 rows, the tiles taken are within 5 % of the best for 46, within 10 % for nine (fp32 dx and
// dW of 2 x 1001 x 777 x 1111 86, best 78; y of 2000 x 4000 x 4000 366, best 336, of 4096 x 4096 x 1000 209, best 196; bf16 y of 300 x 4096 x 500 17.1, best
// 15.9).  The worst: bf16 dx and dW of 512 x 2048 x 2048 38, best 32, by 128 x 128 tiles of planes.
Chosen best_shape(int n, int M, int N, int K, int bf16, bool across, bool planes, bool two = false)
{
    Chosen best{{}, -1};
    if (!planes && !across && is_few(n, M, N, K, bf16)) return Chosen{Shape{false, 32, few_columns(bf16), 1, K, true}, 0};
    for (const Choice& o : kChoices) {
        const double alone = two ? o.two.alone : bf16 ? o.bf16.alone : o.f32.alone, shared = two ? o.two.shared : bf16 ? o.bf16.shared : o.f32.shared;
        if (o.planes != planes || alone == 0 || (o.bm == 32 && (M > 32 || across))) continue;
        const long long tiles = (long long)n * ((M + o.bm - 1) / o.bm) * ((N + o.bn - 1) / o.bn);
        const int unit = bf16 && o.bm == 32 ? 128 : 64;                       // whole slabs of every kernel of these tiles
        for (int s = 1; s <= 64 && (s == 1 || K / s >= unit); ++s) {
            const Shape p = cut(Shape{o.planes, o.bm, o.bn, 1, 0, false}, K, s, unit);
            if (p.splits != s) continue;
            const double each = (double)((tiles * s + 255) / 256);            // tiles of a compute unit
            const double k = each <= o.most ? std::max(alone, each * shared) : each * shared;
            const double cost = std::min(K, p.len) * k * 1e-9 + (each <= o.most ? 1 : each / o.most) * o.tile * 1e-6 + (s > 1 ? 4e-6 + (double)s * n * M * N * 8 / 5e12 : 0);
            if (best.cost < 0 || cost < (s > 1 && best.shape.splits == 1 ? 0.95 : 1) * best.cost) best = Chosen{p, cost};
        }
    }
    return best;
}

struct Work {                      // where things lie in the working memory
    Shape y, dx, dw;
    int ldx, ldz;
    size_t kept, x, w, dz, sums, share, total;
    int blocks, across, depth;     // column sums: row blocks, lanes a row, rows a block
};
// Planes of a 32-bit tensor are its three parts, 6 bytes a value, written once by one launch for x and w; a bf16 tensor is one as it lies, or copied where
// rows of it do not start on 16 bytes or hold whole chunks of eight.  Through registers a tensor is read as it lies; sources there hold eight columns
// at least (tile_product.h), so narrower layers take planes.
// two: dz of bf16 tensors in two parts.
Work plan_of(int n, int rows, int in, int out, int bf16, bool grad, bool packed, bool two)
{
    Work p{};
    p.ldx = up_to(in, 8);
    p.ldz = up_to(out, 8);
    const bool narrow = std::min(in, out) < 8;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    const double nx = (double)n * rows * p.ldx, nw = (double)n * in * p.ldz, nz = (double)n * rows * p.ldz;
    const size_t plane = bf16 ? 2 : 6;
    // of copying values into planes
    auto lay = [&](int cols, double values) { return !bf16 || cols % 8 ? 2e-6 + values * (bf16 ? 4 : 10) / 4e12 : 0.; };
    if (!grad) {
        const Chosen r = best_shape(n, rows, out, in, bf16, false, false), q = best_shape(n, rows, out, in, bf16, false, true);
        p.y = narrow || q.cost + lay(in, nx) + lay(out, nw) + (bf16 ? 0 : 2e-6) < r.cost ? q.shape : r.shape;
        if (p.y.planes) { p.x = take((size_t)nx * plane); p.w = take((size_t)nw * plane); }
        p.share = take(share_bytes(p.y, n, rows, out));
    } else {
        const Chosen rx = best_shape(n, rows, in, out, bf16, false, false, two), rw = best_shape(n, in, out, rows, bf16, true, false, two);
        const Chosen qx = best_shape(n, rows, in, out, bf16, false, true, two), qw = best_shape(n, in, out, rows, bf16, true, true, two);
        if (bf16) {
            p.dx = narrow || qx.cost + lay(out, nw) < rx.cost ? qx.shape : rx.shape;
            p.dw = narrow || qw.cost + lay(packed ? 8 : in, nx) < rw.cost ? qw.shape : rw.shape;
        } else {                                               // dz in one form for both products
            const bool planes = narrow || qx.cost + qw.cost + lay(in, nx) + lay(out, nw) + nz * 2 / 4e12 < rx.cost + rw.cost;
            p.dx = planes ? qx.shape : rx.shape;
            p.dw = planes ? qw.shape : rw.shape;
        }
        if (packed) p.kept = take((size_t)nx * (bf16 ? 2 : 4));
        if (p.dw.planes) p.x = take((size_t)nx * plane);
        if (p.dx.planes) p.w = take((size_t)nw * plane);
        p.dz = take((size_t)nz * (two ? 4 : p.dx.planes || p.dw.planes ? plane : bf16 ? 2 : 4));
        // few rows: one to a line of eight lanes, one block of them and no second launch for db
        p.across = 8;
        while (rows > 32 && p.across < 64 && p.across * 8 < p.ldz) p.across *= 2;
        const long long wide = (p.ldz + p.across * 8 - 1) / (p.across * 8);
        p.depth = rows > 32 ? 256 : 32;
        while (p.depth > 256 / p.across && (long long)n * wide * ((rows + p.depth - 1) / p.depth) < 1024) p.depth /= 2;
        p.blocks = std::max(1, (rows + p.depth - 1) / p.depth);
        p.sums = take((size_t)n * p.blocks * p.ldz * 4);
        p.share = take(std::max(share_bytes(p.dx, n, rows, in), share_bytes(p.dw, n, in, out)));
    }
    p.total = at;
    return p;
}

template <typename T, int BM, int BN, int WM, int WN, bool AA, bool BA, class SA, class SB, class Epi>
hipError_t launch_registers(const SA& a, const SB& b, int n, int M, int N, int K, const Shape& p, const Epi& epi, hipStream_t s)
{
    constexpr int P = std::max(SA::kPlanes, SB::kPlanes);
    constexpr bool wide = P > 1;
    constexpr int KS = BM == 32 ? (wide ? (BA ? 64 : 32) : 128) : P == 2 || (BN == 128 && !wide) ? 64 : 32, NBUF = wide || BM == 32 ? 1 : 2, AHEAD = wide && BM != 32 ? 1 : 2;
    constexpr unsigned kLds = NBUF * (SA::kPlanes * Image<AA, BM, KS>::kPlane + SB::kPlanes * Image<BA, BN, KS>::kPlane);
    if constexpr (Epi::kStaged) static_assert(WM * WN * Epi::template bytes<BN / WN / 32>() <= kLds, "the epilogue's blocks lie in the images");
    const int tm = (M + BM - 1) / BM, tn = (N + BN - 1) / BN;
    const long long total = (long long)n * p.splits * tm * tn;
    if (total == 0) return hipSuccess;
    if (total > 0x7fffff00ll) return hipErrorInvalidValue;
    layer_product_kernel<SA, AA, SB, BA, BM, BN, WM, WN, KS, NBUF, AHEAD, Epi>
        <<<line_grid(die_grid(total), WM * WN * 64), WM * WN * 64, 0, s>>>(a, b, K, tm, tn, p.splits, p.len, (int)total, epi);
    return hipGetLastError();
}
template <int PA, int PB, int BM, int BN, int WM, int WN, bool AA, bool BA, class Epi>
hipError_t launch_planes(const Plane3& a, const Plane3& b, int n, int M, int N, int K, const Shape& p, const Epi& epi, hipStream_t s)
{
    const int tm = (M + BM - 1) / BM, tn = (N + BN - 1) / BN;
    const long long total = (long long)n * p.splits * tm * tn;
    if (total == 0) return hipSuccess;
    if (total > 0x7fffff00ll) return hipErrorInvalidValue;
    layer_planes_kernel<AA, BA, PA, PB, BM, BN, WM, WN, Epi>
        <<<line_grid(die_grid(total), WM * WN * 64), WM * WN * 64, 0, s>>>(a, b, K, tm, tn, p.splits, p.len, (int)total, epi);
    return hipGetLastError();
}
// f(epilogue) launches the product; its shares are added and finished by a second launch
template <typename T, class F> hipError_t whole_or_shares(const Shape& p, int n, int M, int N, const Finish<T>& finish, float* share, hipStream_t s, F&& f)
{
    if (p.splits == 1) return f(FinishTile<T>{finish});
    const int ld = up_to(N, 8);
    const hipError_t e = f(StoreShare<>{share, M, N, ld, M, n, false, false});
    if (e != hipSuccess) return e;
    const long long lines = (long long)n * M, total = lines * (ld / 8);
    finish_shares_kernel<T><<<line_grid((total + 255) / 256, 256), 256, 0, s>>>(share, p.splits, lines * ld, ld, total, finish);
    return hipGetLastError();
}
template <bool AA, bool BA, int PA, int PB, typename T>
hipError_t planes_product(const Plane3& a, const Plane3& b, int n, int M, int N, int K, const Shape& p, const Finish<T>& finish, float* share, hipStream_t s)
{
    return whole_or_shares<T>(p, n, M, N, finish, share, s, [&](const auto& epi) {
        if constexpr (sizeof(T) == 2) {
            if (p.bm == 256) return launch_planes<PA, PB, 256, 256, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
            if (p.bn == 256) return launch_planes<PA, PB, 128, 256, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
            return launch_planes<PA, PB, 128, 128, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        } else return launch_planes<3, 3, 128, 256, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
    });
}
template <bool BA, typename T, class SA, class SB>
hipError_t launch_few(const SA& a, const SB& b, int n, int M, int N, int K, const Finish<T>& finish, hipStream_t s)
{
    constexpr int TN = few_columns(sizeof(T) == 2) / 32, NW = 8;
    const int tm = (M + 31) / 32, tn = (N + 32 * TN - 1) / (32 * TN);
    const long long total = (long long)n * tm * tn;
    layer_few_kernel<SA, SB, BA, TN, NW, T><<<line_grid(die_grid(total), NW * 64), NW * 64, 0, s>>>(a, b, K, tm, tn, (int)total, finish);
    return hipGetLastError();
}
template <bool AA, bool BA, typename T, class SA, class SB>
hipError_t registers_product(const SA& a, const SB& b, int n, int M, int N, int K, const Shape& p, const Finish<T>& finish, float* share, hipStream_t s)
{
    if constexpr (AA)
        if (p.few) return launch_few<BA, T>(a, b, n, M, N, K, finish, s);
    constexpr bool two = SA::kPlanes == 2 || SB::kPlanes == 2;
    return whole_or_shares<T>(p, n, M, N, finish, share, s, [&](const auto& epi) {
        if constexpr (AA)
            if (p.bm == 32) return launch_registers<T, 32, 128, 1, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        if constexpr (!two) {
            if (p.bm == 128) return launch_registers<T, 128, 128, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
            if (p.bn == 128) return launch_registers<T, 64, 128, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        }
        return launch_registers<T, 64, 64, 2, 2, AA, BA>(a, b, n, M, N, K, p, epi, s);
    });
}

// A tensor [n][rows][cols] whose three parts go to out [3][n][rows][ld], zero beyond cols.
struct Parts {
    const float* x;
    long long rep, row;
    int rows, cols, ld;
    long long total, plane;        // chunks of eight; values of a plane
    __bf16* out;
};
Parts parts_of(const Rows& r, int n, int rows, int cols, void* out)
{
    const int ld = up_to(cols, 8);
    const long long plane = (long long)n * rows * ld;
    return Parts{(const float*)r.p, r.rep, r.row, rows, cols, ld, plane / 8, plane, (__bf16*)out};
}
__global__ __launch_bounds__(256) void parts_kernel(Parts first, Parts second)
{
    long long at = line_block() * 256 + threadIdx.x;
    const bool other = at >= first.total;
    const Parts a = other ? second : first;
    if (other) at -= first.total;
    if (at >= a.total) return;
    const int chunks = a.ld / 8;
    const long long line = at / chunks;
    const int c = (int)(at - line * chunks) * 8, k = (int)(line / a.rows), t = (int)(line - (long long)k * a.rows);
    Chunk<float> v;
    u4 part[3];
    v.load(a.x + k * a.rep + t * a.row + c, a.cols - c);
    Source<float>::split(v, part);
#pragma unroll
    for (int s = 0; s < 3; ++s) *(u4*)(a.out + s * a.plane + at * 8) = part[s];
}
hipError_t lay_parts(const Parts& first, const Parts& second, hipStream_t s)
{
    const long long total = first.total + second.total;
    if (total == 0) return hipSuccess;
    parts_kernel<<<line_grid((total + 255) / 256, 256), 256, 0, s>>>(first, second);
    return hipGetLastError();
}
Plane3 plane_of(const Parts& p) { return Plane3{p.out, (long long)p.rows * p.ld, p.plane, p.ld, p.rows, p.ld, nullptr}; }
// a bf16 tensor as a plane: as it lies, or copied to `at`
hipError_t plane_of(const Rows& r, int n, int rows, int cols, void* at, Plane3& out, hipStream_t s)
{
    out = Plane3{(const __bf16*)r.p, r.rep, 0, (int)r.row, rows, cols, nullptr};
    if (is_plane(r, cols)) return hipSuccess;
    const int ld = up_to(cols, 8);
    out = Plane3{(const __bf16*)at, (long long)rows * ld, 0, ld, rows, ld, nullptr};
    return lay_out<__bf16, 1>(n, rows, cols, ld, r, Labelled{nullptr, 0}, nullptr, (__bf16*)at, s);
}

template <typename T> hipError_t forward(const LayerArgs& a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    const Work p = plan_of(a.n, a.rows, a.in, a.out, a.bf16, false, false, false);
    char* work = (char*)a.work;
    float* share = (float*)(work + p.share);
    const Finish<T> finish{(const float*)a.bias.p, a.bias.rep, a.residual, a.pre, a.y, a.rows, a.out, a.act, a.draws};
    if (!p.y.planes)
        return registers_product<true, false, T>(source<T>(a.x, a.rows, a.in), source<T>(a.w, a.in, a.out), a.n, a.rows, a.out, a.in, p.y, finish, share, s);
    Plane3 x, w;
    hipError_t e;
    if constexpr (sizeof(T) == 2) {
        if ((e = plane_of(a.x, a.n, a.rows, a.in, work + p.x, x, s)) != hipSuccess || (e = plane_of(a.w, a.n, a.in, a.out, work + p.w, w, s)) != hipSuccess) return e;
    } else {
        const Parts px = parts_of(a.x, a.n, a.rows, a.in, work + p.x), pw = parts_of(a.w, a.n, a.in, a.out, work + p.w);
        if ((e = lay_parts(px, pw, s)) != hipSuccess) return e;
        x = plane_of(px); w = plane_of(pw);
    }
    return planes_product<true, false, 1, 1, T>(x, w, a.n, a.rows, a.out, a.in, p.y, finish, share, s);
}

// ---- gradient ---------------------------------------------------------------------------------------------------------------
// Two bf16 parts of a float: its sign, exponent and first eight bits, and what is left, rounded.  Both have the float's sign, and neither is zero unless
// the float is (a value that the first part holds whole gets 2^-20 of it as its second), so that their products with an infinity are the infinity that
// the float's product is; an infinity or a NaN is both of its parts.
__device__ __forceinline__ void parts2(const float (&v)[8], u4& high, u4& low)
{
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float top = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v[e]) & 0xffff0000u), left = v[e] - top;
        rest[e] = left != left ? v[e] : left == 0.f ? top * 0x1p-20f : left;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        high[e] = __builtin_bit_cast(unsigned, v[2 * e]) >> 16 | (__builtin_bit_cast(unsigned, v[2 * e + 1]) & 0xffff0000u);
        low[e] = to_bf16x2(rest[2 * e], rest[2 * e + 1]);
    }
}

// dz = D'(dy) a'(pre), eight columns a lane, into [replicas][rows][ld] (PARTS = 1), its two or three bf16 parts into such planes (2, 3) or nowhere (0), and
// the column sums of a block's rows (16 x 1024 x 2048 bf16 with gelu, two parts: 48 us = 5.6 TB/s), a line of `ld` of them a block and sums_rep apart
// from replica to replica: db itself where one block has all rows.  A
// dropped value is zero whatever dy and pre hold there, one that ReLU has switched off whatever dy holds.
template <typename T, int PARTS>
__global__ __launch_bounds__(256) void slope_kernel(const T* dy, long long yrep, long long yrow, const T* pre, long long prep, long long prow, int rows, int cols,
                                                    int ld, int across, int depth, int act, Draws d, void* dz, long long plane, float* sums, long long sums_rep)
{
    __shared__ float part[256][9];
    const int lane = threadIdx.x % across, line = threadIdx.x / across, lines = 256 / across;
    const int c = (blockIdx.x * across + lane) * 8, k = blockIdx.z, first = blockIdx.y * depth, last = min(rows, first + depth);
    const unsigned long long call = d.limit ? call_of(d) : 0ull;
    float sum[8] = {};
    if (c < ld)
        for (int t = first + line; t < last; t += lines) {
            Chunk<T> in, at;
            float v[8], z[8];
            in.load(dy + k * yrep + t * yrow + c, cols - c);
            if (act != kNone) at.load(pre + k * prep + t * prow + c, cols - c);
            in.get(v);
            if (act != kNone) {
                at.get(z);
                if (act == kRelu) each8([&](int e) { v[e] = relu_slope(v[e], z[e]); });
                else if (act == kGelu) each8([&](int e) { v[e] *= slope(z[e], kGelu); });
                else each8([&](int e) { v[e] *= slope(z[e], kSilu); });
            }
            if (d.limit) kept8(d, call, k, t, c, [&](int e, bool kept) { v[e] = kept ? v[e] * d.scale : 0.f; });
            each8([&](int e) { if (c + e >= cols) v[e] = 0.f; sum[e] += v[e]; });
            const long long to = ((long long)k * rows + t) * ld + c;
            if constexpr (PARTS == 1) store_chunk((T*)dz + to, 8, v);
            if constexpr (PARTS == 2) {
                u4 high, low;
                parts2(v, high, low);
                __bf16* out = (__bf16*)dz + to;
                *(u4*)out = high;
                *(u4*)(out + plane) = low;
            }
            if constexpr (PARTS == 3) {
                u2 h[2], m[2], l[2];
                parts3(f4{v[0], v[1], v[2], v[3]}, h[0], m[0], l[0]);
                parts3(f4{v[4], v[5], v[6], v[7]}, h[1], m[1], l[1]);
                __bf16* out = (__bf16*)dz + to;
                *(u4*)out = join8(h[0], h[1]);
                *(u4*)(out + plane) = join8(m[0], m[1]);
                *(u4*)(out + 2 * plane) = join8(l[0], l[1]);
            }
        }
    if (!sums) return;
    each8([&](int e) { part[threadIdx.x][e] = sum[e]; });
    __syncthreads();
    for (int i = threadIdx.x; i < across * 8; i += 256) {
        float v = 0.f;
        for (int r = 0; r < lines; ++r) v += part[r * across + i / 8][i % 8];
        const int col = blockIdx.x * across * 8 + i;
        if (col < cols) sums[k * sums_rep + (long long)blockIdx.y * ld + col] = v;
    }
}
// db from the blocks' sums: 32 columns a workgroup, eight threads a column, each every eighth block, then the eight in order
__global__ __launch_bounds__(256) void column_sums_kernel(const float* sums, int blocks, int ld, int cols, float* db, long long rep)
{
    __shared__ float part[8][32];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, group = threadIdx.x / 32, k = blockIdx.y;
    float v = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (int b = group; b < blocks; b += 8) v += sums[((long long)k * blocks + b) * ld + c];
    }
    part[group][threadIdx.x % 32] = v;
    __syncthreads();
    if (group || c >= cols) return;
#pragma unroll
    for (int g = 1; g < 8; ++g) v += part[g][threadIdx.x % 32];
    db[k * rep + c] = v;
}

// Whether dz of bf16 tensors takes two parts: ReLU's is dy or zero.  Rounded to one, dz adds an error of 1.6e-3 of their norm to dx and dW, as much as their
// own rounding; two parts add none that shows, and cost twice the operations (dx and dW of 8192 x 4096 x 4096 866 us, of one part 469).
inline bool has_two_parts(int act, unsigned drop_limit) { return drop_limit || act == kGelu || act == kSilu; }
template <bool TWO, class S> auto parted(const TwoParts& two, const S& one)
{
    if constexpr (TWO) return two;
    else return one;
}

template <typename T> hipError_t backward(const LayerArgs& a, hipStream_t s)
{
    constexpr bool half = sizeof(T) == 2;
    const bool two = half && has_two_parts(a.act, a.draws.limit);
    const Work p = plan_of(a.n, a.rows, a.in, a.out, a.bf16, true, a.packed.q, two);
    char* work = (char*)a.work;
    float *share = (float*)(work + p.share), *sums = (float*)(work + p.sums);
    const bool want_dx = a.dx.p && a.rows, want_dw = a.dw.p, planes = (want_dx && p.dx.planes) || (want_dw && p.dw.planes);
    hipError_t e = hipSuccess;
    // dz is formed in the working memory; where it is dy itself it is read as it lies, if the products can
    const bool there = a.act == kNone && !a.draws.limit && (!planes || (half && is_plane(a.dy, a.out))), form = (want_dx || want_dw) && !there;
    const long long plane = (long long)a.n * a.rows * p.ldz;
    if (a.rows && (form || a.db.p)) {
        const dim3 grid((unsigned)((p.ldz + p.across * 8 - 1) / (p.across * 8)), (unsigned)p.blocks, (unsigned)a.n);
        auto* kernel = !form ? slope_kernel<T, 0> : half ? (two ? slope_kernel<T, half ? 2 : 1> : slope_kernel<T, 1>) : planes ? slope_kernel<T, half ? 1 : 3> : slope_kernel<T, 1>;
        kernel<<<grid, 256, 0, s>>>((const T*)a.dy.p, a.dy.rep, a.dy.row, (const T*)a.pre.p, a.pre.rep, a.pre.row, a.rows, a.out, p.ldz, p.across, p.depth,
                                    a.act, a.draws, work + p.dz, plane, p.blocks == 1 ? (float*)a.db.p : a.db.p ? sums : nullptr,
                                    p.blocks == 1 ? a.db.rep : (long long)p.blocks * p.ldz);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.db.p && (p.blocks > 1 || a.rows == 0)) {
        column_sums_kernel<<<dim3((unsigned)((a.out + 31) / 32), (unsigned)a.n), 256, 0, s>>>(sums, a.rows ? p.blocks : 0, p.ldz, a.out, (float*)a.db.p, a.db.rep);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    Rows x = a.x;
    if (want_dw && a.packed.q) {                               // the checkpoint's values; columns beyond n_in belong to no row of dW
        x = Rows{work + p.kept, (long long)a.rows * p.ldx, p.ldx};
        if (a.rows && (e = launch_unpack(a.n, a.rows, a.in, half, a.packed.q, x, s)) != hipSuccess) return e;
    }
    const Rows z = there ? a.dy : Rows{work + p.dz, (long long)a.rows * p.ldz, p.ldz};
    const int wz = there ? a.out : p.ldz;
    const Plane3 pz{(const __bf16*)z.p, z.rep, half && !two ? 0 : plane, (int)z.row, a.rows, wz, nullptr};
    const TwoParts tz{(const __bf16*)z.p, z.rep, z.row, a.rows, wz, plane};
    Plane3 px{}, pw{};
    if constexpr (half) {
        if (want_dw && p.dw.planes && (e = plane_of(x, a.n, a.rows, a.packed.q ? p.ldx : a.in, work + p.x, px, s)) != hipSuccess) return e;
        if (want_dx && p.dx.planes && (e = plane_of(a.w, a.n, a.in, a.out, work + p.w, pw, s)) != hipSuccess) return e;
    } else if (planes) {
        const Parts none{}, fx = want_dw ? parts_of(x, a.n, a.rows, a.in, work + p.x) : none, fw = want_dx ? parts_of(a.w, a.n, a.in, a.out, work + p.w) : none;
        if ((e = lay_parts(fx, fw, s)) != hipSuccess) return e;
        px = plane_of(fx); pw = plane_of(fw);
    }
    if (want_dx) {
        const Finish<T> finish = store_only<T>(a.dx, a.rows, a.in);
        const auto w = source<T>(a.w, a.in, a.out);
        if (half && two)
            e = p.dx.planes ? planes_product<true, true, half ? 2 : 1, 1, T>(pz, pw, a.n, a.rows, a.in, a.out, p.dx, finish, share, s)
                            : registers_product<true, true, T>(parted<half>(tz, source<T>(z, a.rows, wz)), w, a.n, a.rows, a.in, a.out, p.dx, finish, share, s);
        else
            e = p.dx.planes ? planes_product<true, true, 1, 1, T>(pz, pw, a.n, a.rows, a.in, a.out, p.dx, finish, share, s)
                            : registers_product<true, true, T>(source<T>(z, a.rows, wz), w, a.n, a.rows, a.in, a.out, p.dx, finish, share, s);
        if (e != hipSuccess) return e;
    }
    if (!want_dw) return hipSuccess;
    const Finish<T> finish = store_only<T>(a.dw, a.in, a.out);
    const auto sx = source<T>(x, a.rows, a.in);
    if (half && two) {
        if (p.dw.planes) return planes_product<false, false, 1, half ? 2 : 1, T>(px, pz, a.n, a.in, a.out, a.rows, p.dw, finish, share, s);
        return registers_product<false, false, T>(sx, parted<half>(tz, source<T>(z, a.rows, wz)), a.n, a.in, a.out, a.rows, p.dw, finish, share, s);
    }
    if (p.dw.planes) return planes_product<false, false, 1, 1, T>(px, pz, a.n, a.in, a.out, a.rows, p.dw, finish, share, s);
    return registers_product<false, false, T>(sx, source<T>(z, a.rows, wz), a.n, a.in, a.out, a.rows, p.dw, finish, share, s);
}

}  // namespace

size_t layer_work_bytes(int n, int rows, int in, int out, int bf16, int act, float drop, bool grad)
{
    const size_t one = plan_of(n, rows, in, out, bf16, false, false, false).total;       // a workspace for the gradient serves the forward pass too
    const bool two = bf16 && has_two_parts(act, drop_limit(drop));
    return grad ? std::max({one, plan_of(n, rows, in, out, bf16, true, false, two).total, plan_of(n, rows, in, out, bf16, true, true, two).total}) : one;
}
hipError_t launch_layer_forward(const LayerArgs& a, hipStream_t s) { return a.bf16 ? forward<__bf16>(a, s) : forward<float>(a, s); }
hipError_t launch_layer_backward(const LayerArgs& a, hipStream_t s) { return a.bf16 ? backward<__bf16>(a, s) : backward<float>(a, s); }

}  // namespace layer
}  // namespace hadfl
