// A dense layer and its gradient, grouped over replicas: y = r + D(a(x W + b)), a an activation, D dropout, r a residual.
//   forward    one product whose epilogue does the rest on 32-bit sums, eight columns of a row at a time; pre = x W + b is left for the
//              gradient where that is asked for
//   gradient   dz = D'(dy) a'(pre) and its column sums db in one pass over dy, then dx = dz W^T and dW = x^T dz
// bf16: dz is rounded to bf16 for the two products (2^-9 of a value, as the outputs themselves are rounded; a second part would double both
// products); db is summed before that.  fp32: operands enter as three bf16 parts, six products (tile_product.h).
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
// Operands in planes of bf16, straight from memory to LDS (direct_product.h: Loader), slabs of 64 k.  A wave reads the operands of a step of 16 k while it
// multiplies the step before, across slabs too: the barrier that frees a slab's image and says that the next one has arrived lies before the slab's
// last step, whose operands are in registers by then, so that the matrix cores have work while the first operands of the next slab are read.
template <bool A_ALONG, bool B_ALONG, int BM, int BN, int WM, int WN, class Epi>
__global__ __launch_bounds__(WM * WN * 64) void layer_planes_kernel(Plane3 a, Plane3 b, int K, int tiles_m, int tiles_n, int splits, int split_len, int total, Epi epi)
{
    constexpr int NT = WM * WN * 64, TM = BM / WM / 32, TN = BN / WN / 32, kSteps = kSlab / 16;
    typedef Loader<A_ALONG, BM, NT> LA;
    typedef Loader<B_ALONG, BN, NT> LB;
    constexpr int kImage = LA::kBytes + LB::kBytes, IMAGES = kImage > 49152 ? 2 : kImage > 32768 ? 3 : 4, kLoads = LA::kLoads + LB::kLoads;
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
    const int k_begin = t.split * split_len, k_end = min(K, k_begin + split_len), slabs = k_begin < k_end ? (k_end - k_begin + kSlab - 1) / kSlab : 0;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) t.acc[i][j] = f16{};
    LA la;
    LB lb;
    la.init(tid, a.ld);
    lb.init(tid, b.ld);

    auto issue = [&](int slab, char* image) {
        la.issue(a, pa, bm, k_begin + slab * kSlab, wave, image);
        lb.issue(b, pb, bn, k_begin + slab * kSlab, wave, image + LA::kBytes);
    };
    bf16x8 fa[2][TM], fb[2][TN];
    auto read = [&](const char* image, int step, int to) {
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[to][i] = LA::read(image, wm + 32 * i, step, t.lane);
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[to][j] = LB::read(image + LA::kBytes, wn + 32 * j, step, t.lane);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                t.acc[i][j] = Epi::kLaneM ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[from][j], fa[from][i], t.acc[i][j], 0, 0, 0)
                                          : __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[from][i], fb[from][j], t.acc[i][j], 0, 0, 0);
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
};
size_t share_bytes(const Shape& p, int n, int M, int N) { return p.splits > 1 ? align256((size_t)p.splits * n * M * up_to(N, 8) * 4) : 0; }

Shape cut(Shape p, int K, int splits, int unit)
{
    p.len = std::max(unit, up_to((K + splits - 1) / splits, unit));
    p.splits = std::max(1, (K + p.len - 1) / p.len);
    return p;
}
// Tiles that there are, with what they cost in nanoseconds a k of a contraction: of a workgroup alone on its compute unit, and of each of several there
// (`most` fit), measured over 64 to 8192 rows, 200 to 4096 inputs and outputs; and in microseconds what a tile costs beside.
struct Choice {
    bool planes;
    int bm, bn, most;
    struct { double alone, shared; } f32, bf16;
    double tile;
};
constexpr Choice kChoices[] = {{false, 32, 128, 3, {23, 15}, {6.3, 5}, 3}, {false, 64, 64, 4, {25, 15.5}, {8.8, 4.9}, 3}, {false, 64, 128, 2, {28, 27}, {7.5, 7.3}, 3},
                               {false, 128, 128, 2, {46, 46}, {10, 11}, 4}, {true, 128, 128, 1, {0, 0}, {7, 9.6}, 4}, {true, 128, 256, 1, {0, 0}, {11.5, 16}, 5},
                               {true, 256, 256, 1, {0, 0}, {21, 28}, 8}};
// The cheapest tiles and shares by that; `lay`: seconds to copy operands into planes first.  A share is written and read at 5 TB/s, and joining them is one more launch, 4 us.  Chosen / best of all, us:
//   bf16  y of 16 x 1024 x 512 x 2048 47.9 / 47.7, 4096 x 1024 x 4096 38.8 / 38.8 (128 x 128 tiles 51), 8192 x 4096 x 4096 232 / 232 (315); dx of the
//         first 39.9 / 39.7 (256 x 256 tiles 55), dW 38.5 / 38.5
//   fp32  the same 205 / 201, 194 / 194, 1490 / 1487, 194 / 192, 191 / 191; 64 x 64 tiles take 250, 252 and 1964 of the first three
Shape best_shape(int n, int M, int N, int K, int bf16, bool across, bool planes, bool registers, double lay)
{
    Shape best{};
    double least = -1;
    for (const Choice& o : kChoices) {
        if ((o.planes ? !planes : !registers) || (o.bm == 32 && (M > 32 || across))) continue;
        const long long tiles = (long long)n * ((M + o.bm - 1) / o.bm) * ((N + o.bn - 1) / o.bn);
        const int unit = bf16 && o.bm == 32 ? 128 : 64;                       // whole slabs of every kernel of these tiles
        const double alone = bf16 ? o.bf16.alone : o.f32.alone, shared = bf16 ? o.bf16.shared : o.f32.shared;
        for (int s = 1; s <= 64 && (s == 1 || K / s >= unit); ++s) {
            const Shape p = cut(Shape{o.planes, o.bm, o.bn, 1, 0}, K, s, unit);
            if (p.splits != s) continue;
            const double each = (double)((tiles * s + 255) / 256);            // tiles of a compute unit
            const double k = each <= o.most ? std::max(alone, each * shared) : each * shared;
            const double cost = std::min(K, p.len) * k * 1e-9 + (each <= o.most ? 1 : each / o.most) * o.tile * 1e-6 + (o.planes ? lay : 0) + (s > 1 ? 4e-6 + (double)s * n * M * N * 8 / 5e12 : 0);
            if (least < 0 || cost < (s > 1 && best.splits == 1 ? 0.95 : 1) * least) { best = p; least = cost; }
        }
    }
    return best;
}

struct Work {                      // where things lie in the working memory
    Shape y, dx, dw;
    int ldx, ldz;
    size_t x, w, dz, sums, share, total;
    int blocks, across, depth;     // column sums: row blocks, lanes a row, rows a block
};
// Sources through registers hold eight columns at least (tile_product.h): narrower tensors are copied into rows of eight.  bf16 operands of products of
// planes are copied where they do not lie as planes do, which shows only at the call.
Work plan_of(int n, int rows, int in, int out, int bf16, bool grad, bool packed)
{
    Work p{};
    p.ldx = up_to(in, 8);
    p.ldz = up_to(out, 8);
    const bool narrow = std::min(in, out) < 8;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    // rows of a size that is no multiple of eight are copied, a launch and their bytes twice
    auto lay = [&](int lines, int cols) { return cols % 8 ? 4e-6 + (double)n * lines * cols * 4 / 4e12 : 0.; };
    auto shape = [&](int M, int N, int K, bool across, double copies) { return best_shape(n, M, N, K, bf16, across, bf16, !bf16 || !narrow, copies); };
    const size_t size = bf16 ? 2 : 4, x = (size_t)n * rows * p.ldx * size, w = (size_t)n * in * p.ldz * size;
    if (!grad) {
        p.y = shape(rows, out, in, false, lay(rows, in) + lay(in, out));
        if (p.y.planes || in < 8) p.x = take(x);
        if (p.y.planes || out < 8) p.w = take(w);
        p.share = take(share_bytes(p.y, n, rows, out));
    } else {
        p.dx = shape(rows, in, out, false, lay(in, out));
        p.dw = shape(in, out, rows, true, packed ? 0. : lay(rows, in));
        if (packed) p.x = take((size_t)n * rows * p.ldx * 2);
        else if (p.dw.planes || in < 8) p.x = take(x);
        if (p.dx.planes || out < 8) p.w = take(w);
        p.dz = take((size_t)n * rows * p.ldz * size);
        p.across = 8;
        while (p.across < 64 && p.across * 8 < p.ldz) p.across *= 2;
        const long long wide = (p.ldz + p.across * 8 - 1) / (p.across * 8);
        p.depth = 256;
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
    constexpr bool wide = SA::kPlanes == 3 || SB::kPlanes == 3;
    constexpr int KS = BM == 32 ? (wide ? (BA ? 64 : 32) : 128) : BN == 128 && !wide ? 64 : 32, NBUF = wide || BM == 32 ? 1 : 2, AHEAD = wide && BM != 32 ? 1 : 2;
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
template <int BM, int BN, int WM, int WN, bool AA, bool BA, class Epi>
hipError_t launch_planes(const Plane3& a, const Plane3& b, int n, int M, int N, int K, const Shape& p, const Epi& epi, hipStream_t s)
{
    const int tm = (M + BM - 1) / BM, tn = (N + BN - 1) / BN;
    const long long total = (long long)n * p.splits * tm * tn;
    if (total == 0) return hipSuccess;
    if (total > 0x7fffff00ll) return hipErrorInvalidValue;
    layer_planes_kernel<AA, BA, BM, BN, WM, WN, Epi>
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
template <bool AA, bool BA>
hipError_t planes_product(const Plane3& a, const Plane3& b, int n, int M, int N, int K, const Shape& p, const Finish<__bf16>& finish, float* share, hipStream_t s)
{
    return whole_or_shares<__bf16>(p, n, M, N, finish, share, s, [&](const auto& epi) {
        if (p.bm == 256) return launch_planes<256, 256, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        if (p.bn == 256) return launch_planes<128, 256, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        return launch_planes<128, 128, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
    });
}
template <bool AA, bool BA, typename T, class SA, class SB>
hipError_t registers_product(const SA& a, const SB& b, int n, int M, int N, int K, const Shape& p, const Finish<T>& finish, float* share, hipStream_t s)
{
    return whole_or_shares<T>(p, n, M, N, finish, share, s, [&](const auto& epi) {
        if (p.bm == 128) return launch_registers<T, 128, 128, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        if constexpr (AA)
            if (p.bm == 32) return launch_registers<T, 32, 128, 1, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        if (p.bn == 64) return launch_registers<T, 64, 64, 2, 2, AA, BA>(a, b, n, M, N, K, p, epi, s);
        return launch_registers<T, 64, 128, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
    });
}

// x [replicas][rows][cols] -> [replicas][rows][8], zero beyond cols
template <typename T>
__global__ __launch_bounds__(256) void widen_kernel(const T* x, long long rep, long long row, int rows, int cols, long long total, T* out)
{
    const long long at = line_block() * 256 + threadIdx.x;
    if (at >= total) return;
    const int k = (int)(at / rows), t = (int)(at - (long long)k * rows);
    Chunk<T> v;
    float f[8];
    v.load(x + k * rep + t * row, cols);
    v.get(f);
    store_chunk(out + at * 8, 8, f);
}
// A tensor [n][rows][cols] as a product takes it: as it lies, or copied to `at`.
template <typename T> hipError_t ready(const Rows& r, int n, int rows, int cols, bool planes, void* at, Rows& out, int& width, hipStream_t s)
{
    out = r;
    width = cols;
    if (planes ? is_plane(r, cols) : cols >= 8) return hipSuccess;
    width = up_to(cols, 8);
    out = Rows{at, (long long)rows * width, width};
    const long long total = (long long)n * rows;
    if (total == 0) return hipSuccess;
    if constexpr (sizeof(T) == 2) return lay_out<__bf16, 1>(n, rows, cols, width, r, Labelled{nullptr, 0}, nullptr, (__bf16*)at, s);
    else {
        widen_kernel<T><<<line_grid((total + 255) / 256, 256), 256, 0, s>>>((const T*)r.p, r.rep, r.row, rows, cols, total, (T*)at);
        return hipGetLastError();
    }
}
Plane3 plane(const Rows& r, int rows, int cols) { return Plane3{(const __bf16*)r.p, r.rep, 0, (int)r.row, rows, cols, nullptr}; }

// C = A B of operands that are ready
template <bool AA, bool BA, typename T, typename TA>
hipError_t product(const Rows& a, int a_rows, int a_cols, const Rows& b, int b_rows, int b_cols, int n, int M, int N, int K, const Shape& p, const Finish<T>& finish,
                   float* share, hipStream_t s)
{
    if constexpr (sizeof(T) == 2)
        if (p.planes) return planes_product<AA, BA>(plane(a, a_rows, a_cols), plane(b, b_rows, b_cols), n, M, N, K, p, finish, share, s);
    return registers_product<AA, BA, T>(source<TA>(a, a_rows, a_cols), source<T>(b, b_rows, b_cols), n, M, N, K, p, finish, share, s);
}

template <typename T> hipError_t forward(const LayerArgs& a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    const Work p = plan_of(a.n, a.rows, a.in, a.out, a.bf16, false, false);
    char* work = (char*)a.work;
    const Finish<T> finish{(const float*)a.bias.p, a.bias.rep, a.residual, a.pre, a.y, a.rows, a.out, a.act, a.draws};
    Rows x, w;
    int wx, ww;
    hipError_t e = ready<T>(a.x, a.n, a.rows, a.in, p.y.planes, work + p.x, x, wx, s);
    if (e == hipSuccess) e = ready<T>(a.w, a.n, a.in, a.out, p.y.planes, work + p.w, w, ww, s);
    if (e != hipSuccess) return e;
    return product<true, false, T, T>(x, a.rows, wx, w, a.in, ww, a.n, a.rows, a.out, a.in, p.y, finish, (float*)(work + p.share), s);
}

// ---- gradient ---------------------------------------------------------------------------------------------------------------
// dz = D'(dy) a'(pre), eight columns a lane, into [replicas][rows][ld] if STORE, and the column sums of a block's rows.  A dropped value is zero
// whatever dy and pre hold there.
template <typename T, bool STORE>
__global__ __launch_bounds__(256) void slope_kernel(const T* dy, long long yrep, long long yrow, const T* pre, long long prep, long long prow, int rows, int cols,
                                                    int ld, int across, int depth, int act, Draws d, T* dz, float* sums)
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
                if (act == kRelu) each8([&](int e) { v[e] *= slope(z[e], kRelu); });
                else if (act == kGelu) each8([&](int e) { v[e] *= slope(z[e], kGelu); });
                else each8([&](int e) { v[e] *= slope(z[e], kSilu); });
            }
            if (d.limit) kept8(d, call, k, t, c, [&](int e, bool kept) { v[e] = kept ? v[e] * d.scale : 0.f; });
            each8([&](int e) { if (c + e >= cols) v[e] = 0.f; sum[e] += v[e]; });
            if constexpr (STORE) store_chunk(dz + ((long long)k * rows + t) * ld + c, 8, v);
        }
    if (!sums) return;
    each8([&](int e) { part[threadIdx.x][e] = sum[e]; });
    __syncthreads();
    for (int i = threadIdx.x; i < across * 8; i += 256) {
        float v = 0.f;
        for (int r = 0; r < lines; ++r) v += part[r * across + i / 8][i % 8];
        const int col = blockIdx.x * across * 8 + i;
        if (col < ld) sums[((long long)k * gridDim.y + blockIdx.y) * ld + col] = v;
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

template <typename T> hipError_t backward(const LayerArgs& a, hipStream_t s)
{
    const Work p = plan_of(a.n, a.rows, a.in, a.out, a.bf16, true, a.packed.q);
    char* work = (char*)a.work;
    float *share = (float*)(work + p.share), *sums = (float*)(work + p.sums);
    const bool want_dx = a.dx.p && a.rows, want_dw = a.dw.p, planes = (want_dx && p.dx.planes) || (want_dw && p.dw.planes);
    hipError_t e = hipSuccess;
    // dz is formed in the working memory; where it is dy itself it is read as it lies, if the products can
    const bool there = a.act == kNone && !a.draws.limit && a.out >= 8 && (!planes || is_plane(a.dy, a.out)), form = (want_dx || want_dw) && !there;
    if (a.rows && (form || a.db.p)) {
        const dim3 grid((unsigned)((p.ldz + p.across * 8 - 1) / (p.across * 8)), (unsigned)p.blocks, (unsigned)a.n);
        auto* kernel = form ? slope_kernel<T, true> : slope_kernel<T, false>;
        kernel<<<grid, 256, 0, s>>>((const T*)a.dy.p, a.dy.rep, a.dy.row, (const T*)a.pre.p, a.pre.rep, a.pre.row, a.rows, a.out, p.ldz, p.across, p.depth,
                                    a.act, a.draws, (T*)(work + p.dz), a.db.p ? sums : nullptr);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.db.p) {
        column_sums_kernel<<<dim3((unsigned)((a.out + 31) / 32), (unsigned)a.n), 256, 0, s>>>(sums, a.rows ? p.blocks : 0, p.ldz, a.out, (float*)a.db.p, a.db.rep);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const Rows z = there ? a.dy : Rows{work + p.dz, (long long)a.rows * p.ldz, p.ldz};
    const int wz = there ? a.out : p.ldz;
    if (want_dx) {
        Rows w;
        int ww;
        if ((e = ready<T>(a.w, a.n, a.in, a.out, p.dx.planes, work + p.w, w, ww, s)) != hipSuccess) return e;
        e = product<true, true, T, T>(z, a.rows, wz, w, a.in, ww, a.n, a.rows, a.in, a.out, p.dx, store_only<T>(a.dx, a.rows, a.in), share, s);
        if (e != hipSuccess) return e;
    }
    if (!want_dw) return hipSuccess;
    const Finish<T> to_dw = store_only<T>(a.dw, a.in, a.out);
    if (a.packed.q) {                                          // the checkpoint's values, exact in bf16; columns beyond n_in belong to no row of dW
        const Rows kept{work + p.x, (long long)a.rows * p.ldx, p.ldx};
        if (a.rows && (e = launch_unpack(a.n, a.rows, a.in, 1, a.packed.q, kept, s)) != hipSuccess) return e;
        return product<false, false, T, __bf16>(kept, a.rows, p.ldx, z, a.rows, wz, a.n, a.in, a.out, a.rows, p.dw, to_dw, share, s);
    }
    Rows x;
    int wx;
    if ((e = ready<T>(a.x, a.n, a.rows, a.in, p.dw.planes, work + p.x, x, wx, s)) != hipSuccess) return e;
    return product<false, false, T, T>(x, a.rows, wx, z, a.rows, wz, a.n, a.in, a.out, a.rows, p.dw, to_dw, share, s);
}

}  // namespace

size_t layer_work_bytes(int n, int rows, int in, int out, int bf16, bool grad)
{
    const size_t one = plan_of(n, rows, in, out, bf16, false, false).total;       // a workspace for the gradient serves the forward pass too
    return grad ? std::max({one, plan_of(n, rows, in, out, bf16, true, false).total, plan_of(n, rows, in, out, bf16, true, true).total}) : one;
}
hipError_t launch_layer_forward(const LayerArgs& a, hipStream_t s) { return a.bf16 ? forward<__bf16>(a, s) : forward<float>(a, s); }
hipError_t launch_layer_backward(const LayerArgs& a, hipStream_t s) { return a.bf16 ? backward<__bf16>(a, s) : backward<float>(a, s); }

}  // namespace layer
}  // namespace hadfl
