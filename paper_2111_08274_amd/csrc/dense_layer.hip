// A dense layer and its gradient, grouped over replicas: y = r + D(a(x W + b)), a an activation, D dropout, r a residual.
//   forward    one product whose epilogue does the rest on 32-bit sums, eight columns of a row at a time; pre = x W + b is left for the
//              gradient where that is asked for
//   gradient   dz = D'(dy) a'(pre) and its column sums db in one pass over dy, then dx = dz W^T and dW = x^T dz
// bf16: dz is rounded to bf16 for the two products (2^-9 of a value, as the outputs themselves are rounded; a second part would double both
// products); db is summed before that.  fp32: operands enter as three bf16 parts, six products (tile_product.h, direct_product.h).
#include "direct_product.h"
#include "layer.h"

namespace hadfl {
namespace layer {

using namespace head;

namespace {

// ---- epilogue -----------------------------------------------------------------------------------------------------------
// eight 32-bit sums of columns n.. of row m to what the layer returns; a null pointer leaves its part out
template <typename T> struct Finish {
    const float* bias;
    long long bias_rep;
    Rows residual, pre, y;
    int rows, cols, act;
    Draws draws;
    __device__ __forceinline__ void operator()(int k, int m, int n, unsigned long long call, float (&v)[8]) const
    {
        if (m >= rows || n >= cols) return;
        const int left = cols - n;
        Chunk<T> add;
        if (residual.p) add.load((const T*)residual.p + k * residual.rep + m * residual.row + n, left);
        if (bias) {
            Chunk<float> b;
            float w[8];
            b.load(bias + k * bias_rep + n, left);
            b.get(w);
            each8([&](int e) { v[e] += w[e]; });
        }
        if (pre.p) store_chunk((T*)pre.p + k * pre.rep + m * pre.row + n, left, v);
        activate8(v, act);
        if (draws.limit) kept8(draws, call, k, m, n, [&](int e, bool kept) { v[e] = kept ? v[e] * draws.scale : 0.f; });
        if (residual.p) {
            float w[8];
            add.get(w);
            each8([&](int e) { v[e] += w[e]; });
        }
        store_chunk((T*)y.p + k * y.rep + m * y.row + n, left, v);
    }
};
// only the store, rounded
template <typename T> Finish<T> store_only(const Rows& y, int rows, int cols)
{
    return Finish<T>{nullptr, 0, {}, {}, y, rows, cols, kNone, Draws{0, 0, 0, nullptr, 0, 1.f}};
}

// A wave's blocks of 32 rows through LDS, as floats: a lane holds four consecutive columns of a row, Finish takes eight.
template <typename T> struct FinishTile {
    static constexpr bool kLaneM = true, kStaged = true, kSums = false;
    template <int TN> static constexpr int pitch() { return TN * 128 + 16; }
    template <int TN> static constexpr int bytes() { return 32 * pitch<TN>(); }
    Finish<T> finish;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t, char* lds) const
    {
        constexpr int kPitch = pitch<TN>(), kAcross = TN * 4;
        char* p = lds + t.wave * bytes<TN>();
        const unsigned long long call = finish.draws.limit ? call_of(finish.draws) : 0ull;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(f4*)(p + (t.lane & 31) * kPitch + (32 * j + 8 * q + 4 * (t.lane >> 5)) * 4) =
                        f4{t.acc[i][j][4 * q], t.acc[i][j][4 * q + 1], t.acc[i][j][4 * q + 2], t.acc[i][j][4 * q + 3]};
#pragma unroll
            for (int u = 0; u < 32 * kAcross / 64; ++u) {
                const int id = u * 64 + t.lane, r = id / kAcross, c = id % kAcross * 8;
                const f4 a = *(const f4*)(p + r * kPitch + c * 4), b = *(const f4*)(p + r * kPitch + c * 4 + 16);
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
                finish(t.rep, t.m0 + 32 * i + r, t.n0 + c, call, v);
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
template <bool A_ALONG, bool B_ALONG, int PA, int PB, int BM, int BN, int WM, int WN, class Epi>
__global__ __launch_bounds__(WM * WN * 64) void layer_planes_kernel(Plane3 a, Plane3 b, int K, int tiles_m, int tiles_n, int splits, int split_len, int total, Epi epi)
{
    direct_tile<A_ALONG, B_ALONG, PA, PB, BM, BN, WM, WN>(a, b, K, tiles_m, tiles_n, splits, split_len, total, epi);
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
    finish(k, t, c, finish.draws.limit ? call_of(finish.draws) : 0ull, v);
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
// operands in planes: products of `pairs` pairs of them
Shape planes_shape(int n, int M, int N, int K, int pairs)
{
    const int slabs = (K + kSlab - 1) / kSlab * pairs;
    auto tiles = [&](int m, int n_) { return (long long)n * ((M + m - 1) / m) * ((N + n_ - 1) / n_); };
    Shape p{true, 256, 256, 1, 0};
    if (tiles(256, 256) < 192) p.bm = p.bn = 128;
    return cut(p, K, best_shares(tiles(p.bm, p.bn), slabs, (double)n * M * N * 4), kSlab);
}
// operands through registers
Shape registers_shape(int n, int M, int N, int K, int bm, int bn)
{
    const long long tiles = (long long)n * ((M + bm - 1) / bm) * ((N + bn - 1) / bn);
    const int splits = (int)std::max<long long>(1, std::min<long long>(512 / std::max<long long>(1, tiles), K / 256));
    return cut(Shape{false, bm, bn, 1, 0}, K, splits, 128);
}

struct Work {                      // where things lie in the working memory
    Shape y, dx, dw;
    int ldx, ldz, planes;
    size_t x, w, dz, sums, share, total;
    int blocks, across, depth;     // column sums: row blocks, lanes a row, rows a block
};
bool few(int rows, int in, int out) { return rows <= 64 && std::min(in, out) >= 8; }

Work plan_of(int n, int rows, int in, int out, int bf16, bool grad)
{
    Work p{};
    p.ldx = up_to(in, 8);
    p.ldz = up_to(out, 8);
    p.planes = bf16 ? 1 : 3;
    const bool small = few(rows, in, out);
    const int pairs = bf16 ? 1 : 6, bm = rows <= 32 ? 32 : 64;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    if (!small || grad) p.x = take((size_t)n * rows * p.ldx * 2 * p.planes);
    if (!small) p.w = take((size_t)n * in * p.ldz * 2 * p.planes);
    if (!grad) {
        p.y = small ? registers_shape(n, rows, out, in, bm, 128) : planes_shape(n, rows, out, in, pairs);
        p.share = take(share_bytes(p.y, n, rows, out));
    } else {
        p.dx = small ? registers_shape(n, rows, in, out, bm, 128) : planes_shape(n, rows, in, out, pairs);
        p.dw = small ? registers_shape(n, in, out, rows, 64, 64) : planes_shape(n, in, out, rows, pairs);
        p.dz = take((size_t)n * rows * p.ldz * (small ? (bf16 ? 2 : 4) : 2 * p.planes));
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
    constexpr int KS = BM == 32 ? (wide ? (BA ? 64 : 32) : 128) : BN == 128 && !wide ? 64 : 32, NBUF = wide || BM == 32 ? 1 : 2, AHEAD = BM == 32 ? 2 : 1;
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
    if constexpr (Epi::kStaged) static_assert(WM * WN * Epi::template bytes<BN / WN / 32>() <= 128 * 1024, "the epilogue's blocks lie in the images");
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
template <int PA, int PB, bool AA, bool BA, typename T>
hipError_t planes_product(const Plane3& a, const Plane3& b, int n, int M, int N, int K, const Shape& p, const Finish<T>& finish, float* share, hipStream_t s)
{
    return whole_or_shares<T>(p, n, M, N, finish, share, s, [&](const auto& epi) {
        if (p.bm == 256) return launch_planes<PA, PB, 256, 256, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
        return launch_planes<PA, PB, 128, 128, 2, 4, AA, BA>(a, b, n, M, N, K, p, epi, s);
    });
}

// a tensor [n][rows][cols] as planes: as it lies, or laid out at `at`
template <typename T, int PL> hipError_t planes_of(const Rows& r, int n, int rows, int cols, __bf16* at, Plane3& out, hipStream_t s)
{
    const int ld = up_to(cols, 8);
    if (PL == 1 && is_plane(r, cols)) {
        out = Plane3{(const __bf16*)r.p, r.rep, 0, (int)r.row, rows, cols, nullptr};
        return hipSuccess;
    }
    out = Plane3{at, (long long)rows * ld, (long long)n * rows * ld, ld, rows, ld, nullptr};
    return lay_out<T, PL>(n, rows, cols, ld, r, Labelled{nullptr, 0}, nullptr, at, s);
}

template <typename T> hipError_t forward(const LayerArgs& a, hipStream_t s)
{
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    if (a.rows == 0) return hipSuccess;
    const Work p = plan_of(a.n, a.rows, a.in, a.out, a.bf16, false);
    char* work = (char*)a.work;
    float* share = (float*)(work + p.share);
    const Finish<T> finish{(const float*)a.bias.p, a.bias.rep, a.residual, a.pre, a.y, a.rows, a.out, a.act, a.draws};
    if (!p.y.planes) {
        const Source<T> x = source<T>(a.x, a.rows, a.in), w = source<T>(a.w, a.in, a.out);
        return whole_or_shares<T>(p.y, a.n, a.rows, a.out, finish, share, s, [&](const auto& epi) {
            if (p.y.bm == 32) return launch_registers<T, 32, 128, 1, 4, true, false>(x, w, a.n, a.rows, a.out, a.in, p.y, epi, s);
            return launch_registers<T, 64, 128, 2, 4, true, false>(x, w, a.n, a.rows, a.out, a.in, p.y, epi, s);
        });
    }
    Plane3 x, w;
    hipError_t e = planes_of<T, PL>(a.x, a.n, a.rows, a.in, (__bf16*)(work + p.x), x, s);
    if (e == hipSuccess) e = planes_of<T, PL>(a.w, a.n, a.in, a.out, (__bf16*)(work + p.w), w, s);
    if (e != hipSuccess) return e;
    return planes_product<PL, PL, true, false, T>(x, w, a.n, a.rows, a.out, a.in, p.y, finish, share, s);
}

// ---- gradient ---------------------------------------------------------------------------------------------------------------
// dz = D'(dy) a'(pre), eight columns a lane, as T rows (OUT = 1, [replicas][rows][ld]), three bf16 parts (3) or not stored (0), and the column
// sums of a block's rows.  A dropped value is zero whatever dy and pre hold there.
template <typename T, int OUT>
__global__ __launch_bounds__(256) void slope_kernel(const T* dy, long long yrep, long long yrow, const T* pre, long long prep, long long prow, int rows, int cols,
                                                    int ld, int across, int depth, int act, Draws d, void* dz, long long plane, float* sums)
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
            const long long to = ((long long)k * rows + t) * ld + c;
            if constexpr (OUT == 1) store_chunk((T*)dz + to, 8, v);
            if constexpr (OUT == 3) {
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
        if (col < ld) sums[((long long)k * gridDim.y + blockIdx.y) * ld + col] = v;
    }
}
// db: the blocks' sums in ascending order
__global__ __launch_bounds__(256) void column_sums_kernel(const float* sums, int blocks, int ld, int cols, float* db, long long rep)
{
    const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.y;
    if (c >= cols) return;
    float v = 0.f;
#pragma unroll 8
    for (int b = 0; b < blocks; ++b) v += sums[((long long)k * blocks + b) * ld + c];
    db[k * rep + c] = v;
}

template <typename T> hipError_t backward(const LayerArgs& a, hipStream_t s)
{
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    const Work p = plan_of(a.n, a.rows, a.in, a.out, a.bf16, true);
    char* work = (char*)a.work;
    float *share = (float*)(work + p.share), *sums = (float*)(work + p.sums);
    void* dz = work + p.dz;
    const bool small = !p.dx.planes, products = a.dx.p || a.dw.p;
    hipError_t e = hipSuccess;
    // dz in the working memory, as the products take it; where it is dy itself only what they cannot read is laid out
    const bool same = a.act == kNone && !a.draws.limit, there = same && (small || (PL == 1 && is_plane(a.dy, a.out)));
    const long long plane = (long long)a.n * a.rows * p.ldz;
    if (a.rows && ((products && !there) || a.db.p)) {
        const dim3 grid((unsigned)((p.ldz + p.across * 8 - 1) / (p.across * 8)), (unsigned)p.blocks, (unsigned)a.n);
        auto* kernel = !products || there ? slope_kernel<T, 0> : small || PL == 1 ? slope_kernel<T, 1> : slope_kernel<T, PL>;
        kernel<<<grid, 256, 0, s>>>((const T*)a.dy.p, a.dy.rep, a.dy.row, (const T*)a.pre.p, a.pre.rep, a.pre.row, a.rows, a.out, p.ldz, p.across, p.depth,
                                    a.act, a.draws, dz, plane, a.db.p ? sums : nullptr);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.db.p) {
        column_sums_kernel<<<dim3((unsigned)((a.out + 255) / 256), (unsigned)a.n), 256, 0, s>>>(sums, a.rows ? p.blocks : 0, p.ldz, a.out, (float*)a.db.p, a.db.rep);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const Rows z = there ? a.dy : Rows{dz, (long long)a.rows * p.ldz, p.ldz};
    const int zcols = there ? a.out : p.ldz;
    const Finish<T> to_dx = store_only<T>(a.dx, a.rows, a.in), to_dw = store_only<T>(a.dw, a.in, a.out);
    Rows kept{work + p.x, (long long)a.rows * p.ldx, p.ldx};   // the checkpoint's values, exact in bf16
    if (a.dw.p && a.packed.q && a.rows && (e = launch_unpack(a.n, a.rows, a.in, 1, a.packed.q, kept, s)) != hipSuccess) return e;
    if (small) {
        const Source<T> g = source<T>(z, a.rows, zcols);
        if (a.dx.p && a.rows) {
            const Source<T> w = source<T>(a.w, a.in, a.out);
            e = whole_or_shares<T>(p.dx, a.n, a.rows, a.in, to_dx, share, s, [&](const auto& epi) {
                if (p.dx.bm == 32) return launch_registers<T, 32, 128, 1, 4, true, true>(g, w, a.n, a.rows, a.in, a.out, p.dx, epi, s);
                return launch_registers<T, 64, 128, 2, 4, true, true>(g, w, a.n, a.rows, a.in, a.out, p.dx, epi, s);
            });
            if (e != hipSuccess) return e;
        }
        if (!a.dw.p) return hipSuccess;
        return whole_or_shares<T>(p.dw, a.n, a.in, a.out, to_dw, share, s, [&](const auto& epi) {
            if (a.packed.q) return launch_registers<T, 64, 64, 2, 2, false, false>(source<__bf16>(kept, a.rows, p.ldx), g, a.n, a.in, a.out, a.rows, p.dw, epi, s);
            return launch_registers<T, 64, 64, 2, 2, false, false>(source<T>(a.x, a.rows, a.in), g, a.n, a.in, a.out, a.rows, p.dw, epi, s);
        });
    }
    const Plane3 g = there ? Plane3{(const __bf16*)a.dy.p, a.dy.rep, 0, (int)a.dy.row, a.rows, a.out, nullptr}
                           : Plane3{(const __bf16*)dz, (long long)a.rows * p.ldz, plane, p.ldz, a.rows, p.ldz, nullptr};
    if (a.dx.p && a.rows) {
        Plane3 w;
        if ((e = planes_of<T, PL>(a.w, a.n, a.in, a.out, (__bf16*)(work + p.w), w, s)) != hipSuccess) return e;
        if ((e = planes_product<PL, PL, true, true, T>(g, w, a.n, a.rows, a.in, a.out, p.dx, to_dx, share, s)) != hipSuccess) return e;
    }
    if (!a.dw.p) return hipSuccess;
    Plane3 x{(const __bf16*)kept.p, kept.rep, 0, p.ldx, a.rows, p.ldx, nullptr};
    if (a.packed.q) return planes_product<1, PL, false, false, T>(x, g, a.n, a.in, a.out, a.rows, p.dw, to_dw, share, s);
    if ((e = planes_of<T, PL>(a.x, a.n, a.rows, a.in, (__bf16*)(work + p.x), x, s)) != hipSuccess) return e;
    return planes_product<PL, PL, false, false, T>(x, g, a.n, a.in, a.out, a.rows, p.dw, to_dw, share, s);
}

}  // namespace

size_t layer_work_bytes(int n, int rows, int in, int out, int bf16, bool grad)
{
    const size_t one = plan_of(n, rows, in, out, bf16, false).total;       // a workspace for the gradient serves the forward pass too
    return grad ? std::max(one, plan_of(n, rows, in, out, bf16, true).total) : one;
}
hipError_t launch_layer_forward(const LayerArgs& a, hipStream_t s) { return a.bf16 ? forward<__bf16>(a, s) : forward<float>(a, s); }
hipError_t launch_layer_backward(const LayerArgs& a, hipStream_t s) { return a.bf16 ? backward<__bf16>(a, s) : backward<float>(a, s); }

}  // namespace layer
}  // namespace hadfl
