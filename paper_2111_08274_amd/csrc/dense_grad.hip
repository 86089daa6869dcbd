// Parameter gradients of a dense layer whose input was kept in 8 bits: dW = x^T dy with x from the checkpoint, db = sum_t dy.
// q * 2^e is exact in bf16, so a bf16 dy needs one product and a 32-bit dy, in three bf16 planes, three.  db comes from the same
// operands as one more product, of ones (tile_product.h).
//   less work   chunks of the checkpoint become bf16 in registers, on their way to LDS (again in every column of tiles)
//   more        the checkpoint is laid out as bf16 first, 3 bytes a value once, and both operands go straight from memory to LDS
#include "direct_product.h"

namespace hadfl {
namespace head {

namespace {

struct Plan {
    bool direct, big;              // big: 256 x 256 tiles, else 128 x 128; not direct: 128 x 128, else 64 x 64
    int ldx, ldy, planes, splits, split_len;
    size_t x, y, share, total;
};

// Laying out costs 3 bytes a value of x (and 10 of a 32-bit dy, which its three planes have to win back over in x out products) and two
// launches; the product after it is faster where there are enough rows and tiles.  Through registers / laid out, us:
//   bf16   packed and multiplied once, operands from memory: 16 x 512 x 512, 512 rows 33 / 33, 1024 rows 52 / 41; 2048 x 2048, 512 rows 29 / 27,
//          1024 rows 44 / 33; 2 x 2048 x 2048, 1024 rows 51 / 54.  Again and again: 2048 x 2048, 2048 rows 44 / 36; 4096 x 4096, 2048 rows
//          110 / 87; 784 x 128, 16384 rows 50 / 60; 8 x 784 x 130, where the larger tiles would be more than half empty, 16384 rows 114 / 191
//   fp32   2048 x 2048, 2048 rows 76 / 89, 8192 rows 241 / 300; 4096 x 4096, 512 rows 65 / 73, 2048 rows 242 / 207; 16 x 1024 x 1024, 8192 rows
//          956 / 1072; 2 x 128 x 4096, 8192 rows 105 / 213
// Through registers 128 x 128 tiles of eight waves convert and read half of what 64 x 64 tiles do (4096 x 4096 bf16, 512 rows 35 us against 50), which
// take few tiles (2 x 128 x 4096 fp32, 128 rows: 7 against 10).
Plan plan_of(int n, int rows, int in, int out, int bf16)
{
    Plan p{};
    auto tiles = [&](int t) { return (long long)n * ((in + t - 1) / t) * ((out + t - 1) / t); };
    const double work = (double)n * rows * in * out;
    p.direct = bf16 ? rows >= 768 && work >= 2e9 && tiles(128) >= 48 && tiles(128) * 4 <= tiles(64) * 1.3
                    : rows >= 1024 && tiles(256) >= 192 && (double)in * out >= 250. * (3. * in + 10. * out);
    p.direct = p.direct || (rows && out < 8);                  // fewer values a row than a chunk: laid out
    p.ldx = (in + 7) / 8 * 8;
    p.ldy = (out + 7) / 8 * 8;
    p.planes = bf16 ? 1 : 3;
    p.big = p.direct ? tiles(256) >= 192 : tiles(128) >= 192 || (rows >= 4096 && tiles(128) >= 100);
    // few tiles: the rows in shares that a second launch adds, for what the compute units hold at a time; where each has a workgroup without
    // them, of 1024 rows at least (300 x 5000 bf16: 1024 rows in one share 19 us, in three 28; 8192 rows 150 and 112)
    const long long have = p.big ? tiles(128) : tiles(64), most = p.big && have >= 256 ? 512 : 768;
    p.splits = p.direct ? best_shares(tiles(p.big ? 256 : 128), (rows + kSlab - 1) / kSlab * p.planes, (double)n * in * out * 4)
                        : (int)std::max<long long>(1, std::min<long long>((most + have - 1) / have, rows / (have < 256 ? 256 : 1024)));
    p.split_len = (((rows + p.splits - 1) / p.splits) + 63) / 64 * 64;
    p.splits = std::max(1, (rows + p.split_len - 1) / std::max(1, p.split_len));
    if (p.direct) {
        p.x = 0;
        p.y = align256((size_t)n * rows * p.ldx * 2);
        p.share = p.y + align256((size_t)n * rows * p.ldy * 2 * p.planes);
    }
    p.total = p.share + (p.splits > 1 ? align256((size_t)p.splits * n * (in + 1) * p.ldy * 4) : 0);
    return p;
}

template <typename T, class Store> hipError_t product(const DenseArgs& a, const Plan& p, const Store& store, hipStream_t s)
{
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    if (!p.direct) {
        const SourcePacked x{a.x, a.rows, a.in};
        const Source<T> dy = source<T>(a.dy, a.rows, a.out);
        const int len = std::max(1, p.split_len);
        if (p.big) return launch_product<128, 128, 2, 4, false, false>(x, dy, a.n, a.in, a.out, a.rows, p.splits, len, store, s);
        return launch_product<64, 64, 2, 2, false, false>(x, dy, a.n, a.in, a.out, a.rows, p.splits, len, store, s);
    }
    __bf16 *wx = (__bf16*)((char*)a.work + p.x), *wy = (__bf16*)((char*)a.work + p.y);
    hipError_t e = launch_unpack(a.n, a.rows, a.in, 1, a.x.q, Rows{wx, (long long)a.rows * p.ldx, p.ldx}, s);
    if (e != hipSuccess) return e;
    const Plane3 x{wx, (long long)a.rows * p.ldx, 0, p.ldx, a.rows, p.ldx, nullptr};
    Plane3 dy{(const __bf16*)a.dy.p, a.dy.rep, 0, (int)a.dy.row, a.rows, a.out, nullptr};
    if (PL == 3 || !is_plane(a.dy, a.out)) {
        if ((e = lay_out<T, PL>(a.n, a.rows, a.out, p.ldy, a.dy, Labelled{nullptr, 0}, nullptr, wy, s)) != hipSuccess) return e;
        dy = Plane3{wy, (long long)a.rows * p.ldy, (long long)a.n * a.rows * p.ldy, p.ldy, a.rows, p.ldy, nullptr};
    }
    if (p.big) return launch_direct<1, PL, 256, 256, 2, 4, false, false>(x, dy, a.n, a.in, a.out, a.rows, p.splits, p.split_len, store, s);
    return launch_direct<1, PL, 128, 128, 2, 4, false, false>(x, dy, a.n, a.in, a.out, a.rows, p.splits, p.split_len, store, s);
}

template <typename T> hipError_t run(const DenseArgs& a, hipStream_t s)
{
    const Plan p = plan_of(a.n, a.rows, a.in, a.out, a.bf16);
    if (p.splits == 1) return product<T>(a, p, StoreTile<float, true>{(float*)a.dw.p, a.dw.rep, a.dw.row, nullptr, a.in, a.out, (float*)a.db.p, a.db.rep}, s);
    float* share = (float*)((char*)a.work + p.share);
    const bool sums = a.db.p;
    const int lines = a.in + (sums ? 1 : 0);
    const hipError_t e = product<T>(a, p, StoreShare<true>{share, a.in, a.out, p.ldy, lines, a.n, false, sums}, s);
    if (e != hipSuccess) return e;
    return join_shares<float>(share, p.splits, a.n, lines, a.out, p.ldy, Labelled{nullptr, 0}, nullptr, a.dw, (float*)a.db.p, a.db.rep, s);
}

}  // namespace

size_t dense_work_bytes(int n, int rows, int in, int out, int bf16) { return plan_of(n, rows, in, out, bf16).total; }

hipError_t launch_dense_grad(const DenseArgs& a, hipStream_t s) { return a.bf16 ? run<__bf16>(a, s) : run<float>(a, s); }

}  // namespace head
}  // namespace hadfl
