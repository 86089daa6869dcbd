// Tiled matrix product on the matrix cores for operands that lie as the matrix cores take them: planes of 16-bit values, rows
// on 16 bytes, whole chunks of eight values.  C[m][n] = sum_k A(m, k) B(n, k).
//
// A plane holds
//   bf16 operands            as they are
//   32-bit operands, 3       three bf16 parts (parts3), against a bf16 operand: three products, nothing is lost
//   32-bit operands, 2       two fp16 parts: with 2^s the power of two that takes the replica's largest finite magnitude to [2^14, 2^15),
//                            y = 2^s x, h = fp16(y), l = fp16(2^11 (y - h)).  Products l h' and h l' first, 2^-11 on the sums, then
//                            h h'; l l', at most 2^-22 of the product, is left out, and l's own rounding is at most 2^-22 of y: a
//                            product is off by 2^-23.5 in the mean square, which is what a 32-bit sum of a few terms loses.  The factor
//                            on l keeps it a normal number, so this holds for magnitudes down to 2^-29 of the largest; below, the
//                            error stays under 2^-50 of the largest.  Three products where three bf16 parts would take six.
//
// Slabs of 64 k go from memory to LDS without passing registers (buffer loads that write LDS), as many slabs ahead of the one
// being multiplied as LDS holds (256 x 256 tiles: one, 128 x 256: two, 128 x 128: three), one barrier a slab.  The LDS image is the slab itself with its 16-byte chunks exchanged within a row, so
// that the operand reads meet every bank once (a load that writes LDS puts the chunks of a wave one after the other: the exchange is in
// the addresses it reads from):
//   along   the contraction runs along the source's rows: [rows][64 k], chunk c of row r at c ^ (r / 2 & 7): two rows are the 64 banks' width
//   across  it runs across them: [64 k][columns], chunk c of row k at c ^ 4 (k & 3); the operand read transposes
// 256 x 256 tiles of eight waves hold 128 x 64 each: 1.5 KiB of LDS reads a matrix instruction of 32 cycles a wave.
#pragma once
#include <algorithm>

#include "tile_product.h"

namespace hadfl {
namespace head {

constexpr int kSlab = 64;

struct Plane3 {                    // an operand: source rows `lines` of `cols` values, `ld` >= cols apart
    const __bf16* p;
    long long rep, plane;
    int ld, lines, cols;
    const unsigned* top;           // two fp16 parts: the replicas' largest magnitudes (bits of a float); null: 1
};

constexpr float kLowScale = 0x1p11f;
// 2^s and 2^-s of two fp16 parts.  A tensor of magnitudes below 2^-112 is scaled by 2^126, which is still exact.
__device__ __forceinline__ float up_scale(unsigned top) { return __builtin_bit_cast(float, (unsigned)min(127 + 14 + 127 - (int)(top >> 23), 253) << 23); }
__device__ __forceinline__ float down_scale(unsigned top) { return __builtin_bit_cast(float, (unsigned)max((int)(top >> 23) - 14, 1) << 23); }
constexpr unsigned kOneBits = 0x3f800000u;
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ unsigned to_f16x2(float a, float b) { return __builtin_bit_cast(unsigned, (h2{(_Float16)a, (_Float16)b})); }
__device__ __forceinline__ void split2(const f4& x, float scale, u2& h, u2& l)
{
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const float a = x[2 * e] * scale, b = x[2 * e + 1] * scale;
        const h2 top{(_Float16)a, (_Float16)b};
        h[e] = __builtin_bit_cast(unsigned, top);
        l[e] = to_f16x2((a - (float)top[0]) * kLowScale, (b - (float)top[1]) * kLowScale);
    }
}
template <bool F16> __device__ __forceinline__ f16 multiply16(const bf16x8& a, const bf16x8& b, const f16& c)
{
    if (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// A bf16 tensor that is a plane as it lies: whole chunks, rows no farther apart than the kernel's 32-bit offsets within a tile reach, and rows that do
// not overlap (a stride of zero would), since what lies beyond a plane's last row is told by its offset alone.
inline bool is_plane(const Rows& r, long long cols) { return chunked(r, 1, cols) && r.row >= cols && r.row <= (1ll << 22); }

typedef __attribute__((address_space(3))) void LdsVoid;
// 16 bytes a lane from b + off to LDS, the wave's lanes one after the other from `at` (the same in all lanes); an offset outside the
// buffer gives zeros.  It has no result in a register; slab_barrier() waits for it.  Written out because the compiler, which cannot
// tell the images apart behind the transposing reads, would wait for every load before the next of those.
__device__ __forceinline__ void load_to_lds(Buffer b, unsigned off, unsigned at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(at), "v"(off), "s"(b) : "memory", "m0");
}

// an address that is the same in all lanes, in scalar registers
__device__ __forceinline__ const __bf16* same(const __bf16* p)
{
    const unsigned long long v = (unsigned long long)p;
    return (const __bf16*)((unsigned long long)__builtin_amdgcn_readfirstlane((unsigned)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((unsigned)v));
}

// BR rows (along) or columns (across) and KS k of an operand, by NT threads.  The exchanges above are those of KS = 64 and BR >= 128; rows of 32 k lie four
// to the banks' width, 64 columns two.
template <bool ALONG, int BR, int NT, int KS = kSlab> struct Loader {
    static constexpr int kBytes = BR * KS * 2, kAcross = ALONG ? KS / 8 : BR / 8, kLoads = kBytes / 16 / NT;
    static constexpr int kStep = NT / kAcross;                 // image rows between a thread's chunks
    static constexpr int kPeriod = ALONG ? 16 : 4;             // rows after which the exchange is the same again
    static_assert((KS == 64 || KS == 32) && BR >= 64, "");
    static __device__ __forceinline__ int place(int r, int c)
    {
        if (ALONG) return KS == 64 ? c ^ (r >> 1 & 7) : c ^ (r >> 2 & 3);
        return BR == 64 ? c ^ ((r & 2) << 1) : c ^ ((r & 3) << 2);
    }
    unsigned off, step;            // of this thread's first chunk, and to its next one
    int kc;                        // along: the chunk's first k
    __device__ __forceinline__ void init(int tid, int ld)
    {
        const int r = tid / kAcross, from = place(r, tid % kAcross);          // its own inverse
        off = (unsigned)(r * ld + from * 8) * 2;
        step = (unsigned)(kStep * ld) * 2;
        kc = from * 8;
    }
    // r0: the tile's first row (along) or column (across)
    __device__ __forceinline__ void issue(const Plane3& s, const __bf16* base, int r0, int k0, int wave, char* image) const
    {
        static_assert(kStep % kPeriod == 0 && kLoads >= 1, "");
        const long long first = ALONG ? (long long)r0 * s.ld : (long long)k0 * s.ld + r0;
        const long long rest = ALONG ? (long long)(s.lines - r0 - 1) * s.ld + s.cols : (long long)(s.lines - k0 - 1) * s.ld + s.cols - r0;
        const Buffer b = buffer(same(base + first), __builtin_amdgcn_readfirstlane((unsigned)min(rest * 2, 0xffffffe0ll)));
        const bool in = !ALONG || k0 + kc < s.cols;
        const unsigned first_byte = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(LdsVoid*)image + wave * 1024);
        unsigned at = off + (ALONG ? (unsigned)k0 * 2 : 0u);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            load_to_lds(b, in ? at : kOutside, first_byte + i * NT * 16);
            at += step;
        }
    }
    // operand of the 32 rows from r0 and the 16 k of step ks
    static __device__ __forceinline__ bf16x8 read(const char* image, int r0, int ks, int lane)
    {
        if (ALONG) {
            const int r = r0 + (lane & 31);
            return *(const bf16x8*)(image + r * KS * 2 + place(lane & 31, ks * 2 + (lane >> 5)) * 16);
        }
        const int k = ks * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2), c = r0 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
        return lds_read_tr8(image, (unsigned)(k * BR * 2 + place(k, c >> 3) * 16 + (c & 7) * 2), BR * 2);
    }
};

// pairs of planes whose products are kept, the small ones first
template <int PA, int PB> struct Pairs;
template <> struct Pairs<1, 1> { static constexpr int kCount = 1; static __device__ int a(int) { return 0; } static __device__ int b(int) { return 0; } };
template <> struct Pairs<1, 3> { static constexpr int kCount = 3; static __device__ int a(int) { return 0; } static __device__ int b(int s) { return 2 - s; } };
template <> struct Pairs<2, 2> {
    static constexpr int kCount = 3;                           // (1,0) (0,1) (0,0)
    static __device__ int a(int s) { return s == 0; }
    static __device__ int b(int s) { return s == 1; }
};

// waits for all but the last N loads of this wave and for its LDS reads, then for the other waves
template <int N> __device__ __forceinline__ void slab_barrier()
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x70);          // vector loads: N, LDS: 0, exports: any
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// a tile's place: groups of eight tiles down m, so that the 32 compute units of a die work on about 8 x 4 tiles that share operands
__device__ __forceinline__ void place_tile(int at, int tiles_m, int tiles_n, int& m, int& n)
{
    constexpr int G = 8;
    const int per = G * tiles_n, g = at / per, in = at - g * per, rows = min(G, tiles_m - g * G);
    n = in / rows;
    m = g * G + in - n * rows;
}

template <bool A_ALONG, bool B_ALONG, int PA, int PB, int BM, int BN, int WM, int WN, class Epi>
__global__ __launch_bounds__(WM * WN * 64) void direct_kernel(Plane3 a, Plane3 b, int K, int tiles_m, int tiles_n, int splits, int split_len,
                                                              int total, Epi epi)
{
    constexpr int NT = WM * WN * 64, TM = BM / WM / 32, TN = BN / WN / 32;
    typedef Loader<A_ALONG, BM, NT> LA;
    typedef Loader<B_ALONG, BN, NT> LB;
    typedef Pairs<PA, PB> P;
    constexpr int kImage = LA::kBytes + LB::kBytes, IMAGES = kImage > 49152 ? 2 : kImage > 32768 ? 3 : 4, kLoads = LA::kLoads + LB::kLoads;
    __shared__ __attribute__((aligned(16))) char images[IMAGES * kImage];

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
    const int k_begin = t.split * split_len, k_end = min(K, k_begin + split_len);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) t.acc[i][j] = f16{};
    if (Epi::kSums) {
#pragma unroll
        for (int j = 0; j < TN; ++j) t.sum[j] = f16{};
    }
    const bool sums = has_sum(epi, t.m0);
    LA la;
    LB lb;
    la.init(tid, a.ld);
    lb.init(tid, b.ld);

    int pair = 0, k0 = k_begin;                                // of the next slab to load
    auto issue = [&](char* image) {
        la.issue(a, pa + P::a(pair) * a.plane, bm, k0, wave, image);
        lb.issue(b, pb + P::b(pair) * b.plane, bn, k0, wave, image + LA::kBytes);
        k0 += kSlab;
        if (k0 >= k_end) { k0 = k_begin; ++pair; }
    };
    auto multiply = [&](const char* image) {
#pragma unroll
        for (int ks = 0; ks < kSlab / 16; ++ks) {
            bf16x8 fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = LA::read(image, wm + 32 * i, ks, t.lane);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = LB::read(image + LA::kBytes, wn + 32 * j, ks, t.lane);
            if (Epi::kSums && sums) {
#pragma unroll
                for (int j = 0; j < TN; ++j) t.sum[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones(), fb[j], t.sum[j], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    t.acc[i][j] = Epi::kLaneM ? multiply16<PA == 2>(fb[j], fa[i], t.acc[i][j]) : multiply16<PA == 2>(fa[i], fb[j], t.acc[i][j]);
        }
    };
    const int low_slabs = 2 * ((k_end - k_begin + kSlab - 1) / kSlab);      // two fp16 parts: those of the products with a low part
    const int slabs = k_begin < k_end ? P::kCount * ((k_end - k_begin + kSlab - 1) / kSlab) : 0;
    // Slab i: its loads are done when at most those of the IMAGES - 2 slabs after it are outstanding (loads finish in order);
    // the barrier says so for all waves, and that all have read the slab before, whose image the next loads take.
    auto turn = [&](int i, char* image, char* free) {
        if (i >= slabs) return;
        if (IMAGES > 2 && i + IMAGES - 2 < slabs) slab_barrier<(IMAGES - 2) * kLoads>();
        else slab_barrier<0>();
        if (i + IMAGES - 1 < slabs) issue(free);
        if (PA == 2 && i == low_slabs) {
#pragma unroll
            for (int x = 0; x < TM; ++x)
#pragma unroll
                for (int y = 0; y < TN; ++y) t.acc[x][y] *= 1.f / kLowScale;
        }
        multiply(image);
    };
#pragma unroll
    for (int i = 0; i < IMAGES - 1; ++i)
        if (i < slabs) issue(images + i * kImage);
    for (int i = 0; i < slabs; i += IMAGES) {
#pragma unroll
        for (int u = 0; u < IMAGES; ++u) turn(i + u, images + u * kImage, images + (u + IMAGES - 1) % IMAGES * kImage);
    }
    if (PA == 2) {                                             // one after the other: their product may be no float
        const float sa = down_scale(a.top ? a.top[t.rep] : kOneBits), sb = down_scale(b.top ? b.top[t.rep] : kOneBits);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) t.acc[i][j] = t.acc[i][j] * sa * sb;
    }
    if constexpr (Epi::kStaged) {
        __syncthreads();                                       // the images are free
        epi(t, images);
    } else epi(t);
}

template <int PA, int PB, int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG, class Epi>
hipError_t launch_direct(const Plane3& a, const Plane3& b, int replicas, int M, int N, int K, int splits, int split_len, const Epi& epi, hipStream_t s)
{
    const int tm = (M + BM - 1) / BM, tn = (N + BN - 1) / BN;
    const long long total = (long long)replicas * splits * tm * tn;
    if (total == 0) return hipSuccess;
    if (total > 0x7fffff00ll) return hipErrorInvalidValue;
    direct_kernel<A_ALONG, B_ALONG, PA, PB, BM, BN, WM, WN, Epi>
        <<<line_grid(die_grid(total), WM * WN * 64), WM * WN * 64, 0, s>>>(a, b, K, tm, tn, splits, split_len, (int)total, epi);
    return hipGetLastError();
}

// Into how many shares a contraction of `slabs` slabs is cut: with t tiles, s shares take ceil(t s / 256) / s rounds of the 256 compute units
// (one workgroup each), 0.85 us a slab of 256 x 256 tiles, and every share costs its bytes written and read, 5 TB/s.  At least four slabs
// a share.  16 x 3 x 3 tiles of 72 slabs: one share 61 us, seven 35.
inline int best_shares(long long tiles, int slabs, double share_bytes)
{
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 64 && (s == 1 || slabs / s >= 4); ++s) {
        const double rounds = (double)((tiles * s + 255) / 256) / s, cost = rounds * slabs * 0.85e-6 + (s > 1 ? s * share_bytes * 2 / 5e12 : 0);
        if (s == 1 || cost < 0.97 * least) { best = s; least = cost; }
    }
    return best;
}

// ---- laying operands out ---------------------------------------------------------------------------------------------
// the largest finite magnitude of every replica's tensor, as a float's bits, joined to what top holds; rows that take no part are left out
struct Magnitudes {
    const float* x;
    long long rep, row;
    int rows, cols;
    Labelled live;
    unsigned* top;
};
__global__ __launch_bounds__(256) inline void largest_kernel(Magnitudes first, Magnitudes second)
{
    Magnitudes a = blockIdx.z ? second : first;
    const int k = blockIdx.y, chunks = (a.cols + 7) / 8;
    const long long total = (long long)a.rows * chunks, step = (long long)gridDim.x * 256;
    if ((long long)blockIdx.x * 256 >= total) return;
    if (a.live.labels) a.live.labels += (long long)k * a.rows;
    unsigned most = 0;
    for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < total; at += step) {
        const int t = (int)(at / chunks), c = (int)(at - (long long)t * chunks) * 8;
        Chunk<float> v;
        v.load(a.x + k * a.rep + t * a.row + c, a.live.at(t) ? a.cols - c : 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned p = v.a[e] & 0x7fffffffu, q = v.b[e] & 0x7fffffffu;
            most = max(most, max(p < 0x7f800000u ? p : 0u, q < 0x7f800000u ? q : 0u));
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = max(most, (unsigned)__shfl_xor((int)most, d));
    __shared__ unsigned waves[4];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x / 64] = most;
    __syncthreads();
    // a maximum: the same in any order; one a workgroup, since additions to one address queue up
    if (threadIdx.x == 0) atomicMax(a.top + k, max(max(waves[0], waves[1]), max(waves[2], waves[3])));
}
__global__ inline void clear_kernel(unsigned* p, int n) { if ((int)threadIdx.x < n) p[threadIdx.x] = 0; }

// x [replicas][rows][cols] -> [planes][replicas][rows][ld], zero beyond cols and in rows that take no part
template <typename T, int PL>
__global__ __launch_bounds__(256) void lay_out_kernel(const T* x, long long rep, long long row, int rows, int cols, int ld, long long total, long long plane,
                                                      Labelled live, const unsigned* top, __bf16* out)
{
    const long long at = line_block() * 256 + threadIdx.x;          // chunk of eight
    if (at >= total) return;
    const int chunks = ld / 8;
    const long long line = at / chunks;
    const int c = (int)(at - line * chunks) * 8, k = (int)(line / rows), t = (int)(line - (long long)k * rows);
    if (live.labels) live.labels += (long long)k * rows;
    Chunk<T> chunk;
    chunk.load(x + k * rep + t * row + c, live.at(t) ? cols - c : 0);
    u4 part[PL];
    if constexpr (PL == 1) part[0] = chunk.a;
    else if constexpr (PL == 3) Source<float>::split(chunk, part);
    else {
        const float scale = up_scale(top[k]);
        u2 h[2], l[2];
        split2(__builtin_bit_cast(f4, chunk.a), scale, h[0], l[0]);
        split2(__builtin_bit_cast(f4, chunk.b), scale, h[1], l[1]);
        part[0] = join8(h[0], h[1]);
        part[1] = join8(l[0], l[1]);
    }
#pragma unroll
    for (int i = 0; i < PL; ++i) *(u4*)(out + i * plane + at * 8) = part[i];
}
template <typename T, int PL>
hipError_t lay_out(int n, int rows, int cols, int ld, const Rows& x, Labelled live, const unsigned* top, __bf16* out, hipStream_t s)
{
    const long long plane = (long long)n * rows * ld, total = plane / 8;
    if (total == 0) return hipSuccess;
    lay_out_kernel<T, PL><<<line_grid((total + 255) / 256, 256), 256, 0, s>>>((const T*)x.p, x.rep, x.row, rows, cols, ld, total, plane, live, top, out);
    return hipGetLastError();
}
inline hipError_t find_largest(int n, const Magnitudes& first, const Magnitudes& second, hipStream_t s)
{
    auto blocks = [](const Magnitudes& a) { return ((long long)a.rows * ((a.cols + 7) / 8) + 255) / 256; };
    const long long most = std::max(blocks(first), blocks(second));
    largest_kernel<<<dim3((unsigned)std::min<long long>(most, std::max(8, 1024 / n)), (unsigned)n, 2), 256, 0, s>>>(first, second);
    return hipGetLastError();
}

// ---- a wave's tile to bf16 rows, through LDS -----------------------------------------------------------------------------
// One block of 32 rows of 32 * TN columns (lanes along m) at a time: a lane writes its four consecutive n, then eight lanes take a row of
// 128 bytes to memory (straight from the registers a store would touch 32 rows, eight bytes each).
template <int TN> struct RowStage {
    static constexpr int kPitch = TN * 64 + 16, kBytes = 32 * kPitch;
    char* p;
    __device__ __forceinline__ void put(int lane, int j, int q, const u2& v) const { *(u2*)(p + (lane & 31) * kPitch + (32 * j + 8 * q + 4 * (lane >> 5)) * 2) = v; }
    // store(row, first column, chunk) for every chunk of eight
    template <class F> __device__ __forceinline__ void take(int lane, F&& store) const
    {
        constexpr int kAcross = TN * 4;
#pragma unroll
        for (int i = 0; i < 32 * kAcross / 64; ++i) {
            const int id = i * 64 + lane, r = id / kAcross, c = id % kAcross;
            store(r, c * 8, *(const u4*)(p + r * kPitch + c * 16));
        }
    }
};
// C times a factor per replica to a bf16 tensor
struct StoreRows {
    static constexpr bool kLaneM = true, kStaged = true, kSums = false;
    __bf16* p;
    long long rep, row;
    const float* factor;
    int M, N;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t, char* lds) const
    {
        const float f = factor[t.rep];
        __bf16* out = p + t.rep * rep;
        const RowStage<TN> stage{lds + t.wave * RowStage<TN>::kBytes};
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    stage.put(t.lane, j, q, u2{to_bf16x2(t.acc[i][j][4 * q] * f, t.acc[i][j][4 * q + 1] * f),
                                               to_bf16x2(t.acc[i][j][4 * q + 2] * f, t.acc[i][j][4 * q + 3] * f)});
            stage.take(t.lane, [&](int r, int c, const u4& v) {
                const int m = t.m0 + 32 * i + r, n = t.n0 + c;
                if (m >= M || n >= N) return;
                __bf16* q = out + m * row + n;
                if (n + 8 <= N) { *(u4any*)q = v; return; }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (n + e < N) ((unsigned short*)q)[e] = (unsigned short)(v[e / 2] >> (16 * (e % 2)));
            });
        }
    }
};

}  // namespace head
}  // namespace hadfl
