// Tiled matrix product on the matrix cores for operands as a caller has them: any size, stride and alignment, 32-bit floats,
// bf16 or an 8-bit checkpoint.  C[m][n] = sum_k A(m, k) B(n, k), what becomes of C is up to an epilogue.
//
// An operand is a source of chunks of eight consecutive values; "along" says whether the contraction runs along a source's
// rows (chunk = eight k of one m) or across them (chunk = eight m of one k).  Chunks go through registers, where what lies
// outside becomes zero and floats become three bf16 planes, to LDS as they are; an operand across its rows is transposed by
// the LDS read.  One or two slabs of the contraction are in flight in registers while the one before is multiplied.
#pragma once
#include "head.h"

namespace hadfl {
namespace head {

using namespace tiles;

// rows without a label take no part, whatever they hold
struct Labelled {
    const int32_t* labels;         // null: every row does
    int classes;
    __device__ __forceinline__ bool at(int t) const { return !labels || (unsigned)labels[t] < (unsigned)classes; }
};

// Three bf16 parts of a float whose sum is the float: h = bf16(x), m = bf16(x - h), l = x - h - m, both differences exact.  No scale, so
// that products of any two magnitudes whose product is a float stay floats; l is no normal bf16 below 2^-107, where the float's lowest
// bits go.  From 3.39e38 on h rounds to infinity, and the parts of it and of an infinity hold a NaN.
__device__ __forceinline__ void parts3(const f4& x, u2& h, u2& m, u2& l)
{
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        float a = x[2 * e], b = x[2 * e + 1];
        h[e] = to_bf16x2(a, b);
        a -= __builtin_bit_cast(float, h[e] << 16); b -= __builtin_bit_cast(float, h[e] & 0xffff0000u);
        m[e] = to_bf16x2(a, b);
        a -= __builtin_bit_cast(float, m[e] << 16); b -= __builtin_bit_cast(float, m[e] & 0xffff0000u);
        l[e] = to_bf16x2(a, b);
    }
}

// A row's last chunk, of fewer than eight values, is loaded as the row's last eight and moved down when it is used; what lies outside
// is loaded from the source's beginning and taken as zero.  So no load of a slab has a branch before it.  Rows hold eight values at least.
__device__ __forceinline__ void move_down(Chunk<float>& v, int by)
{
    u4 a = v.a, b = v.b;
    const u4 none{0, 0, 0, 0};
    if (by & 4) { a = b; b = none; }
    if (by & 2) { a = u4{a[2], a[3], b[0], b[1]}; b = u4{b[2], b[3], 0, 0}; }
    if (by & 1) { a = u4{a[1], a[2], a[3], b[0]}; b = u4{b[1], b[2], b[3], 0}; }
    v.a = a; v.b = b;
}
__device__ __forceinline__ void move_down(Chunk<__bf16>& v, int by)
{
    u4 a = v.a;
    if (by & 4) a = u4{a[2], a[3], 0, 0};
    if (by & 2) a = u4{a[1], a[2], a[3], 0};
    if (by & 1) a = u4{a[0] >> 16 | a[1] << 16, a[1] >> 16 | a[2] << 16, a[2] >> 16 | a[3] << 16, a[3] >> 16};
    v.a = a;
}
template <typename T, bool LABELLED = false> struct Source {
    static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
    struct Raw { Chunk<T> v; int label; bool in; };
    const T* p;
    long long rep, row;
    int rows, cols;
    Labelled live;
    __device__ __forceinline__ void bind(int k) { p += k * rep; if (LABELLED) live.labels += (long long)k * rows; }
    __device__ __forceinline__ Raw load(int r, int c) const
    {
        Raw v;
        v.in = r < rows && c < cols;
        v.label = LABELLED ? live.labels[min(r, rows - 1)] : 0;
        v.v.load(p + (v.in ? r * row + min(c, cols - 8) : 0ll), 8);
        return v;
    }
    // the chunk at column c, some chunk of its slab reaching beyond the row or not
    __device__ __forceinline__ bool has_tail(int c_begin, int c_end) const { return (cols & 7) && c_begin < cols && c_end > cols; }
    __device__ __forceinline__ void planes(Raw v, int c, bool tail, u4 (&out)[kPlanes]) const
    {
        if (tail) move_down(v.v, min(max(c + 8 - cols, 0), 7));
        split(v.v, out);
        const bool on = v.in && (!LABELLED || (unsigned)v.label < (unsigned)live.classes);
#pragma unroll
        for (int s = 0; s < kPlanes; ++s) out[s] = on ? out[s] : u4{0, 0, 0, 0};
    }
    static __device__ __forceinline__ void split(const Chunk<__bf16>& v, u4 (&out)[1]) { out[0] = v.a; }
    static __device__ __forceinline__ void split(const Chunk<float>& v, u4 (&out)[3])
    {
        u2 h[2], m[2], l[2];
        parts3(__builtin_bit_cast(f4, v.a), h[0], m[0], l[0]);
        parts3(__builtin_bit_cast(f4, v.b), h[1], m[1], l[1]);
        out[0] = join8(h[0], h[1]); out[1] = join8(m[0], m[1]); out[2] = join8(l[0], l[1]);
    }
};
template <typename T, bool LABELLED = false> Source<T, LABELLED> source(const Rows& r, int rows, int cols, Labelled live = {nullptr, 0})
{
    return Source<T, LABELLED>{(const T*)r.p, r.rep, r.row, rows, cols, live};
}

struct SourcePacked {              // rows and columns of one replica; the surplus columns of the checkpoint are zero
    static constexpr int kPlanes = 1;
    struct Raw { u2 q; unsigned e; bool in; };
    Packed p;
    int rows, cols;
    __device__ __forceinline__ void bind(int k)
    {
        p.q += (long long)k * rows * p.cols;
        p.e += (long long)k * rows * (p.cols / kGroup);
    }
    __device__ __forceinline__ bool has_tail(int, int) const { return false; }
    __device__ __forceinline__ Raw load(int r, int c) const
    {
        Raw v;
        v.in = r < rows && c < p.cols;
        const long long at = v.in ? r * p.cols + c : 0;
        v.q = *(const u2*)(p.q + at);
        v.e = p.e[at / kGroup];
        return v;
    }
    __device__ __forceinline__ void planes(const Raw& v, int, bool, u4 (&out)[1]) const
    {
        const float unit = group_unit(v.e);                    // q * 2^e has eight significant bits: exact in bf16
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)(int)(int8_t)(v.q[e / 4] >> (8 * (e % 4))) * unit;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[0][e] = v.in ? to_bf16x2(f[2 * e], f[2 * e + 1]) : 0u;
    }
};

// LDS image of one slab of an operand, one plane: along: [BR rows][KS + 8] (rows 16 bytes off a multiple of 32 banks' width),
// across: [KS][BR] with rows an odd multiple of 64 bytes apart, so that the transposing read of 4 rows x 32 columns meets every
// bank once
template <bool ALONG, int BR, int KS> struct Image {
    static constexpr unsigned kPitch = ALONG ? KS * 2 + 16 : BR * 2 % 128 == 0 ? BR * 2 + 64 : BR * 2;
    static constexpr unsigned kPlane = ALONG ? BR * kPitch : KS * kPitch;
    static constexpr int kAcross = ALONG ? KS / 8 : BR / 8;    // chunks in an image row
    static constexpr int kChunks = BR * KS / 8;
    // operand of the 32 rows from r0 and the 16 k of step ks
    static __device__ __forceinline__ bf16x8 read(const char* plane, int r0, int ks, int lane)
    {
        if (ALONG) return *(const bf16x8*)(plane + (r0 + (lane & 31)) * kPitch + (ks * 16 + (lane >> 5) * 8) * 2);
        const unsigned off = (ks * 16 + (lane >> 5) * 8 + (lane & 15) / 4) * kPitch + (r0 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3)) * 2;
        return lds_read_tr8(plane, off, kPitch);
    }
};

// A wave's part of the tile, as an epilogue gets it.  LANE_M: a lane holds one m (m0 + 32 * tm + lane % 32) and the n
// n0 + 32 * tn + 8 * (i / 4) + 4 * (lane / 32) + i % 4 of acc[tm][tn][i]; else n and m change places.
// sum: the columns' sums of B (every row of them the same), in the waves that has_sum() names of an epilogue that asks for them.
template <int TM, int TN> struct Tile {
    f16 acc[TM][TN];
    f16 sum[TN];
    int rep, split, m0, n0, lane, wave, bm, bn;                 // bm, bn: where the workgroup's tile begins
};

// sum_k B(n, k) is one more product, of ones: the first waves of the first row of tiles form it from the operands they hold
template <class Epi> __device__ __forceinline__ bool has_sum(const Epi& epi, int m0)
{
    if constexpr (Epi::kSums) return m0 == 0 && epi.sums;
    return false;
}
__device__ __forceinline__ bf16x8 ones()
{
    constexpr unsigned one2 = 0x3f803f80u;
    return __builtin_bit_cast(bf16x8, (u4{one2, one2, one2, one2}));
}

// One workgroup's tile.
template <class SA, bool A_ALONG, class SB, bool B_ALONG, int BM, int BN, int WM, int WN, int KS, int NBUF, int AHEAD, class Epi>
__device__ __forceinline__ void product_tile(SA a, SB b, int K, int tiles_m, int tiles_n, int splits, int split_len, int total, Epi epi)
{
    constexpr int NT = WM * WN * 64, TM = BM / WM / 32, TN = BN / WN / 32, PA = SA::kPlanes, PB = SB::kPlanes;
    typedef Image<A_ALONG, BM, KS> IA;
    typedef Image<B_ALONG, BN, KS> IB;
    constexpr int NA = (IA::kChunks + NT - 1) / NT, NB = (IB::kChunks + NT - 1) / NT;
    constexpr unsigned kBuf = PA * IA::kPlane + PB * IB::kPlane;
    __shared__ __attribute__((aligned(16))) char smem[NBUF * kBuf];

    const unsigned item = blockIdx.y * gridDim.x + logical_block();
    if (item >= (unsigned)total) return;
    const int tm_i = item % tiles_m, r1 = item / tiles_m, tn_i = r1 % tiles_n, r2 = r1 / tiles_n;
    Tile<TM, TN> t;
    t.split = r2 % splits;
    t.rep = r2 / splits;
    a.bind(t.rep);
    b.bind(t.rep);
    const int tid = threadIdx.x, wave = tid / 64;
    t.lane = tid & 63;
    t.wave = wave;
    const int bm = t.bm = tm_i * BM, bn = t.bn = tn_i * BN, wm = (wave % WM) * TM * 32, wn = (wave / WM) * TN * 32;
    t.m0 = bm + wm;
    t.n0 = bn + wn;
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

    typename SA::Raw ra[AHEAD][NA];
    typename SB::Raw rb[AHEAD][NB];
    auto fetch = [&](int k0, int slot) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int id = tid + i * NT, r = id / IB::kAcross, c = id % IB::kAcross * 8;
            if (IB::kChunks % NT == 0 || id < IB::kChunks) rb[slot][i] = B_ALONG ? b.load(bn + r, k0 + c) : b.load(k0 + r, bn + c);
        }
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int id = tid + i * NT, r = id / IA::kAcross, c = id % IA::kAcross * 8;
            if (IA::kChunks % NT == 0 || id < IA::kChunks) ra[slot][i] = A_ALONG ? a.load(bm + r, k0 + c) : a.load(k0 + r, bm + c);
        }
    };
    auto store = [&](char* buf, int slot, int k0) {
        const bool tail_a = A_ALONG ? a.has_tail(k0, k0 + KS) : a.has_tail(bm, bm + BM), tail_b = B_ALONG ? b.has_tail(k0, k0 + KS) : b.has_tail(bn, bn + BN);
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int id = tid + i * NT, r = id / IA::kAcross, c = id % IA::kAcross;
            if (IA::kChunks % NT == 0 || id < IA::kChunks) {
                u4 p[PA];
                a.planes(ra[slot][i], (A_ALONG ? k0 : bm) + c * 8, tail_a, p);
#pragma unroll
                for (int s = 0; s < PA; ++s) *(u4*)(buf + s * IA::kPlane + r * IA::kPitch + c * 16) = p[s];
            }
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int id = tid + i * NT, r = id / IB::kAcross, c = id % IB::kAcross;
            if (IB::kChunks % NT == 0 || id < IB::kChunks) {
                u4 p[PB];
                b.planes(rb[slot][i], (B_ALONG ? k0 : bn) + c * 8, tail_b, p);
#pragma unroll
                for (int s = 0; s < PB; ++s) *(u4*)(buf + PA * IA::kPlane + s * IB::kPlane + r * IB::kPitch + c * 16) = p[s];
            }
        }
    };
    auto multiply = [&](const char* buf) {
#pragma unroll
        for (int ks = 0; ks < KS / 16; ++ks) {
            bf16x8 fa[TM][PA], fb[TN][PB];
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int s = 0; s < PA; ++s) fa[i][s] = IA::read(buf + s * IA::kPlane, wm + 32 * i, ks, t.lane);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int s = 0; s < PB; ++s) fb[j][s] = IB::read(buf + PA * IA::kPlane + s * IB::kPlane, wn + 32 * j, ks, t.lane);
            if (Epi::kSums && sums) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int s = PB - 1; s >= 0; --s) t.sum[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones(), fb[j][s], t.sum[j], 0, 0, 0);
            }
            // planes i and j with i + j <= 2: what is left out is below 2^-24 of the product
#pragma unroll
            for (int sum = 2; sum >= 0; --sum)                  // the small products first
#pragma unroll
                for (int s = 0; s < PA; ++s) {
                    if (sum - s < 0 || sum - s >= PB) continue;
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j)
                            t.acc[i][j] = Epi::kLaneM ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j][sum - s], fa[i][s], t.acc[i][j], 0, 0, 0)
                                                 : __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i][s], fb[j][sum - s], t.acc[i][j], 0, 0, 0);
                }
        }
    };

#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (k_begin + i * KS < k_end) fetch(k_begin + i * KS, i);
    constexpr int TURNS = AHEAD * NBUF;
    for (int k0 = k_begin; k0 < k_end; k0 += TURNS * KS) {
#pragma unroll
        for (int u = 0; u < TURNS; ++u) {
            const int k = k0 + u * KS;
            if (k >= k_end) break;
            char* buf = smem + u % NBUF * kBuf;
            if (NBUF == 1 && k > k_begin) __syncthreads();     // the slab before has been read
            store(buf, u % AHEAD, k);
            __syncthreads();
            if (k + AHEAD * KS < k_end) fetch(k + AHEAD * KS, u % AHEAD);
            multiply(buf);
        }
    }
    if constexpr (Epi::kStaged) {
        __syncthreads();
        epi(t, smem);
    } else epi(t);
}

template <class SA, bool A_ALONG, class SB, bool B_ALONG, int BM, int BN, int WM, int WN, int KS, int NBUF, int AHEAD, class Epi>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(SA a, SB b, int K, int tiles_m, int tiles_n, int splits, int split_len,
                                                               int total, Epi epi)
{
    product_tile<SA, A_ALONG, SB, B_ALONG, BM, BN, WM, WN, KS, NBUF, AHEAD>(a, b, K, tiles_m, tiles_n, splits, split_len, total, epi);
}

// ---- epilogues that only store ---------------------------------------------------------------------------------
// C to a tensor, times a factor per replica (lanes along n); SUMS: and B's column sums
template <typename T, bool SUMS = false> struct StoreTile {
    static constexpr bool kLaneM = false, kStaged = false, kSums = SUMS;
    T* p;
    long long rep, row;
    const float* factor;           // [replicas] or null
    int M, N;
    float* sums;
    long long sums_rep;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t) const
    {
        const float f = factor ? factor[t.rep] : 1.f;
        T* out = p + t.rep * rep;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = t.n0 + 32 * j + (t.lane & 31);
                if (n >= N) continue;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int m = t.m0 + 32 * i + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4;
                    if (m < M) out[m * row + n] = (T)(t.acc[i][j][e] * f);
                }
            }
        if (SUMS && has_sum(*this, t.m0)) {
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = t.n0 + 32 * j + t.lane;
                if (t.lane < 32 && n < N) sums[t.rep * sums_rep + n] = t.sum[j][0];
            }
        }
    }
};
// C into [split][replica][lines][ld] floats, over or onto what is there; SUMS: B's column sums into line M (lines = M + 1)
template <bool SUMS = false> struct StoreShare {
    static constexpr bool kLaneM = false, kStaged = false, kSums = SUMS;
    float* p;
    int M, N, ld, lines, replicas;
    bool onto, sums;
    template <int TM, int TN> __device__ __forceinline__ void operator()(const Tile<TM, TN>& t) const
    {
        float* out = p + ((long long)t.split * replicas + t.rep) * lines * ld;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = t.n0 + 32 * j + (t.lane & 31);
                if (n >= N) continue;
                float have[16] = {};
                if (onto) {                                    // all loads on their way before the first addition
#pragma unroll
                    for (int e = 0; e < 16; ++e) have[e] = out[(long long)min(t.m0 + 32 * i + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4, M - 1) * ld + n];
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int m = t.m0 + 32 * i + 8 * (e / 4) + 4 * (t.lane >> 5) + e % 4;
                    if (m < M) out[(long long)m * ld + n] = have[e] + t.acc[i][j][e];
                }
            }
        if (SUMS && has_sum(*this, t.m0)) {
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = t.n0 + 32 * j + t.lane;
                if (t.lane < 32 && n < N) out[(long long)M * ld + n] = t.sum[j][0];
            }
        }
    }
};

// A tensor from the shares of a contraction, [splits][replicas][lines][ld] floats, eight columns a thread, times a factor per replica (or
// null); zero in rows that take no part; the last line goes to `last` if that is there.  G threads take the shares of a chunk, each its own in
// ascending order, and are added in ascending order: where there are many shares there are few chunks.
template <typename T, int G>
__global__ __launch_bounds__(256) void join_shares_kernel(const float* share, int splits, long long step, int lines, int cols, int ld, long long total,
                                                          Labelled live, const float* factor, T* out, long long rep, long long row, T* last, long long last_rep)
{
    constexpr int PER = 256 / G;
    __shared__ __attribute__((aligned(16))) float part[G][G > 1 ? PER * 8 : 8];
    const int mine = threadIdx.x % PER, group = threadIdx.x / PER;
    const long long at = line_block() * PER + mine;
    f4 a = {}, b = {};
    if (at < total) {
        const float* src = share + at * 8;
#pragma unroll 8
        for (int s = group; s < splits; s += G) { a += *(const f4*)(src + s * step); b += *(const f4*)(src + s * step + 4); }
    }
    if (G > 1) {
        *(f4*)&part[group][mine * 8] = a;
        *(f4*)&part[group][mine * 8 + 4] = b;
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 1; g < G; ++g) { a += *(const f4*)&part[g][mine * 8]; b += *(const f4*)&part[g][mine * 8 + 4]; }
    }
    if (at >= total) return;
    const int chunks = ld / 8;
    const long long line = at / chunks;
    const int c = (int)(at - line * chunks) * 8, k = (int)(line / lines), t = (int)(line - (long long)k * lines);
    if (live.labels) live.labels += (long long)k * lines;
    const float f = factor ? factor[k] : 1.f;
    const bool on = live.at(t);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = on ? a[e] * f : 0.f; v[4 + e] = on ? b[e] * f : 0.f; }
    store_chunk(last && t == lines - 1 ? last + k * last_rep + c : out + k * rep + t * row + c, cols - c, v);
}
template <typename T>
hipError_t join_shares(const float* share, int splits, int replicas, int lines, int cols, int ld, Labelled live, const float* factor, const Rows& out,
                       T* last, long long last_rep, hipStream_t s)
{
    const long long all = (long long)replicas * lines, total = all * (ld / 8);
    if (total == 0) return hipSuccess;
    auto* kernel = splits > 8 ? join_shares_kernel<T, 8> : join_shares_kernel<T, 1>;
    const int per = splits > 8 ? 32 : 256;
    kernel<<<line_grid((total + per - 1) / per, 256), 256, 0, s>>>(share, splits, all * ld, lines, cols, ld, total, live, factor, (T*)out.p, out.rep, out.row, last, last_rep);
    return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG, class SA, class SB, class Epi>
hipError_t launch_product(const SA& a, const SB& b, int replicas, int M, int N, int K, int splits, int split_len, const Epi& epi, hipStream_t s)
{
    constexpr bool wide = SA::kPlanes == 3 || SB::kPlanes == 3;
    // few rows: memory bound, so more of W on its way at a time and one image, for more workgroups on a compute unit.  32-bit operands: 64 k
    // along W's rows, 32 across (W of 3 x 512 x 26364: 32.6 us against 38.4; the other way round 20 x 128 x 10007: 11.6 against 10.7)
    constexpr int KS = BM == 32 ? (wide ? (B_ALONG ? 64 : 32) : 128) : 32, NBUF = wide || BM == 32 ? 1 : 2, AHEAD = BM == 32 ? 2 : 1;
    const int tm = (M + BM - 1) / BM, tn = (N + BN - 1) / BN;
    const long long total = (long long)replicas * splits * tm * tn;
    if (total == 0) return hipSuccess;
    if (total > 0x7fffff00ll) return hipErrorInvalidValue;
    product_kernel<SA, A_ALONG, SB, B_ALONG, BM, BN, WM, WN, KS, NBUF, AHEAD, Epi>
        <<<line_grid(die_grid(total), WM * WN * 64), WM * WN * 64, 0, s>>>(a, b, K, tm, tn, splits, split_len, (int)total, epi);
    return hipGetLastError();
}

}  // namespace head
}  // namespace hadfl
