// The gated block for prompts and training: both projections, the activation and the product in
// one kernel, and its backward pass. Part of cd_api.hip (its only includer, after cd_adapters.hpp).
//
//   g = x Wg^T, u = x Wu^T, s = 1 / (1 + exp(-g)), h = g s u
//   dg = dh u s (1 + g (1 - s)), du = dh g s
//   dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x
//
// All are products C[m][n] = sum_k M(m, k) N(n, k), n contiguous in C. N's rows are the first operand
// of an MFMA, so that a lane holds four neighbouring n. An operand is stored with k contiguous (x and
// the weights of the first two products, dg and du of dx) or with k across its rows (the weights of
// dx, both operands of the weights' gradients). Either way a tile goes to LDS as it lies in memory,
// 16 bytes a lane without passing registers; a k-contiguous tile is read 16 bytes a lane, the other
// with the transposing LDS reads.
#pragma once

#include "cd_device.hpp"

namespace {

constexpr int kGtMaxDim = 65536, kGtMaxTokens = 1 << 20;
constexpr size_t kGtMaxStride = (size_t)1 << 20;  // row strides: 256 rows stay below 2^30 bytes
constexpr int kGtTerms = 3;                       // bf16 terms of an fp32 number
constexpr int kGtOutside = 0x40000000;            // an offset past every resource: reads zeros
constexpr size_t kGtPartFloats = (size_t)16 << 20;  // place for partial sums (64 MiB)

constexpr int kGtFew = 4096;  // elements of dg that are held in two bf16 terms

enum GtKind { kGtForward, kGtBackward, kGtDx, kGtDw };

struct GtArgs {
    const uint16_t *x;  // [T][m], row stride ldx
    size_t ldx;
    const uint16_t *Wg, *Wu;  // [f][m]
    const uint16_t *dh;       // [T][f], row stride lddh
    size_t lddh;
    int T, m, f;
    int type;    // of out (and of both weight gradients)
    void *out;   // h or dx; dW: the gradient of W_gate
    void *out2;  // dW: the gradient of W_up
    size_t ldo;
    uint16_t *d;  // [terms][T][2][fd]: dg and du of a token side by side
    // f rounded up to 128 bytes, so that rows begin on a cache line (backward of 2000 tokens of 1000 x 3000 in fp32 204 us
    // against 214, of 1000 of 1024 x 2008 53.6 against 55.5)
    int fd;
    int terms;
    float *part;     // their sums (gt_part)
    int mt, nt;      // tiles
    int splits, ktiles;  // dx and dW: workgroups that share a tile, and their tiles of k
};

// a buffer resource over 2^30 bytes at p (uniform): what lies past them reads as zero
__device__ __forceinline__ u32x4 gt_resource(const void *p)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return u32x4{lo, hi, (uint32_t)kGtOutside, 0x00027000u};
}

// 16 bytes a lane from the resource to LDS at `lds` + 16 lane. The builtin would do, but the compiler
// then waits for every load in flight before each LDS read. Nothing is written but LDS and m0, which is
// named: code that the compiler sets it for sets it again behind this. (The warning ignored is that it would not be
// kept for a program that relied on it across the statement.) The waits and barriers are gt_wait's.
// NT: past the caches.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool NT = false>
__device__ __forceinline__ void gt_load_lds(const u32x4 &r, int off, uint32_t lds)
{
    if constexpr (NT)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
                     ::"s"(lds), "v"(off), "s"(r) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     ::"s"(lds), "v"(off), "s"(r) : "memory", "m0");
}
#pragma clang diagnostic pop

// All but the last N loads of this wave have come, and its LDS reads; then every wave's have.
template <int N>
__device__ __forceinline__ void gt_wait()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t gt_lds(const void *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// A tile of R rows (of m or n) x BK columns of k.
//
// KC, k contiguous: rows of BK; 16-byte chunk c of row r sits at c ^ (r & 7), which spreads the 16
// rows of an operand over the banks. Otherwise BK rows of R; the 32-byte slots of row k are permuted
// by k & 3 and bit 3 of k, so that what the lanes of a transposing read take (rows 8 j + 0..3 of one
// slot for 16 lanes, j = lane / 16) lies on different banks.
//
// LINES (KC): rows that begin inside a cache line. A tile then holds whole lines of each row, of which the first
// chunks may belong to the tile of k before, so that its loads take no line twice; products read two tiles in a
// row. Row r begins p8 + r ld8 chunks behind a line's start; its chunks' places in the line are
// permuted by the bits of r that this leaves alike.
template <int R, int BK, bool KC, int THREADS, bool LINES = false>
struct GtTile {
    static constexpr int kRowChunks = (KC ? BK : R) / 8;
    static constexpr int kLoads = R * BK / 8 / THREADS;
    static constexpr int kBytes = R * BK * 2;
    static constexpr int kRowsALoad = THREADS / kRowChunks;
    static_assert(R * BK / 8 % THREADS == 0 && THREADS % kRowChunks == 0, "whole loads");
    static_assert(!KC || kRowsALoad % 8 == 0, "the row's swizzle is the same for every load");
    static_assert(!LINES || KC, "lines of a row");

    int off[kLoads];  // byte offset from the tile's first element
    int k[kLoads];    // k of this thread's chunks
    uint32_t p8, ld8;  // LINES: the operand's address and row length, in chunks

    static __device__ __forceinline__ int slot_key(int k) { return ((k & 3) | (k >> 1 & 4)) & (R / 16 - 1); }

    // LINES: eight rows begin at 8, 4, 2 or 1 places of a line by ld8's factors of 2; r's other bits tell the rest apart
    __device__ __forceinline__ int key(int r) const { return (r & 7) >> (3 - __builtin_ctz(ld8 | 8u)); }

    // p: the operand; valid: its rows (KC) or columns from this tile on
    __device__ __forceinline__ void init(const uint16_t *p, size_t ld, int valid)
    {
        p8 = (uint32_t)(reinterpret_cast<uint64_t>(p) >> 4);
        ld8 = (uint32_t)(ld / 8);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = threadIdx.x / kRowChunks + i * kRowsALoad, pos = threadIdx.x % kRowChunks;
            if (LINES) {
                const int c = (pos ^ key(row)) - (int)((p8 + row * ld8) & 7);
                k[i] = c * 8;
                off[i] = row < valid ? row * (int)ld * 2 + c * 16 + 128 : kGtOutside;  // (from the line before on)
            } else if (KC) {
                const int c = pos ^ (row & 7);
                k[i] = c * 8;
                off[i] = row < valid ? row * (int)ld * 2 + c * 16 : kGtOutside;
            } else {
                const int c = ((pos >> 1) ^ slot_key(row)) * 2 + (pos & 1);
                k[i] = row;
                off[i] = c * 8 < valid ? row * (int)ld * 2 + c * 16 : kGtOutside;
            }
        }
    }

    // the tile at base (uniform), of whose k `left` remain (start: it is the first, LINES)
    template <bool NT = false>
    __device__ __forceinline__ void load(const uint16_t *base, int left, uint32_t lds, bool start = false) const
    {
        const u32x4 r = gt_resource(LINES ? base - 64 : base);
        const uint32_t at = lds + __builtin_amdgcn_readfirstlane(threadIdx.x / cdk::kWave) * 1024;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            gt_load_lds<NT>(r, k[i] < left && (!LINES || !start || k[i] >= 0) ? off[i] : kGtOutside,
                            at + i * (THREADS * 16));
    }

    // the same operand, of LINES: its chunks lie in this tile (at `lds`) and the next
    __device__ __forceinline__ u32x4 read_lines(const char *lds, int next, int r0, int kk) const
    {
        const int lane = threadIdx.x % cdk::kWave, i = lane % 16, c = kk * 4 + lane / 16 + (int)((p8 + i * ld8) & 7);
        return *reinterpret_cast<const u32x4 *>(lds + (c < kRowChunks ? 0 : next) + (r0 + i) * (BK * 2) +
                                                ((c % kRowChunks ^ key(i)) << 4));
    }

    // operand of rows r0..r0 + 15 and k 32 kk..32 kk + 31 (lane: row lane % 16, k 8 (lane / 16)..)
    static __device__ __forceinline__ u32x4 read(const char *lds, int r0, int kk)
    {
        const int lane = threadIdx.x % cdk::kWave, i = lane % 16, j = lane / 16;
        if constexpr (KC) {
            const int r = r0 + i;
            return *reinterpret_cast<const u32x4 *>(lds + r * (BK * 2) + (((kk * 4 + j) ^ (r & 7)) << 4));
        } else {
            const int k = kk * 32 + 8 * j + (i >> 2);
            const char *p = lds + k * (R * 2) + ((r0 / 16) ^ slot_key(k)) * 32 + (i & 3) * 8;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * (R * 2)));
            return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// The workgroup's tile, and its part of k: all tiles of one part after another, an even stretch of them on each
// XCD (blockIdx.x % 8). Neighbours in time there take `group` tiles of m by a stretch of n, so that its L2
// holds what they share. False: no tile.
__device__ __forceinline__ bool gt_place(int block, int mt, int nt, int splits, int &mi, int &ni, int &split)
{
    constexpr int group = 4;
    const int total = mt * nt * splits, per = (total + 7) / 8;
    int t = block % 8 * per + block / 8;
    if (block / 8 >= per || t >= total)
        return false;
    split = splits > 1 ? __builtin_amdgcn_readfirstlane(t / (mt * nt)) : 0;
    t -= split * (mt * nt);
    const int width = group * nt, first = t / width * group, rows = min(group, mt - first);
    // known to be uniform: what follows from them stays in scalar registers
    mi = __builtin_amdgcn_readfirstlane(first + t % width % rows);
    ni = __builtin_amdgcn_readfirstlane(t % width / rows);
    return true;
}

// The tiles of k that a workgroup takes, from `first` on: those of one product (dx: of dg Wg, then of du Wu),
// each with every term of dg and du in turn, the smallest first, so that the other operand's tile comes
// from L2 for all but the first.
template <int KIND, int BK>
struct GtWalk {
    static constexpr bool kTwo = KIND == kGtForward || KIND == kGtBackward;
    const uint16_t *pm, *pn, *pn2;  // m's tile; n's, and the one beside it (kTwo: of W_up)
    int left;                       // k from here on
    int term, product;
    const uint16_t *m1, *n1;        // dx: du's and W_up's first tile

    // n2: from n's tile to the one beside it
    __device__ __forceinline__ void init(const GtArgs &a, int m0, int n0, int n2, int second, int first)
    {
        const size_t plane = (size_t)a.T * 2 * a.fd;
        term = product = 0;
        if constexpr (kTwo) {
            pm = a.x + m0 * a.ldx;
            pn = a.Wg + (size_t)n0 * a.m;
            pn2 = a.Wu + (size_t)n0 * a.m;
            left = a.m;
        } else if constexpr (KIND == kGtDx) {
            const int per = (a.f + BK - 1) / BK, kt = first / a.terms;  // (first: a multiple of the terms)
            const uint16_t *d = a.d + (a.terms - 1) * plane + m0 * (2 * (size_t)a.fd);
            m1 = d + a.fd;
            n1 = a.Wu + n0;
            product = kt >= per;
            pm = (product ? m1 : d) + (size_t)(kt % per) * BK;
            pn = (product ? n1 : a.Wg + n0) + (size_t)(kt % per) * BK * a.m;
            pn2 = pn + n2;
            left = a.f - kt % per * BK;
        } else {
            const int kt = first / a.terms;
            pm = a.d + (a.terms - 1) * plane + (size_t)second * a.fd + m0 + (size_t)kt * BK * 2 * a.fd;
            pn = a.x + n0 + (size_t)kt * BK * a.ldx;
            pn2 = pn + n2;
            left = a.T - kt * BK;
        }
    }

    __device__ __forceinline__ void advance(const GtArgs &a, int n2)
    {
        if constexpr (kTwo) {
            pm += BK;
            pn += BK;
            pn2 += BK;
            left -= BK;
        } else {
            const size_t plane = (size_t)a.T * 2 * a.fd;
            if (++term < a.terms) {
                pm -= plane;
                return;
            }
            term = 0;
            pm += (a.terms - 1) * plane + (KIND == kGtDw ? (size_t)BK * 2 * a.fd : BK);
            pn += (size_t)BK * (KIND == kGtDw ? a.ldx : a.m);
            pn2 = pn + n2;
            left -= BK;
            if (KIND == kGtDx && left <= 0 && product == 0) {
                product = 1;
                pm = m1;
                pn = n1;
                pn2 = pn + n2;
                left = a.f;
            }
        }
    }
};

__device__ __forceinline__ uint64_t gt_pack4(const f32x4_t &v)
{
    return ad_pack(v[0], v[1]) | (uint64_t)ad_pack(v[2], v[3]) << 32;
}

__device__ __forceinline__ void gt_store4(void *out, int type, size_t i, const f32x4_t &v)
{
    if (type == CD_TYPE_F32)
        *reinterpret_cast<f32x4_t *>(static_cast<float *>(out) + i) = v;
    else
        *reinterpret_cast<uint64_t *>(static_cast<uint16_t *>(out) + i) = gt_pack4(v);
}

// Four bf16 a lane of NF neighbouring 16 x 16 tiles (lane: row lane % 16, columns 4 (lane / 16)..), `row` at
// the first column; `left` columns of it exist, none where not ok. Two tiles at a time change hands between
// rows of 16 lanes, so that a lane stores 16 bytes and a row 64 at once: 32-byte pieces cost L2 a request each
// (backward of 1024 tokens of 4096 x 14336 626 us against 651).
template <int NF>
__device__ __forceinline__ void gt_store_tiles(uint16_t *row, bool ok, int left, const uint64_t (&v)[NF])
{
    const int j = threadIdx.x % cdk::kWave / 16;
#pragma unroll
    for (int i = 0; i < NF; i += 2) {
        if constexpr (NF == 1) {
            if (ok && 4 * j < left)
                *reinterpret_cast<uint64_t *>(row + 4 * j) = v[0];
        } else {
            const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)v[i], (uint32_t)v[i + 1], false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(v[i] >> 32), (uint32_t)(v[i + 1] >> 32), false,
                                                             false);
            const int c = 16 * i + j % 2 * 16 + j / 2 * 8;
            if (ok && c < left)
                *reinterpret_cast<u32x4 *>(row + c) = u32x4{lo[0], hi[0], lo[1], hi[1]};
        }
    }
}

// the same of fp32 sums, to out of `type` from element `at` on
template <int NF>
__device__ __forceinline__ void gt_store_sums(void *out, int type, size_t at, bool ok, int left, const f32x4_t (&v)[NF])
{
    const int j = threadIdx.x % cdk::kWave / 16;
    if (type == CD_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < NF; ++i)
            if (ok && 16 * i + 4 * j < left)
                *reinterpret_cast<f32x4_t *>(static_cast<float *>(out) + at + 16 * i + 4 * j) = v[i];
        return;
    }
    uint64_t w[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i)
        w[i] = gt_pack4(v[i]);
    gt_store_tiles(static_cast<uint16_t *>(out) + at, ok, left, w);
}

// 1 / (1 + exp(-g)) to a few units in the last place, on the hardware's exp2 and reciprocal: with the
// library's expf and division the last step of a 256 x 256 tile costs three times the instructions. exp2's
// argument is rounded, for large |g| by more than exp2 itself; its rounding error goes back in as a factor.
// Past 200 it is 0 or 1 (for NaN too: what it multiplies is not finite itself).
__device__ __forceinline__ float gt_sigmoid(float g)
{
    constexpr float log2e = 1.44269502f, rest = 1.92596299e-8f, ln2 = 0.693147182f;
    g = __builtin_amdgcn_fmed3f(g, -200.0f, 200.0f);
    const float t = -g * log2e;
    const float err = fmaf(-g, rest, fmaf(-g, log2e, -t));
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t) * fmaf(err, ln2, 1.0f));
}

// where a split leaves its part: [splits][T][m], or [splits][2][f][m] of the gradients of W_gate and W_up
template <int KIND>
__device__ __forceinline__ float *gt_part(const GtArgs &a, int split, int second)
{
    return a.part + (KIND == kGtDx ? split * (size_t)a.T : (2 * split + second) * (size_t)a.f) * a.m;
}

// What KIND makes of a row's NF tiles (t, n: this lane's row and the first column; ok: the row exists).
template <int NF>
__device__ __forceinline__ void gt_forward(const GtArgs &a, size_t t, int n, bool ok, const f32x4_t (&g)[NF],
                                           const f32x4_t (&u)[NF])
{
    f32x4_t h[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            h[i][r] = g[i][r] * gt_sigmoid(g[i][r]) * u[i][r];
    gt_store_sums(a.out, a.type, t * a.ldo + n, ok, a.f - n, h);
}

__device__ __forceinline__ uint64_t gt_dh(const GtArgs &a, int t, int n)
{
    return *reinterpret_cast<const uint64_t *>(or_zero(t < a.T && n < a.f, a.dh + (size_t)t * a.lddh + n));
}

// dg and du, in a.terms bf16 terms: one is rounded to nearest even, the operand that a bf16 product takes;
// two hold 16 bits, three all of an fp32 number. w: dh.
template <int NF>
__device__ __forceinline__ void gt_backward(const GtArgs &a, size_t t, int n, bool ok, const uint64_t (&w)[NF],
                                            const f32x4_t (&g)[NF], const f32x4_t (&u)[NF])
{
    f32x4_t d[2][NF];
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t p = (uint32_t)(w[i] >> (r / 2 * 32));
            const float dh = r % 2 ? cdk::bf16_hi(p) : cdk::bf16_lo(p);
            const float s = gt_sigmoid(g[i][r]);
            // (dh u first would overflow where the slope brings it back; the slope is at most 1.1)
            d[0][i][r] = dh * (u[i][r] * (s * (1.0f + g[i][r] * (1.0f - s))));
            d[1][i][r] = dh * (g[i][r] * s);
        }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        uint16_t *o = a.d + t * (2 * (size_t)a.fd) + (size_t)q * a.fd + n;
        if (a.terms == 1) {
            gt_store_sums(o, CD_TYPE_BF16, 0, ok, a.f - n, d[q]);
            continue;
        }
        uint64_t out[kGtTerms][NF];
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            uint32_t w3[4][3];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                ad_split(d[q][i][r], w3[r]);
                if (a.terms == 2)  // the second rounded
                    w3[r][1] = ad_pack(__uint_as_float(w3[r][1]) + __uint_as_float(w3[r][2]), 0.0f) << 16;
            }
#pragma unroll
            for (int k = 0; k < kGtTerms; ++k)
                out[k][i] = (w3[0][k] >> 16 | w3[1][k]) | (uint64_t)(w3[2][k] >> 16 | w3[3][k]) << 32;
        }
#pragma unroll
        for (int k = 0; k < kGtTerms; ++k)
            if (k < a.terms)
                gt_store_tiles(o + (size_t)k * a.T * 2 * a.fd, ok, a.f - n, out[k]);
    }
}

// One tile of BM x BN (twice BN for the two projections, of which a lane holds g and u of the same
// elements). WM x WN waves share it, WK of them each a part of every BK columns of k. STAGES tiles
// of k are in LDS, STAGES - 1 of them in flight. One barrier a tile. NT: the weights past the caches.
//
// Few tokens wait for the weights, which long tiles of k (512 bytes of a row at a time) and 64 to 100 KB in
// flight a CU bring at 5.8 to 6.4 TB/s: 4 tokens of 4096 x 11008 31 us, of 8192 x 28672 146. Some hundreds
// wait for their tiles: a CU takes 35 to 45 bytes a ns of them, whatever their shape and the stages (the loads alone, without
// reads and products, 38.8 us of 46.5 at 333 tokens of 3000 x 8008 and 61.5 of 62.1 at 128 of 4096 x 14336; reads and
// products alone 34 and 32, the matrix cores 32 and 19 % busy). Rows that
// do not begin on 128 bytes cost two lines for one (333 tokens of 3000 x 8008 56 us, of 3008 x 8008 43): LINES.
template <int KIND, int BM, int BN, int BK, int WM, int WN, int WK, int STAGES>
constexpr int kGtLds = std::max(STAGES * (BM + (KIND == kGtForward || KIND == kGtBackward ? 2 : 1) * BN) * BK * 2,
                                (WK - 1) * WM * WN * (KIND == kGtForward || KIND == kGtBackward ? 2 : 1) * (BM / WM) *
                                    (BN / WN) * 4);  // the waves' sums

// block: of the grid; lds: kGtLds bytes
template <int KIND, int BM, int BN, int BK, int WM, int WN, int WK, int STAGES, bool NT, bool LINES = false>
__device__ __forceinline__ void gt_tile(const GtArgs &a, int block, char *lds)
{
    constexpr int kThreads = WM * WN * WK * cdk::kWave;
    constexpr bool kTwo = KIND == kGtForward || KIND == kGtBackward;
    constexpr int NP = kTwo ? 2 : 1, FM = BM / WM / 16, FN = BN / WN / 16, KK = BK / 32 / WK;
    using TM = GtTile<BM, BK, KIND != kGtDw, kThreads, LINES>;
    using TN = GtTile<BN, BK, kTwo, kThreads, LINES>;
    constexpr int kStage = TM::kBytes + NP * TN::kBytes;
    constexpr int kFlight = (TM::kLoads + NP * TN::kLoads) * (STAGES - (LINES ? 3 : 2));
    int mi, ni, split;
    if (!gt_place(block, KIND == kGtDw && a.out && a.out2 ? 2 * a.mt : a.mt, a.nt, kTwo ? 1 : a.splits, mi, ni, split))
        return;
    // dW: the tiles of W_gate's gradient, then those of W_up's
    const int second = KIND == kGtDw ? (!a.out || mi >= a.mt) : 0;
    if (KIND == kGtDw && mi >= a.mt)
        mi -= a.mt;
    const int m0 = mi * BM, n0 = ni * BN;
    const int M = KIND == kGtDw ? a.f : a.T, N = kTwo ? a.f : a.m;
    const int K = kTwo ? a.m : KIND == kGtDx ? a.f : a.T;
    const size_t ldm = kTwo ? a.ldx : 2 * (size_t)a.fd, ldn = KIND == kGtDw ? a.ldx : a.m;

    TM tm;
    TN tn;
    tm.init(kTwo ? a.x : a.d, ldm, M - m0);
    tn.init(a.Wg, ldn, N - n0);
    const int first = kTwo ? 0 : split * a.ktiles;  // a split of the tiles of k
    const int all = (K + BK - 1) / BK * (kTwo ? 1 : KIND == kGtDx ? 2 * a.terms : a.terms);
    const int nk = kTwo ? all : min(a.ktiles, all - first);
    GtWalk<KIND, BK> w;
    w.init(a, m0, n0, 0, second, first);
    const uint32_t base = gt_lds(lds);
    const auto issue = [&](int stage) {  // the next tile of k (zeros behind the last)
        const uint32_t at = base + stage * kStage;
        const bool start = LINES && w.left == K;
        tm.load(w.pm, w.left, at, start);
        tn.template load<NT>(w.pn, w.left, at + TM::kBytes, start);
        if constexpr (kTwo)
            tn.template load<NT>(w.pn2, w.left, at + TM::kBytes + TN::kBytes, start);
        w.advance(a, 0);
    };

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / cdk::kWave);
    const int wk = wave % WK, wn = wave / WK % WN, wm = wave / WK / WN;
    f32x4_t acc[NP][FN][FM];
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j)
                acc[p][i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        issue(s);
    int stage = 0;
    for (int t = 0; t < nk; ++t) {
        gt_wait<kFlight>();  // tile t is there (LINES: the next too), and every wave is done with tile t - 1
        issue(stage == 0 ? STAGES - 1 : stage - 1);
        const char *s = lds + stage * kStage;
        const int next = stage + 1 == STAGES ? -stage * kStage : kStage;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            u32x4 vm[FM], vn[NP][FN];
#pragma unroll
            for (int j = 0; j < FM; ++j)
                if constexpr (LINES)
                    vm[j] = tm.read_lines(s, next, (wm * FM + j) * 16, wk * KK + kk);
                else
                    vm[j] = TM::read(s, (wm * FM + j) * 16, wk * KK + kk);
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    const char *sn = s + TM::kBytes + p * TN::kBytes;
                    if constexpr (LINES)
                        vn[p][i] = tn.read_lines(sn, next, (wn * FN + i) * 16, wk * KK + kk);
                    else
                        vn[p][i] = TN::read(sn, (wn * FN + i) * 16, wk * KK + kk);
                }
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int j = 0; j < FM; ++j)
                        acc[p][i][j] = mfma16(vn[p][i], vm[j], acc[p][i][j]);
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    gt_wait<0>();  // no load outlives the workgroup's LDS

    const int lane = threadIdx.x % cdk::kWave;
    if constexpr (WK > 1) {  // the waves' parts of k, added in their order
        f32x4_t *sums = reinterpret_cast<f32x4_t *>(lds);
        const auto at = [&](int w, int p, int i, int j) {
            return ((((w * WM + wm) * WN + wn) * NP + p) * FN + i) * FM * cdk::kWave + j * cdk::kWave + lane;
        };
        if (wk > 0) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int j = 0; j < FM; ++j)
                        sums[at(wk - 1, p, i, j)] = acc[p][i][j];
        }
        __syncthreads();
        if (wk > 0)
            return;
#pragma unroll
        for (int w = 0; w < WK - 1; ++w)
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int j = 0; j < FM; ++j)
                        acc[p][i][j] += sums[at(w, p, i, j)];
    }
    uint64_t dh[FM][FN];  // all loads before the first is used
    if constexpr (KIND == kGtBackward) {
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int i = 0; i < FN; ++i)
                dh[j][i] = gt_dh(a, m0 + (wm * FM + j) * 16 + lane % 16, n0 + (wn * FN + i) * 16 + lane / 16 * 4);
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int m = m0 + (wm * FM + j) * 16 + lane % 16, n = n0 + wn * FN * 16;
        f32x4_t v[NP][FN];
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int i = 0; i < FN; ++i)
                v[p][i] = acc[p][i][j];
        if constexpr (KIND == kGtForward)
            gt_forward(a, m, n, m < M, v[0], v[1]);
        else if constexpr (KIND == kGtBackward)
            gt_backward(a, m, n, m < M, dh[j], v[0], v[1]);
        else if (a.splits > 1)
            gt_store_sums(gt_part<KIND>(a, split, second), CD_TYPE_F32, (size_t)m * a.m + n, m < M, N - n, v[0]);
        else
            gt_store_sums(KIND == kGtDw && second ? a.out2 : a.out, a.type, (size_t)m * a.ldo + n, m < M, N - n, v[0]);
    }
}

template <int KIND, int BM, int BN, int BK, int WM, int WN, int WK, int STAGES, bool NT, bool LINES = false>
__global__ __launch_bounds__(WM *WN *WK *cdk::kWave) void k_gt_product(const GtArgs a)
{
    __shared__ __align__(1024) char lds[kGtLds<KIND, BM, BN, BK, WM, WN, WK, STAGES>];
    gt_tile<KIND, BM, BN, BK, WM, WN, WK, STAGES, NT, LINES>(a, blockIdx.x, lds);
}

constexpr int kGtBackK = 256;  // columns of k of its tiles of dx

// Little work: dx (the first `blocks` of the grid) and the weights' gradients in one launch.
__global__ __launch_bounds__(512) void k_gt_back(const GtArgs x, const GtArgs w, int blocks)
{
    constexpr int kLds = std::max(kGtLds<kGtDx, 64, 64, kGtBackK, 1, 2, 4, 2>, kGtLds<kGtDw, 64, 64, 64, 2, 4, 1, 3>);
    __shared__ __align__(1024) char lds[kLds];
    if ((int)blockIdx.x < blocks)
        gt_tile<kGtDx, 64, 64, kGtBackK, 1, 2, 4, 2, false>(x, blockIdx.x, lds);
    else
        gt_tile<kGtDw, 64, 64, 64, 2, 4, 1, 3, false>(w, (int)blockIdx.x - blocks, lds);
}

// Many tiles: 256 x 256 (256 x 128 of both projections), eight waves, each 64 rows of either half of
// m and 32 of either half of n. A tile of 64 columns of k takes two phases, one for each half of m: read the
// operands and start loading what is needed three phases later, then 32 MFMAs a wave. Waves 0-3
// and 4-7 (one of each on a SIMD) are half a phase apart: while one half multiplies, the other
// reads. A wave's LDS reads have returned when it passes the barrier behind them, so a half tile read
// in phase p may be overwritten by loads of phase p + 1; of the loads the last eight may be in flight.
// MH 1: one half of m alone, 128 x 256, a phase a tile of k and three tiles in LDS; the loads are
// issued two phases before they are read, and six of them may be in flight.
//
// What bounds it is the matrix cores' clock under load (80 % busy in the forward call, 78 in dx) and, where an
// operand has k across its rows, twice as many LDS reads of half the size (61 % in the weights' gradients,
// 1352 us if they were whole reads, 1600 so). 8192 tokens of 4096 x 14336: forward 1284 us (1498 TFLOP/s),
// projections of the backward call 1420 (470 MB are stored, 235 loaded at the end of a tile), dx 1320 to
// 1430, weights 1480 to 1570. Four barriers a phase of 16 MFMAs instead: 1360. Persistent workgroups that load the next
// tile while they store: 1334 and, backward, 4468 against 4262.
template <int KIND, int MH>
__global__ __launch_bounds__(512) void k_gt_large(const GtArgs a)
{
    constexpr int BK = 64, FM = 4, FN = 2, KK = BK / 32, kFlight = MH == 2 ? 8 : 6;
    constexpr bool kTwo = KIND == kGtForward || KIND == kGtBackward;
    using TM = GtTile<128, BK, KIND != kGtDw, 512>;
    using TN = GtTile<128, BK, kTwo, 512>;
    constexpr int kHalf = TM::kBytes, kStages = 4 - MH, kStage = (MH + 2) * kHalf;  // m 0, (m 1,) n 0, n 1
    constexpr int kN0 = MH * kHalf, kN1 = kN0 + kHalf;
    static_assert(TM::kBytes == TN::kBytes && TM::kLoads == 2 && TN::kLoads == 2, "loads of a phase");
    __shared__ __align__(1024) char lds[kStages * kStage];

    int mi, ni, split;
    if (!gt_place(blockIdx.x, KIND == kGtDw && a.out && a.out2 ? 2 * a.mt : a.mt, a.nt, kTwo ? 1 : a.splits, mi, ni,
                  split))
        return;
    const int second = KIND == kGtDw ? (!a.out || mi >= a.mt) : 0;
    if (KIND == kGtDw && mi >= a.mt)
        mi -= a.mt;
    const int m0 = mi * (128 * MH), n0 = ni * (kTwo ? 128 : 256);
    const int M = KIND == kGtDw ? a.f : a.T, N = kTwo ? a.f : a.m;
    const int K = kTwo ? a.m : KIND == kGtDx ? a.f : a.T;
    const size_t ldm = kTwo ? a.ldx : 2 * (size_t)a.fd, ldn = KIND == kGtDw ? a.ldx : a.m;
    const int first = kTwo ? 0 : split * a.ktiles;  // a split of the tiles of k
    const int all = (K + BK - 1) / BK * (kTwo ? 1 : KIND == kGtDx ? 2 * a.terms : a.terms);
    const int nk = kTwo ? all : min(a.ktiles, all - first);

    TM tm[MH];
    TN tn[2];
    tm[0].init(a.x, ldm, M - m0);
    if constexpr (MH == 2)
        tm[1].init(a.x, ldm, M - m0 - 128);
    tn[0].init(a.Wg, ldn, N - n0);
    tn[1].init(a.Wg, ldn, N - n0 - (kTwo ? 0 : 128));
    const size_t mh = KIND == kGtDw ? 128 : 128 * ldm;  // to the second half of m
    GtWalk<KIND, BK> w;
    w.init(a, m0, n0, 128, second, first);
    const uint16_t *pm1;  // the tile of k before w's: its second half of m is loaded next
    int left1;
    const uint32_t base = gt_lds(lds);
    const auto load0 = [&](uint32_t at) {  // all but the second half of m
        tm[0].load(w.pm, w.left, at);
        tn[0].load(w.pn, w.left, at + kN0);
        tn[1].load(w.pn2, w.left, at + kN1);
        pm1 = w.pm + mh;
        left1 = w.left;
        w.advance(a, 128);
    };
    load0(base);
    if constexpr (MH == 2)
        tm[1].load(pm1, left1, base + kHalf);
    load0(base + kStage);

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / cdk::kWave), lane = threadIdx.x % cdk::kWave;
    const int wn = wave % 4, wm = wave / 4;
    f32x4_t acc[2][MH][FN][FM];  // halves of n, of m
#pragma unroll
    for (int p = 0; p < 2 * MH; ++p)
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j)
                acc[p / MH][p % MH][i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 vm[FM][KK], vn[2][FN][KK];
    const auto read_m = [&](const char *s) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int j = 0; j < FM; ++j)
                vm[j][kk] = TM::read(s, (wm * FM + j) * 16, kk);
    };
    const auto read_n = [&](u32x4 (&v)[FN][KK], const char *s) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int i = 0; i < FN; ++i)
                v[i][kk] = TN::read(s, (wn * FN + i) * 16, kk);
    };
    const auto multiply = [&](int hm) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kFlight) : "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int hn = 0; hn < 2; ++hn)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int j = 0; j < FM; ++j)
                        acc[hn][hm][i][j] = mfma16(vn[hn][i][kk], vm[j][kk], acc[hn][hm][i][j]);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kFlight) : "memory");
    if (wm == 1)
        asm volatile("s_barrier" ::: "memory");
    int stage = 0;
    for (int t = 0; t < nk; ++t) {
        const char *s = lds + stage * kStage;
        const uint32_t here = base + stage * kStage;
        const uint32_t other = base + (stage == 0 ? kStages - 1 : stage - 1) * kStage;
        read_n(vn[0], s + kN0);
        read_n(vn[1], s + kN1);
        read_m(s);
        if constexpr (MH == 2) {
            tm[1].load(pm1, left1, other + kHalf);
            multiply(0);
            read_m(s + kHalf);
            load0(here);
            multiply(1);
        } else {
            load0(other);
            multiply(0);
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if (wm == 0)
        asm volatile("s_barrier" ::: "memory");
    gt_wait<0>();  // no load outlives the workgroup's LDS

    uint64_t dh[MH][FM][FN];  // all loads before the first is used
    if constexpr (KIND == kGtBackward) {
#pragma unroll
        for (int hm = 0; hm < MH; ++hm)
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int i = 0; i < FN; ++i)
                    dh[hm][j][i] = gt_dh(a, m0 + hm * 128 + (wm * FM + j) * 16 + lane % 16,
                                         n0 + (wn * FN + i) * 16 + lane / 16 * 4);
    }
#pragma unroll
    for (int hm = 0; hm < MH; ++hm)
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int m = m0 + hm * 128 + (wm * FM + j) * 16 + lane % 16, n = n0 + wn * FN * 16;
            f32x4_t v[2][FN];
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < FN; ++i)
                    v[p][i] = acc[p][hm][i][j];
            if constexpr (KIND == kGtForward) {
                gt_forward(a, m, n, m < M, v[0], v[1]);
            } else if constexpr (KIND == kGtBackward) {
                gt_backward(a, m, n, m < M, dh[hm][j], v[0], v[1]);
            } else {
                void *out = KIND == kGtDw && second ? a.out2 : a.out;
                int type = a.type;
                size_t at = (size_t)m * a.ldo + n;
                if (a.splits > 1) {
                    out = gt_part<KIND>(a, split, second);
                    type = CD_TYPE_F32;
                    at = (size_t)m * a.m + n;
                }
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    gt_store_sums(out, type, at + p * 128, m < M, N - n - p * 128, v[p]);
            }
        }
}

// dx, or the weights' gradients (blockIdx.y), from the parts in their order; four columns a thread
template <int KIND>
__global__ __launch_bounds__(256) void k_gt_sum(const GtArgs a)
{
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4, n = (KIND == kGtDx ? (size_t)a.T : a.f) * a.m;
    void *out = blockIdx.y ? a.out2 : a.out;
    if (i >= n || !out)
        return;
    const float *p = gt_part<KIND>(a, 0, blockIdx.y) + i;
    const size_t step = KIND == kGtDx ? n : 2 * n;
    f32x4_t s = *reinterpret_cast<const f32x4_t *>(p);
#pragma unroll 8
    for (int k = 1; k < a.splits; ++k)
        s += *reinterpret_cast<const f32x4_t *>(p + k * step);
    gt_store4(out, a.type, i / a.m * a.ldo + i % a.m, s);
}

__global__ __launch_bounds__(256) void k_gt_zero(uint32_t *p, size_t words)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (size_t)gridDim.x * 256)
        p[i] = 0u;
}

}  // namespace

struct cd_gated {
    int m, f, max_tokens, device;
    unsigned flags;
    void *ws;
    uint16_t *d;
    float *part;
};

namespace {

int gt_fd(int f) { return (f + 63) / 64 * 64; }

// How many workgroups share a tile of dx or of the weights' gradients: each takes four tiles of k and more.
template <int KIND>
void gt_split(GtArgs &a, int BK, int splits)
{
    a.splits = 1;
    if (KIND != kGtDx && KIND != kGtDw)
        return;
    const int all = KIND == kGtDx ? 2 * ad_ceil(a.f, BK) : ad_ceil(a.T, BK);  // each with all terms
    a.ktiles = a.terms * ad_ceil(all, std::max(1, std::min(splits, all / 4)));
    a.splits = ad_ceil(a.terms * all, a.ktiles);
}

template <int KIND>
void gt_sum(const GtArgs &a, hipStream_t s)
{
    const size_t n = (KIND == kGtDx ? (size_t)a.T : a.f) * a.m;
    if (a.splits > 1)
        k_gt_sum<KIND><<<dim3((unsigned)((n / 4 + 255) / 256), KIND == kGtDx ? 1 : 2), 256, 0, s>>>(a);
}

// workgroups of tiles of bm x bn (of both gradients of weights, as far as they are wanted), of all parts of k
template <int KIND>
int gt_grid(GtArgs &a, int M, int N, int bm, int bn)
{
    a.mt = ad_ceil(M, bm);
    a.nt = ad_ceil(N, bn);
    return ad_ceil(a.mt * a.nt * (KIND == kGtDw && a.out && a.out2 ? 2 : 1) * a.splits, 8) * 8;
}

template <int KIND, int BM, int BN, int BK, int WM, int WN, int WK, int STAGES>
void gt_product(GtArgs a, int M, int N, hipStream_t s, int splits = 1)
{
    gt_split<KIND>(a, BK, splits);
    const int grid = gt_grid<KIND>(a, M, N, BM, BN), block = WM * WN * WK * cdk::kWave;
    // Weights that this launch reads once and that would sweep most of the last-level cache go past it. (The
    // backward call's projections too, though dx reads them again.) dx of several terms reads them once a term, from
    // L2 but for the first, and keeps to the caches; fp32 gradients, captured us a call against going past them:
    // 64 tokens of 8192 x 28672 953 / 1095, of 4096 x 14336 283 / 302, 4 tokens of 4096 x 11008 191 / 201, one of
    // 4096 x 14336 244 / 237.
    constexpr bool weights = KIND != kGtDw && BM <= 64;
    if (weights && a.mt == 1 && (KIND != kGtDx || a.terms == 1) && (size_t)a.f * a.m * 4 > ((size_t)64 << 20))
        k_gt_product<KIND, BM, BN, BK, WM, WN, WK, STAGES, weights><<<grid, block, 0, s>>>(a);
    else
        k_gt_product<KIND, BM, BN, BK, WM, WN, WK, STAGES, false><<<grid, block, 0, s>>>(a);
    if constexpr (KIND == kGtDx || KIND == kGtDw)
        gt_sum<KIND>(a, s);
}

// whether rows begin inside a cache line
bool gt_inside(const uint16_t *p, size_t ld) { return (reinterpret_cast<uintptr_t>(p) | ld * 2) % 128 != 0; }

// Both projections by whole lines. Captured us a call against the same tiles as they lie: 333 tokens of 3000 x 8008
// 47.0 / 55.9, 200 of 2040 x 5504 23.7 / 29.2, 180 of 4088 x 14336 63.8 / 84.1, 32 of 4088 x 14336 44.0 / 52.8, 128 of
// 3000 x 8008 30.3 / 35.1, 40 of 2040 x 5504 14.8 / 16.5, 60 of 2000 x 3000 11.3 / 12.8, 17 of 1000 x 2056 6.6 / 6.5. Not for
// 16 tokens: 8 of 4088 x 14336 40.0 / 43.2, 4 of 1000 x 3000 5.7 / 5.2. The large tiles have no room for the stage
// more that this takes (8192 tokens of 4088 x 14336 1505 us, of 4096 x 14336 1294).
template <int KIND, int BM, int BN, int BK, int WM, int WN, int WK, int STAGES>
void gt_lines(GtArgs a, hipStream_t s)
{
    gt_split<KIND>(a, BK, 1);
    const int grid = gt_grid<KIND>(a, a.T, a.f, BM, BN);
    if (BM <= 64 && a.mt == 1 && (size_t)a.f * a.m * 4 > ((size_t)64 << 20))
        k_gt_product<KIND, BM, BN, BK, WM, WN, WK, STAGES, BM <= 64, true><<<grid, WM * WN * WK * cdk::kWave, 0, s>>>(a);
    else
        k_gt_product<KIND, BM, BN, BK, WM, WN, WK, STAGES, false, true><<<grid, WM * WN * WK * cdk::kWave, 0, s>>>(a);
}

template <int KIND, int MH>
void gt_large(GtArgs a, int M, int N, hipStream_t s, int splits = 1)
{
    gt_split<KIND>(a, 64, splits);
    const int grid = gt_grid<KIND>(a, M, N, 128 * MH, KIND == kGtForward || KIND == kGtBackward ? 128 : 256);
    k_gt_large<KIND, MH><<<grid, 512, 0, s>>>(a);
    if constexpr (KIND == kGtDx || KIND == kGtDw)
        gt_sum<KIND>(a, s);
}

// 256 x 256 against 128 x 256: rounds of workgroups over the CUs, of which the former's take half as long
// again (768 tokens of 4096 x 14336, 2 against 3 rounds, 171 us against 180; 512 tokens of 3000 x 8008, 1 against 1, 85
// against 68).
bool gt_wide(int64_t wide, int64_t narrow) { return 3 * ((wide + 255) / 256) <= 2 * ((narrow + 255) / 256); }

// g and u over T tokens, and what KIND makes of them: the smallest tile that makes one round of
// workgroups over the 256 CUs. Forward, captured us a call (tile: tokens x neurons, of both matrices):
//                                16x16  32x32  64x32  64x64  128x64  192x64  128x128  256x128
//   1 token,    4096 x 14336      41.7   44.9   46.0   42.6    47.5    54.9     57.8     78.6
//   64 tokens,  1024 x 2816        8.6    6.9    7.7    9.3    11.5    13.6     16.0     22.4
//   64 tokens,  3000 x 8008       49.5   34.1   26.6   35.4    42.0    43.7     65.8     70.5
//   128 tokens, 3000 x 8008       87.3   54.0   42.1   35.2    50.1    53.1     72.9     78.0
//   128 tokens, 4096 x 14336     167.1   95.5   90.3   72.7    58.7    63.1     73.7     81.9
//   333 tokens, 3000 x 8008      181    117     97.3   78.2    77.3    55.1     65.9     79.8
//   256 tokens, 4096 x 14336     303    165    140    117      89.2   102       74.1     86.1
//   512 tokens, 4096 x 14336     594    297    260    192     159     150      124       95.5
// (16 x 16 for up to 16 tokens always: what is read there counts; and 64 x 64 for up to 64: 32 tokens of
// 8192 x 28672, 448 tiles, 175 us against 193 of 128 x 128.)
template <int KIND>
void gt_projections(const GtArgs &a, hipStream_t s)
{
    const auto fits = [&](int bm, int bn) { return (int64_t)ad_ceil(a.T, bm) * ad_ceil(a.f, bn) <= 256; };
    const bool lines = gt_inside(a.x, a.ldx) || gt_inside(a.Wg, a.m);
    if (a.T <= 16)
        gt_product<KIND, 16, 16, 256, 1, 1, 4, 3>(a, a.T, a.f, s);
    else if (lines && fits(32, 32))
        gt_lines<KIND, 32, 32, 128, 1, 2, 2, 5>(a, s);
    else if (fits(32, 32))
        gt_product<KIND, 32, 32, 128, 1, 2, 2, 4>(a, a.T, a.f, s);
    else if (lines && fits(64, 32))
        gt_lines<KIND, 64, 32, 128, 2, 2, 1, 5>(a, s);
    else if (fits(64, 32))
        gt_product<KIND, 64, 32, 128, 2, 2, 1, 4>(a, a.T, a.f, s);
    else if (lines && (a.T <= 64 || fits(64, 64)))
        gt_lines<KIND, 64, 64, 64, 2, 4, 1, 6>(a, s);
    else if (a.T <= 64 || fits(64, 64))
        gt_product<KIND, 64, 64, 128, 2, 4, 1, 3>(a, a.T, a.f, s);
    else if (lines && fits(128, 64))
        gt_lines<KIND, 128, 64, 64, 2, 4, 1, 4>(a, s);
    else if (lines && fits(192, 64))
        gt_lines<KIND, 192, 64, 64, 4, 2, 1, 4>(a, s);
    else if (fits(128, 64))
        gt_product<KIND, 128, 64, 64, 2, 4, 1, 3>(a, a.T, a.f, s);
    else if (fits(192, 64))
        gt_product<KIND, 192, 64, 64, 4, 2, 1, 3>(a, a.T, a.f, s);
    else if (fits(128, 128) || !gt_wide((int64_t)ad_ceil(a.T, 256) * ad_ceil(a.f, 128),
                                        (int64_t)ad_ceil(a.T, 128) * ad_ceil(a.f, 128)))
        gt_large<KIND, 1>(a, a.T, a.f, s);
    else
        gt_large<KIND, 2>(a, a.T, a.f, s);
}

// Few tiles of 64 x 64 and many tokens: workgroups that share a tile and fill the CUs twice (their sums take
// at most 512 tiles of the place). Backward us a call, so against whole tiles in one launch with dx: 4392 tokens
// of 168 x 72 19.6 / 31.5, 8000 of 256 x 256 39.6 / 62.8, 3000 of 64 x 512 in fp32 36.9 / 61.0, but 1024 of 256 x 256
// 20.8 / 13.8.
int gt_dw_splits(const GtArgs &a)
{
    const int64_t tiles = (int64_t)ad_ceil(a.f, 64) * ad_ceil(a.m, 64) * 2;
    return tiles <= 128 && a.T * a.terms > 2048 ? (int)(512 / tiles) : 1;
}

// dx and the weights' gradients in one launch, while a tile of dx needs no more than 16 tiles of k and both
// make one or two rounds of workgroups. Captured us a call against launches of their own:
//    37 tokens, 256 x 688 13.7 / 16.6   300, 256 x 1024 17.6 / 20.0   1000, 256 x 2048 28.8 / 35.2
//   with 24 tiles of k: 90, 504 x 952 in fp32 34.1 / 25.8
bool gt_little(const GtArgs &a)
{
    return 2 * a.terms * ad_ceil(a.f, kGtBackK) <= 16 && (int64_t)ad_ceil(a.T, 64) * ad_ceil(a.m, 64) <= 512 &&
           (int64_t)ad_ceil(a.f, 64) * ad_ceil(a.m, 64) * 2 <= 512 && gt_dw_splits(a) == 1;
}

// dx: 64 x 128 tiles, shared by workgroups that fill the CUs twice, or 256 x 256, by what the two were
// measured to take: 0.74 and 1.55 us a tile of k of a round, 2 and 4 around it, and for parts 3 and a write and a
// read of each at 4 TB/s. (Backward us a call, the first against the second: 256 tokens of 1024 x 2816 41 against 52,
// 512 tokens of 4096 x 14336 448 against 386, 655 tokens of 1336 x 6976 in fp32 276 against 244.)
void gt_dx(const GtArgs &a, hipStream_t s)
{
    // workgroups that share a tile: one round over the CUs, and what the place for their sums holds
    const int most = (int)std::min<size_t>(64, kGtPartFloats / ((size_t)a.T * a.m));
    const auto time = [&](int bm, int bn, int slots, double tile, double around, int &splits) {
        const int64_t tiles = (int64_t)ad_ceil(a.T, bm) * ad_ceil(a.m, bn);
        GtArgs b = a;
        gt_split<kGtDx>(b, 64, (int)std::min<int64_t>(most, slots / tiles));
        splits = b.splits;
        const double sums = b.splits > 1 ? 3 + (double)b.splits * a.T * a.m * 8 / 4e6 : 0;
        return (double)((tiles * b.splits + slots - 1) / slots) * (b.ktiles * tile + around) + sums;
    };
    int narrow, wide;
    const double tn = time(64, 128, 512, 0.74, 2, narrow), tw = time(256, 256, 256, 1.55, 4, wide);
    if (tn <= tw)
        gt_product<kGtDx, 64, 128, 64, 2, 2, 1, 3>(a, a.T, a.m, s, narrow);
    else
        gt_large<kGtDx, 2>(a, a.T, a.m, s, wide);
}

// The weights' gradients. Past 512 tiles of 64 x 64: 128 x 128, two workgroups a CU, for few tokens (which
// leave writing to be done: 256 tokens of 4096 x 11008, backward 225 us against 229) and where their rounds
// are shorter than those of 256 x 256, which take 200 where they take 113 (4096 tokens of 2048 x 5504 504
// against 521; of 4096 x 11008 1811 against 1726).
void gt_dw(const GtArgs &a, hipStream_t s)
{
    const auto tiles = [&](int b) { return (int64_t)ad_ceil(a.f, b) * ad_ceil(a.m, b) * 2; };  // of both gradients
    if (tiles(64) <= 512)
        gt_product<kGtDw, 64, 64, 64, 2, 2, 1, 3>(a, a.f, a.m, s, gt_dw_splits(a));
    else if (a.T * a.terms <= 256 || 113 * ((tiles(128) + 511) / 512) <= 200 * ((tiles(256) + 255) / 256))
        gt_product<kGtDw, 128, 128, 64, 2, 2, 1, 2>(a, a.f, a.m, s);
    else
        gt_large<kGtDw, 2>(a, a.f, a.m, s);
}

// what the two calls share; in: the operands that are read, out: those that are written
cd_status gt_check(const cd_gated *p, const AdRows *in, int nin, const AdRows *out, int nout)
{
    for (int i = 0; i < nout; ++i) {
        for (int j = 0; j < nin; ++j)
            if (ad_overlap(out[i], in[j]))
                return CD_EINVAL;
        for (int j = 0; j < i; ++j)
            if (ad_overlap(out[i], out[j]))
                return CD_EINVAL;
    }
    int dev = -1;
    if (hip_status(hipGetDevice(&dev)) != CD_OK)
        return CD_EHIP;
    return dev == p->device ? CD_OK : CD_EINVAL;
}

}  // namespace

extern "C" {

cd_status countdown_gated_create(int d_model, int d_ff, int max_tokens, unsigned flags, cd_gated **out)
{
    if (!out || d_model < 8 || d_model % 8 || d_ff < 8 || d_ff % 8 || max_tokens < 1 ||
        (flags & ~(CD_GATED_TRAIN | CD_GATED_FP32_GRADS)) ||
        ((flags & CD_GATED_FP32_GRADS) && !(flags & CD_GATED_TRAIN)))
        return CD_EINVAL;
    if (d_model > kGtMaxDim || d_ff > kGtMaxDim || max_tokens > kGtMaxTokens)
        return CD_EUNSUPPORTED;
    int dev = -1;
    if (hip_status(hipGetDevice(&dev)) != CD_OK)
        return CD_EHIP;
    cd_gated *p = new (std::nothrow) cd_gated{};
    if (!p)
        return CD_ENOMEM;
    p->m = d_model;
    p->f = d_ff;
    p->max_tokens = max_tokens;
    p->flags = flags;
    p->device = dev;
    if (flags & CD_GATED_TRAIN) {
        // two terms: T d_ff <= kGtFew, and rounding up to 64 makes at most eight times as much of it
        const size_t one = (size_t)max_tokens * 2 * gt_fd(d_ff) * sizeof(uint16_t);
        const size_t planes = flags & CD_GATED_FP32_GRADS ? kGtTerms * one : one + 8 * kGtFew * 2 * sizeof(uint16_t);
        if (hip_status(hipMalloc(&p->ws, planes + kGtPartFloats * sizeof(float))) != CD_OK) {
            delete p;
            return CD_ENOMEM;
        }
        p->d = static_cast<uint16_t *>(p->ws);
        p->part = reinterpret_cast<float *>(static_cast<char *>(p->ws) + planes);
    }
    *out = p;
    return CD_OK;
}

cd_status countdown_gated_destroy(cd_gated *p)
{
    if (!p)
        return CD_OK;
    int dev = -1;
    cd_status st = hip_status(hipGetDevice(&dev));
    if (st == CD_OK)
        st = hip_status(hipSetDevice(p->device));
    if (st == CD_OK)
        st = hip_status(hipDeviceSynchronize());
    if (p->ws && hip_status(hipFree(p->ws)) != CD_OK)
        st = CD_EHIP;
    if (dev >= 0)
        (void)hip_status(hipSetDevice(dev));
    delete p;
    return st;
}

cd_status countdown_gated_forward(cd_gated *p, const uint16_t *x, size_t ldx, int T,
                                  const uint16_t *W_gate, const uint16_t *W_up, int type, void *h,
                                  size_t ldh, void *stream)
{
    if (!p || T < 0 || T > p->max_tokens || (type != CD_TYPE_F32 && type != CD_TYPE_BF16) ||
        !W_gate || !aligned16(W_gate) || !W_up || !aligned16(W_up))
        return CD_EINVAL;
    if (T > 0 && (!x || !aligned16(x) || !ad_ld_ok(ldx, p->m) || !h || !aligned16(h) || !ad_ld_ok(ldh, p->f)))
        return CD_EINVAL;
    const size_t es = ad_size(type), w = (size_t)p->f * p->m * 2;
    const AdRows in[] = {{x, (size_t)p->m * 2, ldx * 2, T}, ad_flat(W_gate, w), ad_flat(W_up, w)};
    const AdRows out[] = {{h, p->f * es, ldh * es, T}};
    const cd_status st = gt_check(p, in, 3, out, 1);
    if (st != CD_OK)
        return st;
    if (T > 0 && ldx > kGtMaxStride)
        return CD_EUNSUPPORTED;
    if (T == 0)
        return CD_OK;
    GtArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.Wg = W_gate;
    a.Wu = W_up;
    a.T = T;
    a.m = p->m;
    a.f = p->f;
    a.type = type;
    a.out = h;
    a.ldo = ldh;
    gt_projections<kGtForward>(a, reinterpret_cast<hipStream_t>(stream));
    return launched(hipGetLastError());
}

cd_status countdown_gated_backward(cd_gated *p, const uint16_t *x, size_t ldx, const uint16_t *dh,
                                   size_t lddh, int T, const uint16_t *W_gate, const uint16_t *W_up,
                                   int type, void *dx, size_t lddx, void *dW_gate, void *dW_up,
                                   void *stream)
{
    if (!p || !(p->flags & CD_GATED_TRAIN) || T < 0 || T > p->max_tokens ||
        (type != CD_TYPE_F32 && type != CD_TYPE_BF16) ||
        (type == CD_TYPE_F32 && !(p->flags & CD_GATED_FP32_GRADS)) ||
        !W_gate || !aligned16(W_gate) || !W_up || !aligned16(W_up) || !aligned16(dW_gate) || !aligned16(dW_up))
        return CD_EINVAL;
    if (T > 0 && (!x || !aligned16(x) || !ad_ld_ok(ldx, p->m) || !dh || !aligned16(dh) || !ad_ld_ok(lddh, p->f) ||
                  (dx && (!aligned16(dx) || !ad_ld_ok(lddx, p->m)))))
        return CD_EINVAL;
    const size_t es = ad_size(type), w = (size_t)p->f * p->m;
    const AdRows in[] = {{x, (size_t)p->m * 2, ldx * 2, T}, {dh, (size_t)p->f * 2, lddh * 2, T},
                         ad_flat(W_gate, w * 2), ad_flat(W_up, w * 2)};
    const AdRows out[] = {{dx, p->m * es, lddx * es, T}, ad_flat(dW_gate, w * es), ad_flat(dW_up, w * es)};
    const cd_status st = gt_check(p, in, 4, out, 3);
    if (st != CD_OK)
        return st;
    if (T > 0 && (ldx > kGtMaxStride || lddh > kGtMaxStride))
        return CD_EUNSUPPORTED;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (T == 0) {
        for (void *g : {dW_gate, dW_up})
            if (g)
                k_gt_zero<<<1024, 256, 0, s>>>(static_cast<uint32_t *>(g), w * es / 4);
        return launched(hipGetLastError());
    }
    if (!dx && !dW_gate && !dW_up)
        return CD_OK;
    GtArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.Wg = W_gate;
    a.Wu = W_up;
    a.dh = dh;
    a.lddh = lddh;
    a.T = T;
    a.m = p->m;
    a.f = p->f;
    a.type = type;
    a.d = p->d;
    a.fd = gt_fd(p->f);
    a.part = p->part;
    // One bf16 term is the operand of a bf16 product: a gradient's 2-norm error is then 1.41 times that of its own
    // rounding, over many independent roundings (2.3e-3 against 1.7e-3). Over few it may by chance be 1.5 times
    // (one token, 64 neurons), and a second term takes the first rounding out. The border is one of cost, 3 us
    // (of 16: 37 tokens, 256 x 688) to 35 (of 145: one token, 4096 x 11008) and twice the products of dx and of the weights'
    // gradients, and of whole outputs, not of rows: on either side, what one token adds to a row of dW has one
    // rounding, beyond the border by up to 2^-8. Who needs more takes fp32 gradients.
    a.terms = type == CD_TYPE_F32 ? kGtTerms : (int64_t)T * a.f <= kGtFew ? 2 : 1;
    gt_projections<kGtBackward>(a, s);
    GtArgs ax = a, aw = a;
    ax.out = dx;
    ax.ldo = lddx;
    aw.out = dW_gate;
    aw.out2 = dW_up;
    aw.ldo = a.m;
    if (gt_little(a)) {
        ax.splits = aw.splits = 1;
        ax.ktiles = 2 * a.terms * ad_ceil(a.f, kGtBackK);
        aw.ktiles = a.terms * ad_ceil(a.T, 64);
        const int nx = dx ? gt_grid<kGtDx>(ax, a.T, a.m, 64, 64) : 0;
        const int nw = dW_gate || dW_up ? gt_grid<kGtDw>(aw, a.f, a.m, 64, 64) : 0;
        k_gt_back<<<nx + nw, 512, 0, s>>>(ax, aw, nx);
    } else {
        if (dx)
            gt_dx(ax, s);
        if (dW_gate || dW_up)
            gt_dw(aw, s);
    }
    return launched(hipGetLastError());
}

}  // extern "C"
