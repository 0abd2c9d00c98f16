// Low-rank adapters of many requests beside a shared projection. Part of cd_api.hip (its
// only includer).
//
//   lat_t = A_a x_t,  y_t = base_t + scale_a B_a lat_t,  a = ids[t]
//   glat_t = scale_a B_a^T dy_t,  dx_t = base_t + A_a^T glat_t
//   dA_a = sum_t glat_t x_t^T,  dB_a = sum_t dy_t (scale_a lat_t)^T
#pragma once

#include "cd_device.hpp"

namespace {

constexpr int kAdMaxDim = 65536, kAdMaxRank = 256, kAdMaxAdapters = 1024;
constexpr int kAdMaxTokens = 1 << 20;
constexpr int kAdDecodeTokens = 16;  // tokens of countdown_adapters_project
constexpr int kAdBlock = 256, kAdWaves = kAdBlock / cdk::kWave;
constexpr size_t kAdPartFloats = (size_t)128 * 1024 * 32;  // place for workgroups' sums (16 MiB)
constexpr int kAdPad = 32;  // tokens of one adapter are padded to the contraction of an MFMA

using cdk::f32x4_t;
using cdk::load16;
using cdk::mfma16;
using cdk::or_zero;
using cdk::u32x4;

// The tokens in the order of their adapters. Adapter a's tokens sit at padded positions
// [first, first + count), first a multiple of kAdPad; those without an adapter are group n.
struct AdGroup {
    int first, count;
};
// A tile of tokens of one group (count 0: an unused slot), or all of them.
struct AdTile {
    int group, first, count, pad;
};

struct AdArgs {
    const uint16_t *x;  // [T][d_in], row stride ldx
    size_t ldx;
    const uint16_t *dy;  // [T][d_out], row stride lddy
    size_t lddy;
    const uint16_t *W;  // [d_out][d_in]
    const int32_t *ids;
    const uint16_t *A;  // [n][rank][d_in]
    const uint16_t *B;  // [n][d_out][rank]
    const float *scale;
    const void *base;
    size_t ldb;
    void *out;  // y or dx
    size_t ldo;
    int type;  // of base and out
    float *dA, *dB;
    int T, n, d_in, d_out, rank;
    // workspace. lat and glat hold scale_a lat_t and glat_t, by token (decode) or position
    float *lat, *glat;
    int *order;       // token at each position
    AdGroup *groups;  // [n + 1]
    AdTile *tiles;
    AdTile *by_size;  // all tokens of each adapter, those with most of them first (training)
    uint16_t *Bt;            // [n][rank][d_out], B transposed (training)
    uint16_t *latT, *glatT;  // lat and glat split in three bf16 terms (ad_term_at; training)
    int tile;    // tokens of a tile: 16 or 32
    float *part; // sums of workgroups that share a gradient's tokens (training)
};

// the wave's number, known to be uniform
__device__ __forceinline__ int ad_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / cdk::kWave); }

__device__ __forceinline__ bool ad_valid(const AdArgs &a, int id) { return (unsigned)id < (unsigned)a.n; }
__device__ __forceinline__ float ad_scale(const AdArgs &a, int id) { return a.scale ? a.scale[id] : 1.0f; }

__device__ __forceinline__ uint32_t ad_pack(float lo, float hi)
{
    return __builtin_bit_cast(uint16_t, (__bf16)lo) |
           (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16;
}

// v = t[0] + t[1] + t[2], each with 8 significant bits cut from what is left: exact, so an
// fp32 factor of a bf16 matrix product costs three products instead of any rounding
__device__ __forceinline__ void ad_split(float v, uint32_t (&t)[3])
{
    t[0] = __float_as_uint(v) & 0xffff0000u;
    float r = fabsf(v) < INFINITY ? v - __uint_as_float(t[0]) : 0.0f;  // infinity and NaN: t[0] alone
    t[1] = __float_as_uint(r) & 0xffff0000u;
    r -= __uint_as_float(t[1]);
    t[2] = __float_as_uint(r) & 0xffff0000u;
}

// the terms of 8 values as MFMA operands
__device__ __forceinline__ void ad_split8(const f32x4_t (&v)[2], u32x4 (&t)[3])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t lo[3], hi[3];
        ad_split(v[i / 2][i % 2 * 2], lo);
        ad_split(v[i / 2][i % 2 * 2 + 1], hi);
#pragma unroll
        for (int k = 0; k < 3; ++k)
            t[k][i] = lo[k] >> 16 | hi[k];
    }
}

// Columns of an 8 x 8 block of bf16 whose rows are r[0..7]: c[j] = column j. It turns 16-byte
// loads along one dimension into MFMA operands that contract over the other.
__device__ __forceinline__ void ad_transpose8(const u32x4 (&r)[8], u32x4 (&c)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c[j][i] = __builtin_amdgcn_perm(r[2 * i + 1][j / 2], r[2 * i][j / 2],
                                            j % 2 ? 0x07060302u : 0x05040100u);
}

// The vector memory unit merges four neighbouring lanes: a load in operand layout, 16 rows on
// 16 neighbouring lanes, takes it 64 cycles a KB (38 GB/s a CU, with two operands less than a
// CU's share of HBM), one whose lanes follow a row 16. So 16 rows x 128 columns come in four
// loads of 4 rows x 256 bytes (lane: row 4 i + lane / 16, columns 8 (lane % 16)) and turn
// into the four operands of those columns in 4 KB of LDS that the wave has to itself. The
// 16-byte chunks of a row are stored in an order of its own (xor), which spreads 16 rows
// over the banks.
constexpr int kAdStage = 256;  // 16-byte chunks

__device__ __forceinline__ void ad_wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ void ad_stage(u32x4 (&v)[4], u32x4 *lds, int lane)
{
    const int m = lane % 16, g = lane / 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        lds[(4 * i + g) * 16 + (m ^ (4 * i + g))] = v[i];
    ad_wave_sync();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = lds[m * 16 + ((4 * i + g) ^ m)];
    ad_wave_sync();
}

// base[t][col, col + 8) as it lies (bf16: in r[0] alone); zeros without a base
__device__ __forceinline__ void ad_base8(const AdArgs &a, bool ok, size_t t, int col, u32x4 (&r)[2])
{
    ok = ok && a.base;
    if (a.type == CD_TYPE_F32) {
        const float *b = static_cast<const float *>(a.base) + t * a.ldb + col;
        r[0] = *reinterpret_cast<const u32x4 *>(or_zero(ok, b));
        r[1] = *reinterpret_cast<const u32x4 *>(or_zero(ok, b + 4));
    } else {
        r[0] = load16(or_zero(ok, static_cast<const uint16_t *>(a.base) + t * a.ldb + col));
    }
}

// out[t][col, col + 8) = base + v (no: the token has no adapter, the base's bits)
__device__ __forceinline__ void ad_store8(const AdArgs &a, size_t t, int col, const u32x4 (&b)[2],
                                          const float (&v)[8], bool no)
{
    u32x4 w[2];
    if (a.type == CD_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i / 4][i % 4] = no ? b[i / 4][i % 4] : __float_as_uint(__uint_as_float(b[i / 4][i % 4]) + v[i]);
        u32x4 *o = reinterpret_cast<u32x4 *>(static_cast<float *>(a.out) + t * a.ldo + col);
        o[0] = w[0];
        o[1] = w[1];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[0][i] = no ? b[0][i] : ad_pack(cdk::bf16_lo(b[0][i]) + v[2 * i], cdk::bf16_hi(b[0][i]) + v[2 * i + 1]);
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.out) + t * a.ldo + col) = w[0];
    }
}

// --------------------------------------------------------- few tokens: one by one

// scale A x of rank k, over a wave
__device__ __forceinline__ float ad_latent(const AdArgs &a, int t, int id, int k)
{
    const uint16_t *p = a.x + (size_t)t * a.ldx, *q = a.A + ((size_t)id * a.rank + k) * a.d_in;
    float s = 0.0f;
#pragma unroll 4
    for (int i = threadIdx.x % cdk::kWave * 8; i < a.d_in; i += cdk::kColsPerLoad)
        s = cdk::dot8(load16(p + i), load16(q + i), s);
    return cdk::wave_sum(s) * ad_scale(a, id);
}

template <bool NT>
__device__ __forceinline__ u32x4 ad_load16(const uint16_t *p)
{
    const u32x4 *q = reinterpret_cast<const u32x4 *>(p);
    return NT ? __builtin_nontemporal_load(q) : *q;
}

// sum over the rank of lat[k] B[a][o][k]
__device__ __forceinline__ float ad_row(const AdArgs &a, int id, int o, const float *lat)
{
    const uint16_t *b = a.B + ((size_t)id * a.d_out + o) * a.rank;
    float s = 0.0f;
#pragma unroll 2
    for (int k = 0; k < a.rank; k += 8) {
        const u32x4 v = load16(b + k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s += lat[k + 2 * i] * cdk::bf16_lo(v[i]) + lat[k + 2 * i + 1] * cdk::bf16_hi(v[i]);
    }
    return s;
}

// out[t][o] = base + v (no: the token has no adapter, the base's bits)
__device__ __forceinline__ void ad_store1(const AdArgs &a, int t, int o, float v, bool no)
{
    const size_t i = (size_t)t * a.ldb + o;
    if (a.type == CD_TYPE_F32) {
        const float *b = static_cast<const float *>(a.base);
        static_cast<float *>(a.out)[(size_t)t * a.ldo + o] = b ? (no ? b[i] : b[i] + v) : v;
    } else {
        const uint16_t *b = static_cast<const uint16_t *>(a.base);
        const uint16_t w = (uint16_t)ad_pack(b ? v + cdk::bf16_lo(b[i]) : v, 0.0f);
        static_cast<uint16_t *>(a.out)[(size_t)t * a.ldo + o] = b && no ? b[i] : w;
    }
}

// lat[t][k]: one wave per (t, k)
__global__ __launch_bounds__(kAdBlock) void k_ad_lat(const AdArgs a)
{
    const int w = blockIdx.x * kAdWaves + ad_wave();
    const int t = w / a.rank, k = w % a.rank;
    if (t >= a.T)
        return;
    const int id = a.ids[t];
    if (!ad_valid(a, id))
        return;
    const float s = ad_latent(a, t, id, k);
    if (threadIdx.x % cdk::kWave == 0)
        a.lat[w] = s;
}

// y = base + B lat: one lane per output, blockIdx.x the token
__global__ __launch_bounds__(kAdBlock) void k_ad_up(const AdArgs a)
{
    const int t = blockIdx.x, o = blockIdx.y * kAdBlock + threadIdx.x, id = a.ids[t];
    if (o >= a.d_out)
        return;
    const bool no = !ad_valid(a, id);
    ad_store1(a, t, o, no ? 0.0f : ad_row(a, id, o, a.lat + t * a.rank), no);
}

// Both in one launch: every workgroup forms its token's latent again, one rank a wave at a
// time, for 1024 outputs. A launch costs the caller's thread 2.9 us and the GPU 1 to 2.
constexpr int kAdTokenBlock = 1024;

__global__ __launch_bounds__(kAdTokenBlock) void k_ad_token(const AdArgs a)
{
    __shared__ float lat[kAdMaxRank];
    const int t = blockIdx.x, o = blockIdx.y * kAdTokenBlock + threadIdx.x, id = a.ids[t];
    const bool no = !ad_valid(a, id);  // uniform
    if (!no) {
        for (int k = ad_wave(); k < a.rank; k += kAdTokenBlock / cdk::kWave) {
            const float s = ad_latent(a, t, id, k);
            if (threadIdx.x % cdk::kWave == 0)
                lat[k] = s;
        }
        __syncthreads();
    }
    if (o < a.d_out)
        ad_store1(a, t, o, no ? 0.0f : ad_row(a, id, o, lat), no);
}

// The backward call on few tokens, without grouping: a workgroup per token forms lat
// (blockIdx.y + kind 0) and glat (1), the next launch everything else.
constexpr int kAdFewTokens = 16, kAdFewRanks = 32;

__global__ __launch_bounds__(kAdTokenBlock) void k_ad_few_latents(const AdArgs a, int kind)
{
    __shared__ float sums[kAdTokenBlock / cdk::kWave][kAdFewRanks];
    const int t = blockIdx.x, id = a.ids[t], wave = ad_wave(), lane = threadIdx.x % cdk::kWave;
    if (!ad_valid(a, id))
        return;
    if (blockIdx.y + kind == 0) {
        for (int k = wave; k < a.rank; k += kAdTokenBlock / cdk::kWave) {
            const float s = ad_latent(a, t, id, k);
            if (lane == 0)
                a.lat[t * a.rank + k] = s;
        }
        return;
    }
    const uint16_t *B = a.B + (size_t)id * a.d_out * a.rank, *dy = a.dy + (size_t)t * a.lddy;
    float acc[kAdFewRanks];
#pragma unroll
    for (int k = 0; k < kAdFewRanks; ++k)
        acc[k] = 0.0f;
#pragma unroll 2
    for (int o = threadIdx.x; o < a.d_out; o += kAdTokenBlock) {
        const float d = cdk::bf16_lo(dy[o]);
#pragma unroll
        for (int c = 0; c < kAdFewRanks / 8; ++c) {
            const u32x4 b = load16(or_zero(8 * c < a.rank, B + (size_t)o * a.rank + 8 * c));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[8 * c + 2 * e] += d * cdk::bf16_lo(b[e]);
                acc[8 * c + 2 * e + 1] += d * cdk::bf16_hi(b[e]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kAdFewRanks; ++k) {
        const float s = cdk::wave_sum(acc[k]);
        if (lane == 0)
            sums[wave][k] = s;
    }
    __syncthreads();
    if ((int)threadIdx.x < a.rank) {
        float s = 0.0f;
        for (int w = 0; w < kAdTokenBlock / cdk::kWave; ++w)
            s += sums[w][threadIdx.x];
        a.glat[t * a.rank + threadIdx.x] = s * ad_scale(a, id);
    }
}

// += f times the 8 bf16 of v
__device__ __forceinline__ void ad_axpy8(float f, const u32x4 &v, float (&acc)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        acc[2 * e] += f * cdk::bf16_lo(v[e]);
        acc[2 * e + 1] += f * cdk::bf16_hi(v[e]);
    }
}

// Workgroups [0, nB) dB, the next nA dA, the others dx; a lane has 8 elements of a row.
__global__ __launch_bounds__(kAdBlock) void k_ad_few_back(const AdArgs a, int nB, int nA)
{
    float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    const int b = blockIdx.x;
    if (b < nB + nA) {  // uniform: one adapter, whose tokens are added in their order
        const bool second = b < nB;
        const int per = (second ? nB : nA) / a.n, i = second ? b : b - nB;
        const int ad = i / per, width = second ? a.d_out * (a.rank / 8) : a.rank * (a.d_in / 8);
        const int at = i % per * kAdBlock + threadIdx.x, lane = threadIdx.x % cdk::kWave;
        static_assert(kAdFewTokens <= cdk::kWave, "a lane for each token");
        const uint64_t mine = cdk::ballot(lane < a.T && a.ids[min(lane, a.T - 1)] == ad);
        if (at >= width)
            return;
        const int row = second ? at / (a.rank / 8) : at / (a.d_in / 8);  // output o, or rank k
        const int col = (second ? at % (a.rank / 8) : at % (a.d_in / 8)) * 8;
        for (uint64_t left = mine; left;) {  // four tokens' loads in flight
            float f[4];
            u32x4 v[4];
            float l[4][8];
            int m = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool ok = left != 0;
                const int t = ok ? __builtin_ctzll(left) : 0;
                left &= left - 1;
                m += ok;
                if (second) {
                    f[q] = cdk::bf16_lo(*or_zero(ok, a.dy + (size_t)t * a.lddy + row));
                    const float *p = a.lat + t * a.rank + col;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        l[q][e] = ok ? p[e] : 0.0f;
                } else {
                    f[q] = *or_zero(ok, a.glat + t * a.rank + row);
                    v[q] = load16(or_zero(ok, a.x + (size_t)t * a.ldx + col));
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (q < m) {
                    if (second)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            acc[e] += f[q] * l[q][e];
                    else
                        ad_axpy8(f[q], v[q], acc);
                }
        }
        float *dst = second ? a.dB + ((size_t)ad * a.d_out + row) * a.rank + col
                            : a.dA + ((size_t)ad * a.rank + row) * a.d_in + col;
        reinterpret_cast<f32x4_t *>(dst)[0] = f32x4_t{acc[0], acc[1], acc[2], acc[3]};
        reinterpret_cast<f32x4_t *>(dst)[1] = f32x4_t{acc[4], acc[5], acc[6], acc[7]};
        return;
    }
    const int per = (a.d_in / 8 + kAdBlock - 1) / kAdBlock, i = b - nB - nA;
    const int t = i / per, col = (i % per * kAdBlock + threadIdx.x) * 8, id = a.ids[t];
    if (col >= a.d_in)
        return;
    const bool no = !ad_valid(a, id);
    u32x4 base[2];
    ad_base8(a, true, t, col, base);
    if (!no) {
        const uint16_t *A = a.A + (size_t)id * a.rank * a.d_in + col;
#pragma unroll 4
        for (int k = 0; k < a.rank; ++k)
            ad_axpy8(a.glat[t * a.rank + k], load16(A + (size_t)k * a.d_in), acc);
    }
    ad_store8(a, t, col, base, acc, no);
}

// y = W x + B lat for up to 16 tokens: a workgroup's eight waves each take an eighth of the
// columns of 16 rows of W (128 at a time, the next 128 in flight), the tokens are the other
// operand; the waves' sums meet in LDS, where the adapters' part is added. Rows past the
// last and tokens past T repeat the last one: they only reach sums of their own.
constexpr int kAdProjBlock = 512, kAdProjWaves = kAdProjBlock / cdk::kWave;
constexpr int kAdOwnLatents = 32;

// OWN: every workgroup forms the latents again, while its first columns of W are on their way.
// NT: W past the caches.
template <bool OWN, bool NT>
__global__ __launch_bounds__(kAdProjBlock) void k_ad_project(const AdArgs a)
{
    __shared__ u32x4 lds[kAdProjWaves][kAdStage];
    __shared__ float own[OWN ? kAdOwnLatents : 1];
    const int lane = threadIdx.x % cdk::kWave, wave = ad_wave();
    const int m = lane % 16, g = lane / 16;
    const int o0 = blockIdx.x * 16;
    const uint16_t *w[4], *x[4];  // this lane's rows
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = a.W + (size_t)min(o0 + 4 * i + g, a.d_out - 1) * a.d_in;
        x[i] = a.x + min(4 * i + g, a.T - 1) * a.ldx;
    }
    // this wave's columns
    const int per = (a.d_in + 128 * kAdProjWaves - 1) / (128 * kAdProjWaves) * 128;
    const int k0 = wave * per, kend = min(a.d_in, k0 + per);
    u32x4 wv[2][4], xv[2][4];
    const auto load = [&](int s, int k) {
        k += 8 * m;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            wv[s][i] = ad_load16<NT>(or_zero(k < a.d_in, w[i] + k));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i == 0 || 4 * i < a.T)
                xv[s][i] = load16(or_zero(k < a.d_in, x[i] + k));
    };
    f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (k0 < kend)
        load(0, k0);
    if constexpr (OWN)
        for (int p = wave; p < a.T * a.rank; p += kAdProjWaves) {
            const int t = p / a.rank, id = a.ids[t];
            const float s = ad_valid(a, id) ? ad_latent(a, t, id, p % a.rank) : 0.0f;
            if (lane == 0)
                own[p] = s;
        }
#pragma unroll 1
    for (int kb = k0; kb < kend; kb += 256) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = kb + s * 128;
            if (k >= kend)
                break;
            if (k + 128 < kend)
                load(1 - s, k + 128);
            ad_stage(wv[s], lds[wave], lane);
            ad_stage(xv[s], lds[wave], lane);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                acc = mfma16(wv[s][u], xv[s][u], acc);
        }
    }
    f32x4_t *sums = reinterpret_cast<f32x4_t *>(&lds[0][0]);
    __syncthreads();
    sums[threadIdx.x] = acc;
    __syncthreads();
    if (threadIdx.x >= 256)
        return;
    const int t = threadIdx.x / 16, r = threadIdx.x % 16, o = o0 + r;  // one output each
    if (t >= a.T || o >= a.d_out)
        return;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < kAdProjWaves; ++i)
        v += sums[i * cdk::kWave + r / 4 * 16 + t][r % 4];
    const int id = a.ids[t];
    if (ad_valid(a, id))
        v += ad_row(a, id, o, (OWN ? own : a.lat) + t * a.rank);
    ad_store1(a, t, o, v, false);
}

// ------------------------------------------------- many tokens: grouped by their adapters

constexpr int kAdSortBlock = 1024, kAdSortWaves = kAdSortBlock / cdk::kWave;

// Workgroup g <= n finds the tokens of group g, in their order, by reading all ids: no
// atomics, no order that depends on timing. Every group's places follow from the number b
// of tokens in lower groups alone: with first = roundup(b) + pad g the next group's first
// is at least first + roundup(count), and with slot b / tile + g its tiles fit as well.
// Workgroups past n transpose B for the backward call.
__global__ __launch_bounds__(kAdSortBlock) void k_ad_group(const AdArgs a)
{
    if ((int)blockIdx.x > a.n) {
        // 128 outputs x 64 ranks, 8 ranks or 8 outputs a thread
        __shared__ uint16_t tile[128][66];
        const int ct = (a.d_out + 127) / 128, rt = (a.rank + 63) / 64;
        const int i = blockIdx.x - a.n - 1;
        const int c0 = i % ct * 128, r0 = i / ct % rt * 64, ad = i / ct / rt;
        const uint16_t *src = a.B + (size_t)ad * a.d_out * a.rank;
        uint16_t *dst = a.Bt + (size_t)ad * a.d_out * a.rank;
        {
            const int o = threadIdx.x / 8, k = threadIdx.x % 8 * 8;
            if (c0 + o < a.d_out && r0 + k < a.rank) {
                const u32x4 v = load16(src + (size_t)(c0 + o) * a.rank + r0 + k);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<uint32_t *>(&tile[o][k + 2 * e]) = v[e];
            }
        }
        __syncthreads();
        const int o = threadIdx.x % 16 * 8, k = threadIdx.x / 16;
        if (c0 + o < a.d_out && r0 + k < a.rank) {
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = tile[o + 2 * e][k] | (uint32_t)tile[o + 2 * e + 1][k] << 16;
            *reinterpret_cast<u32x4 *>(dst + (size_t)(r0 + k) * a.d_out + c0 + o) = v;
        }
        return;
    }
    // A wave counts a run of tokens, 64 at a time, then writes its group's behind those of the
    // waves before it. All ids pass one CU's SIMDs, so instructions an id bound it: 65536
    // tokens 11.3 us, 16384 4.6 (with a check of each lane against the run's end, the id's range
    // in two steps and the comparison made again for the writing 33 and 9.2).
    __shared__ int wl[kAdSortWaves], wm[kAdSortWaves];
    const int grp = blockIdx.x;
    const int lane = threadIdx.x % cdk::kWave, wave = ad_wave();
    const int per = (a.T + kAdSortBlock - 1) / kAdSortBlock * cdk::kWave;
    const int t0 = min(a.T, wave * per), t1 = min(a.T, t0 + per);
    constexpr int kDeep = 16;  // loads in flight
    uint64_t hit[kDeep];       // the group's tokens
    int less = 0, mine = 0;
    const auto count = [&](int t) {
        unsigned of[kDeep];  // (past the run: no group)
        if (t + kDeep * cdk::kWave <= t1) {
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
                of[u] = min((unsigned)a.ids[t + u * cdk::kWave + lane], (unsigned)a.n);
        } else {
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const int i = t + u * cdk::kWave + lane;
                of[u] = min((unsigned)a.ids[min(i, a.T - 1)], (unsigned)a.n);
                of[u] = i < t1 ? of[u] : a.n + 1;
            }
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            hit[u] = cdk::ballot(of[u] == (unsigned)grp);
            less += __popcll(cdk::ballot(of[u] < (unsigned)grp));
            mine += __popcll(hit[u]);
        }
    };
    for (int t = t0; t < t1; t += kDeep * cdk::kWave)
        count(t);
    if (lane == 0) {
        wl[wave] = less;
        wm[wave] = mine;
    }
    __syncthreads();
    int before = 0;
    less = mine = 0;
#pragma unroll
    for (int i = 0; i < kAdSortWaves; ++i) {
        less += wl[i];
        before += i < wave ? wm[i] : 0;
        mine += wm[i];  // the group's count
    }
    const int lower = less, all = mine;
    const int first = (lower + kAdPad - 1) / kAdPad * kAdPad + kAdPad * grp;
    int at = first + before;
    for (int t = t0; t < t1; t += kDeep * cdk::kWave) {
        if (per > kDeep * cdk::kWave)  // (a single batch is still there)
            count(t);
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
            if (hit[u]) {
                if (hit[u] >> lane & 1)
                    a.order[at + cdk::lanes_below(hit[u])] = t + u * cdk::kWave + lane;
                at += __popcll(hit[u]);
            }
    }
    if (threadIdx.x == 0)
        a.groups[grp] = AdGroup{first, all};
    const int slot0 = lower / a.tile + grp, slot1 = (lower + all) / a.tile + grp + 1;
    for (int s = slot0 + threadIdx.x; s < slot1; s += kAdSortBlock) {
        const int off = (s - slot0) * a.tile;
        a.tiles[s] = AdTile{grp, first + off, max(0, min(a.tile, all - off)), 0};
    }
}

// Where the terms of lat lie for the gradients: the operands of 32 positions and 16 ranks
// (lane: rank r % 16, positions 8 (lane / 16) and on) are one run of 1 KB.
__device__ __forceinline__ size_t ad_term_at(const AdArgs &a, size_t p, int s, int r)
{
    const int rts = (a.rank + 15) / 16;
    return ((p / 32 * 3 + s) * rts + r / 16) * 512 + ((p % 32 / 8) * 16 + r % 16) * 8 + p % 8;
}

// a.by_size for 64 adapters, a lane each: its place is the number of adapters that come before
// it, of which every wave counts a part.
template <int WAVES>
__device__ __forceinline__ void ad_by_size(const AdArgs &a, int block, int *before)
{
    const int lane = threadIdx.x % cdk::kWave, wave = ad_wave();
    const int i = block * cdk::kWave + lane;
    const AdGroup mine = a.groups[min(i, a.n - 1)];
    int place = 0;
#pragma unroll 8
    for (int j = wave; j < a.n; j += WAVES) {
        const int other = a.groups[j].count;
        place += other > mine.count || (other == mine.count && j < i);
    }
    before[threadIdx.x] = place;
    __syncthreads();
    if (wave || i >= a.n)
        return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
        place += before[w * cdk::kWave + lane];
    a.by_size[place] = AdTile{i, mine.first, mine.count, 0};
}

// The low-rank latents of a tile (MT * 16 tokens) and RT * 16 ranks (blockIdx.y the ranks;
// blockIdx.z: with both, 0 is glat). The waves split the contraction in blocks of 128
// columns, and their sums meet in LDS. The scale is applied here. Tokens past the tile's last
// and ranks past the last repeat another: they only reach sums of their own, which are not
// stored. At rank 32 bound by reading x (16384 tokens of 4096 in 36 us, 34 without the
// factor's loads; the last call's 134 MB of outputs are written back meanwhile), at rank 64
// by the factor as well, which every XCD reads (8192 tokens of 4096 and 14336 in 8 equal adapters:
// 83 us, 462 MB past L2 at 5.5 TB/s, of them x and dy 302). Neither more blocks in flight nor
// more waves change that; 64 tokens a tile (104 us against 94) and half the ranks a workgroup (97)
// do not pay; and tiles of one adapter on one XCD, whose L2 would hold the factor, cost more on
// the side of x (110): tiles that run at the same time then lie far apart.
template <int MT, int RT, int WAVES>
__global__ __launch_bounds__(WAVES * cdk::kWave, MT + RT <= 4 ? 4 : 2) void k_ad_shrink(const AdArgs a, int kinds)
{
    static_assert(MT * RT <= WAVES, "one sum per thread");
    constexpr int kSums = MT * RT * cdk::kWave;
    constexpr int kDepth = MT + RT <= 2 ? 2 : 1;  // blocks in flight
    __shared__ u32x4 lds[WAVES * (kSums > kAdStage ? kSums : kAdStage)];
    const int spare = blockIdx.x - (a.T / a.tile + a.n + 1);  // workgroups past the tiles: a.by_size
    if (spare >= 0) {
        if (blockIdx.y == 0 && blockIdx.z == 0)
            ad_by_size<WAVES>(a, spare, reinterpret_cast<int *>(lds));
        return;
    }
    const AdTile tile = a.tiles[blockIdx.x];
    const int count = tile.count;
    if (count <= 0 || tile.group == a.n)
        return;
    const bool back = kinds == 3 ? blockIdx.z == 0 : kinds == 2;  // glat
    const int K = back ? a.d_out : a.d_in;
    const uint16_t *src = back ? a.dy : a.x;
    const size_t ld = back ? a.lddy : a.ldx;
    const uint16_t *fac = (back ? a.Bt : a.A) + (size_t)tile.group * a.rank * K;
    const int lane = threadIdx.x % cdk::kWave, wave = ad_wave();
    const int m = lane % 16, g = lane / 16;
    const int r0 = blockIdx.y * RT * 16;
    int xr[MT][4], fr[RT][4];  // this lane's rows
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            xr[i][q] = a.order[tile.first + min(i * 16 + 4 * q + g, count - 1)];
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            fr[j][q] = min(r0 + j * 16 + 4 * q + g, a.rank - 1) * K;
    u32x4 xv[kDepth][MT][4], fv[kDepth][RT][4];
    const auto load = [&](int s, int k) {
        k += 8 * m;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                xv[s][i][q] = load16(or_zero(k < K, src + (size_t)xr[i][q] * ld + k));
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                fv[s][j][q] = load16(or_zero(k < K, fac + (unsigned)(fr[j][q] + k)));
    };
    f32x4_t acc[MT][RT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j)
            acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 *stage = lds + wave * kAdStage;
    constexpr int kStep = 128 * WAVES;
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d)
        if (wave * 128 + d * kStep < K)
            load(d, wave * 128 + d * kStep);
#pragma unroll 1
    for (int kb = wave * 128; kb < K; kb += kDepth * kStep) {
#pragma unroll
        for (int s = 0; s < kDepth; ++s) {
            const int k = kb + s * kStep;
            if (k >= K)
                break;
            if (kDepth == 1)
                load(0, k);
            else if (k + (kDepth - 1) * kStep < K)
                load((s + kDepth - 1) % kDepth, k + (kDepth - 1) * kStep);
#pragma unroll
            for (int j = 0; j < RT; ++j)
                ad_stage(fv[s][j], stage, lane);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                ad_stage(xv[s][i], stage, lane);
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int j = 0; j < RT; ++j)
                        acc[i][j] = mfma16(fv[s][j][u], xv[s][i][u], acc[i][j]);
            }
        }
    }
    f32x4_t *sums = reinterpret_cast<f32x4_t *>(lds);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j)
            sums[wave * kSums + (i * RT + j) * cdk::kWave + lane] = acc[i][j];
    __syncthreads();
    if (threadIdx.x >= kSums)
        return;
    f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        v += sums[w * kSums + threadIdx.x];
    v *= ad_scale(a, tile.group);
    // this thread: token i * 16 + m, ranks r .. r + 3
    const int at = wave / RT * 16 + m;
    const int r = r0 + wave % RT * 16 + g * 4;
    if (at >= count || r >= a.rank)
        return;
    const size_t p = tile.first + at;
    *reinterpret_cast<f32x4_t *>((back ? a.glat : a.lat) + p * a.rank + r) = v;
    uint16_t *terms = back ? a.glatT : a.latT;
    if (!terms)
        return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t s[3];
        ad_split(v[q], s);
#pragma unroll
        for (int k = 0; k < 3; ++k)
            terms[ad_term_at(a, p, k, r + q)] = (uint16_t)(s[k] >> 16);
    }
}

// lat's terms as MFMA operands for a tile's token (m) and K-chunk c
__device__ __forceinline__ void ad_operand(const AdArgs &a, const float *lat, bool ok, size_t p,
                                           int r, u32x4 (&t)[3])
{
    const float *q = or_zero(ok && r < a.rank, lat + p * a.rank + r);
    const f32x4_t v[2] = {*reinterpret_cast<const f32x4_t *>(q),
                          *reinterpret_cast<const f32x4_t *>(ok && r < a.rank ? q + 4 : q)};
    ad_split8(v, t);
}

// A wave's 16 tokens and their latents' terms, the rows of its MFMAs: KC * 32 ranks, KC 0: any
// number, fetched again (from L2) where they are used, since they would not fit the registers
template <int KC>
struct AdTokens {
    int count, group;
    bool no;  // group n: no adapter
    u32x4 lt[KC ? KC : 1][3];
    int first, tok[4];  // rows 4 g + q of the results

    // part: of tile / 16 in each tile; false: nothing to do
    __device__ __forceinline__ bool init(const AdArgs &a, const float *lat, int part, int m, int g)
    {
        const int sub = a.tile / 16;
        const AdTile tile = a.tiles[part / sub];
        first = tile.first + part % sub * 16;
        count = tile.count - part % sub * 16;
        group = tile.group;
        no = group == a.n;
        if (count <= 0 || (no && a.base == a.out))
            return false;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            tok[q] = a.order[first + min(4 * g + q, count - 1)];
#pragma unroll
        for (int c = 0; c < KC; ++c)
            fetch(a, lat, c, m, g);
        return true;
    }
    __device__ __forceinline__ void fetch(const AdArgs &a, const float *lat, int c, int m, int g)
    {
        ad_operand(a, lat, m < count && !no, first + m, c * 32 + g * 8, lt[KC ? c : 0]);
    }
    __device__ __forceinline__ bool live(int g, int q) const { return 4 * g + q < count; }
};

// y = base + B lat for 16 tokens, KC * 32 ranks. Each wave takes steps of 128 outputs: eight
// MFMAs with the tokens as rows and B's rows as columns. Column m of MFMA j is output 8 m + j
// (fp32: 4 m + j % 4 of the half j / 4), so that a lane ends with 16 bytes of a token's row
// and 16 neighbouring lanes with 256. B's rows pass through LDS: 32 ranks of 128 outputs,
// read as they lie. Bound by memory: 16384 tokens of 4096 bf16 outputs, 268 MB, in 58 us
// (4.6 TB/s; a copy runs at 4.8). 32 tokens a wave read B half as often, but need the
// registers of a second wave on the SIMD: 64 to 91 us.
// The launch bounds leave KC 0 in fp32 a spill of 28 bytes: 63 us for 4096 tokens of 4096 outputs at rank
// 128, with two waves a SIMD and no spill 67.
template <int KC, bool F32>
__global__ __launch_bounds__(kAdBlock, KC == 1 && !F32 ? 4 : 3) void k_ad_expand(const AdArgs a)
{
    constexpr int kHalves = F32 ? 2 : 1;
    constexpr int kPad = F32 ? 4 : 8;  // a chunk more every so many rows: 16 columns on 16 banks
    __shared__ u32x4 lds[kAdWaves][128 * 4 + 128 / kPad];
    const int lane = threadIdx.x % cdk::kWave, wave = ad_wave();
    const int m = lane % 16, g = lane / 16;
    AdTokens<KC> tk;
    if (!tk.init(a, a.lat, blockIdx.x, m, g))
        return;
    const uint16_t *B = a.B + (tk.no ? 0 : (size_t)tk.group * a.d_out * a.rank);
    u32x4 *st = lds[wave];
#pragma unroll 1
    for (int o0 = (blockIdx.y * kAdWaves + wave) * 128; o0 < a.d_out; o0 += gridDim.y * kAdWaves * 128) {
        // this lane's columns: cols(h) .. + 8 (fp32: 4)
        const auto cols = [&](int h) { return F32 ? o0 + 64 * h + 4 * m : o0 + 8 * m; };
        u32x4 base[4][kHalves];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const bool ok = a.base && tk.live(g, q) && cols(h) < a.d_out;
                const size_t at = (size_t)tk.tok[q] * a.ldb + cols(h);
                base[q][h] =
                    F32 ? *reinterpret_cast<const u32x4 *>(or_zero(ok, static_cast<const float *>(a.base) + at))
                        : load16(or_zero(ok, static_cast<const uint16_t *>(a.base) + at));
            }
        f32x4_t acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (!tk.no)
#pragma unroll KC ? KC : 1
            for (int c = 0; c < (KC ? KC : (a.rank + 31) / 32); ++c) {
                if (!KC)
                    tk.fetch(a, a.lat, c, m, g);
                const int nch = min(4, a.rank / 8 - 4 * c);  // chunks of a row; uniform
                if (nch <= 0)
                    break;
                const auto place = [&](int i, int &row, int &ch) {
                    const int e = i * cdk::kWave + lane;
                    row = nch == 4 ? e / 4 : nch == 2 ? e / 2 : nch == 1 ? e : e / 3;
                    ch = e - row * nch;
                };
                u32x4 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < 2 * nch) {  // (a row past the last repeats it: sums not stored)
                        int row, ch;
                        place(i, row, ch);
                        v[i] = load16(B + (size_t)min(o0 + row, a.d_out - 1) * a.rank + (4 * c + ch) * 8);
                    }
                ad_wave_sync();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < 2 * nch) {
                        int row, ch;
                        place(i, row, ch);
                        st[row * 4 + ch + row / kPad] = v[i];
                    }
                ad_wave_sync();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int row = F32 ? j / 4 * 64 + 4 * m + j % 4 : 8 * m + j;
                    u32x4 b = st[row * 4 + g + row / kPad];
                    if (g >= nch)  // (ranks past the last)
                        b = cdk::zero16();
#pragma unroll
                    for (int s = 2; s >= 0; --s)
                        acc[j] = mfma16(tk.lt[KC ? c : 0][s], b, acc[j]);
                }
            }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                if (!tk.live(g, q) || cols(h) >= a.d_out)
                    continue;
                u32x4 w = base[q][h];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!tk.no)
                        w[e] = F32 ? __float_as_uint(__uint_as_float(w[e]) + acc[4 * h + e][q])
                                   : ad_pack(cdk::bf16_lo(w[e]) + acc[2 * e][q],
                                             cdk::bf16_hi(w[e]) + acc[2 * e + 1][q]);
                const size_t at = (size_t)tk.tok[q] * a.ldo + cols(h);
                if constexpr (F32)
                    *reinterpret_cast<u32x4 *>(static_cast<float *>(a.out) + at) = w;
                else
                    *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.out) + at) = w;
            }
    }
}

constexpr int kAdBackWaves = 8;  // of the workgroups that compute the gradients

// dx = base + A^T glat: as k_ad_expand, but the factor's rows run along the outputs, so a
// lane loads 8 ranks x 8 columns and transposes them in registers: steps of 128 columns,
// column m of MFMA j is 8 m + j.
template <int KC>
__device__ __forceinline__ void ad_dx(const AdArgs &a, int part, int slice, int slices)
{
    const int lane = threadIdx.x % cdk::kWave, wave = ad_wave();
    const int m = lane % 16, g = lane / 16;
    AdTokens<KC> tk;
    if (!tk.init(a, a.glat, part, m, g))
        return;
    const uint16_t *A = a.A + (tk.no ? 0 : (size_t)tk.group * a.d_in * a.rank);
#pragma unroll 1
    for (int c0 = (slice * kAdBackWaves + wave) * 128; c0 < a.d_in; c0 += slices * kAdBackWaves * 128) {
        const int col = c0 + 8 * m;
        const bool cok = col < a.d_in;
        u32x4 base[4][2];
#pragma unroll
        for (int q = 0; q < 4; ++q)
            ad_base8(a, tk.live(g, q) && cok, tk.tok[q], col, base[q]);
        f32x4_t acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (!tk.no)
#pragma unroll KC ? KC : 1
            for (int c = 0; c < (KC ? KC : (a.rank + 31) / 32); ++c) {
                if (!KC)
                    tk.fetch(a, a.glat, c, m, g);
                u32x4 rows[8], cols[8];
                const bool ok = c * 32 + g * 8 < a.rank && cok;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    rows[e] = load16(or_zero(ok, A + (size_t)(c * 32 + g * 8 + e) * a.d_in + col));
                ad_transpose8(rows, cols);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int s = 2; s >= 0; --s)
                        acc[j] = mfma16(tk.lt[KC ? c : 0][s], cols[j], acc[j]);
            }
        if (cok)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[8] = {acc[0][q], acc[1][q], acc[2][q], acc[3][q],
                                    acc[4][q], acc[5][q], acc[6][q], acc[7][q]};
                if (tk.live(g, q))
                    ad_store8(a, tk.tok[q], col, base[q], v, tk.no);
            }
    }
}

// dA = glat^T x and dB = dy^T lat of one adapter. The contraction runs over the adapter's
// tokens, 32 at a time: a lane loads 8 tokens x 8 columns (the next 32 tokens' in flight) and
// transposes them. A workgroup has 128 columns; its eight waves are WR parts of RT * 16 ranks
// and the rest parts of the tokens, whose sums meet in LDS. Where that leaves CUs without a
// workgroup, `parts` workgroups share the tokens as well, each with sums of its own in
// a.part, and k_ad_sum adds them in order. 4096 tokens of 4096 and 4096 columns at rank 16, in
// equal adapters: 14.4 us (67 MB, 4.7 TB/s); 8192 tokens of 4096 and 14336 at rank 64: 112 us,
// with 363 MB fetched past L2: the columns once (302) and the terms (6 MB, from
// neighbouring columns over and over) where an L2 has not had them. 64 ranks in a wave spill,
// 16 ranks in each of four waves fetch the columns four times through L1; two tiles of
// columns a workgroup, 4 waves, or 64 tokens in flight change little.
template <int RT, int WR, bool DB>
__device__ __forceinline__ void ad_outer(const AdArgs &a, const AdTile &grp, int block, int parts, f32x4_t *lds)
{
    constexpr int WT = kAdBackWaves / WR;
    const int lane = threadIdx.x % cdk::kWave, wave = ad_wave();
    const int m = lane % 16, g = lane / 16;
    const int wt = wave / WR, part = wave % WR;  // tokens; ranks
    const int tokens = block / 8 % parts;        // of the workgroups that share them
    const int width = DB ? a.d_out : a.d_in;
    const int rts = (a.rank + 15) / 16, rgs = (rts + RT * WR - 1) / (RT * WR);
    // eight neighbouring workgroups (one on each XCD) take neighbouring columns
    const int y = block / 8 / parts, rt0 = (y % rgs * WR + part) * RT;
    const int c0 = (y / rgs * 8 + block % 8) * 128, col = c0 + m * 8;
    const uint16_t *src = DB ? a.dy : a.x;
    const size_t ld = DB ? a.lddy : a.ldx;
    const uint16_t *fac = DB ? a.latT : a.glatT;
    const bool cok = col < width;
    f32x4_t acc[RT][8];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 rows[8], f[RT][3];
    // tokens past the group's end load zeros; ranks past the last repeat the last tile's
    const int next = parts * WT * 32;  // from one of this wave's 32 tokens to the next
    int4 ord[2];  // the lane's tokens, of those loaded next
    const auto load_order = [&](int p) {
        if (p >= grp.count)
            return;
        const int4 *o = reinterpret_cast<const int4 *>(a.order + grp.first + p + g * 8);
        ord[0] = o[0];
        ord[1] = o[1];
    };
    const auto load_rows = [&](int p) {
        if (p >= grp.count)
            return;
        const int t[8] = {ord[0].x, ord[0].y, ord[0].z, ord[0].w, ord[1].x, ord[1].y, ord[1].z, ord[1].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool ok = p + g * 8 + e < grp.count && cok;
            rows[e] = load16(or_zero(ok, src + (ok ? (size_t)t[e] * ld : 0) + col));
        }
        load_order(p + next);
    };
    const auto load_term = [&](int p, int s) {
        if (p >= grp.count)
            return;
#pragma unroll
        for (int i = 0; i < RT; ++i)
            f[i][s] = load16(fac + (((size_t)(grp.first + p) / 32 * 3 + s) * rts + min(rt0 + i, rts - 1)) * 512 + lane * 8);
    };
    const int p0 = (tokens * WT + wt) * 32;
    load_order(p0);
    load_rows(p0);
#pragma unroll
    for (int s = 2; s >= 0; --s)
        load_term(p0, s);
#pragma unroll 1
    for (int p = p0; p < grp.count; p += next) {
        u32x4 cols[8];
        ad_transpose8(rows, cols);
        const int left = grp.count - p - g * 8;  // tokens from this lane's first
        if (grp.count - p < 32) {  // what lies past the group's end is not a number of this call
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int s = 0; s < 3; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        f[i][s][e] &= (2 * e < left ? 0xffffu : 0u) | (2 * e + 1 < left ? 0xffff0000u : 0u);
        }
        load_rows(p + next);
#pragma unroll
        for (int s = 2; s >= 0; --s) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < RT; ++i)
                    acc[i][j] = DB ? mfma16(f[i][s], cols[j], acc[i][j]) : mfma16(cols[j], f[i][s], acc[i][j]);
            load_term(p + next, s);
        }
    }
    // the upper half of the token parts hands its sums to the lower, until one has them all
#pragma unroll
    for (int half = WT / 2; half >= 1; half /= 2)
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            f32x4_t *at = lds + ((wt % half * WR + part) * 8) * cdk::kWave + lane;
            __syncthreads();
            if (wt >= half && wt < 2 * half)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    at[j * cdk::kWave] = acc[i][j];
            __syncthreads();
            if (wt < half)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    acc[i][j] += at[j * cdk::kWave];
        }
    if (wt)
        return;
    const size_t whole = (size_t)a.n * a.rank * width;
    float *dst = parts > 1 ? a.part + (DB || !a.dB ? 0 : (size_t)parts * a.n * a.rank * a.d_out) + tokens * whole
                           : DB ? a.dB : a.dA;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        if constexpr (DB) {  // row o = c0 + 8 m + j, ranks 4 g + q
            const int r = (rt0 + i) * 16 + g * 4;
            if (cok && r < a.rank)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<f32x4_t *>(dst + ((size_t)grp.group * a.d_out + col + j) * a.rank + r) =
                        acc[i][j];
        } else {  // row r = m, columns c0 + 8 (4 g + q) + j
            const int r = (rt0 + i) * 16 + m;
            if (r < a.rank)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = c0 + 8 * (4 * g + q);
                    if (c < a.d_in) {
                        f32x4_t *d = reinterpret_cast<f32x4_t *>(dst + ((size_t)grp.group * a.rank + r) * a.d_in + c);
                        d[0] = f32x4_t{acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]};
                        d[1] = f32x4_t{acc[i][4][q], acc[i][5][q], acc[i][6][q], acc[i][7][q]};
                    }
                }
        }
    }
}

// Workgroups take the adapters by their tokens, the most first: nB for dB and nA for dA of each.
// The others compute dx (`slices` of its columns). One launch for small calls' sake, and
// because the kinds wait for different things. A workgroup goes over all tokens of its
// adapter, so one of a large adapter must not start late; and those that run together read
// the same terms. Against the adapters in their own order, side by side (us a launch): 8192 tokens of
// 4096 and 14336, rank 64, 16 uneven requests of 8 adapters 134 against 170; 4096 tokens of
// 4096, rank 16, 4 adapters 31.9 against 38.6. 1024 adapters of 8 tokens each lose (us a call):
// 1243 against 1192.
template <int RT, int WR, int KC>
__global__ __launch_bounds__(kAdBackWaves * cdk::kWave, 2) void k_ad_back(const AdArgs a, int nB, int nA,
                                                                      int parts, int slices)
{
    __shared__ f32x4_t lds[kAdBackWaves / 2 * 8 * cdk::kWave];
    const int b = blockIdx.x, grads = (nB + nA) * a.n;
    if (b >= grads) {
        ad_dx<KC>(a, (b - grads) / slices, (b - grads) % slices, slices);
        return;
    }
    const AdTile grp = a.by_size[b / (nB + nA)];
    const int i = b % (nB + nA);
    if (i < nB)
        ad_outer<RT, WR, true>(a, grp, i, parts, lds);
    else
        ad_outer<RT, WR, false>(a, grp, i - nB, parts, lds);
}

// dB and dA (nb and na elements) from their parts
__global__ __launch_bounds__(kAdBlock) void k_ad_sum(const float *part, int parts, float *dB, size_t nb,
                                                     float *dA, size_t na)
{
    for (size_t i = ((size_t)blockIdx.x * kAdBlock + threadIdx.x) * 4; i < nb + na; i += (size_t)gridDim.x * kAdBlock * 4) {
        const bool b = i < nb;
        const float *p = b ? part + i : part + parts * nb + (i - nb);
        f32x4_t v = *reinterpret_cast<const f32x4_t *>(p);
#pragma unroll 4
        for (int k = 1; k < parts; ++k)
            v += *reinterpret_cast<const f32x4_t *>(p + k * (b ? nb : na));
        *reinterpret_cast<f32x4_t *>(b ? dB + i : dA + (i - nb)) = v;
    }
}

__global__ __launch_bounds__(kAdBlock) void k_ad_zero(float *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * kAdBlock + threadIdx.x; i < n; i += (size_t)gridDim.x * kAdBlock)
        p[i] = 0.0f;
}

// rows of `row` bytes at a stride of ld bytes
struct AdRows {
    const void *p;
    size_t row, ld;
    int n;
};

// Two row arrays share an element, or might: arrays of one stride are compared by their
// columns, others by their ranges.
bool ad_overlap(const AdRows &a, const AdRows &b)
{
    if (!a.p || !b.p || a.n < 1 || b.n < 1)
        return false;
    const size_t na = (a.n - 1) * a.ld + a.row, nb = (b.n - 1) * b.ld + b.row;
    if (!overlaps(a.p, na, b.p, nb))
        return false;
    if (a.ld != b.ld)
        return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const size_t d = y >= x ? (y - x) % a.ld : (a.ld - (x - y) % a.ld) % a.ld;
    return d < a.row || d + b.row > a.ld;
}

AdRows ad_flat(const void *p, size_t bytes) { return {p, bytes, bytes, 1}; }

bool ad_ld_ok(size_t ld, int width) { return ld >= (size_t)width && ld % 8 == 0 && ld <= ((size_t)1 << 32); }

size_t ad_size(int type) { return type == CD_TYPE_F32 ? sizeof(float) : sizeof(uint16_t); }

}  // namespace

struct cd_adapters {
    int d_in, d_out, rank, n, max_tokens, device;
    unsigned flags;
    void *ws;  // everything below lies in it
    float *lat, *glat;
    int *order;
    AdGroup *groups;
    AdTile *tiles;
    AdTile *by_size;
    uint16_t *Bt, *latT, *glatT;
    float *part;
};

namespace {

// Tokens of a tile. Small tiles spread a short batch over the CUs; large ones read the factors
// less often.
int ad_tile(int T) { return T < 8192 ? 16 : 32; }

// the arguments that every call has; out_dim: the columns of base and out (0: neither)
cd_status ad_check(const cd_adapters *p, const AdArgs &a, int out_dim)
{
    if (!p || a.T < 0 || a.T > p->max_tokens || (a.type != CD_TYPE_F32 && a.type != CD_TYPE_BF16))
        return CD_EINVAL;
    if (!a.A || !aligned16(a.A) || !a.B || !aligned16(a.B) ||
        (reinterpret_cast<uintptr_t>(a.scale) & 3u))
        return CD_EINVAL;
    if (a.T > 0 && (!a.x || !aligned16(a.x) || !ad_ld_ok(a.ldx, p->d_in) || !a.ids ||
                    (reinterpret_cast<uintptr_t>(a.ids) & 3u)))
        return CD_EINVAL;
    if (a.T > 0 && out_dim) {
        if (!a.out || !aligned16(a.out) || !ad_ld_ok(a.ldo, out_dim))
            return CD_EINVAL;
        if (a.base && (!aligned16(a.base) || !ad_ld_ok(a.ldb, out_dim)))
            return CD_EINVAL;
    }
    const size_t es = ad_size(a.type), n = p->n, r = p->rank;
    const AdRows base{a.base, out_dim * es, a.ldb * es, a.T};
    const AdRows in[] = {{a.x, (size_t)p->d_in * 2, a.ldx * 2, a.T},
                         {a.dy, (size_t)p->d_out * 2, a.lddy * 2, a.T},
                         ad_flat(a.W, (size_t)p->d_out * p->d_in * 2),
                         {a.ids, 4, 4, a.T},
                         ad_flat(a.A, n * r * p->d_in * 2),
                         ad_flat(a.B, n * r * p->d_out * 2),
                         ad_flat(a.scale, n * 4),
                         base};
    const AdRows out[] = {{out_dim ? a.out : nullptr, out_dim * es, a.ldo * es, a.T},
                          ad_flat(a.dA, n * r * p->d_in * 4),
                          ad_flat(a.dB, n * r * p->d_out * 4)};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 8; ++j) {
            const bool in_place = i == 0 && j == 7 && a.base == a.out && a.ldb == a.ldo;
            if (!in_place && ad_overlap(out[i], in[j]))
                return CD_EINVAL;
        }
        for (int j = 0; j < i; ++j)
            if (ad_overlap(out[i], out[j]))
                return CD_EINVAL;
    }
    int dev = -1;
    if (hip_status(hipGetDevice(&dev)) != CD_OK)
        return CD_EHIP;
    return dev == p->device ? CD_OK : CD_EINVAL;
}

AdArgs ad_args(const cd_adapters *p, const uint16_t *x, size_t ldx, int T, const int32_t *ids,
               const uint16_t *A, const uint16_t *B, const float *scale, int type)
{
    AdArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.ids = ids;
    a.A = A;
    a.B = B;
    a.scale = scale;
    a.type = type;
    a.T = T;
    if (p) {
        a.n = p->n;
        a.d_in = p->d_in;
        a.d_out = p->d_out;
        a.rank = p->rank;
        a.lat = p->lat;
        a.order = p->order;
        a.groups = p->groups;
        a.tiles = p->tiles;
        a.tile = ad_tile(T);
    }
    return a;
}

int ad_ceil(int v, int d) { return (v + d - 1) / d; }

// tiles of the grouped tokens (k_ad_group)
int ad_slots(const AdArgs &a) { return a.T / a.tile + a.n + 1; }

void ad_group(const AdArgs &a, bool transpose, hipStream_t s)
{
    const int more = transpose ? a.n * ad_ceil(a.d_out, 128) * ad_ceil(a.rank, 64) : 0;
    k_ad_group<<<a.n + 1 + more, kAdSortBlock, 0, s>>>(a);
}

// kinds: 1 lat, 2 glat, 3 both
void ad_shrink(const AdArgs &a, int kinds, hipStream_t s)
{
    const int mt = a.tile / 16, slots = ad_slots(a), both = kinds == 3 ? 2 : 1;
    // While 16 ranks a workgroup make no more of them than CUs: so, with sixteen waves each. Rank 32
    // over 13528 columns, 32 tokens (backward, us a call) 24.7 against 29.9, 512 tokens 29.1
    // against 33.8; rank 48 over 4096, 512 tokens (246 workgroups) 32.4 against 33.3, 1024 tokens
    // (438) 43.0 against 39.4. (The backward call counts both latents, whichever it needs: a
    // gradient's sums are the same alone and together.)
    const bool few = slots * (a.dy ? 2 : 1) * ad_ceil(a.rank, 16) <= 256;
    const int rt = a.rank <= 16 || few ? 1 : a.rank <= 32 ? 2 : 4;
    const dim3 grid(slots + (a.by_size ? ad_ceil(a.n, cdk::kWave) : 0), ad_ceil(a.rank, rt * 16), both);
#define AD_SHRINK(M, R, W) \
    if (mt == M && rt == R && few == (W == 16)) \
        k_ad_shrink<M, R, W><<<grid, W * cdk::kWave, 0, s>>>(a, kinds)
    AD_SHRINK(1, 1, 16);
    AD_SHRINK(1, 1, 8);
    AD_SHRINK(1, 2, 8);
    AD_SHRINK(1, 4, 8);
    AD_SHRINK(2, 1, 8);
    AD_SHRINK(2, 2, 8);
    AD_SHRINK(2, 4, 8);
#undef AD_SHRINK
}

// Slices of the columns, 128 to each of `waves` waves, so that `parts` tiles make about 2048 workgroups.
int ad_slices(int width, int waves, int parts)
{
    return std::max(1, std::min(ad_ceil(width, 128 * waves), ad_ceil(2048, parts)));
}

// y from the latents
void ad_expand(const AdArgs &a, hipStream_t s)
{
    const int parts = ad_slots(a) * (a.tile / 16);
    const dim3 grid(parts, ad_slices(a.d_out, kAdWaves, parts));
#define AD_EXPAND(K) \
    if (a.type == CD_TYPE_F32) \
        k_ad_expand<K, true><<<grid, kAdBlock, 0, s>>>(a); \
    else \
        k_ad_expand<K, false><<<grid, kAdBlock, 0, s>>>(a)
    if (a.rank <= 32) {
        AD_EXPAND(1);
    } else if (a.rank <= 64) {
        AD_EXPAND(2);
    } else {
        AD_EXPAND(0);
    }
#undef AD_EXPAND
}

// dx, dA and dB, as far as they are wanted, from the latents
template <int RT, int WR, int KC>
void ad_back(const AdArgs &a, hipStream_t s)
{
    constexpr int WT = kAdBackWaves / WR;
    const int rgs = ad_ceil(a.rank, RT * WR * 16);
    // With fewer gradient tiles than half the CUs, the tokens are shared: at least two times 32
    // for each wave, and no more parts than fit their place. (Counted for dA and dB, whichever is
    // wanted: the sums' order is the same alone and together.)
    const int tiles128 = a.n * rgs * (ad_ceil(a.d_in, 128) + ad_ceil(a.d_out, 128));
    const size_t whole = (size_t)a.n * a.rank * (a.d_in + a.d_out);
    int parts = 1;
    if (tiles128 <= 128 && (a.dA || a.dB))
        parts = std::max(1, (int)std::min<size_t>({(size_t)(256 / tiles128), (size_t)(a.T / (2 * 32 * WT)),
                                                   kAdPartFloats / whole}));
    const int nA = a.dA ? rgs * ad_ceil(a.d_in, 8 * 128) * 8 * parts : 0;
    const int nB = a.dB ? rgs * ad_ceil(a.d_out, 8 * 128) * 8 * parts : 0;
    const int tiles = ad_slots(a) * (a.tile / 16);
    const int slices = a.out ? ad_slices(a.d_in, kAdBackWaves, tiles) : 1;
    const int nX = a.out ? tiles * slices : 0;
    k_ad_back<RT, WR, KC><<<a.n * (nB + nA) + nX, kAdBackWaves * cdk::kWave, 0, s>>>(a, nB, nA, parts, slices);
    if (parts > 1)
        k_ad_sum<<<std::min<size_t>(1024, (whole / 4 + kAdBlock - 1) / kAdBlock), kAdBlock, 0, s>>>(
            a.part, parts, a.dB, a.dB ? (size_t)a.n * a.rank * a.d_out : 0, a.dA,
            a.dA ? (size_t)a.n * a.rank * a.d_in : 0);
}

}  // namespace

extern "C" {

cd_status countdown_adapters_create(int d_in, int d_out, int rank, int n_adapters, int max_tokens,
                                    unsigned flags, cd_adapters **out)
{
    if (!out || d_in < 8 || d_in % 8 || d_out < 8 || d_out % 8 || rank < 8 || rank % 8 ||
        n_adapters < 1 || max_tokens < 1 || (flags & ~CD_ADAPTERS_TRAIN))
        return CD_EINVAL;
    if (d_in > kAdMaxDim || d_out > kAdMaxDim || rank > kAdMaxRank || n_adapters > kAdMaxAdapters ||
        max_tokens > kAdMaxTokens)
        return CD_EUNSUPPORTED;
    int dev = -1;
    if (hip_status(hipGetDevice(&dev)) != CD_OK)
        return CD_EHIP;
    cd_adapters *p = new (std::nothrow) cd_adapters{};
    if (!p)
        return CD_ENOMEM;
    p->d_in = d_in;
    p->d_out = d_out;
    p->rank = rank;
    p->n = n_adapters;
    p->max_tokens = max_tokens;
    p->flags = flags;
    p->device = dev;
    const bool train = flags & CD_ADAPTERS_TRAIN;
    const size_t pos = (size_t)(max_tokens + kAdPad - 1) / kAdPad * kAdPad + kAdPad * (n_adapters + 1);
    const size_t lat = pos * rank * sizeof(float);
    const size_t terms = 3 * pos * ((rank + 15) / 16 * 16) * sizeof(uint16_t);
    const size_t tiles = ((size_t)max_tokens / 16 + n_adapters + 1) * sizeof(AdTile);
    const size_t groups = (n_adapters + 1) * sizeof(AdGroup);
    const size_t copy = (size_t)n_adapters * rank * d_out * sizeof(uint16_t);
    const size_t parts[] = {lat,   pos * sizeof(int),  tiles,             groups,
                            train ? lat : 0, train ? terms : 0, train ? terms : 0, train ? copy : 0,
                            train ? kAdPartFloats * sizeof(float) : 0,
                            train ? n_adapters * sizeof(AdTile) : 0};
    size_t at[11] = {0};
    for (int i = 0; i < 10; ++i)
        at[i + 1] = at[i] + (parts[i] + 255) / 256 * 256;
    if (hip_status(hipMalloc(&p->ws, at[10])) != CD_OK) {
        delete p;
        return CD_ENOMEM;
    }
    char *ws = static_cast<char *>(p->ws);
    p->lat = reinterpret_cast<float *>(ws + at[0]);
    p->order = reinterpret_cast<int *>(ws + at[1]);
    p->tiles = reinterpret_cast<AdTile *>(ws + at[2]);
    p->groups = reinterpret_cast<AdGroup *>(ws + at[3]);
    if (train) {
        p->glat = reinterpret_cast<float *>(ws + at[4]);
        p->latT = reinterpret_cast<uint16_t *>(ws + at[5]);
        p->glatT = reinterpret_cast<uint16_t *>(ws + at[6]);
        p->Bt = reinterpret_cast<uint16_t *>(ws + at[7]);
        p->part = reinterpret_cast<float *>(ws + at[8]);
        p->by_size = reinterpret_cast<AdTile *>(ws + at[9]);
    }
    *out = p;
    return CD_OK;
}

cd_status countdown_adapters_destroy(cd_adapters *p)
{
    if (!p)
        return CD_OK;
    int dev = -1;
    cd_status st = hip_status(hipGetDevice(&dev));
    if (st == CD_OK)
        st = hip_status(hipSetDevice(p->device));
    if (st == CD_OK)
        st = hip_status(hipDeviceSynchronize());
    if (hip_status(hipFree(p->ws)) != CD_OK)
        st = CD_EHIP;
    if (dev >= 0)
        (void)hip_status(hipSetDevice(dev));
    delete p;
    return st;
}

cd_status countdown_adapters_project(cd_adapters *p, const uint16_t *x, size_t ldx, int T,
                                     const uint16_t *W, const int32_t *ids, const uint16_t *A,
                                     const uint16_t *B, const float *scale, int type, void *y,
                                     size_t ldy, void *stream)
{
    AdArgs a = ad_args(p, x, ldx, T, ids, A, B, scale, type);
    a.W = W;
    a.out = y;
    a.ldo = ldy;
    if (!W || !aligned16(W))
        return CD_EINVAL;
    const cd_status st = ad_check(p, a, p ? p->d_out : 0);
    if (st != CD_OK)
        return st;
    if (T > kAdDecodeTokens)
        return CD_EUNSUPPORTED;
    if (T == 0)
        return CD_OK;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    // Few latents every workgroup forms for itself, one after another, before its sums are whole;
    // with more workgroups than the CUs hold at once (512) that comes twice. Captured / eager us a call
    // against a launch of their own:
    //   16 latents, 4096 -> 4096  8.4 /  8.2 against  9.0 /  9.2   4096 -> 14336 28.5 / 28.8 against 22.6 / 23.0
    //   32 latents, 1000 -> 4096  5.4 /  7.3 against  5.2 / 10.2   4096 ->  4096 10.7 / 10.6 against  9.1 /  9.9
    //   64 latents, 1000 -> 4096  7.8 /  7.7 against  5.3 /  9.7
    const int latents = T * a.rank;
    const bool own = latents <= kAdOwnLatents && latents * a.d_in <= 1 << 16 && a.d_out <= 512 * 16;
    // A W that would sweep most of the last-level cache goes past it: 117 MB (4096 x 14336, 8
    // tokens) 24.7 us against 27.1; 48 MB that was still there from the last call, 14.9 against 11.9.
    const bool nt = (size_t)a.d_in * a.d_out * sizeof(uint16_t) > ((size_t)64 << 20);
    if (!own)
        k_ad_lat<<<ad_ceil(T * a.rank, kAdWaves), kAdBlock, 0, s>>>(a);
#define AD_PROJECT(O, N) \
    if (own == O && nt == N) \
        k_ad_project<O, N><<<ad_ceil(a.d_out, 16), kAdProjBlock, 0, s>>>(a)
    AD_PROJECT(false, false);
    AD_PROJECT(false, true);
    AD_PROJECT(true, false);
    AD_PROJECT(true, true);
#undef AD_PROJECT
    return launched(hipGetLastError());
}

cd_status countdown_adapters_add(cd_adapters *p, const uint16_t *x, size_t ldx, int T,
                                 const int32_t *ids, const uint16_t *A, const uint16_t *B,
                                 const float *scale, int type, const void *base, size_t ldb,
                                 void *y, size_t ldy, void *stream)
{
    AdArgs a = ad_args(p, x, ldx, T, ids, A, B, scale, type);
    a.base = base;
    a.ldb = ldb;
    a.out = y;
    a.ldo = ldy;
    const cd_status st = ad_check(p, a, p ? p->d_out : 0);
    if (st != CD_OK || T == 0)
        return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    // How the tokens are taken (us an eager call, fp32 y, tokens 8 / 64 / 256 / 1024):
    //                          one launch            two launches          grouped
    //   4096 -> 4096, rank 16   8.4  8.3 12.5  41.6  11.2 11.5 11.0  28.0  14.8 15.4 15.7 21.5
    //   1024 -> 4096, rank 64   8.3  9.2 27.0 101.3  10.8 10.7 22.1  77.7  16.1 17.2 17.8 23.7
    //   4096 -> 4096, rank 64  13.0 19.0 49.2 179.9   9.8 10.9 31.8  97.3  21.0 21.7 22.9 33.2
    // By token, every one reads its adapter again: once, or A again for each 1024 outputs, 16
    // ranks at a time. The bounds below are where the columns cross. (Captured, where a second
    // launch costs 1.6 us and not 2.9, rank 32 and more would rather take two: 5.2 against 7.2 for
    // 4096 -> 4096, 16 tokens.) Two launches and grouped, captured: T r (d_in + d_out) of 40 M 11.0
    // against 19.8 (4096 -> 1024, rank 128, 64 tokens) to 22.7 against 18.3 (1024 -> 4096); of 59 to 67 M
    // 27.0 against 15.7 (256 -> 688, rank 64, 1024 tokens) to 16.5 against 14.6 (4096 -> 4096, rank 32, 256).
    // They count products, not the workgroup and the round trips that every token costs, and so come
    // late for narrow layers and thousands of tokens. One launch, two and grouped, captured:
    //   256 -> 256 rank 8, 2048 tokens  8.2  7.9 11.5   4096 13.5 11.6 12.2    8192 24.5 19.1 14.3
    //    64 ->  64 rank 16, 2048 tokens 9.0  9.9 11.4   4096 15.2 15.2 11.5   16384 51.3 47.5 14.8
    // From 1024 -> 1024, rank 16 on they hold there too: 2048 tokens 14.1 15.6 15.4.
    const int64_t down = (int64_t)a.rank * a.d_in, up = (int64_t)a.rank * a.d_out;
    const int slices = ad_ceil(a.d_out, kAdTokenBlock);
    if (a.rank <= 64 && down <= 3 << 16 && T * (slices * down + up) < 3 << 24) {
        k_ad_token<<<dim3(T, slices), kAdTokenBlock, 0, s>>>(a);
    } else if (T * (down + up) < 3 << 24) {
        k_ad_lat<<<ad_ceil(T * a.rank, kAdWaves), kAdBlock, 0, s>>>(a);
        k_ad_up<<<dim3(T, ad_ceil(a.d_out, kAdBlock)), kAdBlock, 0, s>>>(a);
    } else {
        ad_group(a, false, s);
        ad_shrink(a, 1, s);
        ad_expand(a, s);
    }
    return launched(hipGetLastError());
}

cd_status countdown_adapters_backward(cd_adapters *p, const uint16_t *x, size_t ldx,
                                      const uint16_t *dy, size_t lddy, int T, const int32_t *ids,
                                      const uint16_t *A, const uint16_t *B, const float *scale,
                                      int type, const void *base, size_t ldb, void *dx,
                                      size_t lddx, float *dA, float *dB, void *stream)
{
    AdArgs a = ad_args(p, x, ldx, T, ids, A, B, scale, type);
    a.dy = dy;
    a.lddy = lddy;
    a.base = dx ? base : nullptr;
    a.ldb = ldb;
    a.out = dx;
    a.ldo = lddx;
    a.dA = dA;
    a.dB = dB;
    if (!p || !(p->flags & CD_ADAPTERS_TRAIN) || !aligned16(dA) || !aligned16(dB) ||
        (T > 0 && (!dy || !aligned16(dy) || !ad_ld_ok(lddy, p->d_out))))
        return CD_EINVAL;
    const cd_status st = ad_check(p, a, dx ? p->d_in : 0);
    if (st != CD_OK)
        return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (T == 0) {
        if (dA)
            k_ad_zero<<<1024, kAdBlock, 0, s>>>(dA, (size_t)a.n * a.rank * a.d_in);
        if (dB)
            k_ad_zero<<<1024, kAdBlock, 0, s>>>(dB, (size_t)a.n * a.rank * a.d_out);
        return launched(hipGetLastError());
    }
    const bool back = dx || dA;
    if (!back && !dB)
        return CD_OK;
    a.glat = p->glat;
    a.Bt = p->Bt;
    a.latT = p->latT;
    a.glatT = dA ? p->glatT : nullptr;
    a.part = p->part;
    a.by_size = dA || dB ? p->by_size : nullptr;
    // Two launches instead of three while a workgroup reads a token's factors in a moment, and the
    // tokens of one adapter, one after another in its rows' sums, are few. Captured / eager us a call
    // against the three:
    //    1 token,  4096 -> 4096 rank 16, one adapter  10.1 / 10.8 against 13.1 / 13.7
    //    8 tokens, 4096 -> 4096 rank 16, one adapter  12.6 / 13.0 against 13.0 / 13.9 (16: 16.1 against 13.4)
    //   16 tokens, 4096 -> 4096 rank 16, four         11.1 / 11.5 against 16.4 / 17.2
    //    1 token,  2048 -> 14336, one: rank 24        15.5 / 15.8 against 20.9 / 21.5, rank 32 22.3 / 22.6 against 21.1 / 21.6
    //    8 tokens, 4096 -> 4096 rank 32, one adapter  14.8 / 15.1 against 14.8 / 15.4
    //    8 tokens, 4096 -> 4096 rank 40, one adapter  19.9 / 20.2 against 14.4 / 15.1 (256 -> 688 15.8 against 12.1)
    if (T <= std::min(kAdFewTokens, 8 * a.n) && a.rank <= kAdFewRanks &&
        a.rank * std::max(a.d_in, a.d_out) <= 3 << 17) {
        k_ad_few_latents<<<dim3(T, back && dB ? 2 : 1), kAdTokenBlock, 0, s>>>(a, dB ? 0 : 1);
        const int nB = dB ? a.n * ad_ceil(a.d_out * (a.rank / 8), kAdBlock) : 0;
        const int nA = dA ? a.n * ad_ceil(a.rank * (a.d_in / 8), kAdBlock) : 0;
        const int nX = dx ? T * ad_ceil(a.d_in / 8, kAdBlock) : 0;
        k_ad_few_back<<<nB + nA + nX, kAdBlock, 0, s>>>(a, nB, nA);
        return launched(hipGetLastError());
    }
    ad_group(a, back, s);
    ad_shrink(a, (dB ? 1 : 0) + (back ? 2 : 0), s);
    if (a.rank <= 16)
        ad_back<1, 1, 1>(a, s);
    else if (a.rank <= 32)
        ad_back<2, 1, 1>(a, s);
    else if (a.rank <= 64)
        ad_back<2, 2, 2>(a, s);
    else
        ad_back<2, 2, 0>(a, s);
    return launched(hipGetLastError());
}

}  // extern "C"
