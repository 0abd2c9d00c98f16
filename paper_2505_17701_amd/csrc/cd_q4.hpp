// Decode products with 4-bit weights and a bf16 scale for each group of columns of a row. Part of
// cd_api.hip (its only includer, after cd_adapters.hpp).
//
//   w[r][c] = scale[r][c / G] code[r][c], code in -8..7, G in {32, 64, 128}
//   project: y_t = base_t + W x_t       gated: h_t = SiLU(Wg x_t) * (Wu x_t)
//
// Up to 16 tokens, the columns of a 16 x 16 x 32 MFMA: the weights, a quarter of bf16's bytes, are
// streamed once for all of them. A 4-bit code c + 8 put into the upper mantissa bits of a bf16 16.0
// is exactly 24 + c, two instructions for a pair of weights; the 24 goes again with one more product,
// of -24 and the same tokens, that the sums of a group start from. Sums are fp32, the group's scale
// multiplies a group's sum, not its weights.
//
// Packed layout: blocks of 16 rows x 128 columns, the blocks of 16 rows one after another. A block is
// 1024 bytes of codes and 32 for each of its 128 / G groups (the 16 rows' scales). Lane l = 16 j + i of
// a wave owns bytes 16 l..16 l + 15: word w holds row i, columns 32 w + 8 j + e; the code of e = 2 p lies
// at bits 4 p, that of e = 2 p + 1 at bits 16 + 4 p, each as c + 8. So a wave's load is 1 KB on end
// and each word is an operand. Rows and columns that pad the matrix have code 0 and scale 0.
#pragma once

#include "cd_device.hpp"

namespace {

constexpr int kQ4MaxDim = 65536, kQ4Tokens = 16;
constexpr int kQ4Rows = 16, kQ4Cols = 128;  // of a block
constexpr int kQ4Waves = 8, kQ4Block = kQ4Waves * cdk::kWave;
constexpr int kQ4Flight = 4;  // blocks of a wave (and matrix) in flight
constexpr int kQ4XUnits = 4096;  // 16-byte units of the tokens in LDS

__host__ __device__ constexpr int q4_block(int group) { return 1024 + 32 * (kQ4Cols / group); }

struct Q4Args {
    const uint16_t *x;
    size_t ldx;
    const uint8_t *W, *W2;  // packed (gated: W_gate, W_up)
    int T, rows, cols;
    const void *base;
    size_t ldb;
    void *out;
    size_t ldo;
    int type;   // of base and out
    int chunk;  // columns that LDS holds of each token
};

template <int NM, int G>
struct Q4Block {  // what a lane holds of a block of each of NM matrices
    u32x4 code[NM];
    uint64_t scale[NM][kQ4Cols / G];
};

template <int NM, int G, bool NT>
__device__ __forceinline__ void q4_load(Q4Block<NM, G> &b, const uint8_t *const (&w)[NM], int kt)
{
    const int lane = threadIdx.x % cdk::kWave;
#pragma unroll
    for (int q = 0; q < NM; ++q) {
        const uint8_t *p = w[q] + (size_t)kt * q4_block(G);
        b.code[q] = ad_load16<NT>(reinterpret_cast<const uint16_t *>(p + lane * 16));
#pragma unroll
        for (int g = 0; g < kQ4Cols / G; ++g)
            b.scale[q][g] = *reinterpret_cast<const uint64_t *>(p + 1024 + g * 32 + lane / 16 * 8);
    }
}

// the 8 weights of a word as an MFMA operand, each 24 too large
__device__ __forceinline__ u32x4 q4_operand(uint32_t w)
{
    constexpr uint32_t mask = 0x00780078u, one = 0x41804180u;
    return u32x4{(w << 3 & mask) | one, (w >> 1 & mask) | one, (w >> 5 & mask) | one, (w >> 9 & mask) | one};
}

// A workgroup per 16 rows; its waves take the blocks of a row tile in turn.
template <int NM, int G, bool NT>
__global__ __launch_bounds__(kQ4Block) void k_q4(const Q4Args a)
{
    __shared__ u32x4 xs[kQ4XUnits + kQ4Tokens];
    const int wave = ad_wave(), lane = threadIdx.x % cdk::kWave, i16 = lane % 16, j = lane / 16;
    const int nkt = (a.cols + kQ4Cols - 1) / kQ4Cols;
    const size_t tile = (size_t)blockIdx.x * nkt * q4_block(G);
    const uint8_t *w[NM];
    w[0] = a.W + tile;
    if constexpr (NM > 1)
        w[1] = a.W2 + tile;

    Q4Block<NM, G> blk[kQ4Flight];
#pragma unroll
    for (int d = 0; d < kQ4Flight; ++d)
        q4_load<NM, G, NT>(blk[d], w, min(wave + d * kQ4Waves, nkt - 1));
    f32x4_t y[NM];
#pragma unroll
    for (int q = 0; q < NM; ++q)
        y[q] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int units = a.chunk / 8, stride = units + 1;  // (+ 1: 16 tokens' units on different banks)
    const u32x4 *xr = xs + min(i16, a.T - 1) * stride + j;  // lanes past the tokens read the last one's
    const uint32_t m24 = 0xC1C0C1C0u;
    const u32x4 minus24 = {m24, m24, m24, m24};

    const int steps = (nkt + kQ4Waves - 1) / kQ4Waves, held = a.chunk / (kQ4Cols * kQ4Waves);
    for (int n0 = 0; n0 < steps; n0 += kQ4Flight) {
#pragma unroll
        for (int d = 0; d < kQ4Flight; ++d) {
            const int n = n0 + d, k = n * kQ4Waves + wave;  // (uniform; n for the workgroup)
            if (n >= steps)
                break;
            if (n % held == 0) {  // the next columns of the tokens
                const int c0 = n * kQ4Waves * kQ4Cols;
                if (n)
                    __syncthreads();
                for (int u = threadIdx.x; u < a.T * units; u += kQ4Block) {
                    const int t = u / units, c = u % units;
                    xs[t * stride + c] = load16(or_zero(c0 + c * 8 < a.cols, a.x + t * a.ldx + c0 + c * 8));
                }
                __syncthreads();
            }
            if (k < nkt) {
                const u32x4 *xp = xr + (n % held * kQ4Waves + wave) * (kQ4Cols / 8);
                u32x4 xv[4];
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    xv[s] = xp[4 * s];
#pragma unroll
                for (int g = 0; g < kQ4Cols / G; ++g) {
                    f32x4_t start = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int s = 0; s < G / 32; ++s)
                        start = mfma16(minus24, xv[g * (G / 32) + s], start);
#pragma unroll
                    for (int q = 0; q < NM; ++q) {
                        f32x4_t acc = start;
#pragma unroll
                        for (int s = 0; s < G / 32; ++s)
                            acc = mfma16(q4_operand(blk[d].code[q][g * (G / 32) + s]), xv[g * (G / 32) + s], acc);
                        const uint32_t lo = (uint32_t)blk[d].scale[q][g], hi = (uint32_t)(blk[d].scale[q][g] >> 32);
                        y[q][0] += acc[0] * cdk::bf16_lo(lo);
                        y[q][1] += acc[1] * cdk::bf16_hi(lo);
                        y[q][2] += acc[2] * cdk::bf16_lo(hi);
                        y[q][3] += acc[3] * cdk::bf16_hi(hi);
                    }
                }
            }
            q4_load<NM, G, NT>(blk[d], w, min(k + kQ4Flight * kQ4Waves, nkt - 1));
        }
    }
    f32x4_t *sums = reinterpret_cast<f32x4_t *>(xs);  // [NM][waves][lane]
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NM; ++q)
        sums[(q * kQ4Waves + wave) * cdk::kWave + lane] = y[q];
    __syncthreads();
    const int row = blockIdx.x * kQ4Rows + j * 4;
    if (wave > 0 || i16 >= a.T || row >= a.rows)
        return;
#pragma unroll
    for (int q = 0; q < NM; ++q)
        for (int v = 1; v < kQ4Waves; ++v)
            y[q] += sums[(q * kQ4Waves + v) * cdk::kWave + lane];
    float o[4];
    if constexpr (NM > 1) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            o[r] = cdk::silu(y[0][r]) * y[1][r];
    } else {
        const size_t at = i16 * a.ldb + row;
        if (!a.base) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                o[r] = y[0][r];
        } else if (a.type == CD_TYPE_F32) {
            const f32x4_t b = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(a.base) + at);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                o[r] = b[r] + y[0][r];
        } else {
            const uint64_t b = *reinterpret_cast<const uint64_t *>(static_cast<const uint16_t *>(a.base) + at);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                o[r] = __uint_as_float((uint32_t)(b >> (16 * r)) << 16) + y[0][r];
        }
    }
    gt_store4(a.out, a.type, i16 * a.ldo + row, o);
}

// The four words' place of 8 columns (c: a multiple of 8) of a row, and its scale's.
__device__ __forceinline__ size_t q4_word_at(int row, int c, int nkt, int group)
{
    return ((size_t)(row / kQ4Rows) * nkt + c / kQ4Cols) * q4_block(group) +
           (16 * (c % 32 / 8) + row % kQ4Rows) * 16 + c % kQ4Cols / 32 * 4;
}

__device__ __forceinline__ size_t q4_scale_at(int row, int g, int nkt, int group)
{
    const int c = g * group;
    return ((size_t)(row / kQ4Rows) * nkt + c / kQ4Cols) * q4_block(group) + 1024 +
           c % kQ4Cols / group * 32 + row % kQ4Rows * 2;
}

__device__ __forceinline__ uint32_t q4_word(const int (&code)[8])
{
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        w |= (uint32_t)(code[e] + 8 & 15) << (e / 2 * 4 + e % 2 * 16);
    return w;
}

struct Q4PackArgs {
    const uint16_t *W;  // [rows][cols] bf16, row stride ldw; or
    size_t ldw;
    const int8_t *codes;    // [rows][cols] and
    const uint16_t *scale;  // [rows][groups]
    int rows, cols, group;
    uint8_t *out;
};

// One thread per row and group of the padded matrix. W is quantised to the nearest code with the
// scale max |w| / 7 of its group, rounded to bf16.
__global__ __launch_bounds__(256) void k_q4_pack(const Q4PackArgs a)
{
    const int nkt = (a.cols + kQ4Cols - 1) / kQ4Cols, groups = nkt * (kQ4Cols / a.group);
    const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(id / groups), g = (int)(id % groups), c0 = g * a.group;
    if (row >= (a.rows + kQ4Rows - 1) / kQ4Rows * kQ4Rows)
        return;
    const int end = row < a.rows ? min(a.group, a.cols - c0) : 0;  // columns of the matrix (<= 0: none)
    uint16_t scale = 0;
    float div = 0.0f;
    if (a.W) {
        const uint16_t *w = a.W + row * a.ldw + c0;
        float top = 0.0f;
        bool bad = false;
        for (int c = 0; c < end; ++c) {
            const float v = fabsf(cdk::bf16_lo(w[c]));
            bad |= !(v < INFINITY);
            top = fmaxf(top, v);
        }
        scale = bad ? 0x7fc0 : (uint16_t)ad_pack(top / 7.0f, 0.0f);  // a number that is not finite: NaN
        div = bad ? 0.0f : cdk::bf16_lo(scale);
    } else if (end > 0) {
        scale = a.scale[(size_t)row * ((a.cols + a.group - 1) / a.group) + g];
    }
    for (int c = 0; c < a.group; c += 8) {
        int code[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            code[e] = 0;
            if (c + e >= end)
                continue;
            if (!a.W)
                code[e] = a.codes[(size_t)row * a.cols + c0 + c + e];
            else if (div > 0.0f)
                code[e] = (int)fminf(fmaxf(rintf(cdk::bf16_lo(a.W[row * a.ldw + c0 + c + e]) / div), -8.0f), 7.0f);
        }
        *reinterpret_cast<uint32_t *>(a.out + q4_word_at(row, c0 + c, nkt, a.group)) = q4_word(code);
    }
    *reinterpret_cast<uint16_t *>(a.out + q4_scale_at(row, g, nkt, a.group)) = scale;
}

// W[row][c..c + 7] = scale code, rounded to bf16
__global__ __launch_bounds__(256) void k_q4_unpack(const uint8_t *packed, int rows, int cols, int group,
                                                   uint16_t *W, size_t ldw)
{
    const int nkt = (cols + kQ4Cols - 1) / kQ4Cols;
    const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(id / (cols / 8)), c = (int)(id % (cols / 8)) * 8;
    if (row >= rows)
        return;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(packed + q4_word_at(row, c, nkt, group));
    const float s = cdk::bf16_lo(*reinterpret_cast<const uint16_t *>(packed + q4_scale_at(row, c / group, nkt, group)));
    u32x4 o;
#pragma unroll
    for (int p = 0; p < 4; ++p)
        o[p] = ad_pack(s * (float)((int)(w >> (4 * p) & 15) - 8), s * (float)((int)(w >> (16 + 4 * p) & 15) - 8));
    *reinterpret_cast<u32x4 *>(W + row * ldw + c) = o;
}

cd_status q4_shape(int rows, int cols, int group)
{
    if (rows < 8 || rows % 8 || cols < 8 || cols % 8 || (group != 32 && group != 64 && group != 128))
        return CD_EINVAL;
    return rows > kQ4MaxDim || cols > kQ4MaxDim ? CD_EUNSUPPORTED : CD_OK;
}

size_t q4_bytes(int rows, int cols, int group)
{
    return (size_t)ad_ceil(rows, kQ4Rows) * ad_ceil(cols, kQ4Cols) * q4_block(group);
}

template <int NM, int G>
void q4_launch(const Q4Args &a, hipStream_t s)
{
    const int grid = ad_ceil(a.rows, kQ4Rows);
    if (NM * q4_bytes(a.rows, a.cols, G) > ((size_t)64 << 20))
        k_q4<NM, G, true><<<grid, kQ4Block, 0, s>>>(a);
    else
        k_q4<NM, G, false><<<grid, kQ4Block, 0, s>>>(a);
}

template <int NM>
cd_status q4_run(Q4Args a, int group, hipStream_t s)
{
    const int whole = ad_ceil(a.cols, kQ4Cols * kQ4Waves) * kQ4Cols * kQ4Waves;
    a.chunk = std::min(whole, kQ4XUnits / a.T / (kQ4Cols * kQ4Waves / 8) * (kQ4Cols * kQ4Waves));
    if (group == 32)
        q4_launch<NM, 32>(a, s);
    else if (group == 64)
        q4_launch<NM, 64>(a, s);
    else
        q4_launch<NM, 128>(a, s);
    return launched(hipGetLastError());
}

cd_status q4_check(const Q4Args &a, int group, bool gated)
{
    const cd_status st = q4_shape(a.rows, a.cols, group);
    if (st == CD_EINVAL || a.T < 0 || (a.type != CD_TYPE_F32 && a.type != CD_TYPE_BF16) || !a.W || !aligned16(a.W) ||
        (gated && (!a.W2 || !aligned16(a.W2))))
        return CD_EINVAL;
    if (st != CD_OK)
        return st;
    if (a.T > 0 && (!a.x || !aligned16(a.x) || !ad_ld_ok(a.ldx, a.cols) || !a.out || !aligned16(a.out) ||
                    !ad_ld_ok(a.ldo, a.rows) || (a.base && (!aligned16(a.base) || !ad_ld_ok(a.ldb, a.rows)))))
        return CD_EINVAL;
    const size_t es = ad_size(a.type), w = q4_bytes(a.rows, a.cols, group);
    const AdRows out{a.out, a.rows * es, a.ldo * es, a.T}, base{a.base, a.rows * es, a.ldb * es, a.T};
    if (ad_overlap(out, {a.x, (size_t)a.cols * 2, a.ldx * 2, a.T}) || ad_overlap(out, ad_flat(a.W, w)) ||
        ad_overlap(out, ad_flat(a.W2, w)) || (!(a.base == a.out && a.ldb == a.ldo) && ad_overlap(out, base)))
        return CD_EINVAL;
    return a.T > kQ4Tokens ? CD_EUNSUPPORTED : CD_OK;
}

cd_status q4_pack(const Q4PackArgs &a, hipStream_t s)
{
    const size_t threads = (size_t)ad_ceil(a.rows, kQ4Rows) * kQ4Rows * ad_ceil(a.cols, kQ4Cols) * (kQ4Cols / a.group);
    k_q4_pack<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
    return launched(hipGetLastError());
}

}  // namespace

extern "C" {

size_t countdown_q4_bytes(int rows, int cols, int group)
{
    return q4_shape(rows, cols, group) == CD_OK ? q4_bytes(rows, cols, group) : 0;
}

cd_status countdown_q4_quantize(const uint16_t *W, size_t ldw, int rows, int cols, int group, void *packed,
                                void *stream)
{
    const cd_status st = q4_shape(rows, cols, group);
    if (st == CD_EINVAL || !W || !aligned16(W) || !packed || !aligned16(packed))
        return CD_EINVAL;
    if (st != CD_OK)
        return st;
    if (!ad_ld_ok(ldw, cols) || ad_overlap({W, (size_t)cols * 2, ldw * 2, rows},
                                           ad_flat(packed, q4_bytes(rows, cols, group))))
        return CD_EINVAL;
    return q4_pack({W, ldw, nullptr, nullptr, rows, cols, group, static_cast<uint8_t *>(packed)},
                   reinterpret_cast<hipStream_t>(stream));
}

cd_status countdown_q4_pack(const int8_t *codes, const uint16_t *scale, int rows, int cols, int group,
                            void *packed, void *stream)
{
    const cd_status st = q4_shape(rows, cols, group);
    if (st == CD_EINVAL || !codes || !aligned16(codes) || !scale || !aligned16(scale) || !packed ||
        !aligned16(packed))
        return CD_EINVAL;
    if (st != CD_OK)
        return st;
    const AdRows out = ad_flat(packed, q4_bytes(rows, cols, group));
    if (ad_overlap(out, ad_flat(codes, (size_t)rows * cols)) ||
        ad_overlap(out, ad_flat(scale, (size_t)rows * ad_ceil(cols, group) * 2)))
        return CD_EINVAL;
    return q4_pack({nullptr, 0, codes, scale, rows, cols, group, static_cast<uint8_t *>(packed)},
                   reinterpret_cast<hipStream_t>(stream));
}

cd_status countdown_q4_unpack(const void *packed, int rows, int cols, int group, uint16_t *W, size_t ldw,
                              void *stream)
{
    const cd_status st = q4_shape(rows, cols, group);
    if (st == CD_EINVAL || !W || !aligned16(W) || !packed || !aligned16(packed))
        return CD_EINVAL;
    if (st != CD_OK)
        return st;
    if (!ad_ld_ok(ldw, cols) || ad_overlap({W, (size_t)cols * 2, ldw * 2, rows},
                                           ad_flat(packed, q4_bytes(rows, cols, group))))
        return CD_EINVAL;
    const size_t threads = (size_t)rows * (cols / 8);
    k_q4_unpack<<<(unsigned)((threads + 255) / 256), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(
        static_cast<const uint8_t *>(packed), rows, cols, group, W, ldw);
    return launched(hipGetLastError());
}

cd_status countdown_q4_project(const uint16_t *x, size_t ldx, int T, const void *W, int d_in, int d_out,
                               int group, int type, const void *base, size_t ldb, void *y, size_t ldy,
                               void *stream)
{
    const Q4Args a{x, ldx, static_cast<const uint8_t *>(W), nullptr, T, d_out, d_in, base, ldb, y, ldy, type, 0};
    const cd_status st = q4_check(a, group, false);
    return st != CD_OK || T == 0 ? st : q4_run<1>(a, group, reinterpret_cast<hipStream_t>(stream));
}

cd_status countdown_q4_gated(const uint16_t *x, size_t ldx, int T, const void *W_gate, const void *W_up,
                             int d_model, int d_ff, int group, int type, void *h, size_t ldh, void *stream)
{
    const Q4Args a{x, ldx, static_cast<const uint8_t *>(W_gate), static_cast<const uint8_t *>(W_up), T, d_ff,
                   d_model, nullptr, 0, h, ldh, type, 0};
    const cd_status st = q4_check(a, group, true);
    return st != CD_OK || T == 0 ? st : q4_run<2>(a, group, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
