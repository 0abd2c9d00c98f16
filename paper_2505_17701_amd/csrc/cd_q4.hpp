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
// Roundings are thus those of sums over 24 + code: 2-norm errors of 4096 columns 0.9e-7 to 1.2e-7 with codes over -8..7
// (fp32 sums of the weights themselves 2.6e-7), but 1.5e-7 (G 32) to 5.2e-7 (G 128) with codes of -1..1 (1.3e-7),
// and zero codes need not give 0. Sums of 24 and of 24 + code side by side, and their difference, give 0 there; other
// errors are then up to twice as large, and G 32 up to 9 % slower (16 tokens of 8192 -> 28672 gated 77 us against 70).
//
// Packed layout: blocks of 16 rows x 128 columns, the blocks of 16 rows one after another in groups of eight
// (the last group may have fewer): the codes of a group's blocks, 1024 bytes each, then their
// scales, 32 bytes for each of the 128 / G groups of columns of a block (16 rows). Lane l = 16 j + i of
// a wave owns bytes 16 l..16 l + 15 of a block's codes: word w holds row i, columns 32 w + 8 j + e; the code of
// e = 2 p lies at bits 4 p, that of e = 2 p + 1 at bits 16 + 4 p, each as c + 8. So a wave's load is 1 KB
// on end and each word is an operand. Rows and columns that pad the matrix have code 0 and scale 0.
#pragma once

#include "cd_device.hpp"

namespace {

constexpr int kQ4MaxDim = 65536, kQ4Tokens = 16;
constexpr int kQ4Rows = 16, kQ4Cols = 128;  // of a block

constexpr int kQ4Group = 8;  // blocks whose codes lie together

__host__ __device__ constexpr int q4_block(int group) { return 1024 + 32 * (kQ4Cols / group); }

// byte offsets of a block's codes and scales from its row tile of nkt blocks (at most 512 of 1152 bytes)
__host__ __device__ constexpr int q4_codes_at(int kt, int group)
{
    return kt / kQ4Group * kQ4Group * q4_block(group) + kt % kQ4Group * 1024;
}

__host__ __device__ constexpr int q4_scales_at(int kt, int nkt, int group)
{
    const int first = kt / kQ4Group * kQ4Group, n = nkt - first < kQ4Group ? nkt - first : kQ4Group;
    return first * q4_block(group) + n * 1024 + (kt - first) * 32 * (kQ4Cols / group);
}

struct Q4Args {
    const uint16_t *x;
    size_t ldx;
    const uint8_t *W, *W2;  // packed (gated: W_gate, W_up)
    int T, rows, cols;
    const void *base;
    size_t ldb;
    void *out;
    size_t ldo;
    int type;  // of base and out
};

// the 8 weights of a word as an MFMA operand, each 24 too large
__device__ __forceinline__ u32x4 q4_operand(uint32_t w, uint32_t mask, uint32_t one)
{
    return u32x4{(w << 3 & mask) | one, (w >> 1 & mask) | one, (w >> 5 & mask) | one, (w >> 9 & mask) | one};
}

// out of four rows
__device__ __forceinline__ void q4_store(const Q4Args &a, int t, int row, const f32x4_t &y)
{
    f32x4_t o = y;
    const size_t at = t * a.ldb + row;
    if (a.base && a.type == CD_TYPE_F32) {
        const f32x4_t b = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(a.base) + at);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            o[r] += b[r];
    } else if (a.base) {
        const uint64_t b = *reinterpret_cast<const uint64_t *>(static_cast<const uint16_t *>(a.base) + at);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            o[r] += __uint_as_float((uint32_t)(b >> (16 * r)) << 16);
    }
    gt_store4(a.out, a.type, t * a.ldo + row, o);
}

// Stages of LDS: what leaves two workgroups a CU, if that is three, else three; at most four (each costs
// its loads before the first product)
__host__ __device__ constexpr int q4_stages(int stage)
{
    const int n = 80 * 1024 / stage;
    return n < 3 ? 3 : n < 4 ? n : 4;
}

// Bound by the stream of the codes and, with many tokens, by that of the tokens (each workgroup reads them
// all from L2; two row tiles a part halve that): 8192 -> 28672 gated at one token, 242 MB, 46 us (5.2 TB/s; the
// same loads without products 43, a plain stream 35); 4096 -> 11008 gated at 13 tokens, 51 MB, 19.6 (the loads alone
// 16.4, products alone 12.3); 14336 -> 4096 at 1, 8 and 16 tokens 11.0, 12.6 and 14.3, the loads alone 8.4, 11.9 and 13.7
// (products alone 8.7 to 9). Deeper rings, tokens whole in LDS and twice the waves measured the same or slower.
//
// A part is 16 rows of both matrices (gated), or NM x 16 rows of one; a workgroup takes part after part. A
// step is 1024 columns, a block of each of NM row tiles for each wave; its codes, scales and tokens go to
// LDS without passing registers, kStages - 1 steps ahead, the next part's while the last one ends.
// XT: the tokens that LDS has room for.
template <int NM, int G, int XT, int WAVES, bool GATED, bool NT>
__global__ __launch_bounds__(WAVES *cdk::kWave) void k_q4(const Q4Args a)
{
    constexpr int kStep = WAVES * kQ4Cols, kHalf = cdk::kWave * 8;  // columns of a step, of a load
    constexpr int kScale = 32 * (kQ4Cols / G), kCodes = WAVES * NM * 1024, kScales = WAVES * NM * kScale;
    constexpr int kXRow = kStep * 2 + 16;  // (+ 16: 16 tokens' columns on different banks)
    constexpr int kStage = kCodes + kScales + XT * kXRow;
    constexpr int XL = XT / 4;  // the loads of tokens that a wave makes for a step
    constexpr int kStages = q4_stages(kStage);
    static_assert(XL * WAVES >= XT * (kStep / kHalf) && WAVES % NM == 0 && (kStages - 2) * (NM + 1 + XL) < 64, "loads");
    __shared__ __align__(1024) char lds[kStages * kStage];
    const int wave = ad_wave(), lane = threadIdx.x % cdk::kWave, i16 = lane % 16, j = lane / 16;
    const int nkt = (a.cols + kQ4Cols - 1) / kQ4Cols, steps = (nkt + WAVES - 1) / WAVES;
    const int tiles = (a.rows + kQ4Rows - 1) / kQ4Rows;
    const int parts = (tiles + (GATED ? 0 : NM - 1)) / (GATED ? 1 : NM);
    const uint8_t *w[NM];  // the row tiles that are loaded next
    int ahead = blockIdx.x, next = 0;  // their part, and the step
    const auto begin = [&]() {
#pragma unroll
        for (int q = 0; q < NM; ++q) {
            const int tile = GATED ? ahead : min(ahead * NM + q, tiles - 1);
            w[q] = (GATED && q ? a.W2 : a.W) + (size_t)tile * nkt * q4_block(G);
        }
    };
    begin();
    // Load i of the tokens: 64 lanes of 8 columns of one of them. With many tokens every wave makes as
    // many loads a step (past the last token that one again) and takes the scales of NM blocks; with few, waves
    // without a token make fewer, and wave q takes all scales of matrix q. (One way for all: 8192 -> 28672 gated at
    // one token 48.7 us against 46.8, 3000 -> 8008 at 16 tokens 7.6 against 7.4.)
    constexpr bool kEven = XL > 2;
    constexpr int kPer = kStep / kHalf;
    const uint16_t *xp[XL];
    int xcol[XL], xloads = 0;
    uint32_t xat[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int n = min(wave + i * WAVES, kPer * a.T - 1);
        xloads += kEven || wave + i * WAVES < kPer * a.T;
        xp[i] = a.x + n / kPer * a.ldx;
        xcol[i] = n % kPer * kHalf + lane * 8;
        xat[i] = kCodes + kScales + n / kPer * kXRow + n % kPer * 1024;
    }
    const int sq = kEven ? wave % NM : wave, sfirst = kEven ? wave / NM * NM : 0;
    constexpr int kSLanes = (kEven ? NM : WAVES) * kScale / 16;
    const int loads = xloads + (kEven || wave < NM);
    const auto wait = [&]() {  // the loads of the last kStages - 2 steps may be in flight
#pragma unroll
        for (int n = kEven ? XL + 1 : 0; n <= XL + 1; ++n)
            if (kEven || loads == n)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages - 2) * (NM + n)) : "memory");
        asm volatile("s_barrier" ::: "memory");
    };
    const uint32_t base = gt_lds(lds);
    const auto issue = [&](int stage) {
        const uint32_t at = base + stage * kStage;
        const int first = next * WAVES, kt = first + wave;
        const bool in = ahead < parts;  // uniform
#pragma unroll
        for (int q = 0; q < NM; ++q)
            gt_load_lds<NT>(gt_resource(w[q] + q4_codes_at(kt, G)), in && kt < nkt ? lane * 16 : kGtOutside,
                            at + (q * WAVES + wave) * 1024);
        if ((kEven || wave < NM) && lane < kSLanes) {
            const u32x4 r = gt_resource((sq ? w[NM - 1] : w[0]) + q4_scales_at(first + sfirst, nkt, G));
            gt_load_lds<NT>(r, in && lane * 16 < (nkt - first - sfirst) * kScale ? lane * 16 : kGtOutside,
                            at + kCodes + (sq * WAVES + sfirst) * kScale);
        }
#pragma unroll
        for (int i = 0; i < XL; ++i)
            if (kEven || i < xloads)
                gt_load_lds(gt_resource(xp[i]),
                            next * kStep + xcol[i] < a.cols ? (next * kStep + xcol[i]) * 2 : kGtOutside, at + xat[i]);
        if (++next == steps) {
            next = 0;
            ahead += gridDim.x;
            begin();
        }
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        issue(s);

    const uint32_t m24 = 0xC1C0C1C0u;
    const u32x4 minus24 = {m24, m24, m24, m24};
    // In registers, which the compiler cannot see through: as literals they would cost an instruction more a pair.
    uint32_t mask, one;
    asm("s_mov_b32 %0, 0x00780078" : "=s"(mask));
    asm("v_mov_b32 %0, 0x41804180" : "=v"(one));
    // lanes past the tokens read the last one's
    const int xread = kCodes + kScales + min(i16, a.T - 1) * kXRow + wave * (kQ4Cols * 2) + j * 16;
    int stage = 0;
    for (int part = blockIdx.x; part < parts; part += gridDim.x) {
        f32x4_t y[NM];
#pragma unroll
        for (int q = 0; q < NM; ++q)
            y[q] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        char *done = lds;  // the last step's codes
        for (int n = 0; n < steps; ++n) {
            wait();
            issue(stage == 0 ? kStages - 1 : stage - 1);
            char *s = done = lds + stage * kStage;
            stage = stage + 1 == kStages ? 0 : stage + 1;
            u32x4 xv[4], code[NM];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                xv[k] = *reinterpret_cast<const u32x4 *>(s + xread + k * 64);
#pragma unroll
            for (int q = 0; q < NM; ++q)
                code[q] = *reinterpret_cast<const u32x4 *>(s + (q * WAVES + wave) * 1024 + lane * 16);
#pragma unroll
            for (int g = 0; g < kQ4Cols / G; ++g) {
                f32x4_t start = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < G / 32; ++k)
                    start = mfma16(minus24, xv[g * (G / 32) + k], start);
#pragma unroll
                for (int q = 0; q < NM; ++q) {
                    const uint64_t scale =
                        *reinterpret_cast<const uint64_t *>(s + kCodes + (q * WAVES + wave) * kScale + g * 32 + j * 8);
                    f32x4_t acc = start;
#pragma unroll
                    for (int k = 0; k < G / 32; ++k)
                        acc = mfma16(q4_operand(code[q][g * (G / 32) + k], mask, one), xv[g * (G / 32) + k], acc);
                    const uint32_t lo = (uint32_t)scale, hi = (uint32_t)(scale >> 32);
                    y[q][0] += acc[0] * cdk::bf16_lo(lo);
                    y[q][1] += acc[1] * cdk::bf16_hi(lo);
                    y[q][2] += acc[2] * cdk::bf16_lo(hi);
                    y[q][3] += acc[3] * cdk::bf16_hi(hi);
                }
            }
        }
        // The waves' sums, each over the codes that it alone read. (They are read before the next barrier,
        // and overwritten by loads after it.)
#pragma unroll
        for (int q = 0; q < NM; ++q)
            reinterpret_cast<f32x4_t *>(done)[(q * WAVES + wave) * cdk::kWave + lane] = y[q];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (GATED ? wave > 0 : wave >= NM)
            continue;
        const auto total = [&](int q) {
            const f32x4_t *sums = reinterpret_cast<const f32x4_t *>(done) + q * WAVES * cdk::kWave + lane;
            f32x4_t v = sums[0];
#pragma unroll
            for (int k = 1; k < WAVES; ++k)
                v += sums[k * cdk::kWave];
            return v;
        };
        const int row = (GATED ? part : part * NM + wave) * kQ4Rows + j * 4;
        if (i16 >= a.T || row >= a.rows)
            continue;
        if constexpr (GATED) {
            const f32x4_t g = total(0), u = total(1);
            q4_store(a, i16, row, f32x4_t{g[0] * gt_sigmoid(g[0]) * u[0], g[1] * gt_sigmoid(g[1]) * u[1],
                                          g[2] * gt_sigmoid(g[2]) * u[2], g[3] * gt_sigmoid(g[3]) * u[3]});
        } else {
            q4_store(a, i16, row, total(wave));
        }
    }
    gt_wait<0>();  // no load outlives the workgroup's LDS
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

// A wave's block: tile of rows, block of columns; a lane has row `row` and the chunks of 8 columns col + 32 w,
// w = 0..3, one word of codes each.
struct Q4Place {
    int tile, kt, row, col;
    size_t base;  // the row tile's first byte

    __device__ __forceinline__ Q4Place(int nkt, int group)
    {
        const int lane = threadIdx.x % cdk::kWave;
        const size_t id = (size_t)blockIdx.x * (256 / cdk::kWave) + ad_wave();
        tile = (int)(id / nkt);
        kt = (int)(id % nkt);
        row = tile * kQ4Rows + lane % 16;
        col = kt * kQ4Cols + lane / 16 * 8;
        base = (size_t)tile * nkt * q4_block(group);
    }
};

// A wave a block. W is quantised to the nearest code with the scale max |w| / 7 of its group, rounded to
// bf16. Bound by memory: 28672 x 8192, 189 us, from given codes 138 (a thread for each group of a row 7478 and 749).
__global__ __launch_bounds__(256) void k_q4_pack(const Q4PackArgs a)
{
    const int nkt = (a.cols + kQ4Cols - 1) / kQ4Cols, lane = threadIdx.x % cdk::kWave;
    const Q4Place p(nkt, a.group);
    if (p.tile * kQ4Rows >= a.rows)
        return;
    bool in[4];
    u32x4 v[4], out;
    uint32_t scale[4];  // of each chunk's group
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int c = p.col + 32 * w, g = c / a.group;
        in[w] = p.row < a.rows && c < a.cols;
        v[w] = u32x4{0u, 0u, 0u, 0u};
        scale[w] = 0u;
        if (in[w] && a.W) {
            v[w] = load16(a.W + p.row * a.ldw + c);
        } else if (in[w]) {
            const uint64_t q = *reinterpret_cast<const uint64_t *>(a.codes + (size_t)p.row * a.cols + c);
            v[w][0] = (uint32_t)q;
            v[w][1] = (uint32_t)(q >> 32);
        }
        if (!a.W && p.row < a.rows && g * a.group < a.cols)
            scale[w] = a.scale[(size_t)p.row * ((a.cols + a.group - 1) / a.group) + g];
    }
    if (a.W) {
        uint32_t top[4];  // the largest magnitude, as bits: they order like their numbers, infinity and NaN last
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            top[w] = 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top[w] = max(top[w], max(v[w][e] & 0x7fffu, v[w][e] >> 16 & 0x7fffu));
            top[w] = max(top[w], (uint32_t)__shfl_xor((int)top[w], 16));
            top[w] = max(top[w], (uint32_t)__shfl_xor((int)top[w], 32));
        }
        if (a.group > 32) {
            top[0] = top[1] = max(top[0], top[1]);
            top[2] = top[3] = max(top[2], top[3]);
        }
        if (a.group > 64)
            top[0] = top[1] = top[2] = top[3] = max(top[0], top[2]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {  // a number that is not finite: NaN
            scale[w] = top[w] >= 0x7f80u ? 0x7fc0u : ad_pack(__uint_as_float(top[w] << 16) / 7.0f, 0.0f) & 0xffffu;
            const float div = __uint_as_float(scale[w] << 16);
            int code[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = e % 2 ? cdk::bf16_hi(v[w][e / 2]) : cdk::bf16_lo(v[w][e / 2]);
                code[e] = div > 0.0f ? (int)fminf(fmaxf(rintf(x / div), -8.0f), 7.0f) : 0;
            }
            out[w] = q4_word(code);
        }
    } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            int code[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                code[e] = (int)(v[w][e / 4] >> (8 * (e % 4)));
            out[w] = q4_word(code);
        }
    }
    *reinterpret_cast<u32x4 *>(a.out + p.base + q4_codes_at(p.kt, a.group) + lane * 16) = out;
    uint16_t *scales = reinterpret_cast<uint16_t *>(a.out + p.base + q4_scales_at(p.kt, nkt, a.group));
#pragma unroll
    for (int w = 0; w < 4; ++w)
        if (lane / 16 == w && w % (a.group / 32) == 0)
            scales[w / (a.group / 32) * kQ4Rows + lane % 16] = (uint16_t)scale[w];
}

// W = scale code, rounded to bf16; a wave a block. 28672 x 8192: 147 us (590 MB; a thread for each word 160).
__global__ __launch_bounds__(256) void k_q4_unpack(const uint8_t *packed, int rows, int cols, int group,
                                                   uint16_t *W, size_t ldw)
{
    const int nkt = (cols + kQ4Cols - 1) / kQ4Cols, lane = threadIdx.x % cdk::kWave;
    const Q4Place p(nkt, group);
    if (p.tile * kQ4Rows >= rows)
        return;
    const u32x4 code = *reinterpret_cast<const u32x4 *>(packed + p.base + q4_codes_at(p.kt, group) + lane * 16);
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(packed + p.base + q4_scales_at(p.kt, nkt, group));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float s = cdk::bf16_lo(scales[32 * w / group * kQ4Rows + lane % 16]);
        u32x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            o[q] = ad_pack(s * (float)((int)(code[w] >> (4 * q) & 15) - 8),
                           s * (float)((int)(code[w] >> (16 + 4 * q) & 15) - 8));
        if (p.row < rows && p.col + 32 * w < cols)
            *reinterpret_cast<u32x4 *>(W + p.row * ldw + p.col + 32 * w) = o;
    }
}

// workgroups of four waves, a wave for each block
unsigned q4_blocks(int rows, int cols)
{
    return (unsigned)(((size_t)ad_ceil(rows, kQ4Rows) * ad_ceil(cols, kQ4Cols) + 3) / 4);
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

template <int NM, int G, int XT, int W, bool GATED>
void q4_launch(const Q4Args &a, int parts, hipStream_t s)
{
    // persistent: as many workgroups as run at once
    constexpr int stage = W * NM * q4_block(G) + XT * (W * kQ4Cols * 2 + 16);
    const int grid = std::min(parts, 256 * (160 * 1024 / (q4_stages(stage) * stage)));
    if ((GATED ? 2 : 1) * q4_bytes(a.rows, a.cols, G) > ((size_t)64 << 20))
        k_q4<NM, G, XT, W, GATED, true><<<grid, W * cdk::kWave, 0, s>>>(a);
    else
        k_q4<NM, G, XT, W, GATED, false><<<grid, W * cdk::kWave, 0, s>>>(a);
}

// Many tokens and more parts than CUs: two workgroups of four waves a CU, whose steps are half as large
// (16 tokens, 4096 -> 11008 gated 17.3 us against 19.2; 14336 -> 4096, 256 parts, 16.3 against 14.0).
template <int NM, int G, int XT, bool GATED>
void q4_launch(const Q4Args &a, hipStream_t s)
{
    const int parts = ad_ceil(a.rows, kQ4Rows * (GATED ? 1 : NM));
    if (XT > 8 && parts > 256)
        q4_launch<NM, G, XT, (XT > 8 ? 4 : 8), GATED>(a, parts, s);
    else
        q4_launch<NM, G, XT, 8, GATED>(a, parts, s);
}

template <int NM, int G, bool GATED>
void q4_launch(const Q4Args &a, hipStream_t s)
{
    constexpr bool few = GATED || NM == 1;  // (two row tiles of one matrix: from five tokens on)
    if (few && a.T <= 4)
        q4_launch<NM, G, few ? 4 : 8, GATED>(a, s);
    else if (a.T <= 8)
        q4_launch<NM, G, 8, GATED>(a, s);
    else
        q4_launch<NM, G, 16, GATED>(a, s);
}

template <int NM, bool GATED>
cd_status q4_run(const Q4Args &a, int group, hipStream_t s)
{
    if (group == 32)
        q4_launch<NM, 32, GATED>(a, s);
    else if (group == 64)
        q4_launch<NM, 64, GATED>(a, s);
    else
        q4_launch<NM, 128, GATED>(a, s);
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
    k_q4_pack<<<q4_blocks(a.rows, a.cols), 256, 0, s>>>(a);
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
    k_q4_unpack<<<q4_blocks(rows, cols), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(
        static_cast<const uint8_t *>(packed), rows, cols, group, W, ldw);
    return launched(hipGetLastError());
}

cd_status countdown_q4_project(const uint16_t *x, size_t ldx, int T, const void *W, int d_in, int d_out,
                               int group, int type, const void *base, size_t ldb, void *y, size_t ldy,
                               void *stream)
{
    const Q4Args a{x, ldx, static_cast<const uint8_t *>(W), nullptr, T, d_out, d_in, base, ldb, y, ldy, type};
    const cd_status st = q4_check(a, group, false);
    if (st != CD_OK || T == 0)
        return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    // Two row tiles a workgroup, which then read the tokens once, where there are enough of either (16
    // tokens, 4096 -> 14336 12.7 us against 15.4, 6144 7.6 against 8.2, 4096 7.4 against 6.2; one token, 4096 ->
    // 14336 11.5 against 10.8).
    return T > 4 && d_out >= 6144 ? q4_run<2, false>(a, group, s) : q4_run<1, false>(a, group, s);
}

cd_status countdown_q4_gated(const uint16_t *x, size_t ldx, int T, const void *W_gate, const void *W_up,
                             int d_model, int d_ff, int group, int type, void *h, size_t ldh, void *stream)
{
    const Q4Args a{x, ldx, static_cast<const uint8_t *>(W_gate), static_cast<const uint8_t *>(W_up), T, d_ff,
                   d_model, nullptr, 0, h, ldh, type};
    const cd_status st = q4_check(a, group, true);
    return st != CD_OK || T == 0 ? st : q4_run<2, true>(a, group, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
