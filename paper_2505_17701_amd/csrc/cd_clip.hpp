// The global gradient norm over many tensors, and clipping. Part of cd_api.hip (its only
// includer).
//
//   norm = sqrt(sum g^2),   out = g * min(1, max_norm / norm).
//
// The scale depends on every gradient, so gradients that do not fit the caches are read
// twice and written once; nothing else moves. Squares are formed and added in fp64: the
// product of two fp32 values is exact there, no gradient overflows, and the sum's order is
// fixed (a chunk's elements by thread, the threads of a workgroup by a tree, the
// workgroups' sums by index), so the norm has the same bits whatever the timing.
#pragma once

#include <algorithm>
#include <vector>

#include "cd_device.hpp"

namespace {

constexpr int kClipTensors = 96;        // tensors per launch: the table is a kernel argument (3 KB)
// bytes per step of a workgroup: eight 16-byte vectors for each thread, which the norm has in flight
// together (the scaling loads each behind the store before it, since the two may be one tensor). 671 MB of
// fp32 gradients 142 + 226 us, with twice as many 146 + 232; 67 MB of bf16 14.3 us, with half as many 16.8
constexpr unsigned kClipChunk = 32768;
// workgroups per launch of the norm, at most: its registers let 1024 run at once. With 1024 as the most
// (a call in a graph): the norm of 671 MB of fp32 120.5 us, the same, of 67 MB of bf16 17.1 against 17.9; clipping
// the 671 MB 374 against 371
constexpr unsigned kClipGroups = 2048;
constexpr unsigned kClipScaleGroups = 768;  // where they also write: 512 take 273 us for 671 MB, 768 227, 1024 230, 2048 248
constexpr int kClipBlock = 256;

struct ClipEntry {
    const void *grad;
    void *out;
    uint64_t count;
    uint32_t chunk0;  // its first chunk
    uint32_t type;
};

struct ClipTable {
    int n;
    unsigned chunk[2];  // elements of a chunk, by type
    uint64_t chunks;  // of all tensors
    ClipEntry entry[kClipTensors];
};

struct ClipChunk {
    int t;           // entry
    uint64_t first;  // its first element
    unsigned n;      // elements
};

// the tensor and range of chunk c
__device__ __forceinline__ ClipChunk clip_chunk(const ClipTable &a, unsigned c)
{
    int lo = 0, hi = a.n - 1;  // the last tensor whose first chunk is <= c
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.entry[mid].chunk0 <= c)
            lo = mid;
        else
            hi = mid - 1;
    }
    ClipChunk r;
    r.t = lo;
    const unsigned chunk = a.chunk[a.entry[lo].type];
    r.first = (uint64_t)(c - a.entry[lo].chunk0) * chunk;
    const uint64_t left = a.entry[lo].count - r.first;
    r.n = left < chunk ? (unsigned)left : chunk;
    return r;
}

// elements of a chunk before the first 16-byte boundary of p
template <class T>
__device__ __forceinline__ unsigned clip_lead(const T *p, unsigned n)
{
    return min(n, (unsigned)((16u - (unsigned)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) /
                      (unsigned)sizeof(T));
}

__device__ __forceinline__ double square(float v) { return (double)v * (double)v; }
__device__ __forceinline__ float clip_value(float v) { return v; }
__device__ __forceinline__ float clip_value(uint16_t v) { return cdk::bf16_lo(v); }
template <class T>
__device__ __forceinline__ void square16(const cdk::u32x4 &v, double (&s)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if constexpr (sizeof(T) == 4) {
            s[i] += square(__uint_as_float(v[i]));
        } else {
            s[i] += square(cdk::bf16_lo(v[i]));
            s[i] += square(cdk::bf16_hi(v[i]));
        }
}

// (thread `at` of BLOCK, here and below)
template <int BLOCK, class T>
__device__ __forceinline__ double clip_squares(const T *p, unsigned n, unsigned at)
{
    constexpr unsigned kVec = 16 / sizeof(T);
    const unsigned lead = clip_lead(p, n), vecs = (n - lead) / kVec, done = lead + vecs * kVec;
    const cdk::u32x4 *v = reinterpret_cast<const cdk::u32x4 *>(p + lead);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if (at < lead)
        s[0] += square(clip_value(p[at]));
#pragma unroll 8
    for (unsigned i = at; i < vecs; i += BLOCK)
        square16<T>(v[i], s);
    if (at < n - done)
        s[1] += square(clip_value(p[done + at]));
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// sum over the workgroup, in every thread (butterflies: the same bits everywhere)
template <int BLOCK>
__device__ __forceinline__ double clip_block_sum(double s)
{
    constexpr int kWaves = BLOCK / cdk::kWave;
    __shared__ double waves[kWaves];
#pragma unroll
    for (int d = 1; d < cdk::kWave; d *= 2)
        s += __shfl_xor(s, d);
    if (threadIdx.x % cdk::kWave == 0)
        waves[threadIdx.x / cdk::kWave] = s;
    __syncthreads();
    s = waves[threadIdx.x % kWaves];
#pragma unroll
    for (int d = 1; d < kWaves; d *= 2)
        s += __shfl_xor(s, d);
    return s;
}

// sum of squares of every step-th chunk from `first` on, over BLOCK threads' own parts
template <int BLOCK>
__device__ __forceinline__ double clip_sum(const ClipTable &a, unsigned first, unsigned step, unsigned at)
{
    double s = 0.0;
    for (unsigned c = first; c < a.chunks; c += step) {
        const ClipChunk k = clip_chunk(a, c);
        const void *grad = a.entry[k.t].grad;
        s += a.entry[k.t].type == CD_TYPE_F32
                 ? clip_squares<BLOCK>(static_cast<const float *>(grad) + k.first, k.n, at)
                 : clip_squares<BLOCK>(static_cast<const uint16_t *>(grad) + k.first, k.n, at);
    }
    return s;
}

__global__ __launch_bounds__(kClipBlock) void k_clip_norm(const ClipTable a, double *part)
{
    const double s = clip_block_sum<kClipBlock>(clip_sum<kClipBlock>(a, blockIdx.x, gridDim.x, threadIdx.x));
    if (threadIdx.x == 0)
        part[blockIdx.x] = s;
}

// The sum of the workgroups' sums, in every thread. Each workgroup of the launch that needs it
// adds them for itself (16 KB from L2 for the 96 tensors of one launch): a counter that tells one workgroup
// it is the last makes every other flush its L2 first (2032 of them: 70 us for 67 MB of gradients).
__device__ __forceinline__ double clip_total(const double *part, unsigned parts)
{
    double s = 0.0;
    for (unsigned i = threadIdx.x; i < parts; i += kClipBlock)
        s += part[i];
    return clip_block_sum<kClipBlock>(s);
}

__global__ __launch_bounds__(kClipBlock) void k_clip_total(const double *part, unsigned parts,
                                                           double *norm_out)
{
    const double s = clip_total(part, parts);
    if (threadIdx.x == 0)
        *norm_out = sqrt(s);
}

// The scale max_norm / norm as an fp32 factor and a power of two: below fp32's normal numbers
// (gradients of 3e38 clipped to 1) the quotient alone would lose its bits, or all of it
struct ClipCoef {
    float f;
    int e;  // 0 for the usual quotient, and out = grad * f
};

// a norm that is not finite scales nothing
__device__ __forceinline__ ClipCoef clip_coef(double norm, double max_norm)
{
    if (!(norm > max_norm && norm < (double)INFINITY))
        return {1.0f, 0};
    const double c = max_norm / norm;
    if (c >= (double)__FLT_MIN__)
        return {(float)c, 0};
    return {(float)__builtin_amdgcn_frexp_mant(c), __builtin_amdgcn_frexp_exp(c)};
}

__device__ __forceinline__ bool clip_same(const ClipCoef &c) { return c.f == 1.0f && c.e == 0; }

__device__ __forceinline__ uint32_t bf16_bits(float v)
{
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}
__device__ __forceinline__ float clip_round(float v, float) { return v; }
__device__ __forceinline__ uint16_t clip_round(float v, uint16_t) { return (uint16_t)bf16_bits(v); }

template <class T>
__device__ __forceinline__ cdk::u32x4 scale16(cdk::u32x4 v, float coef)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = sizeof(T) == 4 ? __float_as_uint(__uint_as_float(v[i]) * coef)
                              : bf16_bits(cdk::bf16_lo(v[i]) * coef) |
                                    bf16_bits(cdk::bf16_hi(v[i]) * coef) << 16;
    return v;
}

// coef 1 copies the bits (a NaN's among them)
template <int BLOCK, class T>
__device__ __forceinline__ void clip_scale(const T *p, T *o, unsigned n, const ClipCoef &coef, unsigned at)
{
    constexpr unsigned kVec = 16 / sizeof(T);
    const bool same = clip_same(coef);
    if (coef.e || ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(o)) & 15u) != 0) {
        for (unsigned i = at; i < n; i += BLOCK)
            o[i] = same ? p[i] : clip_round(__builtin_amdgcn_ldexpf(clip_value(p[i]) * coef.f, coef.e), T{});
        return;
    }
    const unsigned lead = clip_lead(p, n), vecs = (n - lead) / kVec, done = lead + vecs * kVec;
    const cdk::u32x4 *v = reinterpret_cast<const cdk::u32x4 *>(p + lead);
    cdk::u32x4 *w = reinterpret_cast<cdk::u32x4 *>(o + lead);
    if (at < lead)
        o[at] = same ? p[at] : clip_round(clip_value(p[at]) * coef.f, T{});
#pragma unroll 8
    for (unsigned i = at; i < vecs; i += BLOCK)
        w[i] = same ? v[i] : scale16<T>(v[i], coef.f);
    if (at < n - done)
        o[done + at] =
            same ? p[done + at] : clip_round(clip_value(p[done + at]) * coef.f, T{});
}

// (BACK: the last chunks first. The norm read them last, they may still be in the last cache)
template <int BLOCK, bool BACK>
__device__ __forceinline__ void clip_scale_all(const ClipTable &a, const ClipCoef &coef, unsigned first,
                                               unsigned step, unsigned at)
{
    for (unsigned c = first; c < a.chunks; c += step) {
        const ClipChunk k = clip_chunk(a, BACK ? (unsigned)a.chunks - 1 - c : c);
        const void *grad = a.entry[k.t].grad;
        void *out = a.entry[k.t].out;
        if (!out || (clip_same(coef) && out == grad))
            continue;
        if (a.entry[k.t].type == CD_TYPE_F32)
            clip_scale<BLOCK>(static_cast<const float *>(grad) + k.first,
                              static_cast<float *>(out) + k.first, k.n, coef, at);
        else
            clip_scale<BLOCK>(static_cast<const uint16_t *>(grad) + k.first,
                              static_cast<uint16_t *>(out) + k.first, k.n, coef, at);
    }
}

// (total: where the sum is kept for the launches that follow, as their only part; else null)
__global__ __launch_bounds__(kClipBlock) void k_clip_scale(const ClipTable a, const double *part,
                                                           unsigned parts, double max_norm,
                                                           double *norm_out, double *total)
{
    const double sum = clip_total(part, parts), norm = sqrt(sum);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (norm_out)
            *norm_out = norm;
        if (total)
            *total = sum;
    }
    clip_scale_all<kClipBlock, true>(a, clip_coef(norm, max_norm), blockIdx.x, gridDim.x, threadIdx.x);
}

// Few elements: one workgroup does it all in one launch, each of its waves on chunks of its
// own (a smaller chunk, so that every wave has one). The first chunk stays in the wave's registers
// between the norm and the scaling (65536 fp32: 6.9 us a launch, 10.6 when it is read again).
// With more elements two launches over many CUs are faster (us a call, captured / eager): 131072 fp32
// 8.4 / 11.1 against 13.8 / 14.0, 65536 fp32 8.1 / 11.7 against 6.6 / 8.9.
constexpr int kClipOneBlock = 1024, kClipOneWaves = kClipOneBlock / cdk::kWave;
constexpr unsigned kClipOneChunk = 4096, kClipOneElements = 65536, kClipOneChunks = 32;
constexpr int kClipHeld = kClipOneChunk * sizeof(float) / 16 / cdk::kWave;  // 16-byte vectors a lane

// clip_squares over a wave (the same order), which keeps the vectors
template <class T>
__device__ __forceinline__ double clip_hold(const T *p, unsigned n, unsigned lane, cdk::u32x4 (&v)[kClipHeld])
{
    constexpr unsigned kVec = 16 / sizeof(T);
    const unsigned lead = clip_lead(p, n), vecs = (n - lead) / kVec, done = lead + vecs * kVec;
    const cdk::u32x4 *q = reinterpret_cast<const cdk::u32x4 *>(p + lead);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int u = 0; u < kClipHeld * (int)sizeof(T) / 4; ++u)
        v[u] = lane + u * cdk::kWave < vecs ? q[lane + u * cdk::kWave] : cdk::zero16();
    if (lane < lead)
        s[0] += square(clip_value(p[lane]));
#pragma unroll
    for (int u = 0; u < kClipHeld * (int)sizeof(T) / 4; ++u)
        square16<T>(v[u], s);
    if (lane < n - done)
        s[1] += square(clip_value(p[done + lane]));
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// clip_scale from the kept vectors
template <class T>
__device__ __forceinline__ void clip_scale_held(const T *p, T *o, unsigned n, const ClipCoef &coef, unsigned lane,
                                                const cdk::u32x4 (&v)[kClipHeld])
{
    constexpr unsigned kVec = 16 / sizeof(T);
    const bool same = clip_same(coef);
    if (!o || (same && o == p))
        return;
    if (coef.e || ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(o)) & 15u) != 0) {
        clip_scale<cdk::kWave>(p, o, n, coef, lane);
        return;
    }
    const unsigned lead = clip_lead(p, n), vecs = (n - lead) / kVec, done = lead + vecs * kVec;
    cdk::u32x4 *w = reinterpret_cast<cdk::u32x4 *>(o + lead);
    if (lane < lead)
        o[lane] = same ? p[lane] : clip_round(clip_value(p[lane]) * coef.f, T{});
#pragma unroll
    for (int u = 0; u < kClipHeld * (int)sizeof(T) / 4; ++u)
        if (lane + u * cdk::kWave < vecs)
            w[lane + u * cdk::kWave] = same ? v[u] : scale16<T>(v[u], coef.f);
    if (lane < n - done)
        o[done + lane] = same ? p[done + lane] : clip_round(clip_value(p[done + lane]) * coef.f, T{});
}

__global__ __launch_bounds__(kClipOneBlock) void k_clip_one(const ClipTable a, double max_norm,
                                                            double *norm_out)
{
    const unsigned lane = threadIdx.x % cdk::kWave;
    const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / cdk::kWave);
    const ClipChunk k = clip_chunk(a, min(wave, (unsigned)a.chunks - 1));
    const bool mine = wave < a.chunks, f32 = a.entry[k.t].type == CD_TYPE_F32;
    const void *grad = a.entry[k.t].grad;
    void *out = a.entry[k.t].out;
    const float *p32 = static_cast<const float *>(grad) + k.first;
    const uint16_t *p16 = static_cast<const uint16_t *>(grad) + k.first;
    cdk::u32x4 v[kClipHeld];
    double s = 0.0;
    if (mine)
        s = f32 ? clip_hold(p32, k.n, lane, v) : clip_hold(p16, k.n, lane, v);
    s += clip_sum<cdk::kWave>(a, wave + kClipOneWaves, kClipOneWaves, lane);
    const double norm = sqrt(clip_block_sum<kClipOneBlock>(s));
    if (norm_out && threadIdx.x == 0)
        *norm_out = norm;
    const ClipCoef coef = clip_coef(norm, max_norm);
    if (mine && f32)
        clip_scale_held(p32, out ? static_cast<float *>(out) + k.first : nullptr, k.n, coef, lane, v);
    else if (mine)
        clip_scale_held(p16, out ? static_cast<uint16_t *>(out) + k.first : nullptr, k.n, coef, lane, v);
    clip_scale_all<cdk::kWave, false>(a, coef, wave + kClipOneWaves, kClipOneWaves, lane);
}

size_t clip_size(int type) { return type == CD_TYPE_F32 ? sizeof(float) : sizeof(uint16_t); }

struct ClipSpan {
    uintptr_t lo, hi;
    int tensor;  // (-1: the norm)
    bool operator<(const ClipSpan &o) const { return lo < o.lo; }
};

// outputs share no memory with each other, with *norm or with another tensor's gradient
bool clip_disjoint(const cd_grad *g, int n, bool scaled, const double *norm)
{
    std::vector<ClipSpan> outs;
    outs.reserve(n + 1);
    for (int i = 0; i < n; ++i)
        if (g[i].count && g[i].out && (scaled || g[i].out != g[i].grad)) {
            const uintptr_t lo = reinterpret_cast<uintptr_t>(g[i].out);
            outs.push_back({lo, lo + g[i].count * clip_size(g[i].type), i});
        }
    if (norm) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(norm);
        outs.push_back({lo, lo + sizeof(double), -1});
    }
    std::sort(outs.begin(), outs.end());
    for (size_t i = 1; i < outs.size(); ++i)
        if (outs[i].lo < outs[i - 1].hi)
            return false;
    for (int i = 0; i < n; ++i) {
        if (!g[i].count)
            continue;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(g[i].grad);
        const uintptr_t hi = lo + g[i].count * clip_size(g[i].type);
        // the outputs are disjoint: those that end after lo and start before hi
        auto o = std::upper_bound(outs.begin(), outs.end(), ClipSpan{lo, 0, -1});
        if (o != outs.begin() && (o - 1)->hi > lo)
            --o;
        for (; o != outs.end() && o->lo < hi; ++o)
            if (o->lo != lo || o->tensor != i)
                return false;
    }
    return true;
}

}  // namespace

struct cd_clip {
    int device, max_tensors;
    double *total; // the sum of all squares
    double *part;  // workgroups' sums of every launch
};

extern "C" {

cd_status countdown_clip_create(int max_tensors, cd_clip **out)
{
    if (!out || max_tensors < 1)
        return CD_EINVAL;
    if (max_tensors > 65536)
        return CD_EUNSUPPORTED;
    int dev = -1;
    if (hip_status(hipGetDevice(&dev)) != CD_OK)
        return CD_EHIP;
    cd_clip *p = new (std::nothrow) cd_clip{};
    if (!p)
        return CD_ENOMEM;
    p->device = dev;
    p->max_tensors = max_tensors;
    const size_t launches = (max_tensors + kClipTensors - 1) / kClipTensors;
    void *ws = nullptr;
    if (hip_status(hipMalloc(&ws, (1 + launches * kClipGroups) * sizeof(double))) != CD_OK) {
        delete p;
        return CD_ENOMEM;
    }
    p->total = static_cast<double *>(ws);
    p->part = p->total + 1;
    *out = p;
    return CD_OK;
}

cd_status countdown_clip_destroy(cd_clip *p)
{
    if (!p)
        return CD_OK;
    int dev = -1;
    cd_status st = hip_status(hipGetDevice(&dev));
    if (st == CD_OK)
        st = hip_status(hipSetDevice(p->device));
    if (st == CD_OK)
        st = hip_status(hipDeviceSynchronize());
    if (hip_status(hipFree(p->total)) != CD_OK)
        st = CD_EHIP;
    if (dev >= 0)
        (void)hip_status(hipSetDevice(dev));
    delete p;
    return st;
}

cd_status countdown_clip_grads(cd_clip *p, const cd_grad *grads, int n, double max_norm,
                               double *norm, void *stream)
{
    if (!p || n < 0 || n > p->max_tensors || (n && !grads) || !(max_norm >= 0.0) ||
        (reinterpret_cast<uintptr_t>(norm) & 7u))
        return CD_EINVAL;
    const bool scaled = max_norm < (double)INFINITY;
    bool writes = false;
    uint64_t elements = 0;
    for (int i = 0; i < n; ++i) {
        const cd_grad &g = grads[i];
        if (g.type != CD_TYPE_F32 && g.type != CD_TYPE_BF16)
            return CD_EINVAL;
        if (!g.count)
            continue;
        const uintptr_t odd = clip_size(g.type) - 1;
        if (!g.grad || (reinterpret_cast<uintptr_t>(g.grad) & odd) ||
            (reinterpret_cast<uintptr_t>(g.out) & odd) || (scaled && !g.out))
            return CD_EINVAL;
        if (g.count > ((uint64_t)1 << 38))  // a launch's chunks are counted in 32 bits
            return CD_EUNSUPPORTED;
        elements += g.count;
        writes |= g.out && (scaled || g.out != g.grad);
    }
    try {
        if (!clip_disjoint(grads, n, scaled, norm))
            return CD_EINVAL;
    } catch (const std::bad_alloc &) {
        return CD_ENOMEM;
    }
    int dev = -1;
    if (hip_status(hipGetDevice(&dev)) != CD_OK)
        return CD_EHIP;
    if (dev != p->device)
        return CD_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    // the next tensors that are not empty, as many as a launch takes, in chunks of so many fp32
    // and bf16 elements; returns the number of chunks
    const auto fill = [&](ClipTable &a, int &i, unsigned f32, unsigned bf16) {
        uint64_t chunks = 0;
        a.n = 0;
        a.chunk[CD_TYPE_F32] = f32;
        a.chunk[CD_TYPE_BF16] = bf16;
        for (; i < n && a.n < kClipTensors; ++i) {
            if (!grads[i].count)
                continue;
            a.entry[a.n++] = ClipEntry{grads[i].grad, grads[i].out, grads[i].count,
                                       (uint32_t)chunks, (uint32_t)grads[i].type};
            const unsigned chunk = a.chunk[grads[i].type];
            chunks += (grads[i].count + chunk - 1) / chunk;
        }
        a.chunks = chunks;
        return chunks;
    };
    ClipTable a;
    if (elements <= kClipOneElements) {
        int i = 0;
        const uint64_t chunks = fill(a, i, kClipOneChunk, kClipOneChunk);
        if (i == n && chunks && chunks <= kClipOneChunks) {
            k_clip_one<<<1, kClipOneBlock, 0, s>>>(a, max_norm, norm);
            return launched(hipGetLastError());
        }
    }
    // the norm of every launch's tensors, then the scaling
    unsigned parts = 0;
    const double *part = p->part;
    for (int pass = 0; pass < (writes ? 2 : 1); ++pass) {
        int i = 0;
        do {
            const uint64_t chunks = fill(a, i, kClipChunk / sizeof(float), kClipChunk / sizeof(uint16_t));
            const unsigned grid = (unsigned)std::min<uint64_t>(chunks, pass ? kClipScaleGroups : kClipGroups);
            if (!grid)
                continue;
            if (pass == 0) {
                k_clip_norm<<<grid, kClipBlock, 0, s>>>(a, p->part + parts);
                parts += grid;
            } else {
                // with many tensors the sums are added up by the first launch alone
                double *total = part == p->part && i < n ? p->total : nullptr;
                k_clip_scale<<<grid, kClipBlock, 0, s>>>(a, part, parts, max_norm, norm, total);
                norm = nullptr;  // written by the first
                part = p->total;
                parts = 1;
            }
            if (launched(hipGetLastError()) != CD_OK)
                return CD_EHIP;
        } while (i < n);
    }
    if (norm) {
        k_clip_total<<<1, kClipBlock, 0, s>>>(p->part, parts, norm);
        return launched(hipGetLastError());
    }
    return CD_OK;
}

}  // extern "C"
