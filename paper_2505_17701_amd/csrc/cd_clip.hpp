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

constexpr int kClipTensors = 96;        // tensors per launch: the table is a kernel argument (2.8 KB)
constexpr unsigned kClipChunk = 16384;  // elements per step of a workgroup
constexpr unsigned kClipGroups = 2048;  // workgroups per launch: 8 on each CU
constexpr int kClipBlock = 256;

struct ClipTable {
    const void *grad[kClipTensors];
    void *out[kClipTensors];
    uint64_t count[kClipTensors];
    uint32_t chunk0[kClipTensors + 1];  // first chunk of each tensor
    uint8_t type[kClipTensors];
    int n;
};

struct ClipChunk {
    int t;           // tensor
    uint64_t first;  // its first element
    unsigned n;      // elements
};

// the tensor and range of chunk c (uniform over the workgroup)
__device__ __forceinline__ ClipChunk clip_chunk(const ClipTable &a, unsigned c)
{
    int lo = 0, hi = a.n - 1;  // the last tensor whose first chunk is <= c
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.chunk0[mid] <= c)
            lo = mid;
        else
            hi = mid - 1;
    }
    ClipChunk r;
    r.t = lo;
    r.first = (uint64_t)(c - a.chunk0[lo]) * kClipChunk;
    const uint64_t left = a.count[lo] - r.first;
    r.n = left < kClipChunk ? (unsigned)left : kClipChunk;
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
__device__ __forceinline__ double square16(const cdk::u32x4 &v)
{
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        s += sizeof(T) == 4 ? square(__uint_as_float(v[i]))
                            : square(cdk::bf16_lo(v[i])) + square(cdk::bf16_hi(v[i]));
    return s;
}

template <class T>
__device__ __forceinline__ double clip_squares(const T *p, unsigned n)
{
    constexpr unsigned kVec = 16 / sizeof(T);
    const unsigned lead = clip_lead(p, n), vecs = (n - lead) / kVec, done = lead + vecs * kVec;
    const cdk::u32x4 *v = reinterpret_cast<const cdk::u32x4 *>(p + lead);
    double s = 0.0;
    if (threadIdx.x < lead)
        s += square(clip_value(p[threadIdx.x]));
#pragma unroll 8
    for (unsigned i = threadIdx.x; i < vecs; i += kClipBlock)
        s += square16<T>(v[i]);
    if (threadIdx.x < n - done)
        s += square(clip_value(p[done + threadIdx.x]));
    return s;
}

// sum over the workgroup, in thread 0
__device__ __forceinline__ double clip_block_sum(double s)
{
    __shared__ double waves[kClipBlock / cdk::kWave];
#pragma unroll
    for (int d = 1; d < cdk::kWave; d *= 2)
        s += __shfl_xor(s, d);
    __syncthreads();
    if (threadIdx.x % cdk::kWave == 0)
        waves[threadIdx.x / cdk::kWave] = s;
    __syncthreads();
    s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kClipBlock / cdk::kWave; ++w)
            s += waves[w];
    return s;
}

// sums of squares by workgroup
__global__ __launch_bounds__(kClipBlock) void k_clip_norm(const ClipTable a, double *part)
{
    double s = 0.0;
    for (unsigned c = blockIdx.x; c < a.chunk0[a.n]; c += gridDim.x) {
        const ClipChunk k = clip_chunk(a, c);
        s += a.type[k.t] == CD_TYPE_F32
                 ? clip_squares(static_cast<const float *>(a.grad[k.t]) + k.first, k.n)
                 : clip_squares(static_cast<const uint16_t *>(a.grad[k.t]) + k.first, k.n);
    }
    s = clip_block_sum(s);
    if (threadIdx.x == 0)
        part[blockIdx.x] = s;
}

// The norm from the workgroups' sums, in every thread. Each workgroup that needs it adds
// them for itself (at most 16 KB a launch, from L2): a counter that tells one workgroup it is the last
// makes every other flush its L2 first (2032 of them: 70 us for 67 MB of gradients).
__device__ __forceinline__ double clip_total(const double *part, unsigned parts)
{
    __shared__ double total;
    double s = 0.0;
    for (unsigned i = threadIdx.x; i < parts; i += kClipBlock)
        s += part[i];
    s = clip_block_sum(s);
    if (threadIdx.x == 0)
        total = sqrt(s);
    __syncthreads();
    return total;
}

__global__ __launch_bounds__(kClipBlock) void k_clip_total(const double *part, unsigned parts,
                                                           double *norm_out)
{
    const double norm = clip_total(part, parts);
    if (threadIdx.x == 0)
        *norm_out = norm;
}

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
template <class T>
__device__ __forceinline__ void clip_scale(const T *p, T *o, unsigned n, float coef)
{
    constexpr unsigned kVec = 16 / sizeof(T);
    const bool same = coef == 1.0f;
    if (((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(o)) & 15u) != 0) {
        for (unsigned i = threadIdx.x; i < n; i += kClipBlock)
            o[i] = same ? p[i] : clip_round(clip_value(p[i]) * coef, T{});
        return;
    }
    const unsigned lead = clip_lead(p, n), vecs = (n - lead) / kVec, done = lead + vecs * kVec;
    const cdk::u32x4 *v = reinterpret_cast<const cdk::u32x4 *>(p + lead);
    cdk::u32x4 *w = reinterpret_cast<cdk::u32x4 *>(o + lead);
    if (threadIdx.x < lead)
        o[threadIdx.x] = same ? p[threadIdx.x] : clip_round(clip_value(p[threadIdx.x]) * coef, T{});
#pragma unroll 8
    for (unsigned i = threadIdx.x; i < vecs; i += kClipBlock)
        w[i] = same ? v[i] : scale16<T>(v[i], coef);
    if (threadIdx.x < n - done)
        o[done + threadIdx.x] =
            same ? p[done + threadIdx.x] : clip_round(clip_value(p[done + threadIdx.x]) * coef, T{});
}

__global__ __launch_bounds__(kClipBlock) void k_clip_scale(const ClipTable a, const double *part,
                                                           unsigned parts, double max_norm,
                                                           double *norm_out)
{
    const double norm = clip_total(part, parts);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0)
        *norm_out = norm;
    // a norm that is not finite scales nothing
    const float coef =
        norm > max_norm && norm < (double)INFINITY ? (float)(max_norm / norm) : 1.0f;
    for (unsigned c = blockIdx.x; c < a.chunk0[a.n]; c += gridDim.x) {
        const ClipChunk k = clip_chunk(a, c);
        if (!a.out[k.t] || (coef == 1.0f && a.out[k.t] == a.grad[k.t]))
            continue;
        if (a.type[k.t] == CD_TYPE_F32)
            clip_scale(static_cast<const float *>(a.grad[k.t]) + k.first,
                       static_cast<float *>(a.out[k.t]) + k.first, k.n, coef);
        else
            clip_scale(static_cast<const uint16_t *>(a.grad[k.t]) + k.first,
                       static_cast<uint16_t *>(a.out[k.t]) + k.first, k.n, coef);
    }
}

size_t clip_size(int type) { return type == CD_TYPE_F32 ? sizeof(float) : sizeof(uint16_t); }

struct ClipSpan {
    uintptr_t lo, hi;
    const void *grad;  // the tensor's own gradient
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
            outs.push_back({lo, lo + g[i].count * clip_size(g[i].type), g[i].grad});
        }
    if (norm) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(norm);
        outs.push_back({lo, lo + sizeof(double), nullptr});
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
        auto o = std::upper_bound(outs.begin(), outs.end(), ClipSpan{lo, 0, nullptr});
        if (o != outs.begin() && (o - 1)->hi > lo)
            --o;
        for (; o != outs.end() && o->lo < hi; ++o)
            if (o->lo != lo || o->hi != hi || o->grad != g[i].grad)
                return false;
    }
    return true;
}

}  // namespace

struct cd_clip {
    int device, max_tensors;
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
    if (hip_status(hipMalloc(&ws, launches * kClipGroups * sizeof(double))) != CD_OK) {
        delete p;
        return CD_ENOMEM;
    }
    p->part = static_cast<double *>(ws);
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
    if (hip_status(hipFree(p->part)) != CD_OK)
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
    // The norm of every launch's tensors, then the scaling; a launch's table holds the
    // tensors that are not empty.
    unsigned parts = 0;
    for (int pass = 0; pass < (writes ? 2 : 1); ++pass) {
        int i = 0;
        do {
            ClipTable a;
            a.n = 0;
            uint64_t chunks = 0;
            for (; i < n && a.n < kClipTensors; ++i) {
                if (!grads[i].count)
                    continue;
                a.grad[a.n] = grads[i].grad;
                a.out[a.n] = grads[i].out;
                a.count[a.n] = grads[i].count;
                a.type[a.n] = (uint8_t)grads[i].type;
                a.chunk0[a.n++] = (uint32_t)chunks;
                chunks += (grads[i].count + kClipChunk - 1) / kClipChunk;
            }
            a.chunk0[a.n] = (uint32_t)chunks;
            const unsigned grid = (unsigned)std::min<uint64_t>(chunks, kClipGroups);
            if (!grid)
                continue;
            if (pass == 0) {
                k_clip_norm<<<grid, kClipBlock, 0, s>>>(a, p->part + parts);
                parts += grid;
            } else {
                k_clip_scale<<<grid, kClipBlock, 0, s>>>(a, p->part, parts, max_norm, norm);
                norm = nullptr;  // written by the first
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
