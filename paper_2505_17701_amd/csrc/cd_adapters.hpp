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
    float *lat, *glat;  // [T][rank]; both without scale_a
    int T, n, d_in, d_out, rank;
};

__device__ __forceinline__ float ad_load(const void *p, int type, size_t i)
{
    return type == CD_TYPE_F32 ? static_cast<const float *>(p)[i]
                               : cdk::bf16_lo(static_cast<const uint16_t *>(p)[i]);
}
__device__ __forceinline__ void ad_store(void *p, int type, size_t i, float v)
{
    if (type == CD_TYPE_F32)
        static_cast<float *>(p)[i] = v;
    else
        static_cast<uint16_t *>(p)[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
}

__device__ __forceinline__ bool ad_valid(const AdArgs &a, int id) { return (unsigned)id < (unsigned)a.n; }
__device__ __forceinline__ float ad_scale(const AdArgs &a, int id) { return a.scale ? a.scale[id] : 1.0f; }

// dot product of two bf16 rows of n (a multiple of 8) columns, over a wave
__device__ __forceinline__ float ad_dot(const uint16_t *p, const uint16_t *q, int n)
{
    float s = 0.0f;
    for (int i = threadIdx.x % cdk::kWave * 8; i < n; i += cdk::kColsPerLoad)
        s = cdk::dot8(cdk::load16(p + i), cdk::load16(q + i), s);
    return cdk::wave_sum(s);
}

// lat[t][k]: one wave per (t, k)
__global__ __launch_bounds__(kAdBlock) void k_ad_lat(const AdArgs a)
{
    const size_t w = (size_t)blockIdx.x * kAdWaves + threadIdx.x / cdk::kWave;
    const size_t t = w / a.rank;
    if (t >= (size_t)a.T)
        return;
    const int k = (int)(w % a.rank), id = a.ids[t];
    if (!ad_valid(a, id))
        return;
    const float v = ad_dot(a.x + t * a.ldx, a.A + ((size_t)id * a.rank + k) * a.d_in, a.d_in);
    if (threadIdx.x % cdk::kWave == 0)
        a.lat[w] = v;
}

// out[t][o] = base or W x_t, + scale B lat: one wave per (t, o) with W, else one lane
template <bool PROJECT>
__global__ __launch_bounds__(kAdBlock) void k_ad_out(const AdArgs a)
{
    const size_t i = (size_t)blockIdx.x * (PROJECT ? kAdWaves : kAdBlock) +
                     threadIdx.x / (PROJECT ? cdk::kWave : 1);
    const size_t t = i / a.d_out, o = i % a.d_out;
    if (t >= (size_t)a.T)
        return;
    float v = 0.0f;
    if constexpr (PROJECT) {
        v = ad_dot(a.x + t * a.ldx, a.W + o * a.d_in, a.d_in);
        if (threadIdx.x % cdk::kWave != 0)
            return;
    }
    const int id = a.ids[t];
    if (ad_valid(a, id)) {
        const uint16_t *b = a.B + ((size_t)id * a.d_out + o) * a.rank;
        float s = 0.0f;
        for (int k = 0; k < a.rank; ++k)
            s += a.lat[t * a.rank + k] * cdk::bf16_lo(b[k]);
        v += ad_scale(a, id) * s;
    }
    if (a.base)
        v += ad_load(a.base, a.type, t * a.ldb + o);
    ad_store(a.out, a.type, t * a.ldo + o, v);
}

// glat[t][k] (without the scale): one wave per (t, k)
__global__ __launch_bounds__(kAdBlock) void k_ad_glat(const AdArgs a)
{
    const size_t w = (size_t)blockIdx.x * kAdWaves + threadIdx.x / cdk::kWave;
    const size_t t = w / a.rank;
    if (t >= (size_t)a.T)
        return;
    const int k = (int)(w % a.rank), id = a.ids[t];
    if (!ad_valid(a, id))
        return;
    float s = 0.0f;
    for (int o = threadIdx.x % cdk::kWave; o < a.d_out; o += cdk::kWave)
        s += cdk::bf16_lo(a.dy[t * a.lddy + o]) *
             cdk::bf16_lo(a.B[((size_t)id * a.d_out + o) * a.rank + k]);
    s = cdk::wave_sum(s);
    if (threadIdx.x % cdk::kWave == 0)
        a.glat[w] = s;
}

// dx[t][i]: one lane each
__global__ __launch_bounds__(kAdBlock) void k_ad_dx(const AdArgs a)
{
    const size_t w = (size_t)blockIdx.x * kAdBlock + threadIdx.x;
    const size_t t = w / a.d_in, i = w % a.d_in;
    if (t >= (size_t)a.T)
        return;
    const int id = a.ids[t];
    float v = 0.0f;
    if (ad_valid(a, id)) {
        for (int k = 0; k < a.rank; ++k)
            v += a.glat[t * a.rank + k] * cdk::bf16_lo(a.A[((size_t)id * a.rank + k) * a.d_in + i]);
        v *= ad_scale(a, id);
    }
    if (a.base)
        v += ad_load(a.base, a.type, t * a.ldb + i);
    ad_store(a.out, a.type, t * a.ldo + i, v);
}

// dA (DB false) and dB: one lane per element, over the tokens
template <bool DB>
__global__ __launch_bounds__(kAdBlock) void k_ad_grad(const AdArgs a)
{
    const size_t w = (size_t)blockIdx.x * kAdBlock + threadIdx.x;
    const size_t d = DB ? a.d_out : a.d_in, id = w / (d * a.rank), at = w % (d * a.rank);
    if (id >= (size_t)a.n)
        return;
    const size_t k = DB ? at % a.rank : at / d, i = DB ? at / a.rank : at % d;
    float v = 0.0f;
    bool used = false;  // (an adapter without tokens has a zero gradient whatever its scale)
    for (int t = 0; t < a.T; ++t)
        if (a.ids[t] == (int)id) {
            used = true;
            v += DB ? a.lat[(size_t)t * a.rank + k] * cdk::bf16_lo(a.dy[t * a.lddy + i])
                    : a.glat[(size_t)t * a.rank + k] * cdk::bf16_lo(a.x[t * a.ldx + i]);
        }
    (DB ? a.dB : a.dA)[w] = used ? v * ad_scale(a, (int)id) : 0.0f;
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

unsigned ad_blocks(size_t items, size_t per) { return (unsigned)((items + per - 1) / per); }

}  // namespace

struct cd_adapters {
    int d_in, d_out, rank, n, max_tokens, device;
    unsigned flags;
    float *lat, *glat;
};

namespace {

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
                         ad_flat(a.ids, (size_t)a.T * 4),
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
        a.lat = p->lat;
        a.glat = p->glat;
        a.n = p->n;
        a.d_in = p->d_in;
        a.d_out = p->d_out;
        a.rank = p->rank;
    }
    return a;
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
    const size_t lat = (size_t)max_tokens * rank * sizeof(float);
    void *ws = nullptr;
    if (hip_status(hipMalloc(&ws, flags & CD_ADAPTERS_TRAIN ? 2 * lat : lat)) != CD_OK) {
        delete p;
        return CD_ENOMEM;
    }
    p->lat = static_cast<float *>(ws);
    p->glat = flags & CD_ADAPTERS_TRAIN ? p->lat + lat / sizeof(float) : nullptr;
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
    if (hip_status(hipFree(p->lat)) != CD_OK)
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
    k_ad_lat<<<ad_blocks((size_t)T * a.rank, kAdWaves), kAdBlock, 0, s>>>(a);
    k_ad_out<true><<<ad_blocks((size_t)T * a.d_out, kAdWaves), kAdBlock, 0, s>>>(a);
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
    k_ad_lat<<<ad_blocks((size_t)T * a.rank, kAdWaves), kAdBlock, 0, s>>>(a);
    k_ad_out<false><<<ad_blocks((size_t)T * a.d_out, kAdBlock), kAdBlock, 0, s>>>(a);
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
    if (dB && T > 0)
        k_ad_lat<<<ad_blocks((size_t)T * a.rank, kAdWaves), kAdBlock, 0, s>>>(a);
    if ((dx || dA) && T > 0)
        k_ad_glat<<<ad_blocks((size_t)T * a.rank, kAdWaves), kAdBlock, 0, s>>>(a);
    if (dx && T > 0)
        k_ad_dx<<<ad_blocks((size_t)T * a.d_in, kAdBlock), kAdBlock, 0, s>>>(a);
    if (dA)
        k_ad_grad<false><<<ad_blocks((size_t)a.n * a.rank * a.d_in, kAdBlock), kAdBlock, 0, s>>>(a);
    if (dB)
        k_ad_grad<true><<<ad_blocks((size_t)a.n * a.rank * a.d_out, kAdBlock), kAdBlock, 0, s>>>(a);
    return launched(hipGetLastError());
}

}  // extern "C"
