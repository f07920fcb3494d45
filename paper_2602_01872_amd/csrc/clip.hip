// Clipping of a gradient that lies in many tensors by its global norm:
//   norm = sqrt(sum over all tensors of g^2),  c = 1 if norm <= max_norm else max_norm / norm,  out = c g  (in the tensor's type).
//
// The squares are added in fp64 (an fp32 square overflows from 1.8e19 on, and a model has 10^8 of them).  Two launches, whatever the number of
// tensors: the first leaves a partial sum for every workgroup, in the second every workgroup adds those up again, in the same order, and scales its
// share.  Both are bound by memory: the gradient is read twice and written once.  What the first launch read last is still in the 256 MB last-level cache, so the
// second goes through the pieces from the end, and its stores pass that cache by: 158 MB of gradient 106 -> 91 us (5.2 TB/s over its three passes), 451 MB 288 -> 243,
// stores alone 92 and 267, the order alone 107 and 281.  0.7 MB: 3.0 + 3.6 us, two launches' latency.
#include "common.h"

#include <new>

namespace grp {
namespace {

struct ClipPiece {              // a run of one tensor's elements
    const void* src;
    void* dst;
    int32_t count;
    int32_t bf16;
};
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_WGS_MOST = 2048;           // partial sums that every workgroup of the second launch reads: eight a thread
constexpr int64_t CLIP_PIECE_LEAST = 2048;    // elements of a piece: eight a thread
constexpr int64_t CLIP_ELEMENTS_MOST = (int64_t)1 << 38;      // more than the memory of a GPU in the narrowest type

}  // namespace
}  // namespace grp

struct grp_gradients_s {
    int64_t pieces = 0;
    int32_t per_wg = 1, wgs = 1;
    int64_t elements = 0;
    double bytes = 0.0;
    grp::ClipPiece* piece = nullptr;        // device
    double* part = nullptr;                 // device, [wgs]
};

namespace grp {
namespace {

// One workgroup's sum, in every thread; the order is fixed.
__device__ __forceinline__ double wg_sum(double s, double* lds /*[4]*/) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// f(values, first element, count) of the units of 16 bytes of a piece, then of what is left element by element.
template <class F> __device__ __forceinline__ void for_units(const ClipPiece& p, F f) {
    const int V = p.bf16 ? 8 : 4, units = p.count / V;
    for (int u = threadIdx.x; u < units; u += CLIP_THREADS) {
        float v[8];
        if (p.bf16) {
            const u32x4_any t = *reinterpret_cast<const u32x4_any*>((const uint16_t*)p.src + (int64_t)u * 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(t[i] << 16); v[2 * i + 1] = __uint_as_float(t[i] & 0xFFFF0000u); }
            f(v, u * 8, 8);
        } else {
            const u32x4_any t = *reinterpret_cast<const u32x4_any*>((const float*)p.src + (int64_t)u * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(t[i]); v[4 + i] = 0.f; }
            f(v, u * 4, 4);
        }
    }
    for (int i = units * V + threadIdx.x; i < p.count; i += CLIP_THREADS) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        v[0] = p.bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p.src)[i] << 16) : ((const float*)p.src)[i];
        f(v, i, 1);
    }
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_squares_kernel(const ClipPiece* __restrict__ piece, int64_t pieces, int per_wg, double* __restrict__ part) {
    __shared__ double lds[4];
    double s = 0.0;
    const int64_t end = (int64_t)(blockIdx.x + 1) * per_wg < pieces ? (int64_t)(blockIdx.x + 1) * per_wg : pieces;
    for (int64_t i = (int64_t)blockIdx.x * per_wg; i < end; ++i)
        for_units(piece[i], [&](const float (&v)[8], int, int) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)v[e], (double)v[e], s);
        });
    s = wg_sum(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(CLIP_THREADS) void clip_scale_kernel(const ClipPiece* __restrict__ piece, int64_t pieces, int per_wg,
                                                                  const double* __restrict__ part, double max_norm, float* __restrict__ norm_out) {
    __shared__ double lds[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += CLIP_THREADS) s += part[i];
    const double norm = sqrt(wg_sum(s, lds));
    const float c = norm <= max_norm ? 1.f : (float)(max_norm / norm);       // (a NaN norm: NaN everywhere, as the formula has it)
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm_out) *norm_out = (float)norm;
    const int64_t b = gridDim.x - 1 - blockIdx.x;
    const int64_t end = (b + 1) * per_wg < pieces ? (b + 1) * per_wg : pieces;
    for (int64_t i = end - 1; i >= b * per_wg; --i) {
        const ClipPiece p = piece[i];
        if (p.src == p.dst && c == 1.f) continue;                            // in place, and nothing to change
        for_units(p, [&](const float (&v)[8], int at, int n) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = v[e] * c;
            if (n == 8) {
                u32x4_any t;
#pragma unroll
                for (int k = 0; k < 4; ++k) t[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{o[2 * k], o[2 * k + 1]}), bf16x2));
                __builtin_nontemporal_store(t, reinterpret_cast<u32x4_any*>((uint16_t*)p.dst + at));
            } else if (n == 4) {
                __builtin_nontemporal_store(u32x4_any{__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3])},
                                            reinterpret_cast<u32x4_any*>((float*)p.dst + at));
            } else if (p.bf16) {
                ((__bf16*)p.dst)[at] = (__bf16)o[0];
            } else {
                ((float*)p.dst)[at] = o[0];
            }
        });
    }
}

}  // namespace
}  // namespace grp

extern "C" grp_status grp_gradients_destroy(grp_gradients_t* g) {
    if (!g) return GRP_OK;
    grp::pool_free(g->piece);
    grp::pool_free(g->part);
    delete g;
    return GRP_OK;
}

extern "C" grp_status grp_gradients_create(int32_t tensors, const void* const* src, void* const* dst, const int64_t* counts, const int32_t* dtypes,
                                           grp_gradients_t** out) {
    using namespace grp;
    if (!out) return fail(GRP_EINVAL, "grp_gradients_create: out is null");
    *out = nullptr;
    if (tensors < 0 || (tensors > 0 && (!src || !counts || !dtypes))) return fail(GRP_EINVAL, "grp_gradients_create: null argument");
    int64_t total = 0;
    double bytes = 0.0;
    for (int32_t i = 0; i < tensors; ++i) {
        if (counts[i] < 0) return fail(GRP_EINVAL, "grp_gradients_create: tensor %d has %lld elements", i, (long long)counts[i]);
        if (dtypes[i] != GRP_DTYPE_FP32 && dtypes[i] != GRP_DTYPE_BF16) return fail(GRP_EINVAL, "grp_gradients_create: tensor %d: bad type", i);
        if (counts[i] > 0 && (!src[i] || (dst && !dst[i]))) return fail(GRP_EINVAL, "grp_gradients_create: tensor %d is null", i);
        const size_t el = dtypes[i] == GRP_DTYPE_BF16 ? 2 : 4;
        if ((uintptr_t)src[i] % el || (dst && (uintptr_t)dst[i] % el)) return fail(GRP_EINVAL, "grp_gradients_create: tensor %d is not aligned to its elements", i);
        if (counts[i] > CLIP_ELEMENTS_MOST - total) return fail(GRP_EUNSUPPORTED, "grp_gradients_create: more than 2^38 elements");
        total += counts[i];
        bytes += (double)el * counts[i];
    }
    grp_gradients_t* g = nullptr;
    try {
        // pieces so long that the workgroups get one each up to 2^22 elements, then several of 2^13
        const int64_t length = std::min<int64_t>(1 << 13, std::max<int64_t>(CLIP_PIECE_LEAST, round_up(cdiv(total, CLIP_WGS_MOST), 2048)));
        std::vector<ClipPiece> list;
        for (int32_t i = 0; i < tensors; ++i)
            for (int64_t at = 0; at < counts[i]; at += length) {
                const size_t el = dtypes[i] == GRP_DTYPE_BF16 ? 2 : 4;
                list.push_back({(const char*)src[i] + at * el, (char*)(dst ? dst[i] : const_cast<void*>(src[i])) + at * el,
                                (int32_t)std::min<int64_t>(length, counts[i] - at), dtypes[i] == GRP_DTYPE_BF16});
            }
        g = new grp_gradients_t();
        g->pieces = (int64_t)list.size();
        g->per_wg = (int32_t)std::max<int64_t>(1, cdiv(g->pieces, CLIP_WGS_MOST));
        g->wgs = (int32_t)std::max<int64_t>(1, cdiv(g->pieces, g->per_wg));
        g->elements = total;
        g->bytes = bytes;
        if (pool_alloc((void**)&g->piece, std::max<size_t>(1, list.size()) * sizeof(ClipPiece)) != hipSuccess ||
            pool_alloc((void**)&g->part, sizeof(double) * g->wgs) != hipSuccess) {
            (void)hipGetLastError();
            grp_gradients_destroy(g);
            return fail(GRP_ENOMEM, "grp_gradients_create: device allocation failed");
        }
        if (!list.empty()) {
            const hipError_t e = hipMemcpy(g->piece, list.data(), list.size() * sizeof(ClipPiece), hipMemcpyHostToDevice);
            if (e != hipSuccess) {
                grp_gradients_destroy(g);
                return fail(GRP_EHIP, "grp_gradients_create: %s", hipGetErrorString(e));
            }
        }
    } catch (const std::bad_alloc&) {
        grp_gradients_destroy(g);
        return fail(GRP_ENOMEM, "grp_gradients_create: host allocation failed");
    }
    *out = g;
    return GRP_OK;
}

extern "C" grp_status grp_clip_gradients(const grp_gradients_t* g, double max_norm, float* norm_out, void* stream) {
    using namespace grp;
    if (!g) return fail(GRP_EINVAL, "grp_clip_gradients: null handle");
    if (!(max_norm > 0.0)) return fail(GRP_EINVAL, "grp_clip_gradients: max_norm must be positive");
    hipStream_t st = (hipStream_t)stream;
    {
        ProfScope ps("clip_squares", st, 2.0 * g->elements, g->bytes);
        hipLaunchKernelGGL(clip_squares_kernel, dim3((unsigned)g->wgs), dim3(CLIP_THREADS), 0, st, g->piece, g->pieces, g->per_wg, g->part);
        GRP_LAUNCH_CHECK();
    }
    ProfScope ps("clip_scale", st, (double)g->elements, 2.0 * g->bytes);
    hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)g->wgs), dim3(CLIP_THREADS), 0, st, g->piece, g->pieces, g->per_wg, g->part, max_norm, norm_out);
    GRP_LAUNCH_CHECK();
    return GRP_OK;
}
