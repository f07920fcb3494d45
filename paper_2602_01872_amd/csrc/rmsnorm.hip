// Root-mean-square norm of rows, with the residual's addition before it and 8-bit rows behind it, and its gradient.
//
//   h = x + r                 rho = 1 / sqrt(mean_c h_c^2 + eps)             y_c = h_c rho w_c
//   8-bit rows:  s = max(max_c |y_c| / 448, 2^-126),  q_c = e4m3(y_c / s)    (448: the largest e4m3 number)
//   gradient, u_c = dy_c w_c:   dh_c = rho u_c - h_c rho^3 mean(u h) + g_c,   dw_c = sum over rows of dy_c h_c rho
//
// All arithmetic is fp32 (y is made from the sum x + r before that is rounded to h's type).  What bounds these kernels is memory: every input is
// read once and every output written once, 16 bytes a lane, a row held in registers by the 8 .. 64 lanes of a wavefront or by a whole workgroup.
//   Measured: 3e5 x 256 fp32 with the residual to bf16 183 us (5.9 TB/s), 8192 x 8192 bf16 with the residual to 8 bits 93 us (5.1 TB/s), 1e5 x 1004 bf16 to 8 bits
// without a norm 53 us (5.7 TB/s), the gradient over 3e5 x 256 with the residual's 200 us (5.4 TB/s, 5 us of it the sum over 1024 workgroups' rows for the weight).
// Odd widths: 3e5 rows of 257 instead of 256 bf16 150 and 104 us, fp32 223 and 209, the gradient bf16 132 and 119, fp32 281 and 199 (its lanes are half empty);
// 8192 rows of 8191 instead of 8192 bf16 to 8 bits 116 and 93, bf16 125 and 93, fp32 the same, the gradient bf16 153 and 118, fp32 187 and 185.
#include "common.h"

namespace grp {
namespace {

typedef __bf16 bf16_t;
struct fp8_t { uint8_t v; };

constexpr float E4M3_MAX = 448.f, TINY_SCALE = 0x1p-126f;

template <typename T> __device__ __forceinline__ float widen(T v) { return (float)v; }

// V consecutive elements from any element's address on, as fp32 (V elements of the narrower type are 16 bytes; V = 1 where rows are narrower than that).
template <int V, typename T> __device__ __forceinline__ void load_v(const T* p, float (&f)[V]) {
    if constexpr (V == 1) {
        f[0] = widen(p[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < V; k += 4) {
            const u32x4_any t = *reinterpret_cast<const u32x4_any*>(p + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[k + i] = __uint_as_float(t[i]);
        }
    } else {
        uint32_t t[V / 2];
        if constexpr (V == 8) {
            const u32x4_any a = *reinterpret_cast<const u32x4_any*>(p);
            t[0] = a.x; t[1] = a.y; t[2] = a.z; t[3] = a.w;
        } else {
            const u32x2_any a = *reinterpret_cast<const u32x2_any*>(p);
            t[0] = a.x; t[1] = a.y;
        }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            f[2 * i] = __uint_as_float(t[i] << 16);
            f[2 * i + 1] = __uint_as_float(t[i] & 0xFFFF0000u);
        }
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{a, b}), bf16x2)); }

template <int V, typename T> __device__ __forceinline__ void store_v(T* p, const float (&f)[V]) {
    if constexpr (V == 1) {
        if constexpr (sizeof(T) == 1) p->v = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[0], 0, false);
        else p[0] = (T)f[0];
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < V; k += 4)
            *reinterpret_cast<u32x4_any*>(p + k) = u32x4_any{__float_as_uint(f[k]), __float_as_uint(f[k + 1]), __float_as_uint(f[k + 2]), __float_as_uint(f[k + 3])};
    } else if constexpr (sizeof(T) == 2) {
        if constexpr (V == 8)
            *reinterpret_cast<u32x4_any*>(p) = u32x4_any{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
        else
            *reinterpret_cast<u32x2_any*>(p) = u32x2_any{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
    } else {
        uint32_t t[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
            t[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
        }
        if constexpr (V == 8) *reinterpret_cast<u32x2_b*>(p) = u32x2_b{t[0], t[1]};
        else *reinterpret_cast<u32_b*>(p) = t[0];
    }
}

// Sums (or unsigned maxima) over the G lanes of a row; G = 64 * waves: by way of LDS, which is read until the workgroup's next barrier: an array for each call.
template <int G, typename T, class Op> __device__ __forceinline__ T row_reduce(T v, Op op, T* lds /*[G / 64]*/) {
#pragma unroll
    for (int o = 1; o < (G < 64 ? G : 64); o <<= 1) v = op(v, __shfl_xor(v, o, 64));
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < G / 64; ++w) v = op(v, lds[w]);
    }
    return v;
}

// A row's columns as units of V: unit u starts at column u V, but the last one at width - V, where its first `skip` elements belong to the unit
// before (they count as zero in sums, and are stored twice with the same value).  No lane reads or writes past a row, at any width >= V.
template <int V> struct UnitAt {
    int64_t at;
    int skip;             // V: no such unit
    UnitAt() = default;
    __device__ __forceinline__ UnitAt(int u, int width) {
        const int c0 = u * V;
        at = c0 < width ? c0 : 0;
        skip = c0 < width ? 0 : V;
        if (c0 < width && c0 + V > width) { at = width - V; skip = c0 + V - width; }
    }
};

struct NormArgs {
    int64_t rows;
    int32_t width;
    const void* x;
    int64_t ldx;
    const void* r;            // or null
    int64_t ldr;
    const float* weight;      // or null
    float eps;
    void* h;                  // or null
    int64_t ldh;
    void* y;
    int64_t ldy;
    float* scale;
};

constexpr int norm_threads(int G) { return G > 256 ? G : 256; }

}  // namespace
// Rows of G lanes each that one launch takes: a launch holds fewer than 2^32 work-items.
int64_t norm_rows_of_launch(int G) { return (int64_t)((1u << 31) / norm_threads(G)) * (norm_threads(G) / G); }
namespace {

// G lanes a row, P units a lane.
template <typename XT, typename YT, bool NORM, int V, int G, int P>
__global__ __launch_bounds__(norm_threads(G)) void rmsnorm_kernel(NormArgs a) {
    constexpr int ROWS = norm_threads(G) / G;
    __shared__ float lds_sum[G > 64 ? G / 64 : 1];
    __shared__ uint32_t lds_max[G > 64 ? G / 64 : 1];
    const int l = threadIdx.x & (G - 1);
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / G;
    if (G <= 64 && row >= a.rows) return;                       // (whole groups of lanes; larger G: one row a workgroup)
    const XT* x = (const XT*)a.x + row * a.ldx;
    float h[P][V];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const UnitAt<V> u(p * G + l, a.width);
        if (u.skip < V) {
            load_v<V>(x + u.at, h[p]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) h[p][e] = 0.f;
        }
    }
    if (a.r) {
        const XT* r = (const XT*)a.r + row * a.ldr;
        float t[P][V];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const UnitAt<V> u(p * G + l, a.width);
            if (u.skip < V) {
                load_v<V>(r + u.at, t[p]);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) t[p][e] = 0.f;
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) h[p][e] += t[p][e];
    }
    float rho = 1.f;
    if constexpr (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const UnitAt<V> u(p * G + l, a.width);
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) s = e >= u.skip ? fmaf(h[p][e], h[p][e], s) : s;
            ss += s;
        }
        ss = row_reduce<G>(ss, [](float p, float q) { return p + q; }, lds_sum);
        rho = rsqrtf(ss / (float)a.width + a.eps);
    }
    if (a.h) {                                                  // (every load of the row has returned: its sums are known)
        XT* ho = (XT*)a.h + row * a.ldh;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const UnitAt<V> u(p * G + l, a.width);
            if (u.skip < V) store_v<V>(ho + u.at, h[p]);
        }
    }
    YT* yo = (YT*)a.y + row * a.ldy;
    if constexpr (NORM) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const UnitAt<V> u(p * G + l, a.width);
            float w[V];
            if (a.weight && u.skip < V) {
                load_v<V>(a.weight + u.at, w);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) w[e] = 1.f;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) h[p][e] = h[p][e] * rho * w[e];
        }
    }
    if constexpr (sizeof(YT) == 1) {
        // The bits of |y| order as the numbers do, with infinity above them and NaN above that: a row with a NaN has the scale NaN.
        uint32_t most = 0;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const UnitAt<V> u(p * G + l, a.width);
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const uint32_t b = __float_as_uint(h[p][e]) & 0x7FFFFFFFu;
                m = m > b ? m : b;
            }
            if (u.skip < V) most = most > m ? most : m;          // (a lane without a unit has 0 rho, which is NaN where rho is infinite)
        }
        most = row_reduce<G>(most, [](uint32_t p, uint32_t q) { return p > q ? p : q; }, lds_max);
        float s = __uint_as_float(most) / E4M3_MAX;
        s = s < TINY_SCALE ? TINY_SCALE : s;
        if (l == 0) a.scale[row] = s;
        if (s >= 0x1p-100f && s <= 0x1p120f) {
            // y / s by the reciprocal, corrected by its remainder: the quotient rounded once, without a division for every element
            const float inv = 1.f / s;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float q = h[p][e] * inv;
                    h[p][e] = fmaf(fmaf(-q, s, h[p][e]), inv, q);
                }
        } else {                                                // infinities, NaN, rows of very small numbers
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < V; ++e) h[p][e] = h[p][e] / s;
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const UnitAt<V> u(p * G + l, a.width);
        if (u.skip < V) store_v<V>(yo + u.at, h[p]);
    }
}

// Lanes and units for rows of `units` units: the fewest lanes that hold a row in one unit each up to a wavefront, then two units a lane (the gradient, which
// keeps five values of every column: half a wavefront and four), then workgroups.  f(G, P) gets them as constants; false: too wide.  us, this and another:
//   3e5 x 256 bf16 norm 105, a quarter of the lanes with four units 117; 3e5 x 500 200 and 242; 1e5 x 1004 norm, 64 lanes with two 148, 32 with four 159, 256 with
//   one 164; its gradient, 32 with four 157, 64 with two 183; 2e4 x 4096 norm, 256 with two 116, 1024 with one 138; 8192 x 8192, 1024 with one 93, 256 with four 104.
// On both sides of each border, bf16, 2^26 elements, norm and gradient:
//   128 units, 64 with two (32 with four) 95 and 104, 256 with one 107 and 115; 129, 256 with one 116 and 121, 64 with four 103 and 124; 192 91 and 102, 100 and 106
//   256 units, 256 with one 89 and 105, with two 90 and 106;  257, with two 106 and 117, with four 124 and 173
//   513 units, 256 with four 107 and 132, 1024 with one 121 and 134;  768, 101 and 114, 95 and 121;  769, 1024 with one 97 and 125, 256 with four 109 and 124
//   1024 units, 1024 with one 92 and 117, with two 94 and 150
// fp32 rows are within 4 % of the better one, but for the gradient of 65 .. 128 units: 32 with four 122 .. 100, 64 with two 93 .. 90.  Above 2048 units the gradient's registers
// no longer hold a row: 8192 x 16384 bf16 251 us (4.3 TB/s), 8192 x 32768 1530 us (1.4 TB/s).
template <int I> using int_c = std::integral_constant<int, I>;
template <bool GRAD, class F> bool for_row_shape(int64_t units, F f) {
    if (units <= 8) f(int_c<8>(), int_c<1>());
    else if (units <= 16) f(int_c<16>(), int_c<1>());
    else if (units <= 32) f(int_c<32>(), int_c<1>());
    else if (units <= 64) f(int_c<64>(), int_c<1>());
    else if (units <= 128) f(int_c<GRAD ? 32 : 64>(), int_c<GRAD ? 4 : 2>());
    else if (units <= 256) f(int_c<256>(), int_c<1>());
    else if (units <= 512) f(int_c<256>(), int_c<2>());
    else if (units <= 768) f(int_c<256>(), int_c<4>());
    else if (units <= 1024) f(int_c<1024>(), int_c<1>());
    else if (units <= 2048) f(int_c<1024>(), int_c<2>());
    else if (units <= 4096) f(int_c<1024>(), int_c<4>());
    else if (units <= 8192) f(int_c<1024>(), int_c<8>());
    else return false;
    return true;
}

template <typename XT, typename YT, bool NORM> grp_status launch_norm(const NormArgs& a, hipStream_t st) {
    constexpr int V = 16 / sizeof(XT);
    auto go = [&](auto v, auto G, auto P) {
        constexpr int rows = norm_threads(G) / G;
        const int64_t most = norm_rows_of_launch(G);
        for (int64_t at = 0; at < a.rows; at += most) {
            NormArgs b = a;
            b.rows = std::min(most, a.rows - at);
            b.x = (const XT*)a.x + at * a.ldx;
            if (a.r) b.r = (const XT*)a.r + at * a.ldr;
            if (a.h) b.h = (XT*)a.h + at * a.ldh;
            b.y = (YT*)a.y + at * a.ldy;
            if (a.scale) b.scale = a.scale + at;
            hipLaunchKernelGGL((rmsnorm_kernel<XT, YT, NORM, decltype(v)::value, decltype(G)::value, decltype(P)::value>), dim3((unsigned)cdiv(b.rows, rows)),
                               dim3(norm_threads(G)), 0, st, b);
        }
    };
    if (a.width < V) go(int_c<1>(), int_c<8>(), int_c<1>());
    else for_row_shape<false>(cdiv(a.width, V), [&](auto G, auto P) { if constexpr (V * decltype(P)::value <= 32) go(int_c<V>(), G, P); });
    GRP_LAUNCH_CHECK();
    return GRP_OK;
}

// ------------------------------------------------------------------ gradient
struct NormGradArgs {
    int64_t rows;
    int32_t width;
    const void* dy;
    int64_t lddy;
    const void* h;
    int64_t ldh;
    const float* weight;
    float eps;
    const void* g;
    int64_t ldg;
    void* dh;
    int64_t lddh;
    float* part;              // [gridDim.x x units V], or null
    int32_t ld_part;
};

// A workgroup takes the rows b ROWS .. + ROWS - 1, then those gridDim.x ROWS further on, and so on; every lane adds up the weight's gradient of its own columns.
template <typename DT, typename HT, int V, int G, int P>
__global__ __launch_bounds__(norm_threads(G)) void rmsnorm_grad_kernel(NormGradArgs a) {
    constexpr int ROWS = norm_threads(G) / G;
    __shared__ float lds_red[2][2][G > 64 ? G / 64 : 1];        // (a row's sums are read until the next barrier: two sets in turn)
    const int l = threadIdx.x & (G - 1);
    float dw[P][V], w[P][V];
    UnitAt<V> at[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        at[p] = UnitAt<V>(p * G + l, a.width);
        if (a.weight && at[p].skip < V) {
            load_v<V>(a.weight + at[p].at, w[p]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) w[p][e] = 1.f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) dw[p][e] = 0.f;
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / G; row < a.rows; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        float h[P][V], d[P][V], t[P][V];
        const HT* hp = (const HT*)a.h + row * a.ldh;
        const DT* dp = (const DT*)a.dy + row * a.lddy;
        const HT* gp = a.g ? (const HT*)a.g + row * a.ldg : nullptr;
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int e = 0; e < V; ++e) h[p][e] = d[p][e] = t[p][e] = 0.f;
            if (at[p].skip < V) {
                load_v<V>(hp + at[p].at, h[p]);
                load_v<V>(dp + at[p].at, d[p]);
                if (gp) load_v<V>(gp + at[p].at, t[p]);
            }
        }
        float ss = 0.f, sd = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool mine = e >= at[p].skip;
                ss = mine ? fmaf(h[p][e], h[p][e], ss) : ss;
                sd = mine ? fmaf(d[p][e] * w[p][e], h[p][e], sd) : sd;
            }
        auto add = [](float p, float q) { return p + q; };
        if constexpr (G > 64) {
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) { ss += __shfl_xor(ss, o, 64); sd += __shfl_xor(sd, o, 64); }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // dh may be h or g: no wavefront writes before all have read (the last unit reads another's columns too)
            if ((threadIdx.x & 63) == 0) { lds_red[turn][0][threadIdx.x >> 6] = ss; lds_red[turn][1][threadIdx.x >> 6] = sd; }
            __syncthreads();
            ss = lds_red[turn][0][0];
            sd = lds_red[turn][1][0];
#pragma unroll
            for (int k = 1; k < G / 64; ++k) { ss += lds_red[turn][0][k]; sd += lds_red[turn][1][k]; }
        } else {
            ss = row_reduce<G>(ss, add, (float*)nullptr);
            sd = row_reduce<G>(sd, add, (float*)nullptr);
        }
        const float rho = rsqrtf(ss / (float)a.width + a.eps);
        // dh = rho (u - v mean(u v)) + g, v = h rho: rho^3 leaves fp32's range where |h| is 10^13 or 10^-13 and its product with h mean(u h) does not
        const float k = rho * (rho * (sd / (float)a.width));
        HT* out = (HT*)a.dh + row * a.lddh;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float v = h[p][e] * rho;
                dw[p][e] = e >= at[p].skip ? fmaf(d[p][e], v, dw[p][e]) : 0.f;
                o[e] = fmaf(-v, k, rho * (d[p][e] * w[p][e])) + t[p][e];
            }
            if (at[p].skip < V) store_v<V>(out + at[p].at, o);
        }
    }
    if (!a.part) return;
    float* mine = a.part + (int64_t)blockIdx.x * a.ld_part;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (at[p].skip < V)
#pragma unroll
                for (int e = 0; e < V; ++e) mine[(p * G + l) * V + e] = dw[p][e];
    } else {
        __shared__ float sums[ROWS][G * P * V + 1];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[threadIdx.x / G][(p * G + l) * V + e] = dw[p][e];
        __syncthreads();
        for (int c = threadIdx.x; c < a.ld_part; c += 256) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < ROWS; ++k) s += sums[k][c];
            mine[c] = s;
        }
    }
}

// dweight[c] = sum over the workgroups of part[b][c's place]: 16 columns and 64 slices of the workgroups each, added in a fixed order.
__global__ __launch_bounds__(1024) void rmsnorm_grad_sum_kernel(const float* __restrict__ part, int count, int ld, int width, int V, float* __restrict__ dw) {
    __shared__ float sums[64][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4;
    const int u = c / V;
    const int at = (u + 1) * V > width && width >= V ? u * V + c - (width - V) : c;      // (the last unit is kept from its own first column on)
    float s = 0.f;
    if (c < width) {
        int b = slice;
        for (; b + 7 * 64 < count; b += 8 * 64) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = part[(int64_t)(b + 64 * i) * ld + at];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        for (; b < count; b += 64) s += part[(int64_t)b * ld + at];
    }
    sums[slice][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x < 16 && c < width) {
        float t = 0.f;
        for (int k = 0; k < 64; ++k) t += sums[k][threadIdx.x];
        dw[c] = t;
    }
}

struct GradPlan { int V, units, wgs; };
GradPlan grad_plan(int64_t rows, int32_t width, bool wide /*both types bf16*/) {
    GradPlan p;
    p.V = width < 8 ? 1 : wide ? 8 : 4;
    p.units = (int)cdiv(width, p.V);
    int rows_wg = 1;
    for_row_shape<true>(p.units, [&](auto G, auto) { rows_wg = norm_threads(G) / G; });
    // 1024 workgroups: of 256 threads four a CU, as many as run at once; of 1024 threads (rows of more than 768 units) one or two a CU run at a time
    p.wgs = (int)std::min<int64_t>(1024, cdiv(rows, rows_wg));
    return p;
}
size_t grad_part_bytes(const GradPlan& p) { return (size_t)p.wgs * p.units * p.V * sizeof(float); }

template <typename DT, typename HT> grp_status launch_norm_grad(NormGradArgs a, const GradPlan& p, float* dweight, hipStream_t st) {
    constexpr int V = sizeof(DT) == 2 && sizeof(HT) == 2 ? 8 : 4;
    auto go = [&](auto v, auto G, auto P) {
        hipLaunchKernelGGL((rmsnorm_grad_kernel<DT, HT, decltype(v)::value, decltype(G)::value, decltype(P)::value>), dim3((unsigned)p.wgs),
                           dim3(norm_threads(G)), 0, st, a);
    };
    if (p.V == 1) go(int_c<1>(), int_c<8>(), int_c<1>());
    else for_row_shape<true>(p.units, [&](auto G, auto P) { if constexpr (V * decltype(P)::value <= 32) go(int_c<V>(), G, P); });
    GRP_LAUNCH_CHECK();
    if (dweight) {
        hipLaunchKernelGGL(rmsnorm_grad_sum_kernel, dim3((unsigned)cdiv(a.width, 16)), dim3(1024), 0, st, a.part, p.wgs, a.ld_part, a.width, p.V, dweight);
        GRP_LAUNCH_CHECK();
    }
    return GRP_OK;
}

bool float_type(int32_t t) { return t == GRP_DTYPE_FP32 || t == GRP_DTYPE_BF16; }
double bytes_of(int32_t t) { return t == GRP_DTYPE_FP32 ? 4.0 : t == GRP_DTYPE_BF16 ? 2.0 : 1.0; }
bool off_grid(const void* p, int32_t type) { return type != GRP_DTYPE_E4M3 && (uintptr_t)p % (type == GRP_DTYPE_BF16 ? 2 : 4) != 0; }
constexpr int32_t WIDEST = 32768;

grp_status check_rows(const char* who, int64_t rows, int32_t width) {
    if (rows < 0 || width < 1) return fail(GRP_EINVAL, "%s: rows = %lld, width = %d", who, (long long)rows, width);
    if (width > WIDEST) return fail(GRP_EUNSUPPORTED, "%s: rows of %d (at most %d)", who, width, WIDEST);
    if (rows > ((int64_t)1 << 31)) return fail(GRP_EUNSUPPORTED, "%s: more than 2^31 rows", who);
    return GRP_OK;
}

template <bool NORM> grp_status norm_by_type(const NormArgs& a, int32_t xt, int32_t yt, hipStream_t st) {
    auto go = [&](auto x) -> grp_status {
        typedef decltype(x) XT;
        if constexpr (NORM) {
            if (yt == GRP_DTYPE_FP32) return launch_norm<XT, float, true>(a, st);
            if (yt == GRP_DTYPE_BF16) return launch_norm<XT, bf16_t, true>(a, st);
        }
        return launch_norm<XT, fp8_t, NORM>(a, st);
    };
    return xt == GRP_DTYPE_FP32 ? go(float()) : go(bf16_t());
}

}  // namespace
}  // namespace grp

extern "C" grp_status grp_rmsnorm(int64_t rows, int32_t width, const void* x, int64_t ldx, int32_t x_dtype, const void* r, int64_t ldr,
                                  const float* weight, float eps, void* h, int64_t ldh, void* y, int64_t ldy, int32_t y_dtype, float* scale,
                                  void* stream) {
    using namespace grp;
    GRP_TRY(check_rows("grp_rmsnorm", rows, width));
    if (!float_type(x_dtype) || (!float_type(y_dtype) && y_dtype != GRP_DTYPE_E4M3)) return fail(GRP_EINVAL, "grp_rmsnorm: bad type");
    if (ldx < width || ldy < width || (r && ldr < width) || (h && ldh < width)) return fail(GRP_EINVAL, "grp_rmsnorm: a pitch is below the width");
    if (!(eps >= 0.f)) return fail(GRP_EINVAL, "grp_rmsnorm: eps must not be negative");
    if (rows == 0) return GRP_OK;
    if (!x || !y || (y_dtype == GRP_DTYPE_E4M3 && !scale)) return fail(GRP_EINVAL, "grp_rmsnorm: null argument");
    if (off_grid(x, x_dtype) || off_grid(r, x_dtype) || off_grid(h, x_dtype) || off_grid(y, y_dtype) || off_grid(weight, GRP_DTYPE_FP32) ||
        (y_dtype == GRP_DTYPE_E4M3 && off_grid(scale, GRP_DTYPE_FP32)))
        return fail(GRP_EINVAL, "grp_rmsnorm: a pointer is not aligned to its elements");
    if (rows > 1 && h && ((h == x && ldh != ldx) || (h == r && ldh != ldr))) return fail(GRP_EINVAL, "grp_rmsnorm: h in place of x or r needs its pitch");
    NormArgs a{rows, width, x, ldx, r, ldr, weight, eps, h, ldh, y, ldy, scale};
    ProfScope ps("rmsnorm", (hipStream_t)stream, 6.0 * rows * width,
                 (double)rows * width * (bytes_of(x_dtype) * (1 + (r ? 1 : 0) + (h ? 1 : 0)) + bytes_of(y_dtype)));
    return norm_by_type<true>(a, x_dtype, y_dtype, (hipStream_t)stream);
}

extern "C" grp_status grp_quantize_rows(int64_t rows, int32_t width, const void* x, int64_t ldx, int32_t x_dtype, void* q, int64_t ldq, float* scale,
                                        void* stream) {
    using namespace grp;
    GRP_TRY(check_rows("grp_quantize_rows", rows, width));
    if (!float_type(x_dtype)) return fail(GRP_EINVAL, "grp_quantize_rows: bad type");
    if (ldx < width || ldq < width) return fail(GRP_EINVAL, "grp_quantize_rows: a pitch is below the width");
    if (rows == 0) return GRP_OK;
    if (!x || !q || !scale) return fail(GRP_EINVAL, "grp_quantize_rows: null argument");
    if (off_grid(x, x_dtype) || off_grid(scale, GRP_DTYPE_FP32)) return fail(GRP_EINVAL, "grp_quantize_rows: a pointer is not aligned to its elements");
    NormArgs a{rows, width, x, ldx, nullptr, 0, nullptr, 0.f, nullptr, 0, q, ldq, scale};
    ProfScope ps("quantize_rows", (hipStream_t)stream, 6.0 * rows * width, (double)rows * width * (bytes_of(x_dtype) + 1.0));
    return norm_by_type<false>(a, x_dtype, GRP_DTYPE_E4M3, (hipStream_t)stream);
}

extern "C" size_t grp_rmsnorm_backward_workspace_bytes(int64_t rows, int32_t width) {
    using namespace grp;
    if (rows <= 0 || width < 1 || width > WIDEST) return 0;
    return std::max(grad_part_bytes(grad_plan(rows, width, false)), grad_part_bytes(grad_plan(rows, width, true)));
}

extern "C" grp_status grp_rmsnorm_backward(int64_t rows, int32_t width, const void* dy, int64_t lddy, int32_t dy_dtype, const void* h, int64_t ldh,
                                           int32_t h_dtype, const float* weight, float eps, const void* g, int64_t ldg, void* dh, int64_t lddh,
                                           float* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace grp;
    GRP_TRY(check_rows("grp_rmsnorm_backward", rows, width));
    if (!float_type(dy_dtype) || !float_type(h_dtype)) return fail(GRP_EINVAL, "grp_rmsnorm_backward: bad type");
    if (lddy < width || ldh < width || lddh < width || (g && ldg < width)) return fail(GRP_EINVAL, "grp_rmsnorm_backward: a pitch is below the width");
    if (!(eps >= 0.f)) return fail(GRP_EINVAL, "grp_rmsnorm_backward: eps must not be negative");
    hipStream_t st = (hipStream_t)stream;
    if (rows == 0) return dweight ? launch_fill_zero(dweight, sizeof(float) * width, st) : GRP_OK;
    if (!dy || !h || !dh) return fail(GRP_EINVAL, "grp_rmsnorm_backward: null argument");
    if (off_grid(dy, dy_dtype) || off_grid(h, h_dtype) || off_grid(g, h_dtype) || off_grid(dh, h_dtype) || off_grid(weight, GRP_DTYPE_FP32) ||
        off_grid(dweight, GRP_DTYPE_FP32) || (dweight && off_grid(workspace, GRP_DTYPE_FP32)))
        return fail(GRP_EINVAL, "grp_rmsnorm_backward: a pointer is not aligned to its elements");
    if (rows > 1 && ((dh == h && lddh != ldh) || (dh == g && lddh != ldg))) return fail(GRP_EINVAL, "grp_rmsnorm_backward: dh in place of h or g needs its pitch");
    const GradPlan p = grad_plan(rows, width, dy_dtype == GRP_DTYPE_BF16 && h_dtype == GRP_DTYPE_BF16);
    if (dweight && (!workspace || workspace_bytes < grad_part_bytes(p)))
        return fail(GRP_EWORKSPACE, "grp_rmsnorm_backward: workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : (size_t)0, grad_part_bytes(p));
    NormGradArgs a{rows, width, dy, lddy, h, ldh, weight, eps, g, ldg, dh, lddh, dweight ? (float*)workspace : nullptr, p.units * p.V};
    ProfScope ps("rmsnorm_backward", st, 12.0 * rows * width, (double)rows * width * (bytes_of(dy_dtype) + bytes_of(h_dtype) * (g ? 3 : 2)));
    if (dy_dtype == GRP_DTYPE_FP32)
        return h_dtype == GRP_DTYPE_FP32 ? launch_norm_grad<float, float>(a, p, dweight, st) : launch_norm_grad<float, bf16_t>(a, p, dweight, st);
    return h_dtype == GRP_DTYPE_FP32 ? launch_norm_grad<bf16_t, float>(a, p, dweight, st) : launch_norm_grad<bf16_t, bf16_t>(a, p, dweight, st);
}
