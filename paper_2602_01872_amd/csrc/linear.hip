// Linear layers in bf16 and in 8 bits on the matrix cores, with what stands around them in a residual block, and their gradients:
//
//   forward   z = A W + b  (8 bits: row m of A times a_scale[m], column n of W times w_scale[n]),  c = act(z) + r       sum over k
//   dx        dA = (dZ W^T) act'(zin)                                                                                     sum over n
//   dw        dW = A^T dZ,  db = column sums of dZ                                                                        sum over the rows
//
// The 8-bit matrix instructions cut, of every eight products, what is below 2^-13 of the largest (measured on single instructions; rms 1.3e-5 of the
// result on normal deviates).  Beside the rounding of a bf16 result (rms 1.6e-3) that is nothing, and they run at twice the rate; for fp32 results
// e4m3 numbers are widened to bf16, which holds them exactly, and multiplied as those (8192^3 384 us and 717, 4096^3 56 and 105).
//
// All are D[i, j] = sum_s P(i, s) Q(s, j): an operand either has s contiguous ("rows": A, dZ, the 8-bit weights) or its output index ("columns": W of the
// forward product, both operands of dw).  Products are accumulated in fp32 by the matrix unit.  Three kernels make them: tiles (linear_kernel, with
// linear_sum_kernel where the sums are split), a few rows (linear_few_kernel), and many rows with short sums or rows at odd places (linear_tall_kernel); which one is
// plan_of's choice.
//
// Tiles.  A workgroup of WI x WJ wavefronts makes 16 FI WI rows and 64 WJ columns; a step takes 128 bytes of s (64 bf16, 128 e4m3 numbers) of both operands
// through LDS, two steps' tiles in turn, so that a step's loads have the whole step before to arrive.
//   rows     LDS row o (output index) has 128 bytes, eight places of 16; a lane's operand of a matrix instruction is one (bf16) or two (8 bits) places
//   columns  LDS row s has the tile's output indices; ds_read_b64_tr_b16 turns four rows of 16 around into a lane's four consecutive s
// Places are permuted by some bits of the row (swizzle) so that the 16 lanes of a group read different banks.
//   The instruction's rows are D's columns: lane (g, t) holds D[i + t, j + 16 g + 4 f + e], e < 4, for the wavefront's fragments f < 4: 16 consecutive columns.
//   Measured, 8192^3 with inputs that stay in the caches, on several cards: forward 770 - 800 us (1370 - 1430 TFLOP/s), dx 780 - 810, dw 800, 8 bits 370 - 385 (2860 - 2990);
// the matrix unit is busy 53 - 68 % of the cycles, a third of the rest goes to the loads (660 us without any), 256 x 256 tiles against 128 x 128: 790 and 1040 us (forward).
#include "common.h"

namespace grp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

enum LinearOp { FWD_BF16, FWD_E4M3 /* bf16 results */, FWD_E4M3_WIDE /* fp32 results */, GRAD_X, GRAD_W };
constexpr bool is_e4m3(int op) { return op == FWD_E4M3 || op == FWD_E4M3_WIDE; }
constexpr bool is_forward(int op) { return op == FWD_BF16 || is_e4m3(op); }
constexpr int elem_size(int op) { return is_e4m3(op) ? 1 : 2; }
constexpr bool p_columns(int op) { return op == GRAD_W; }
constexpr bool q_columns(int op) { return op == GRAD_W || op == FWD_BF16; }

struct LinearArgs {
    const void* P;
    int64_t ldp;
    const void* Q;
    int64_t ldq;
    int64_t end_p, end_q;             // bytes of the operands, to the end of their last rows
    int64_t I, S;                     // rows of D, length of the sums
    int32_t J;                        // columns of D
    const float *a_scale, *w_scale, *bias;
    int32_t act;
    const void* r;                    // of c's type, or null
    int64_t ldr;
    void* c;
    int64_t ldc;
    int32_t c_bf16;
    void* z;                          // forward: out, or null; dx: zin
    int64_t ldz;
    float* db;                        // dw
    float* part;                      // [splits][rows of D (dw: one more, db)][ld_part] when splits > 1
    int32_t splits, ld_part;
    int64_t steps_per_split;
    int32_t tiles_i, tiles_j;
};

// ------------------------------------------------------------------ epilogue
// Phi(-|z|) of the normal distribution: exp(-z^2 / 2) times erfcx(|z| / sqrt 2) / 2, the latter as t P(t), t = 1 / (1 + 0.3 |z|), with P fitted to
// its relative error over all |z| (1.5e-7).  As evaluated it is off by 4e-7 of itself, and by the roundings of the exponent z^2 / 2 (up to 7.5e-8 z^2): 4.6e-7 where
// |z| < 1, 1.4e-6 up to 5, 7.4e-6 at 13, measured.  One exponential, one reciprocal and nine multiply-adds; e: exp(-z^2 / 2), which the slope needs too.
//   (With the library's erff and expf and a division, the epilogue of 8192 x 4096 results over sums of 4096 took 60 of 296 us, and 85 of 522 us for silu.)
__device__ __forceinline__ float normal_tail(float z, float& e) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(z), 1.f));
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    float p = 0.03567504137754440f;
    p = fmaf(p, t, -0.15720410645008087f);
    p = fmaf(p, t, 0.20635513961315155f);
    p = fmaf(p, t, -0.05368502438068390f);
    p = fmaf(p, t, 0.12856230139732360f);
    p = fmaf(p, t, 0.09991330653429031f);
    p = fmaf(p, t, 0.12075398117303848f);
    p = fmaf(p, t, 0.11962929368019104f);
    return e * (p * t);
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f)); }

template <int ACT> __device__ __forceinline__ float act_of(float z) {
    if constexpr (ACT == GRP_ACT_RELU) return z <= 0.f ? 0.f : z;              // (NaN stays)
    if constexpr (ACT == GRP_ACT_GELU) {
        float e;
        const float q = normal_tail(z, e);
        return z * (z > 0.f ? 1.f - q : q);
    }
    if constexpr (ACT == GRP_ACT_SILU) return z * sigmoid(z);
    return z;
}
template <int ACT> __device__ __forceinline__ float slope_of(float z) {
    if constexpr (ACT == GRP_ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    if constexpr (ACT == GRP_ACT_GELU) {
        float e;
        const float q = normal_tail(z, e);
        return fmaf(z * 0.39894228040143268f, e, z > 0.f ? 1.f - q : q);
    }
    if constexpr (ACT == GRP_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    return 1.f;
}
template <class F> __device__ __forceinline__ void for_act(int act, F f) {
    switch (act) {
        case GRP_ACT_RELU: f(std::integral_constant<int, GRP_ACT_RELU>()); break;
        case GRP_ACT_GELU: f(std::integral_constant<int, GRP_ACT_GELU>()); break;
        case GRP_ACT_SILU: f(std::integral_constant<int, GRP_ACT_SILU>()); break;
        default: break;
    }
}

// N (4, 8 or 16) consecutive elements of which the first n exist (the others as zeros), as they lie in memory.
template <int N, bool BF16> struct RowPart {
    uint32_t w[BF16 ? N / 2 : N];
    __device__ __forceinline__ void load(const void* p, int n) {
        constexpr int W = BF16 ? N / 2 : N;
        if (n >= N) {
            if constexpr (W % 4 == 0) {
#pragma unroll
                for (int k = 0; k < W; k += 4) {
                    const u32x4_any t = *reinterpret_cast<const u32x4_any*>((const char*)p + 4 * k);
                    w[k] = t.x; w[k + 1] = t.y; w[k + 2] = t.z; w[k + 3] = t.w;
                }
            } else {
                const u32x2_any t = *reinterpret_cast<const u32x2_any*>(p);
                w[0] = t.x; w[1] = t.y;
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < W; ++k) w[k] = 0;
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < n) {
                if constexpr (BF16) w[e / 2] |= (uint32_t)((const uint16_t*)p)[e] << (16 * (e % 2));
                else w[e] = ((const uint32_t*)p)[e];
            }
    }
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (BF16) return __uint_as_float(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        return __uint_as_float(w[e]);
    }
};
template <int N, bool BF16> __device__ __forceinline__ void store_row(void* p, int n, const float (&f)[N]) {
    if (n >= N) {
        uint32_t w[BF16 ? N / 2 : N];
        constexpr int W = BF16 ? N / 2 : N;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            if constexpr (BF16) w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{f[2 * k], f[2 * k + 1]}), bf16x2));
            else w[k] = __float_as_uint(f[k]);
        }
        if constexpr (W % 4 == 0) {
#pragma unroll
            for (int k = 0; k < W; k += 4) *reinterpret_cast<u32x4_any*>((char*)p + 4 * k) = u32x4_any{w[k], w[k + 1], w[k + 2], w[k + 3]};
        } else {
            *reinterpret_cast<u32x2_any*>(p) = u32x2_any{w[0], w[1]};
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < n) {
            if constexpr (BF16) ((__bf16*)p)[e] = (__bf16)f[e];
            else ((float*)p)[e] = f[e];
        }
}

// What depends on the columns alone.
template <int OP, int N> struct ColumnTerms {
    RowPart<N, false> bias, ws;
    ColumnTerms() = default;
    __device__ __forceinline__ ColumnTerms(const LinearArgs& a, int j, bool whole = false) {
        const int n = whole ? N : a.J - j;
        if constexpr (is_forward(OP)) {
#pragma unroll
            for (int e = 0; e < N; ++e) bias.w[e] = 0;
            if (a.bias) bias.load(a.bias + j, n);
        }
        if constexpr (is_e4m3(OP)) {
#pragma unroll
            for (int e = 0; e < N; ++e) ws.w[e] = 0x3F800000u;
            if (a.w_scale) ws.load(a.w_scale + j, n);
        }
    }
};

// What a row of D takes besides: the residual (forward) or the pre-activation (dx).  BF16: its type.
template <int OP> __device__ __forceinline__ bool takes_more(const LinearArgs& a) {
    return is_forward(OP) ? a.r != nullptr : OP == GRAD_X && a.act != GRP_ACT_NONE;
}
template <int OP, int N, bool BF16> __device__ __forceinline__ void load_more(const LinearArgs& a, int64_t i, int j, RowPart<N, BF16>& t, bool whole = false) {
    const int64_t at = is_forward(OP) ? i * a.ldr + j : i * a.ldz + j;
    t.load((const char*)(is_forward(OP) ? a.r : a.z) + at * (BF16 ? 2 : 4), whole ? N : a.J - j);
}

// D[i, j .. j + N - 1], all terms of the sums in v, to the outputs; more: takes_more, then t is load_more's.  ACT: the activation where it is known (-1: not),
// WHOLE: all N columns exist.
template <int OP, int N, bool BF16, int ACT = -1, bool WHOLE = false>
__device__ __forceinline__ void finish(const LinearArgs& a, int64_t i, int j, float (&v)[N], const ColumnTerms<OP, N>& col, bool more, const RowPart<N, BF16>& t) {
    const int n = WHOLE ? N : a.J - j;
    if (n <= 0) return;
    auto with_act = [&](auto f) {
        if constexpr (ACT < 0) for_act(a.act, f);
        else if constexpr (ACT != GRP_ACT_NONE) f(std::integral_constant<int, ACT>());
    };
    if constexpr (is_forward(OP)) {
        if constexpr (is_e4m3(OP)) {
            const float as = a.a_scale ? a.a_scale[i] : 1.f;
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = v[e] * as * col.ws[e];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += col.bias[e];
        if (a.z) store_row<N, true>((uint16_t*)a.z + i * a.ldz + j, n, v);
        with_act([&](auto act) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = act_of<decltype(act)::value>(v[e]);
        });
        if (more)
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += t[e];
        store_row<N, BF16>((char*)a.c + (i * a.ldc + j) * (BF16 ? 2 : 4), n, v);
    } else {
        if (more)
            with_act([&](auto act) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] *= slope_of<decltype(act)::value>(t[e]);
            });
        if (a.c_bf16) store_row<N, true>((uint16_t*)a.c + i * a.ldc + j, n, v);
        else store_row<N, false>((float*)a.c + i * a.ldc + j, n, v);
    }
}
// f(the type of `t` above as a constant)
template <int OP, class F> __device__ __forceinline__ void for_more_type(const LinearArgs& a, F f) {
    if constexpr (OP == GRAD_X || OP == FWD_E4M3) f(std::true_type());
    else if constexpr (OP == GRAD_W || OP == FWD_E4M3_WIDE) f(std::false_type());
    else if (a.c_bf16) f(std::true_type());
    else f(std::false_type());
}

// ------------------------------------------------------------------ tiles
// Where place `pos` (16 bytes) of LDS row `row` comes from; an involution.  T: output indices of the tile.
template <bool COLUMNS, bool IS_Q, int T> __device__ __forceinline__ int swizzle(int pos, int row) {
    if constexpr (!COLUMNS)
        return IS_Q ? pos ^ (((row >> 1) & 1) | ((row >> 3) & 6))      // its lanes read rows 16 q + 4 f + e, q and e < 4
                    : pos ^ ((row >> 1) & 7);                          //                rows t < 16
    else if constexpr (IS_Q)
        return T >= 128 ? pos ^ ((row & 1) | ((row & 2) << 2)) : pos ^ ((row >> 1) & 1);
    else
        return T >= 128 ? pos ^ (((row & 3) << 1) | (row & 8)) : pos ^ ((row & 2) | ((row >> 1) & 4));
}

// v moved down by some elements of ES bytes, zeros above them.
template <int ES> __device__ __forceinline__ u32x4_al moved_down(u32x4_al v, int64_t elements) {
    const int bits = elements < 16 / ES ? (int)elements * ES * 8 : 128;
    uint64_t lo = ((uint64_t)v.y << 32) | v.x, hi = ((uint64_t)v.w << 32) | v.z;
    if (bits > 0) {
        lo = bits >= 128 ? 0 : bits >= 64 ? hi >> (bits & 63) : (lo >> bits) | (hi << (64 - bits));
        hi = bits >= 64 ? 0 : hi >> bits;
    }
    return u32x4_al{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// 16 bytes from any byte on, by loads of whole dwords and a shift at the end: 16 bytes a lane at 2-byte boundaries take the address unit more than twice
// as long as at 4-byte ones (3e5 x 65 by 65 x 65 63 us, 66 x 66 33).  Each dword that is read holds some of the 16 bytes.
struct AnyUnit {
    u32x4_al x;
    uint32_t y, shift;
    __device__ __forceinline__ void load(const char* p) {
        const uint32_t m = (uint32_t)(uintptr_t)p & 3;
        const char* const at = p - m;
        typedef uint32_t u32x4_4 __attribute__((ext_vector_type(4), aligned(4)));
        x = (u32x4_al)*reinterpret_cast<const u32x4_4*>(at);
        y = *reinterpret_cast<const uint32_t*>(at + (m ? 16 : 12));
        shift = m * 8;
    }
    __device__ __forceinline__ u32x4_al value() const {
        return u32x4_al{__builtin_amdgcn_alignbit(x.y, x.x, shift), __builtin_amdgcn_alignbit(x.z, x.y, shift), __builtin_amdgcn_alignbit(x.w, x.z, shift),
                        __builtin_amdgcn_alignbit(y, x.w, shift)};
    }
};

struct PlainUnit {
    u32x4_al x;
    __device__ __forceinline__ void load(const char* p) { x = (u32x4_al)*reinterpret_cast<const u32x4_b*>(p); }
    __device__ __forceinline__ u32x4_al value() const { return x; }
};

// 16 bytes of a row of n elements of ES bytes from element `at` on; what is past its end as zeros.  One load, at any byte, that stays in the row: the last
// units are read from the row's last 16 bytes and moved down.
template <int ES> __device__ __forceinline__ u32x4_al load_part(const char* row, int64_t at, int64_t n) {
    constexpr int V = 16 / ES;
    u32x4_al v = {0, 0, 0, 0};
    if (n >= V) {
        const int64_t from = at <= n - V ? at : n - V;
        v = (u32x4_al)*reinterpret_cast<const u32x4_b*>(row + from * ES);
        return at > from ? moved_down<ES>(v, at - from) : v;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (at + e < n) {
            const uint32_t x = ES == 2 ? (uint32_t)((const uint16_t*)row)[at + e] : (uint32_t)((const uint8_t*)row)[at + e];
            v[e * ES / 4] |= x << (8 * (e * ES % 4));
        }
    return v;
}

// Unit u (16 bytes, in the order of LDS) of an operand's tile that starts at output index o0 and s0.
template <int ES, bool COLUMNS, bool IS_Q, int T>
__device__ __forceinline__ u32x4_al load_unit(const void* base, int64_t ld, int64_t o0, int64_t O, int64_t s0, int64_t S, int u) {
    if constexpr (!COLUMNS) {
        const int row = u >> 3, at = swizzle<COLUMNS, IS_Q, T>(u & 7, row);
        const int64_t o = o0 + row < O ? o0 + row : O - 1;                               // (a row past the end: any; it is not stored)
        return load_part<ES>((const char*)base + o * ld * ES, s0 + at * (16 / ES), S);
    } else {
        const int row = u / (T / 8), at = swizzle<COLUMNS, IS_Q, T>(u % (T / 8), row);
        const int64_t s = s0 + row < S ? s0 + row : S - 1;
        return load_part<ES>((const char*)base + s * ld * ES, s0 + row < S ? o0 + at * 8 : O, O);
    }
}

// 16 bytes a lane from buffer `rsrc` at `off` to LDS, a wavefront's 64 places in a row from byte `lds` on.  (Inline: the compiler would wait for it before
// any other read of LDS.  No register is written; who reads the tile waits for vmcnt(0) before the barrier that is before it.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, __amdgpu_buffer_rsrc_t rsrc, uint32_t off) {
    uint32_t m0;                     // (written in here: nothing that the compiler keeps in m0 outlives this)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds" : "={m0}"(m0) : "s"(lds), "v"(off), "s"(rsrc) : "memory");
}

// 16 e4m3 numbers in bf16 (exact).
struct Wide8 {
    bf16x8 v[2];
    Wide8() = default;
    __device__ __forceinline__ explicit Wide8(u32x4_al x) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x2 t[4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                t[2 * k] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * h + k], 1.f, false);
                t[2 * k + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * h + k], 1.f, true);
            }
            v[h] = bf16x8{t[0][0], t[0][1], t[1][0], t[1][1], t[2][0], t[2][1], t[3][0], t[3][1]};
        }
    }
};

// Which tile a workgroup makes, and of which split.  Workgroups go round the eight XCDs in turn: each of these gets a run of tiles (all of one split, then
// the next), in bands of eight rows of tiles, so that the tiles that an XCD makes at one time share their operands in its L2.
__device__ __forceinline__ void tile_of(unsigned b, unsigned all, int tiles_i, int tiles_j, int& ti, int& tj, unsigned& split) {
    const unsigned xcd = b % 8, q = all / 8, r = all % 8, tiles = (unsigned)tiles_i * (unsigned)tiles_j;
    unsigned n = xcd * q + (xcd < r ? xcd : r) + b / 8;
    split = n / tiles;
    n %= tiles;
    const unsigned band = 8u * (unsigned)tiles_j, first = n / band * 8, rows = (unsigned)tiles_i - first < 8 ? (unsigned)tiles_i - first : 8, in = n % band;
    ti = (int)(first + in % rows);
    tj = (int)(in / rows);
}

// What a lane reads of a fragment at once: all 128 bytes of s (its part: 32) for the 8-bit instruction, else half of them.
template <int OP> using FragOf = std::conditional_t<OP == FWD_E4M3, intx8, u32x4_al>;
template <int OP> __device__ __forceinline__ void multiply(const FragOf<OP>& q, const FragOf<OP>& p, floatx4& c) {
    if constexpr (OP == FWD_E4M3) {
        c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(q, p, c, 0, 0, 0, 0, 0, 0);
    } else if constexpr (OP == FWD_E4M3_WIDE) {
        const Wide8 qw(q), pw(p);
#pragma unroll
        for (int h = 0; h < 2; ++h) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qw.v[h], pw.v[h], c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, p), c, 0, 0, 0);
    }
}

// DMA: rows of both operands are whole units of 16 bytes and begin on them.
template <int OP, int WI, int WJ, int FI, bool DMA> __global__ __launch_bounds__(64 * WI * WJ, 2) void linear_kernel(LinearArgs a) {
    constexpr int ES = elem_size(OP), NT = 64 * WI * WJ, TI = 16 * FI * WI, TJ = 64 * WJ, STEP = 128 / ES;
    constexpr bool PC = p_columns(OP), QC = q_columns(OP);
    constexpr int UP = TI * 8 / NT, UQ = TJ * 8 / NT, STAGE = (TI + TJ) * 128;
    __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, t = lane & 15;
    const int wi = wave / WJ, wj = wave % WJ;
    int ti, tj;
    unsigned split;
    tile_of(blockIdx.x, gridDim.x, a.tiles_i, a.tiles_j, ti, tj, split);
    const int64_t i0 = (int64_t)ti * TI, j0 = (int64_t)tj * TJ;
    const int64_t s_begin = split * a.steps_per_split * STEP;
    const int64_t s_end = s_begin + a.steps_per_split * STEP < a.S ? s_begin + a.steps_per_split * STEP : a.S;

    // A lane's offset into the tile for each of its units.  DMA: the buffers begin at the tile and end with the operand (what is past the end arrives as
    // zeros).  Else: raw registers between two steps; rows past the end are the last one.
    uint32_t off[UP + UQ];
    u32x4_al raw[DMA ? 1 : UP + UQ];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
#pragma unroll
    for (int n = 0; n < UP + UQ; ++n) {
        const bool p = n < UP;
        const int u = (p ? n : n - UP) * NT + threadIdx.x, per = p ? (PC ? TI / 8 : 8) : (QC ? TJ / 8 : 8);
        int row = u / per;
        const int at = p ? swizzle<PC, false, TI>(u % per, row) : swizzle<QC, true, TJ>(u % per, row);
        if (!DMA && !(p ? PC : QC)) {
            const int64_t most = (p ? a.I - i0 : a.J - j0) - 1;
            row = row < most ? row : (int)most;
        }
        off[n] = (uint32_t)row * ((uint32_t)(p ? a.ldp : a.ldq) * ES) + (uint32_t)at * 16;
    }
    auto buffer = [&](const void* base, int64_t ld, bool columns, int64_t o0, int64_t end, int64_t s0) {
        const int64_t at = (columns ? s0 * ld + o0 : o0 * ld + s0) * ES;
        const int64_t left = s0 >= s_end ? 0 : end - at < 0x7FFFFFF0 ? end - at : 0x7FFFFFF0;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>((const char*)base + at), 0, (int)left, 0x00020000);
    };
    // A stage is asked for in UP + UQ pieces (of one load a lane): `aim` says what the next ones are of.
    __amdgpu_buffer_rsrc_t rsrc_p, rsrc_q;
    int64_t aim_s = s_begin;
    auto aim = [&](int64_t s0) {
        aim_s = s0;
        if constexpr (DMA) {
            rsrc_p = buffer(a.P, a.ldp, PC, i0, a.end_p, s0);
            rsrc_q = buffer(a.Q, a.ldq, QC, j0, a.end_q, s0);
        }
    };
    auto piece = [&](int n, int buf) {
        const bool p = n < UP;
        const int u = (p ? n : n - UP) * NT + threadIdx.x;
        if constexpr (DMA) {
            uint32_t o = off[n];
            if (aim_s + STEP > a.S && !(p ? PC : QC)) {            // places of "rows" past the end of the sums: past the buffer
                const int at = p ? swizzle<PC, false, TI>(u & 7, u >> 3) : swizzle<QC, true, TJ>(u & 7, u >> 3);
                o = at * (16 / ES) < a.S - aim_s ? o : 0x80000000u;
            }
            load_to_lds(lds0 + buf * STAGE + ((p ? n * NT : TI * 8 + (n - UP) * NT) + wave * 64) * 16, p ? rsrc_p : rsrc_q, o);
        }
    };
    auto pieces = [&](int from, int to, int buf) {
        if constexpr (DMA) {
#pragma unroll
            for (int n = 0; n < UP + UQ; ++n)
                if (n >= from && n < to) piece(n, buf);
        } else {                                                   // all at once
            const bool inside = aim_s + STEP <= a.S;               // no unit reaches past the end of a row
            if (inside && (!PC || i0 + TI <= a.I) && a.ldp < ((int64_t)1 << 23)) {
                const char* base = (const char*)a.P + (PC ? aim_s * a.ldp + i0 : i0 * a.ldp + aim_s) * ES;
#pragma unroll
                for (int n = 0; n < UP; ++n) raw[n] = (u32x4_al)*reinterpret_cast<const u32x4_b*>(base + off[n]);
            } else {
#pragma unroll
                for (int n = 0; n < UP; ++n) raw[n] = load_unit<ES, PC, false, TI>(a.P, a.ldp, i0, a.I, aim_s, a.S, n * NT + threadIdx.x);
            }
            if (inside && (!QC || j0 + TJ <= a.J) && a.ldq < ((int64_t)1 << 23)) {
                const char* base = (const char*)a.Q + (QC ? aim_s * a.ldq + j0 : j0 * a.ldq + aim_s) * ES;
#pragma unroll
                for (int n = 0; n < UQ; ++n) raw[UP + n] = (u32x4_al)*reinterpret_cast<const u32x4_b*>(base + off[UP + n]);
            } else {
#pragma unroll
                for (int n = 0; n < UQ; ++n) raw[UP + n] = load_unit<ES, QC, true, TJ>(a.Q, a.ldq, j0, a.J, aim_s, a.S, n * NT + threadIdx.x);
            }
        }
    };
    auto put = [&](int buf) {
        if constexpr (!DMA) {
#pragma unroll
            for (int n = 0; n < UP + UQ; ++n)
                *reinterpret_cast<u32x4_al*>(lds + buf * STAGE + ((n < UP ? n * NT : TI * 8 + (n - UP) * NT) + threadIdx.x) * 16) = raw[n];
        }
    };

    floatx4 acc[FI][4], sums[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[i][f] = floatx4{0.f, 0.f, 0.f, 0.f};
        sums[f] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const bool make_sums = OP == GRAD_W && ti == 0 && wi == 0 && a.db;

    // byte of a lane's part of fragment f at half s of the step (columns: of its rows 4 half ..)
    auto at_p = [&](int f, int s, int half) {
        if constexpr (PC) {
            const int row = 32 * s + 8 * g + 4 * half + (t >> 2);
            return row * (TI * 2) + 16 * swizzle<PC, false, TI>((wi * FI + f) * 2 + ((t >> 1) & 1), row) + 8 * (t & 1);
        } else {
            const int row = (wi * FI + f) * 16 + t;
            return row * 128 + 16 * swizzle<PC, false, TI>(4 * s + g, row);
        }
    };
    auto at_q = [&](int f, int s, int half) {
        if constexpr (QC) {
            const int row = 32 * s + 8 * g + 4 * half + (t >> 2);
            return TI * 128 + row * (TJ * 2) + 16 * swizzle<QC, true, TJ>(wj * 8 + (t & 3) * 2 + (f >> 1), row) + 8 * (f & 1);
        } else {
            const int row = wj * 64 + (t >> 2) * 16 + f * 4 + (t & 3);
            return TI * 128 + row * 128 + 16 * swizzle<QC, true, TJ>(4 * s + g, row);
        }
    };
    typedef FragOf<OP> Frag;
    constexpr int PHASES = OP == FWD_E4M3 ? 1 : 2;
    auto read = [&](const char* buf, auto columns, auto at, int f, int s) -> Frag {
        if constexpr (OP == FWD_E4M3) {
            const u32x4_al lo = *reinterpret_cast<const u32x4_al*>(buf + at(f, 0, 0)), hi = *reinterpret_cast<const u32x4_al*>(buf + at(f, 1, 0));
            return __builtin_bit_cast(intx8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else if constexpr (decltype(columns)::value) {
            typedef shortx4 __attribute__((address_space(3))) * tr_ptr;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(buf + at(f, s, 0)));
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(buf + at(f, s, 1)));
            return __builtin_bit_cast(u32x4_al, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const u32x4_al*>(buf + at(f, s, 0));
        }
    };
    auto read_p = [&](const char* buf, int s, int i) { return read(buf, std::integral_constant<bool, PC>(), at_p, i, s); };
    auto read_q = [&](const char* buf, int s, int f) { return read(buf, std::integral_constant<bool, QC>(), at_q, f, s); };
    if (s_begin < s_end) {
        // A step's last TAIL rows of fragments are multiplied behind the barrier that gives its stage free, column by column; a column's operand of the next
        // step is read as soon as it is no longer needed.  So neither the barrier nor the latency of LDS leaves the matrix unit without work.
        //   The loads of the step after the next go between the products, EARLY of them behind the barrier and the others among the next step's first rows: a
        // wavefront that asks for all of them at once is held up until the address unit has taken the 64 KB that all eight ask for.  (8192^3, us, all at once /
        // spread: dx 865 / 843, forward 871 / 804, dw 892 / 822, e4m3 420 / 393; of these a quarter, a half, three quarters behind the barrier: dx 859, 822,
        // 829, e4m3 405, 409, 384.)  A wavefront that has its operands goes before one that asks for some: dx 822 -> 798.
        constexpr int TAIL = FI > 4 ? 3 : 2, ALL = UP + UQ, EARLY = OP == FWD_E4M3 ? ALL * 3 / 4 : ALL / 2;
        Frag q[4], p[4];
        aim(s_begin);
        pieces(0, ALL, 0);
        put(0);
        aim(s_begin + STEP);
        if constexpr (DMA) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (DMA || s_begin + STEP < s_end) pieces(0, DMA ? EARLY : ALL, 1);
        __syncthreads();
#pragma unroll
        for (int f = 0; f < 4; ++f) q[f] = read_q(lds, 0, f);
        p[0] = read_p(lds, 0, 0);
        int buf = 0;
        for (int64_t s0 = s_begin; s0 < s_end; s0 += STEP, buf ^= 1) {
            const char *const here = lds + buf * STAGE, *const next = lds + (buf ^ 1) * STAGE;
#pragma unroll
            for (int s = 0; s < PHASES; ++s) {
#pragma unroll
                for (int i = 0; i < FI - TAIL; ++i) {
                    constexpr int ROWS = FI - TAIL, MORE = ALL - EARLY, EACH = (MORE + ROWS - 1) / ROWS;
                    p[(i + 1) % 4] = read_p(here, s, i + 1);
                    if (DMA && s == 0) pieces(EARLY + i * EACH, EARLY + (i + 1) * EACH, buf ^ 1);
                    __builtin_amdgcn_s_setprio(1);
#pragma unroll
                    for (int f = 0; f < 4; ++f) multiply<OP>(q[f], p[i % 4], acc[i][f]);
                    __builtin_amdgcn_s_setprio(0);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int i = FI - TAIL + 1; i < FI; ++i) p[i % 4] = read_p(here, s, i);
                const bool ends = s == PHASES - 1;
                if (ends) {
                    if (!DMA && s0 + STEP < s_end) put(buf ^ 1);
                    if constexpr (DMA) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the next step's stage
                    __syncthreads();                                                        // all have read this one, and all see the next
                    aim(s0 + 2 * STEP);
                    if (!DMA && s0 + 2 * STEP < s_end) pieces(0, ALL, buf);
                }
                const char* const then = ends ? next : here;                     // (after the last step: what is there; nobody uses it)
                const int then_s = ends ? 0 : s + 1;
                p[FI % 4] = read_p(then, then_s, 0);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    if (DMA && ends) pieces(f * EARLY / 4, (f + 1) * EARLY / 4, buf);
#pragma unroll
                    for (int i = FI - TAIL; i < FI; ++i) multiply<OP>(q[f], p[i % 4], acc[i][f]);
                    if constexpr (OP == GRAD_W) {
                        if (make_sums) {
                            const bf16x8 one = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
                            multiply<OP>(q[f], __builtin_bit_cast(u32x4_al, one), sums[f]);
                        }
                    }
                    q[f] = read_q(then, then_s, f);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if constexpr (DMA) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                  // (no load may write LDS when it is another workgroup's)
    }

    // Out by way of LDS, 32 rows of the wavefront's 64 columns at a time, in its own part of it: a wavefront then loads and stores whole lines (128 bytes of
    // eight rows, or 256 of four).  Straight from the registers, 64 bytes of 16 rows at a time, fp32 results of 65536 x 4096 (K = 256) took 419 us, now 297.
    __syncthreads();
    constexpr int PITCH = 68, BATCHES = FI / 2;
    static_assert(2 * STAGE / (WI * WJ) >= 32 * PITCH * 4, "32 rows of every wavefront fit LDS");
    float* const mine = (float*)(lds + wave * (2 * STAGE / (WI * WJ)));
    const int64_t row0 = i0 + wi * FI * 16;
    const int col0 = (int)j0 + wj * 64;
    auto batch = [&](int b) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int f = 0; f < 4; ++f) *reinterpret_cast<floatx4*>(mine + (16 * i + t) * PITCH + 16 * g + 4 * f) = acc[2 * b + i][f];
    };
    // unit u of a batch: N columns a lane of 64 N / 64 rows
    auto unit = [&](auto n, int u, float (&v)[decltype(n)::value]) {
        constexpr int N = decltype(n)::value;
        const float* p = mine + (u * N + lane / (64 / N)) * PITCH + lane % (64 / N) * N;
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const floatx4 x = *reinterpret_cast<const floatx4*>(p + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k + e] = x[e];
        }
    };
    if (a.splits > 1) {
        const int64_t rows = a.I + (OP == GRAD_W ? 1 : 0);
        float* const part = a.part + (int64_t)split * rows * a.ld_part;
        const int col = col0 + lane % 16 * 4;
#pragma unroll
        for (int b = 0; b < BATCHES; ++b) {
            batch(b);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                float v[4];
                unit(std::integral_constant<int, 4>(), u, v);
                const int64_t row = row0 + 32 * b + 4 * u + lane / 16;
                if (row < a.I && col < a.ld_part) *reinterpret_cast<floatx4*>(part + row * a.ld_part + col) = floatx4{v[0], v[1], v[2], v[3]};
            }
        }
        if (OP == GRAD_W && make_sums && t == 0 && col0 + 16 * g < a.ld_part)
#pragma unroll
            for (int f = 0; f < 4; ++f) *reinterpret_cast<floatx4*>(part + a.I * a.ld_part + col0 + 16 * g + 4 * f) = sums[f];
        return;
    }
    auto rows_out = [&](auto type, auto activation, auto all_columns) {
        constexpr bool BF16 = decltype(type)::value, WHOLE = decltype(all_columns)::value;
        constexpr int N = BF16 ? 8 : 4, UNITS = 32 / N, ACT = decltype(activation)::value;
        constexpr int AHEAD = !BF16 ? 1 : OP == GRAD_X ? BATCHES : BATCHES < 2 ? BATCHES : 2;      // batches whose further terms are on their way: what registers allow
        const bool more = takes_more<OP>(a);
        const int col = col0 + lane % (64 / N) * N;
        const bool here = col < a.J;
        ColumnTerms<OP, N> terms;
        if (here) terms = ColumnTerms<OP, N>(a, col, WHOLE);
        RowPart<N, BF16> further[AHEAD][UNITS];
        auto ask = [&](int b) {
            if (more && here)
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    const int64_t row = row0 + 32 * b + u * N + lane / (64 / N);
                    if (row < a.I) load_more<OP>(a, row, col, further[b % AHEAD][u], WHOLE);
                }
        };
#pragma unroll
        for (int b = 0; b < AHEAD; ++b) ask(b);
#pragma unroll
        for (int b = 0; b < BATCHES; ++b) {
            batch(b);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                float v[N];
                unit(std::integral_constant<int, N>(), u, v);
                const int64_t row = row0 + 32 * b + u * N + lane / (64 / N);
                if (here && row < a.I) finish<OP, N, BF16, ACT, WHOLE>(a, row, col, v, terms, more, further[b % AHEAD][u]);
            }
            if (b + AHEAD < BATCHES) ask(b + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // One run of code for each activation where a lane's columns all exist or none does: a small product spends a good part of its time on fetching code for
    // the first time (512 x 256, K = 256 8.1 -> 7.1 us; 3e5 x 256 of K = 256 142 -> 134).
    for_more_type<OP>(a, [&](auto type) {
        if (col0 + 64 > a.J && a.J % (decltype(type)::value ? 8 : 4) != 0) {
            rows_out(type, std::integral_constant<int, -1>(), std::false_type());
        } else if (OP == GRAD_W || a.act == GRP_ACT_NONE) {
            rows_out(type, std::integral_constant<int, GRP_ACT_NONE>(), std::true_type());
        } else {
            if constexpr (OP != GRAD_W) for_act(a.act, [&](auto act) { rows_out(type, act, std::true_type()); });
        }
    });
    if (OP == GRAD_W && make_sums && t == 0) {
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = sums[e >> 2][e & 3];
        const int col = col0 + 16 * g;
        if (col < a.J) store_row<16, false>(a.db + col, a.J - col, v);
    }
}

// The partial results of all splits, added in a fixed order, to the outputs: four columns a thread, and SLICES threads for each, which take a run of the splits
// and are added in LDS.  (dw of 256 x 256 in 127 splits: 64 workgroups and 10.5 us with one, 7.7 us with eight.)
template <int OP, int SLICES> __global__ __launch_bounds__(256) void linear_sum_kernel(LinearArgs a) {
    constexpr int EACH = 256 / SLICES;
    __shared__ floatx4 sums[SLICES > 1 ? SLICES : 1][SLICES > 1 ? EACH : 1];
    const int quads = a.ld_part / 4, slice = threadIdx.x / EACH;
    const int64_t at = (int64_t)blockIdx.x * EACH + threadIdx.x % EACH, row = at / quads, rows = a.I + (OP == GRAD_W ? 1 : 0);
    const int j = (int)(at % quads) * 4;
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
    if (row < rows) {
        const float* p = a.part + row * a.ld_part + j;
        const int per = (a.splits + SLICES - 1) / SLICES, first = slice * per, end = first + per < a.splits ? first + per : a.splits;
        if (first < end)
            in_order(first, end, [&](int k) { return *reinterpret_cast<const floatx4*>(p + (int64_t)k * rows * a.ld_part); },
                     [&](floatx4 v, bool on) { if (on) s += v; });
    }
    if constexpr (SLICES > 1) {
        sums[slice][threadIdx.x % EACH] = s;
        __syncthreads();
        if (slice > 0) return;
#pragma unroll
        for (int k = 1; k < SLICES; ++k) s += sums[k][threadIdx.x];
    }
    if (row >= rows) return;
    float v[4] = {s[0], s[1], s[2], s[3]};
    if (OP == GRAD_W && row == a.I) {
        if (a.db) store_row<4, false>(a.db + j, a.J - j, v);
        return;
    }
    for_more_type<OP>(a, [&](auto type) {
        RowPart<4, decltype(type)::value> terms;
        const bool more = takes_more<OP>(a);
        if (more) load_more<OP>(a, row, j, terms);
        finish<OP, 4, decltype(type)::value>(a, row, j, v, ColumnTerms<OP, 4>(a, j), more, terms);
    });
}

// ------------------------------------------------------------------ few rows
// Products of at most 64 rows are bound by reading W once.  A workgroup of sixteen wavefronts makes 16 MI rows and 16 F columns; every wavefront takes blocks
// of 128 bytes of s (all sixteen together consecutive ones) straight into registers, several in flight, and the sixteen sums are added in LDS: one
// launch, however long the sums.  W by columns: 32 F bytes of 32 / F rows a load, turned around by way of LDS of the wavefront's own (with loads of
// four bytes, which need no turning but byte permutations, a row times 4096 x 4096 took 14.1 us, now 11.7).  F = 1 where W has no more than 4096 columns, so that every
// CU has a workgroup: the same 8.9 us (3.8 TB/s, of which some 2 us are the launch); 8192 columns, K = 4096 19.3 and, F = 2, 16.2.
//   Lane (g, t) has D[t, 16 f + 4 g + e] in fragment f.
template <int OP, int F> struct FewBlock {                  // a lane's part of 128 bytes of s
    static constexpr int ES = elem_size(OP), STEP = 128 / ES;
    static constexpr bool QC = q_columns(OP);
    u32x4_al q[2 * F];  // rows: fragment f's halves at 2 f, 2 f + 1;  columns: row lane / 2F + 32 k / F of the block at k, columns 8 (lane % 2F) ..

    // jc, down: where a lane's columns begin and how far they are moved down (QC); jr: the lane's rows of Q, existing ones
    __device__ __forceinline__ void load(const LinearArgs& a, int64_t s0, int lane, int64_t jc, const int64_t (&jr)[F], bool whole) {
        if constexpr (QC) {
#pragma unroll
            for (int k = 0; k < 2 * F; ++k) {
                const int64_t s = s0 + 32 / F * k + lane / (2 * F);
                q[k] = u32x4_al{0, 0, 0, 0};
                if (whole || s < a.S) q[k] = (u32x4_al)*reinterpret_cast<const u32x4_b*>((const uint16_t*)a.Q + s * a.ldq + jc);
            }
        } else {
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int h = 0; h < 2; ++h) q[2 * f + h] = part_of(a.Q, a.ldq, jr[f], s0, a.S, 4 * h + (lane >> 4), whole);
        }
    }
    static __device__ __forceinline__ u32x4_al part_of(const void* base, int64_t ld, int64_t o, int64_t s0, int64_t S, int at, bool whole) {
        const int64_t s = s0 + at * (16 / ES);
        const char* row = (const char*)base + o * ld * ES;
        if (whole) return (u32x4_al)*reinterpret_cast<const u32x4_b*>(row + s * ES);
        return load_part<ES>(row, s, S);
    }
};

constexpr int FEW_WAVES = 16;
template <int OP, int MI, int F> __global__ __launch_bounds__(64 * FEW_WAVES) void linear_few_kernel(LinearArgs a) {
    typedef FewBlock<OP, F> Block;
    constexpr int STEP = Block::STEP, U = MI == 1 ? 4 : MI == 2 ? 2 : 1;
    constexpr bool QC = Block::QC;
    constexpr int PITCH = 16 * F + 4, OWN = QC && 16 * MI * PITCH < 512 * F ? 512 * F : 16 * MI * PITCH;       // a wavefront's LDS, in floats: a block to turn, then its sums
    __shared__ __attribute__((aligned(16))) float part[FEW_WAVES * OWN];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, t = lane & 15;
    // workgroups b and b + 8 run on one XCD: those that share the lines of W's rows (of 64 columns) do
    constexpr unsigned SHARE = 4 / F;
    const unsigned nb = (unsigned)a.tiles_j, b = blockIdx.x, whole_groups = nb / (8 * SHARE) * (8 * SHARE);
    const unsigned col_block = b < whole_groups ? b / (8 * SHARE) * (8 * SHARE) + (b % 8) * SHARE + (b / 8) % SHARE : b;
    char* const turn = (char*)(part + wave * OWN);
    const int64_t j0 = (int64_t)col_block * 16 * F, i0 = (int64_t)blockIdx.y * 16 * MI;
    const int64_t j = j0 + 8 * (lane % (2 * F)), jc = j <= a.J - 8 ? j : a.J - 8;      // (the last columns from the row's last 16 bytes, moved down)
    const bool edge = j0 + 16 * F > a.J;
    int64_t jr[F];
#pragma unroll
    for (int f = 0; f < F; ++f) jr[f] = j0 + 16 * f + t < a.J ? j0 + 16 * f + t : a.J - 1;
    int64_t row[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) row[i] = i0 + 16 * i + t < a.I ? i0 + 16 * i + t : a.I - 1;

    floatx4 acc[MI][F];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int f = 0; f < F; ++f) acc[i][f] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto take = [&](auto count, int64_t s0, bool whole) {
        constexpr int N = decltype(count)::value;
        Block q[N];
        u32x4_al p[N][MI][2];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            q[n].load(a, s0 + n * STEP, lane, jc, jr, whole);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) p[n][i][h] = Block::part_of(a.P, a.ldp, row[i], s0 + n * STEP, a.S, 4 * h + g, whole);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (QC) {
#pragma unroll
                for (int k = 0; k < 2 * F; ++k) {
                    const u32x4_al v = edge ? moved_down<2>(q[n].q[k], j - jc) : q[n].q[k];
                    *reinterpret_cast<u32x4_al*>(turn + 1024 * k + 16 * lane) = v;       // (rows of 32 F bytes)
                }
                __builtin_amdgcn_wave_barrier();                     // (a wavefront's accesses to LDS are made in order)
            }
#pragma unroll
            for (int f = 0; f < F; ++f) {
                if constexpr (OP == FWD_E4M3) {
                    const intx8 w = __builtin_bit_cast(intx8, __builtin_shufflevector(q[n].q[2 * f], q[n].q[2 * f + 1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int i = 0; i < MI; ++i)
                        multiply<OP>(w, __builtin_bit_cast(intx8, __builtin_shufflevector(p[n][i][0], p[n][i][1], 0, 1, 2, 3, 4, 5, 6, 7)), acc[i][f]);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        u32x4_al w;
                        if constexpr (QC) {
                            typedef shortx4 __attribute__((address_space(3))) * tr_ptr;
                            const char* at = turn + (32 * h + 8 * g + (t >> 2)) * (32 * F) + 32 * f + 8 * (t & 3);
                            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(at + 4 * 32 * F));
                            w = __builtin_bit_cast(u32x4_al, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                        } else {
                            w = q[n].q[2 * f + h];
                        }
#pragma unroll
                        for (int i = 0; i < MI; ++i) multiply<OP>(w, p[n][i][h], acc[i][f]);
                    }
                }
            }
            if constexpr (QC) __builtin_amdgcn_wave_barrier();
        }
    };
    const int64_t full = a.S / STEP;
    int64_t k = (int64_t)wave * U;
    for (; k + U <= full; k += FEW_WAVES * U) take(std::integral_constant<int, U>(), k * STEP, true);
    for (int64_t end = k + U; k < end && k * STEP < a.S; ++k) take(std::integral_constant<int, 1>(), k * STEP, k < full);

#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int f = 0; f < F; ++f) *reinterpret_cast<floatx4*>(part + wave * OWN + (16 * i + t) * PITCH + 16 * f + 4 * g) = acc[i][f];
    __syncthreads();
    const int r = threadIdx.x / (4 * F), c4 = threadIdx.x % (4 * F) * 4;
    if (r >= 16 * MI || i0 + r >= a.I || j0 + c4 >= a.J) return;
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) s += *reinterpret_cast<const floatx4*>(part + w * OWN + r * PITCH + c4);
    float v[4] = {s[0], s[1], s[2], s[3]};
    for_more_type<OP>(a, [&](auto type) {
        RowPart<4, decltype(type)::value> terms;
        const bool more = takes_more<OP>(a);
        if (more) load_more<OP>(a, i0 + r, (int)j0 + c4, terms);
        finish<OP, 4, decltype(type)::value>(a, i0 + r, (int)j0 + c4, v, ColumnTerms<OP, 4>(a, (int)j0 + c4), more, terms);
    });
}

// ------------------------------------------------------------------ many rows, short sums
// Products of many rows with sums of at most 1024 bytes are bound by their rows, not by arithmetic, and in tiles a workgroup mostly waits: for its first loads,
// for its last stores.  Here W stays: a workgroup keeps up to 128 KB of it (blocks of 64 columns) in LDS, and each of its eight wavefronts walks over rows, 16 at a
// time, on its own: their 16 x S operands come straight into registers, one walk ahead, no barrier in the loop, and 64 columns after the other are
// multiplied and stored.  Over 3e5 rows, GELU and residual (ReLU alone), us, tiles and this: 64 by 64 42 and 26 (29 and 16), K = 256 by 47 93 and 64 (61 and 47); 256 by 256
// 135 and 140 (84 and 101).  It takes rows at any alignment (ODD: that are no whole dwords): 65 by 65 74 and 52 (56 and 33); 8192 rows of them 15.6 and 7.5.
//   CHUNKS: of 64 bytes of s; BLOCKS: of 64 columns that LDS has room for at CHUNKS.  fp32 results: fragment f has columns 16 f + t, so that a store has 64
// bytes of a row; bf16: lane g has 16 columns, 32 bytes of its row.
constexpr int TALL_WAVES = 8;
template <int OP, int CHUNKS, bool CF32, bool ODD, int LDS_KB> __global__ __launch_bounds__(64 * TALL_WAVES, 2) void linear_tall_kernel(LinearArgs a, int blocks, int64_t rows_16) {
    static_assert(OP == FWD_BF16 || OP == GRAD_X, "bf16 operands");
    constexpr bool QC = q_columns(OP);
    constexpr int STEPS = (CHUNKS + 1) / 2, BLOCK = STEPS * 64 * 128, BLOCKS = LDS_KB * 1024 / BLOCK;
    __shared__ __attribute__((aligned(16))) char lds[BLOCKS * BLOCK];
    __shared__ float lds_bias[BLOCKS * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, t = lane & 15;
    const int64_t j0 = (int64_t)blockIdx.y * blocks * 64;
    const int mine = (int)((a.J - j0 + 63) / 64) < blocks ? (int)((a.J - j0 + 63) / 64) : blocks;

    for (int u = threadIdx.x; u < mine * (BLOCK / 16); u += 64 * TALL_WAVES) {
        const int b = u / (BLOCK / 16), step = u % (BLOCK / 16) / 512;
        *reinterpret_cast<u32x4_al*>(lds + u * 16) = load_unit<2, QC, !CF32, 64>(a.Q, a.ldq, j0 + b * 64, a.J, step * 64, a.S, u % 512);
    }
    if constexpr (OP == FWD_BF16)
        for (int c = threadIdx.x; c < mine * 64; c += 64 * TALL_WAVES) lds_bias[c] = a.bias && j0 + c < a.J ? a.bias[j0 + c] : 0.f;
    __syncthreads();

    auto operand = [&](int b, int f, int chunk) -> bf16x8 {
        const char* const L = lds + b * BLOCK + (chunk >> 1) * (64 * 128);
        const int s = chunk & 1;
        if constexpr (QC) {
            typedef shortx4 __attribute__((address_space(3))) * tr_ptr;
            auto at = [&](int half) {
                const int row = 32 * s + 8 * g + 4 * half + (t >> 2);
                const int place = CF32 ? f * 2 + ((t >> 1) & 1) : (t & 3) * 2 + (f >> 1);
                return row * 128 + 16 * swizzle<true, !CF32, 64>(place, row) + 8 * (CF32 ? t & 1 : f & 1);
            };
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(L + at(0))), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(L + at(1)));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int row = CF32 ? f * 16 + t : (t >> 2) * 16 + f * 4 + (t & 3);
            return *reinterpret_cast<const bf16x8*>(L + row * 128 + 16 * swizzle<false, !CF32, 64>(4 * s + g, row));
        }
    };
    constexpr int ALWAYS = CHUNKS > 2 ? CHUNKS / 2 : 0;              // chunks that every S of this kernel has (two chunks: S >= 8)
    const int inside = (int)(a.S / 32), most = (int)a.S - 8;         // chunks that no row ends in; where a row's last 16 bytes begin
    std::conditional_t<ODD, AnyUnit, PlainUnit> p[CHUNKS];
    u32x4_al now[CHUNKS];
    auto ask = [&](int64_t r) {
        const int64_t i = r * 16 + t < a.I ? r * 16 + t : a.I - 1;   // (a row past the end: any; it is not stored)
        const char* const row = (const char*)a.P + i * a.ldp * 2;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = c * 32 + g * 8, from = c < ALWAYS || at < most ? at : most;      // (the last ones from the row's last 16 bytes)
            p[c].load(row + from * 2);
        }
    };
    const bool more = takes_more<OP>(a);
    const int64_t first = (int64_t)blockIdx.x * TALL_WAVES + wave, stride = (int64_t)gridDim.x * TALL_WAVES;
    if (first < rows_16) ask(first);
    for (int64_t r = first; r < rows_16; r += stride) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            now[c] = p[c].value();
            if (c >= ALWAYS && c >= inside) now[c] = moved_down<2>(now[c], c * 32 + g * 8 > most ? c * 32 + g * 8 - most : 0);
        }
        const int64_t row = r * 16 + t;
        constexpr bool TB = OP == GRAD_X || !CF32;                   // the type of what a row takes besides
        constexpr int N = CF32 ? 4 : 16, PARTS = CF32 ? 4 : 1;
        RowPart<N, TB> further[PARTS];
        auto ask_more = [&](int b) {
#pragma unroll
            for (int f = 0; f < PARTS; ++f) {
                const int col = (int)j0 + b * 64 + (CF32 ? 16 * f + 4 * g : 16 * g);
                if (more && row < a.I && col < a.J) load_more<OP>(a, row, col, further[f]);
            }
        };
        ask_more(0);
        if (r + stride < rows_16) ask(r + stride);
        for (int b = 0; b < mine; ++b) {
            floatx4 acc[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) acc[f] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int f = 0; f < 4; ++f)
                    acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(b, f, c), __builtin_bit_cast(bf16x8, now[c]), acc[f], 0, 0, 0);
            RowPart<N, TB> these[PARTS];
#pragma unroll
            for (int f = 0; f < PARTS; ++f) these[f] = further[f];
            if (b + 1 < mine) ask_more(b + 1);
#pragma unroll
            for (int f = 0; f < PARTS; ++f) {
                const int in = b * 64 + (CF32 ? 16 * f + 4 * g : 16 * g), col = (int)j0 + in;
                if (row < a.I && col < a.J) {
                    ColumnTerms<OP, N> terms;
                    if constexpr (OP == FWD_BF16)
#pragma unroll
                        for (int e = 0; e < N; ++e) terms.bias.w[e] = __float_as_uint(lds_bias[in + e]);
                    float v[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] = acc[CF32 ? f : e >> 2][e & 3];
                    finish<OP, N, TB>(a, row, col, v, terms, more, these[f]);
                }
            }
        }
    }
}

// ------------------------------------------------------------------ rows that are no whole units
// An operand's rows copied to whole units of 16 bytes, zeros behind them: tiles of such rows go straight into LDS, where others come by way of registers
// (8192 x 4096, K = 4096 211 us, with rows of 4097 549: for 2 x 33 MB more the first is had again).
struct PackOperand {
    const void* from;
    int64_t ld, rows, length;           // elements
    void* to;
    int64_t units;                      // of a row
};
template <int ES> __global__ __launch_bounds__(256) void linear_pack_kernel(PackOperand a, PackOperand b) {
    const uint32_t all = (uint32_t)(a.rows * a.units), both = all + (uint32_t)(b.rows * b.units);
    for (uint32_t u0 = blockIdx.x * 1024 + threadIdx.x; u0 < both; u0 += gridDim.x * 1024) {
        u32x4_al v[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {                        // four loads on their way
            const uint32_t u = u0 + k * 256, in = u < all ? u : u - all;
            if (u >= both) break;
            const PackOperand& o = u < all ? a : b;
            const uint32_t row = in / (uint32_t)o.units, at = in - row * (uint32_t)o.units;
            v[k] = load_part<ES>((const char*)o.from + row * o.ld * ES, at * (16 / ES), o.length);
        }
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t u = u0 + k * 256;
            if (u < both) reinterpret_cast<u32x4_al*>((u < all ? a : b).to)[u < all ? u : u - all] = v[k];
        }
    }
}
constexpr int64_t MOST_PACKED = (int64_t)3 << 30;       // units of both operands, which are counted in 32 bits

// ------------------------------------------------------------------ host
struct LinearPlan {
    int shape = 0;                      // of LINEAR_TILES
    int few = 0, few_columns = 0;       // fragments of rows and columns of linear_few_kernel (0: tiles)
    bool tall = false;                  // linear_tall_kernel, whatever the alignment
    size_t packed_p = 0, packed_q = 0;  // bytes of the operands' copies as whole units (0: none)
    int64_t steps = 0, per_split = 0;
    int32_t tiles_j = 0, splits = 1, ld_part = 0;
    size_t bytes = 0;
};
// The tiles there are, and what a step of 128 bytes of one takes, in us, with one workgroup on a CU and with as many as fit there; what a tile takes
// besides (measured on products of K = 64 .. 4096 over 128 .. 3e5 rows).
struct TileShape { int i, j, most, threads; float step[3], besides; };
constexpr TileShape LINEAR_TILES[] = {{64, 128, 3, 128, {0.50f, 0.55f, 0.78f}, 1.5f}, {128, 128, 2, 256, {0.62f, 0.95f, 0.f}, 2.f}, {256, 256, 1, 512, {1.6f, 0.f, 0.f}, 6.f}};
constexpr int CUS = 256;
// Whether a launch of so many workgroups of `threads` holds fewer than 2^32 work-items, which is the limit.
bool launch_holds(double workgroups, int threads) { return workgroups * threads < 4294967296.0; }

// What linear_tall_kernel can take.
bool may_be_tall(int op, int64_t S) { return (op == FWD_BF16 || op == GRAD_X) && S >= 8 && (S <= 256 || (S <= 512 && S % 2 == 0)); }

// The tile and the number of splits of the sums with the least time by a model of it: workgroups in rounds of what fits the CUs, 15 TB/s for the tiles' loads,
// and for splits a second launch that reads the partial sums (1.5 us; two launches cost the host 9.5).  Against the best of all tiles and splits, on 90
// products (forward of 128 .. 3e5 rows and dw): forward 1.3 % slower in the mean and 13 % at most, dw 2.0 % and 26 %.
//   Examples, us: forward 512 x 4096, K = 4096: 128 x 128 in 2 splits 38, unsplit 47, 256 x 256 (4) 50; 8192 x 4096, K = 4096: 256 x 256 211, 128 x 128 258; 512 x 256,
// K = 256: 64 x 128 8.0, 256 x 256 15.8; dw over 8192 rows, 256 x 256: 64 x 128 in 16 splits 13.7, unsplit 81.
//   By way of registers (rows that are no whole units): 128 x 128 tiles, whose step then takes 2.1 us alone and 3.1 with another on the CU, and 9 us at least.
double search_tiles(LinearPlan& p, int op, int64_t I, int32_t J, bool registers) {
    double best = 0.0;
    const double extra = op == GRAD_W ? 1.0 : 0.0;
    for (int shape = registers ? 1 : 0; shape < (registers ? 2 : 3); ++shape) {
        const TileShape& t = LINEAR_TILES[shape];
        const double tiles = (double)cdiv(I, t.i) * (double)cdiv(J, t.j);
        for (int64_t splits = 1; splits <= p.steps && splits <= 512 && (splits == 1 || tiles * splits <= 16.0 * CUS); splits *= 2) {
            const int64_t per = cdiv(p.steps, splits), real = cdiv(p.steps, per);
            const double work = tiles * real;
            double rounds = 1.0;
            const int on = (int)std::min<double>(t.most, ceil(work / CUS));
            if (work > (double)CUS * t.most) {
                rounds = work / ((double)CUS * t.most);
                rounds = rounds < 4.0 ? ceil(rounds) : rounds + 0.5;
            }
            const double step = registers ? 1.1 + on : (double)t.step[on - 1];
            double us = (registers ? 7.0 : 3.5) + std::max(rounds * (per * step + t.besides * (0.5 + 0.5 * on)), work * per * (t.i + t.j) * 128.0 / 15e6);
            if (real > 1) us = std::max(9.5, us + 1.5 + ((double)I + extra) * J * 4.0 * real / 3e6 + 0.02 * real);
            if (best == 0.0 || us < best) {
                best = us;
                p.shape = shape;
                p.per_split = per;
                p.splits = (int32_t)real;
            }
        }
    }
    return best;
}

LinearPlan plan_of(int op, int64_t I, int32_t J, int64_t S) {
    LinearPlan p;
    p.steps = std::max<int64_t>(1, cdiv(S, 128 / elem_size(op)));
    const int64_t s_bytes = S * elem_size(op);
    // Few rows: one launch, as long as the sums are not so long that tiles in splits, two launches, are faster.  Forward of bf16, J = 4096, us, this and tiles:
    // 1 row, K = 4096 8.9 and 10.9, K = 8192 17.6 and 16.6; 32 rows, K = 2048 8.3 and 10.8, K = 4096 15.1 and 14.0; 64 rows, K = 1024 (J = 256) 7.0 and 9.3, K = 2048
    // (J = 1024) 11.0 and 10.0.
    const int few_columns = J <= 16 * CUS ? 1 : 2;
    if (op != GRAD_W && I <= 64 && J >= 8 && s_bytes <= (I <= 16 ? 8 : I <= 32 ? 6 : 3) * 1024 && launch_holds((double)cdiv(J, 16 * few_columns), 64 * FEW_WAVES)) {
        p.few = I <= 16 ? 1 : I <= 32 ? 2 : 4;
        p.few_columns = few_columns;
        p.tiles_j = (int32_t)cdiv(J, 16 * p.few_columns);
        return p;
    }
    const int V = 16 / elem_size(op);
    const int64_t length_p = p_columns(op) ? I : S, length_q = q_columns(op) ? J : S;      // of the operands' rows
    const bool odd_p = length_p % V != 0, odd_q = length_q % V != 0;                       // that are no whole units
    auto take_tall = [&] {
        p.tall = true;
        p.splits = 1;
        p.shape = 1;                    // (rows of more than 256 that begin at odd elements are left to tiles, unsplit)
        p.per_split = p.steps;
        return p;
    };
    if (!odd_p && !odd_q) {
        if (may_be_tall(op, S) && I >= 8192 && J <= 128 && s_bytes <= 512) return take_tall();
        search_tiles(p, op, I, J, false);
    } else {
        // as they are, or copied to whole units first (a launch, and 4.5 TB/s both ways), or with W in LDS, which takes them at any alignment
        auto copy = [&](int64_t rows, int64_t length) { return (double)rows * (double)round_up(length, V) * elem_size(op); };
        const double copy_p = odd_p ? p_columns(op) ? copy(S, I) : copy(I, S) : 0.0, copy_q = odd_q ? q_columns(op) ? copy(S, J) : copy(J, S) : 0.0;
        LinearPlan whole = p;
        double packed = search_tiles(whole, op, I, J, false), tiles = search_tiles(p, op, I, J, true);
        if (may_be_tall(op, S)) {
            // A wavefront's 16 rows and 64 columns take 0.3 us of a CU up to S = 128, 0.42 up to 256, then 0.35 + 0.0011 S; tiles are held to 4 TB/s for A and for C and
            // one tensor like it.  us, this and the better tiles: 512 rows, 65 -> 1025 7.1 and 15.4; 3e5, 65 -> 65 52 and 74, 500 -> 129 192 and 291; 44 713, 376 -> 8175
            // 983 and 670.
            const double memory = ((double)I * S * 2.0 + (double)I * J * 4.0) / 4e6;
            const double tall = 6.5 + std::max(1.0, (double)cdiv(I, 16) * (double)cdiv(J, 64) / CUS) * (S <= 128 ? 0.3 : S <= 256 ? 0.42 : 0.35 + 0.0011 * S);
            packed = std::max(packed, memory);
            tiles = std::max(tiles, memory);
            if (tall < std::min(tiles, packed + 3.5 + 2.0 * (copy_p + copy_q) / 4.5e6)) return take_tall();
        }
        packed += 3.5 + 2.0 * (copy_p + copy_q) / 4.5e6;
        if (tiles > packed && copy_p + copy_q < 16.0 * MOST_PACKED && length_p < (1 << 20) && length_q < (1 << 20)) {
            p = whole;
            p.packed_p = (size_t)round_up((int64_t)copy_p, 256);
            p.packed_q = (size_t)round_up((int64_t)copy_q, 256);
        }
    }
    p.ld_part = (int32_t)round_up(J, 16);
    if (p.splits > 1) p.bytes = (size_t)round_up(p.splits * (I + (op == GRAD_W ? 1 : 0)) * p.ld_part * (int64_t)sizeof(float), 256);
    return p;
}

// Whether rows of n elements, `ld` apart, are whole units of 16 bytes that begin on them (and a tile's offsets fit 31 bits).
bool whole_units(const void* p, int64_t ld, int64_t n, int es) {
    return (uintptr_t)p % 16 == 0 && ld * es % 16 == 0 && n * es % 16 == 0 && ld * es < (1 << 22);
}

// How a product is made: the kernel and its launch, from sizes, pitches and alignment.
enum LinearKind { FEW, TALL, TILES };
struct LinearWay {
    LinearPlan plan;
    LinearKind kind = TILES;
    bool units_p = false, units_q = false, pack = false;     // operands whose rows are whole units; whether the others are copied to such
    bool dma = false;                    // tiles straight into LDS
    int shape = 0;                       // of LINEAR_TILES
    bool odd = false;                    // TALL: rows that are no whole dwords
    int chunks = 0, kb = 0, blocks = 0;  //       of 64 bytes of s; of LDS; of 64 columns of a workgroup
    double x = 0.0;                      // workgroups
    int64_t y = 1;
    int threads = 0;
    bool fits = true;                    // a launch holds them
};
LinearWay way_of(int op, const LinearArgs& a) {
    LinearWay w;
    w.plan = plan_of(op, a.I, a.J, a.S);
    const LinearPlan& p = w.plan;
    if (p.few) {
        w.kind = FEW;
        w.x = p.tiles_j;
        w.y = cdiv(a.I, 16 * p.few);
        w.threads = 64 * FEW_WAVES;
        return w;
    }
    const int es = elem_size(op);
    w.units_p = whole_units(a.P, a.ldp, p_columns(op) ? a.I : a.S, es);
    w.units_q = whole_units(a.Q, a.ldq, q_columns(op) ? a.J : a.S, es);
    w.odd = (uintptr_t)a.P % 4 != 0 || a.ldp % 2 != 0;
    if ((p.tall || (may_be_tall(op, a.S) && !(w.units_p && w.units_q) && !p.packed_p && !p.packed_q)) && (a.S <= 256 || !w.odd)) {
        const int64_t walks = cdiv(cdiv(a.I, 16), TALL_WAVES);
        w.chunks = a.S <= 64 ? 2 : a.S <= 128 ? 4 : a.S <= 256 ? 8 : 16;
        const int block_kb = w.chunks / 2 * 8;
        const int64_t columns = cdiv(a.J, 64);
        // as much of W as fits, but a workgroup for every CU
        w.blocks = (int)std::min<int64_t>(std::min<int64_t>(columns, 128 / block_kb), std::max<int64_t>(1, columns * std::min<int64_t>(walks, CUS) / CUS));
        w.kb = w.blocks * block_kb <= 64 ? 64 : 128;
        w.y = cdiv(columns, w.blocks);
        w.x = (double)std::min<int64_t>(walks, round_up(cdiv((int64_t)CUS * (w.kb == 64 ? 2 : 1), w.y), 8));
        w.threads = 64 * TALL_WAVES;
        if (w.y <= 65535) {              // (more columns are left to tiles)
            w.kind = TALL;
            return w;
        }
        w.y = 1;
    }
    w.pack = (p.packed_p || p.packed_q) && (w.units_p || p.packed_p) && (w.units_q || p.packed_q);
    w.dma = w.pack || (w.units_p && w.units_q);
    w.shape = w.dma ? p.shape : 1;       // by way of registers: those of 128 x 128 tiles suffice
    const TileShape& t = LINEAR_TILES[w.shape];
    w.x = (double)cdiv(a.I, t.i) * (double)cdiv(a.J, t.j) * p.splits;
    w.threads = t.threads;
    w.fits = launch_holds(w.x, w.threads);
    return w;
}

template <int OP> grp_status run_linear(const char* who, const char* name, LinearArgs a, double bytes, void* ws, size_t ws_bytes, hipStream_t st) {
    constexpr int ES = elem_size(OP);
    const LinearWay w = way_of(OP, a);
    const LinearPlan& p = w.plan;
    if (!w.fits) return fail(GRP_EUNSUPPORTED, "%s: %lld x %d results are more than a launch holds", who, (long long)a.I, a.J);
    const size_t need = p.bytes + p.packed_p + p.packed_q;
    if (need && (!ws || ws_bytes < need)) return fail(GRP_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws ? ws_bytes : (size_t)0, need);
    if (need && (uintptr_t)ws % 16) return fail(GRP_EINVAL, "%s: workspace is not 16-byte aligned", who);
    const double flops = 2.0 * (double)a.I * a.J * a.S;
    const dim3 grid((unsigned)w.x, (unsigned)w.y), group((unsigned)w.threads);
    if constexpr (OP != GRAD_W)
        if (w.kind == FEW) {
            ProfScope ps(name, st, flops, bytes);
            auto go = [&](auto kernel) { a.tiles_j = p.tiles_j; hipLaunchKernelGGL(kernel, grid, group, 0, st, a); };
            if (p.few == 1) { if (p.few_columns == 1) go(linear_few_kernel<OP, 1, 1>); else go(linear_few_kernel<OP, 1, 2>); }
            else if (p.few == 2) { if (p.few_columns == 1) go(linear_few_kernel<OP, 2, 1>); else go(linear_few_kernel<OP, 2, 2>); }
            else { if (p.few_columns == 1) go(linear_few_kernel<OP, 4, 1>); else go(linear_few_kernel<OP, 4, 2>); }
            GRP_LAUNCH_CHECK();
            return GRP_OK;
        }
    if constexpr (OP == FWD_BF16 || OP == GRAD_X)
        if (w.kind == TALL) {
            ProfScope ps(name, st, flops, bytes);
            auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, group, 0, st, a, w.blocks, cdiv(a.I, 16)); };
            auto by_type = [&](auto c, auto lds) {
                constexpr int C = decltype(c)::value, KB = decltype(lds)::value;
                auto by_row = [&](auto o) {
                    if (a.c_bf16) go(linear_tall_kernel<OP, C, false, decltype(o)::value, KB>);
                    else go(linear_tall_kernel<OP, C, true, decltype(o)::value, KB>);
                };
                if (!w.odd) by_row(std::false_type());
                else if constexpr (C <= 8) by_row(std::true_type());
            };
            auto by_lds = [&](auto c) {
                if (w.kb == 64) by_type(c, std::integral_constant<int, 64>());
                else by_type(c, std::integral_constant<int, 128>());
            };
            if (w.chunks == 2) by_lds(std::integral_constant<int, 2>());
            else if (w.chunks == 4) by_lds(std::integral_constant<int, 4>());
            else if (w.chunks == 8) by_lds(std::integral_constant<int, 8>());
            else by_lds(std::integral_constant<int, 16>());
            GRP_LAUNCH_CHECK();
            return GRP_OK;
        }
    const int64_t length_p = p_columns(OP) ? a.I : a.S, length_q = q_columns(OP) ? a.J : a.S;
    a.end_p = (((p_columns(OP) ? a.S : a.I) - 1) * a.ldp + length_p) * ES;
    a.end_q = (((q_columns(OP) ? a.S : a.J) - 1) * a.ldq + length_q) * ES;
    if (w.pack) {
        char* at = (char*)ws + p.bytes;
        PackOperand o[2] = {};
        auto copy = [&](PackOperand& k, const void*& from, int64_t& ld, int64_t& end, bool columns, int64_t O, int64_t length, size_t size) {
            k = PackOperand{from, ld, columns ? a.S : O, length, at, cdiv(length * ES, 16)};
            from = at;
            ld = k.units * 16 / ES;
            end = k.rows * k.units * 16;
            at += size;
        };
        if (!w.units_p) copy(o[0], a.P, a.ldp, a.end_p, p_columns(OP), a.I, length_p, p.packed_p);
        if (!w.units_q) copy(o[1], a.Q, a.ldq, a.end_q, q_columns(OP), a.J, length_q, p.packed_q);
        const int64_t all = o[0].rows * o[0].units + o[1].rows * o[1].units;
        if (all > 0) {
            ProfScope ps("linear_pack", st, 0.0, 32.0 * all);
            hipLaunchKernelGGL((linear_pack_kernel<ES>), dim3((unsigned)std::min<int64_t>(cdiv(all, 1024), 8192)), dim3(256), 0, st, o[0], o[1]);
            GRP_LAUNCH_CHECK();
        }
    }
    a.part = (float*)ws;
    a.splits = p.splits;
    a.ld_part = p.ld_part;
    a.steps_per_split = p.per_split;
    a.tiles_i = (int32_t)cdiv(a.I, LINEAR_TILES[w.shape].i);
    a.tiles_j = (int32_t)cdiv(a.J, LINEAR_TILES[w.shape].j);
    {
        ProfScope ps(name, st, flops, bytes);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, group, 0, st, a); };
        if (!w.dma) go(linear_kernel<OP, 2, 2, 4, false>);
        else if (w.shape == 0) go(linear_kernel<OP, 1, 2, 4, true>);
        else if (w.shape == 1) go(linear_kernel<OP, 2, 2, 4, true>);
        else go(linear_kernel<OP, 2, 4, 8, true>);
        GRP_LAUNCH_CHECK();
    }
    if (p.splits > 1) {
        const int64_t rows = a.I + (OP == GRAD_W ? 1 : 0);
        ProfScope ps("linear_sum", st, 0.0, 4.0 * rows * a.J * (p.splits + 1.0));
        const int64_t quads = rows * (p.ld_part / 4);
        if (p.splits >= 16 && quads <= 256 * CUS)              // (more have workgroups enough)
            hipLaunchKernelGGL((linear_sum_kernel<OP, 8>), dim3((unsigned)cdiv(quads, 32)), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((linear_sum_kernel<OP, 1>), dim3((unsigned)cdiv(quads, 256)), dim3(256), 0, st, a);
        GRP_LAUNCH_CHECK();
    }
    return GRP_OK;
}

}  // namespace
// What a product D[I x J] with sums of S runs as, as numbers: op is a LinearOp; out: kind, then few: fragments of rows and of columns, tall: chunks, odd rows
// and LDS, tiles: shape (3: by way of registers), splits and copied operands; then workgroups, the second dimension's, and threads.  False: refused.
bool linear_way(int op, int64_t I, int32_t J, int64_t S, const void* P, int64_t ldp, const void* Q, int64_t ldq, int64_t (&out)[7]) {
    LinearArgs a = {};
    a.P = P; a.ldp = ldp; a.Q = Q; a.ldq = ldq; a.I = I; a.J = J; a.S = S;
    const LinearWay w = way_of(op, a);
    const bool few = w.kind == FEW, tall = w.kind == TALL;
    out[0] = w.kind;
    out[1] = few ? w.plan.few : tall ? w.chunks : w.dma ? w.shape : 3;
    out[2] = few ? w.plan.few_columns : tall ? w.odd : w.plan.splits;
    out[3] = few ? 0 : tall ? w.kb : w.pack;
    out[4] = w.fits ? (int64_t)w.x : -1;
    out[5] = w.y;
    out[6] = w.threads;
    return w.fits;
}
namespace {

bool aligned_to(const void* p, int32_t dtype) { return dtype == GRP_DTYPE_E4M3 || (uintptr_t)p % (dtype == GRP_DTYPE_BF16 ? 2 : 4) == 0; }
grp_status check_sizes(const char* who, int64_t m, int32_t n, int32_t k) {
    if (m < 0 || n < 1 || k < 1) return fail(GRP_EINVAL, "%s: M = %lld, N = %d, K = %d", who, (long long)m, n, k);
    return GRP_OK;
}

}  // namespace
}  // namespace grp

extern "C" size_t grp_linear_workspace_bytes(int32_t kind, int64_t m, int32_t n, int32_t k, int32_t dtype) {
    using namespace grp;
    if (m < 0 || n < 1 || k < 1) return 0;
    if (kind != GRP_LINEAR_FORWARD && kind != GRP_LINEAR_DX && kind != GRP_LINEAR_DW) return 0;
    const LinearPlan p = kind == GRP_LINEAR_FORWARD ? plan_of(dtype == GRP_DTYPE_E4M3 ? FWD_E4M3 : FWD_BF16, m, n, k)
                         : kind == GRP_LINEAR_DX    ? plan_of(GRAD_X, m, k, n)
                                                    : plan_of(GRAD_W, k, n, m);
    return p.bytes + p.packed_p + p.packed_q;
}

extern "C" grp_status grp_linear(int64_t m, int32_t n, int32_t k, const void* a, int64_t lda, const void* w, int64_t ldw, int32_t dtype,
                                 const float* a_scale, const float* w_scale, const float* bias, int32_t act, const void* r, int64_t ldr, void* c,
                                 int64_t ldc, int32_t c_dtype, void* z, int64_t ldz, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace grp;
    GRP_TRY(check_sizes("grp_linear", m, n, k));
    const bool e8 = dtype == GRP_DTYPE_E4M3;
    if (!e8 && dtype != GRP_DTYPE_BF16) return fail(GRP_EINVAL, "grp_linear: operands are bf16 or e4m3");
    if (c_dtype != GRP_DTYPE_FP32 && c_dtype != GRP_DTYPE_BF16) return fail(GRP_EINVAL, "grp_linear: c is fp32 or bf16");
    if (act < GRP_ACT_NONE || act > GRP_ACT_SILU) return fail(GRP_EINVAL, "grp_linear: bad activation %d", act);
    if (lda < k || ldw < (e8 ? k : n) || ldc < n || (r && ldr < n) || (z && ldz < n)) return fail(GRP_EINVAL, "grp_linear: a pitch is below the row's length");
    if (!e8 && (a_scale || w_scale)) return fail(GRP_EINVAL, "grp_linear: scales belong to 8-bit operands");
    if (m == 0) return GRP_OK;
    if (!a || !w || !c) return fail(GRP_EINVAL, "grp_linear: null argument");
    if (!aligned_to(a, dtype) || !aligned_to(w, dtype) || !aligned_to(c, c_dtype) || !aligned_to(r, c_dtype) || !aligned_to(z, GRP_DTYPE_BF16) ||
        !aligned_to(bias, GRP_DTYPE_FP32) || !aligned_to(a_scale, GRP_DTYPE_FP32) || !aligned_to(w_scale, GRP_DTYPE_FP32))
        return fail(GRP_EINVAL, "grp_linear: a pointer is not aligned to its elements");
    if (m > 1 && r == c && ldr != ldc) return fail(GRP_EINVAL, "grp_linear: C in place of r needs its pitch");
    LinearArgs x = {};
    x.P = a; x.ldp = lda; x.Q = w; x.ldq = ldw; x.I = m; x.J = n; x.S = k;
    x.a_scale = a_scale; x.w_scale = w_scale; x.bias = bias; x.act = act; x.r = r; x.ldr = ldr;
    x.c = c; x.ldc = ldc; x.c_bf16 = c_dtype == GRP_DTYPE_BF16; x.z = z; x.ldz = ldz;
    const double es = e8 ? 1.0 : 2.0, cs = x.c_bf16 ? 2.0 : 4.0;
    const double bytes = ((double)m * k + (double)n * k) * es + (double)m * n * (cs * (r ? 2 : 1) + (z ? 2 : 0));
    if (e8 && x.c_bf16) return run_linear<FWD_E4M3>("grp_linear", "linear_e4m3", x, bytes, workspace, workspace_bytes, (hipStream_t)stream);
    if (e8) return run_linear<FWD_E4M3_WIDE>("grp_linear", "linear_e4m3_wide", x, bytes, workspace, workspace_bytes, (hipStream_t)stream);
    return run_linear<FWD_BF16>("grp_linear", "linear_bf16", x, bytes, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" grp_status grp_linear_dx(int64_t m, int32_t n, int32_t k, const void* dz, int64_t lddz, const void* w, int64_t ldw, int32_t act,
                                    const void* zin, int64_t ldzin, void* da, int64_t ldda, int32_t da_dtype, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    using namespace grp;
    GRP_TRY(check_sizes("grp_linear_dx", m, n, k));
    if (da_dtype != GRP_DTYPE_FP32 && da_dtype != GRP_DTYPE_BF16) return fail(GRP_EINVAL, "grp_linear_dx: da is fp32 or bf16");
    if (act < GRP_ACT_NONE || act > GRP_ACT_SILU) return fail(GRP_EINVAL, "grp_linear_dx: bad activation %d", act);
    const bool slope = act != GRP_ACT_NONE;
    if (lddz < n || ldw < n || ldda < k || (slope && ldzin < k)) return fail(GRP_EINVAL, "grp_linear_dx: a pitch is below the row's length");
    if (m == 0) return GRP_OK;
    if (!dz || !w || !da || (slope && !zin)) return fail(GRP_EINVAL, "grp_linear_dx: null argument");
    if (!aligned_to(dz, GRP_DTYPE_BF16) || !aligned_to(w, GRP_DTYPE_BF16) || !aligned_to(da, da_dtype) || (slope && !aligned_to(zin, GRP_DTYPE_BF16)))
        return fail(GRP_EINVAL, "grp_linear_dx: a pointer is not aligned to its elements");
    LinearArgs x = {};
    x.P = dz; x.ldp = lddz; x.Q = w; x.ldq = ldw; x.I = m; x.J = k; x.S = n;
    x.act = act; x.z = slope ? const_cast<void*>(zin) : nullptr; x.ldz = ldzin;
    x.c = da; x.ldc = ldda; x.c_bf16 = da_dtype == GRP_DTYPE_BF16;
    const double bytes = 2.0 * ((double)m * n + (double)k * n) + (double)m * k * ((x.c_bf16 ? 2.0 : 4.0) + (slope ? 2.0 : 0.0));
    return run_linear<GRAD_X>("grp_linear_dx", "linear_dx", x, bytes, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" grp_status grp_linear_dw(int64_t m, int32_t n, int32_t k, const void* a, int64_t lda, const void* dz, int64_t lddz, float* dw, int64_t lddw,
                                    float* db, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace grp;
    GRP_TRY(check_sizes("grp_linear_dw", m, n, k));
    if (lda < k || lddz < n || lddw < n) return fail(GRP_EINVAL, "grp_linear_dw: a pitch is below the row's length");
    if (!dw || (m > 0 && (!a || !dz))) return fail(GRP_EINVAL, "grp_linear_dw: null argument");
    if (!aligned_to(a, GRP_DTYPE_BF16) || !aligned_to(dz, GRP_DTYPE_BF16) || !aligned_to(dw, GRP_DTYPE_FP32) || !aligned_to(db, GRP_DTYPE_FP32))
        return fail(GRP_EINVAL, "grp_linear_dw: a pointer is not aligned to its elements");
    LinearArgs x = {};
    x.P = a; x.ldp = lda; x.Q = dz; x.ldq = lddz; x.I = k; x.J = n; x.S = m;
    x.c = dw; x.ldc = lddw; x.db = db;
    const double bytes = 2.0 * (double)m * ((double)n + k) + 4.0 * ((double)n * k + n);
    return run_linear<GRAD_W>("grp_linear_dw", "linear_dw", x, bytes, workspace, workspace_bytes, (hipStream_t)stream);
}
