// Answering with the trained layer (paper Section 3.1: W holds one row per class, Section 3.2: the fc forward): rows as 8-bit codes
// in the order in which matrix instructions take them, logits of a batch against every class from those codes, and the
// penalties, biases and masks that requests bring.
#include "../../include/class_logits.h"
#include "ks_common.h"
#include <type_traits>

typedef int32_t cl_i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t cl_i32x16 __attribute__((ext_vector_type(16)));

#define CL_NT 256
#define CL_PIECE 1024 /* bytes of a piece: 32 rows x 32 codes, the operand of one 32x32x32 matrix instruction */
#define CL_GROUP 64   /* classes whose two blocks of codes lie next to each other, every other class in each */

// ------------------------------------------------------------------------------------------------
// rows -> codes
// ------------------------------------------------------------------------------------------------
template <typename IN> struct ClRow; // four: elements at byte `at` of a row as a buffer, 0 where it has ended
template <> struct ClRow<float> {
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    template <int AUX> static __device__ __forceinline__ float4 four(__amdgpu_buffer_rsrc_t row, int at) {
        return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(row, at, 0, AUX));
    }
};
template <> struct ClRow<uint16_t> {
    static __device__ __forceinline__ float one(const uint16_t *p) { return ks_bf2f(*p); }
    template <int AUX> static __device__ __forceinline__ float4 four(__amdgpu_buffer_rsrc_t row, int at) {
        const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(row, at, 0, AUX));
        return make_float4(ks_bf2f(v.x & 0xFFFFu), ks_bf2f(v.x >> 16), ks_bf2f(v.y & 0xFFFFu), ks_bf2f(v.y >> 16));
    }
};
template <> struct ClRow<int8_t> {
    static __device__ __forceinline__ float one(const int8_t *p) { return (float)*p; }
    template <int AUX> static __device__ __forceinline__ float4 four(__amdgpu_buffer_rsrc_t row, int at) {
        const uint32_t v = __builtin_amdgcn_raw_buffer_load_b32(row, at, 0, AUX);
        return make_float4((float)(int8_t)v, (float)(int8_t)(v >> 8), (float)(int8_t)(v >> 16), (float)(int8_t)(v >> 24));
    }
};
// the first `left` of four elements one by one, 0 for the others
template <typename IN> __device__ __forceinline__ float4 cl_load_few(const IN *p, int left) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (left > 0) v.x = ClRow<IN>::one(p);
    if (left > 1) v.y = ClRow<IN>::one(p + 1);
    if (left > 2) v.z = ClRow<IN>::one(p + 2);
    if (left > 3) v.w = ClRow<IN>::one(p + 3);
    return v;
}

// 127 v / a to the nearest integer, halves to even, where it is one of t's two neighbours: |v| * 254 and (2 lo + 1) a are exact in F, fp64 for fp32
// rows (32 bits each), fp32 for bf16 (16; both by 2^-10, which keeps them in range).
template <typename F> __device__ __forceinline__ uint32_t cl_code(float v, float t, F a) {
    const int lo = (int)fabsf(t);
    const F l = (F)fabsf(v) * (F)(254.0 / 1024), r = (F)(2 * lo + 1) * (F)(1.0 / 1024) * a;
    const int m = l > r || (l == r && (lo & 1)) ? lo + 1 : lo;
    return (v < 0.f ? -m : m) & 255;
}
// Four codes as bytes.  inv, 127 / a rounded to fp32, is off by 2^-24 of itself, so t = v * inv by less than 2^-17 (|t| <= 127); added to 1.5 * 2^23
// it is rounded once, to an integer in the low bits.  Where t lies within 2^-16 of the middle of two (one fp32 value
// in 30,000), cl_code decides.
template <typename F> __device__ __forceinline__ uint32_t cl_codes(float4 v, float inv, F a) {
    const float whole = 12582912.f;
    const float r0 = fmaf(v.x, inv, whole), r1 = fmaf(v.y, inv, whole), r2 = fmaf(v.z, inv, whole), r3 = fmaf(v.w, inv, whole);
    const float d0 = fmaf(v.x, inv, whole - r0), d1 = fmaf(v.y, inv, whole - r1), d2 = fmaf(v.z, inv, whole - r2), d3 = fmaf(v.w, inv, whole - r3);
    uint32_t q = __builtin_amdgcn_perm(__builtin_amdgcn_perm(__float_as_uint(r3), __float_as_uint(r2), 0x0c0c0400u),
                                       __builtin_amdgcn_perm(__float_as_uint(r1), __float_as_uint(r0), 0x0c0c0400u), 0x05040100u);
    if (fmaxf(fmaxf(fabsf(d0), fabsf(d1)), fmaxf(fabsf(d2), fabsf(d3))) > 0.5f - 0x1p-16f)
        q = cl_code(v.x, v.x * inv, a) | cl_code(v.y, v.y * inv, a) << 8 | cl_code(v.z, v.z * inv, a) << 16 | cl_code(v.w, v.w * inv, a) << 24;
    return q;
}
// Reductions of N = 1 or 4 values a lane over the wavefront at once.  Of four, every lane passes two on to its neighbour and keeps two, then
// one and one; lanes of equal number modulo 4 then hold the same value's parts, and go on four and eight lanes apart, and from row
// to row by exchange (row_bcast, as in ks_wave_sum, would hand on lane 15's value only): 7 steps for four values instead of 24.
// Value i ends up in lane 63, or in lane 60 + i / 2 + i % 2 * 2.
struct ClMaxI {
    typedef int T;
    static __device__ __forceinline__ int op(int a, int b) { return max(a, b); }
    template <int CTRL, int ROWS> static __device__ __forceinline__ int move(int v) { return KS_DPP(0, v, CTRL, ROWS); }
    static __device__ __forceinline__ int with_row(int v) { // op of the two rows of 16 of a half, in both
        const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return op((int)s[0], (int)s[1]);
    }
    static __device__ __forceinline__ int with_half(int v) { // op of the two halves, in both
        const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return op((int)s[0], (int)s[1]);
    }
    static __device__ __forceinline__ int lane(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
};
struct ClSumD {
    typedef double T;
    static __device__ __forceinline__ double op(double a, double b) { return a + b; }
    template <int CTRL, int ROWS> static __device__ __forceinline__ double move(double v) {
        return __hiloint2double(KS_DPP(0, __double2hiint(v), CTRL, ROWS), KS_DPP(0, __double2loint(v), CTRL, ROWS));
    }
    static __device__ __forceinline__ double with_row(double v) {
        const auto lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
        return op(__hiloint2double((int)hi[0], (int)lo[0]), __hiloint2double((int)hi[1], (int)lo[1]));
    }
    static __device__ __forceinline__ double with_half(double v) {
        const auto lo = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
        return op(__hiloint2double((int)hi[0], (int)lo[0]), __hiloint2double((int)hi[1], (int)lo[1]));
    }
    static __device__ __forceinline__ double lane(double v, int l) {
        return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), l), __builtin_amdgcn_readlane(__double2loint(v), l));
    }
};
template <class R, int N> __device__ __forceinline__ void cl_wave_reduce(typename R::T (&t)[N]) { // no value is below 0: 0 is neutral
    static_assert(N == 1 || N == 4, "");
    typename R::T v = t[0];
    if constexpr (N == 4) {
        const bool b0 = threadIdx.x & 1, b1 = threadIdx.x & 2;
        const typename R::T u0 = R::op(b0 ? t[2] : t[0], R::template move<0xB1, 0xf>(b0 ? t[0] : t[2])); // quad_perm [1, 0, 3, 2]
        const typename R::T u1 = R::op(b0 ? t[3] : t[1], R::template move<0xB1, 0xf>(b0 ? t[1] : t[3]));
        v = R::op(b1 ? u1 : u0, R::template move<0x4E, 0xf>(b1 ? u0 : u1)); // quad_perm [2, 3, 0, 1]
    } else {
        v = R::op(v, R::template move<0x111, 0xf>(v));
        v = R::op(v, R::template move<0x112, 0xf>(v));
    }
    v = R::op(v, R::template move<0x114, 0xf>(v));
    v = R::op(v, R::template move<0x118, 0xf>(v));
    v = R::with_half(R::with_row(v));
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = R::lane(v, N == 1 ? 63 : 60 + i / 2 + i % 2 * 2);
}

// A workgroup takes RB consecutive slots (32: a whole block, or 8) of a block of 32 rows, each of its eight wavefronts RB / 8 of them at
// the same time, and NP * 256 elements of a row at a time: they stay in registers from the search for the largest to the
// codes (longer rows are read twice), the codes go through LDS so that RB * 16 bytes in a row are stored.
// What bounds it: the rows in, the codes out: 390,625 x 512 fp32 with norms 182 us (1.0 GB at 5.5 TB/s), bf16 135 (0.6 GB at 4.4 TB/s: the ties of
// values of 8 bits, 8 % of the time, and the sums of squares), int8 69; few rows: the launch and one row's way through it, 3 us.
// Wavefronts per SIMD: fp32 rows of 257 .. 512 elements do not fit into 64 registers (with 8 of them 192 us, with 6 182).
#define CLQ_NT 512
template <int RB, int NP, typename IN, bool VEC>
__global__ void __launch_bounds__(CLQ_NT, RB * NP < 64 ? 8 : RB * NP > 64 ? 4 : sizeof(IN) == 4 ? 6 : 8)
cl_quantize_kernel(const IN *__restrict__ V, int64_t n, int D, int64_t ldv, uint32_t flags, int8_t *__restrict__ codes,
                   float *__restrict__ row_scale, int64_t blk0, int stream_out) { // blk0: the launch's first block
    constexpr int RW = RB / 8, DC = NP * 256, HALF = RB * 16 + 16; // rows of a wavefront; elements at a time; bytes of a half of a piece and padding that spreads the halves over the banks
    __shared__ __attribute__((aligned(16))) char lds[DC / 16 * HALF];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t blk = blk0 + blockIdx.x / (32 / RB);
    const int slot0 = blockIdx.x % (32 / RB) * RB, kb = (D + 31) / 32;
    constexpr bool RAW = sizeof(IN) == 1;
    // many rows of more than 1 KB pass by the caches (100,000 x 1,024 fp32: 82 us, 92 through them; but x 128: 75, 71, and rows that are read twice gain by them)
    constexpr int AUX = RB == 32 && NP > 1 ? 2 : 0;
    const auto row_of = [&](int i) __attribute__((always_inline)) {
        const int slot = slot0 + wave * RW + i;
        return flags & KS_QUANT_CLASSES ? (blk >> 1) * CL_GROUP + 2 * slot + (blk & 1) : blk * 32 + slot;
    };
    float4 x[RW][NP];
    const auto load = [&](int d0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < RW; ++i) {
            const int64_t row = row_of(i);
            const IN *v = V + (row < n ? row : n - 1) * ldv;
            const int len = row < n ? D : 0;
            if (VEC) { // whole fours as a buffer that ends with the last of them, which needs no branch
                const __amdgpu_buffer_rsrc_t whole = __builtin_amdgcn_make_buffer_rsrc((void *)v, 0, (len & ~3) * (int)sizeof(IN), 0x00020000);
#pragma unroll
                for (int e = 0; e < NP; ++e) x[i][e] = ClRow<IN>::template four<AUX>(whole, (d0 + e * 256 + lane * 4) * (int)sizeof(IN));
            }
            if (!VEC || (D & 3))
#pragma unroll
                for (int e = 0; e < NP; ++e) {
                    const int d = d0 + e * 256 + lane * 4;
                    if (!VEC || (d < len && d + 4 > len)) x[i][e] = cl_load_few(v + d, len - d);
                }
        }
    };
    int top[RW];  // bits of the largest |v|: ordered as the values, NaN above infinity
    double ss[RW];
#pragma unroll
    for (int i = 0; i < RW; ++i) { top[i] = 0; ss[i] = 0.0; }
    if (!RAW)
        for (int d0 = 0; d0 < D; d0 += DC) {
            load(d0);
#pragma unroll
            for (int i = 0; i < RW; ++i)
#pragma unroll
                for (int e = 0; e < NP; ++e) {
                    const float4 v = x[i][e];
                    top[i] = max(max(top[i], max(__float_as_int(v.x) & 0x7FFFFFFF, __float_as_int(v.y) & 0x7FFFFFFF)),
                                 max(__float_as_int(v.z) & 0x7FFFFFFF, __float_as_int(v.w) & 0x7FFFFFFF));
                    if (flags & KS_QUANT_NORMALIZE) {
                        ss[i] = __builtin_fma((double)v.x, (double)v.x, ss[i]);
                        ss[i] = __builtin_fma((double)v.y, (double)v.y, ss[i]);
                        ss[i] = __builtin_fma((double)v.z, (double)v.z, ss[i]);
                        ss[i] = __builtin_fma((double)v.w, (double)v.w, ss[i]);
                    }
                }
        }
    if (!RAW) cl_wave_reduce<ClMaxI>(top);
    if (flags & KS_QUANT_NORMALIZE) cl_wave_reduce<ClSumD>(ss);
    // the divisions and the root of row i in the lanes i modulo RW, all rows at once
    int my_top = top[0];
    double my_ss = ss[0];
#pragma unroll
    for (int i = 1; i < RW; ++i)
        if (lane % RW == i) { my_top = top[i]; my_ss = ss[i]; }
    const double my_a = my_top < 0x7F800000 ? (double)__int_as_float(my_top) : 0.0; // not finite: codes 0
    const float up = my_a < 0x1p-100 ? 0x1p100f : 1.f; // rows of which 127 / a might be no fp32 number
    const float my_inv = my_a > 0.0 ? (float)(127.0 / (my_a * up)) : 0.f;
    if (!RAW) {
        double scale = my_a / 127.0;
        if ((flags & KS_QUANT_NORMALIZE) && my_a > 0.0) scale /= sqrt(my_ss);
        const int64_t row = row_of(lane % RW);
        if (lane < RW && row < n) row_scale[row] = my_top < 0x7F800000 ? (float)scale : __int_as_float(0x7FC00000);
    }
    typedef std::conditional_t<sizeof(IN) == 4, double, float> F;
    F a[RW];
    float inv[RW];
#pragma unroll
    for (int i = 0; i < RW; ++i) {
        a[i] = (F)ClSumD::lane(my_a, i);
        inv[i] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_inv), i));
    }
    for (int d0 = 0; d0 < D; d0 += DC) {
        if (RAW || D > DC) load(d0);
        const int len = min(DC, kb * 32 - d0); // a multiple of 32
#pragma unroll
        for (int i = 0; i < RW; ++i)
#pragma unroll
            for (int e = 0; e < NP; ++e) {
                const int d = e * 256 + lane * 4;
                float4 v = x[i][e];
                F ai = a[i];
                if (!RAW && ai < (F)0x1p-100) {
                    v.x *= 0x1p100f; v.y *= 0x1p100f; v.z *= 0x1p100f; v.w *= 0x1p100f;
                    ai *= (F)0x1p100;
                }
                const uint32_t q = RAW ? ((int)v.x & 255) | ((int)v.y & 255) << 8 | ((int)v.z & 255) << 16 | (uint32_t)(int)v.w << 24
                                       : a[i] > 0 ? cl_codes(v, inv[i], ai) : 0;
                if (d < len) *(uint32_t *)(lds + (d >> 4) * HALF + (wave * RW + i) * 16 + (d & 15)) = q;
            }
        __syncthreads();
        int8_t *out = codes + (blk * kb + d0 / 32) * CL_PIECE + slot0 * 16;
        for (int e = threadIdx.x; e < len / 16 * RB; e += CLQ_NT) { // 16 bytes each: row e % RB of half-piece e / RB
            const cl_i32x4 q = *(const cl_i32x4 *)(lds + e / RB * HALF + e % RB * 16);
            cl_i32x4 *const to = (cl_i32x4 *)(out + (int64_t)(e / RB) * 512 + e % RB * 16);
            if (stream_out) __builtin_nontemporal_store(q, to);
            else *to = q;
        }
        if (d0 + DC < D) __syncthreads();
    }
}

extern "C" size_t class_codes_bytes(int64_t n, int D, uint32_t flags) {
    if (n < 1 || n >= (int64_t)1 << 31 || D < 1 || D > KS_MAX_INT8_D) return 0;
    const int64_t rows = flags & KS_QUANT_CLASSES ? ks_ceil_div(n, CL_GROUP) * CL_GROUP : ks_ceil_div(n, 32) * 32;
    return (size_t)rows * ((D + 31) / 32 * 32);
}

template <typename IN, bool VEC>
static void cl_quantize(const void *V, int64_t n, int D, int64_t ldv, uint32_t flags, int8_t *codes, float *row_scale, hipStream_t st) {
    const int64_t blocks = flags & KS_QUANT_CLASSES ? ks_ceil_div(n, CL_GROUP) * 2 : ks_ceil_div(n, 32);
    // codes of 4 MB (an XCD's cache) or more pass by the caches (390,625 x 512 int8: 65 us, 98 through them; then its product of fp32
    // rows and 64 samples: 234 us together, 239)
    const int stream_out = blocks * ((D + 31) / 32) >= 4096;
    const auto go = [&](auto kernel, int rb) { // a launch's threads are counted in 32 bits
        for (int64_t b0 = 0; b0 < blocks; b0 += 1 << 20)
            hipLaunchKernelGGL(kernel, dim3((unsigned)((blocks - b0 < 1 << 20 ? blocks - b0 : 1 << 20) * (32 / rb))), dim3(CLQ_NT), 0, st, (const IN *)V,
                               n, D, ldv, flags, codes, row_scale, b0, stream_out);
    };
    // whole blocks where there are enough of them and a wavefront holds four rows; else a row a wavefront
    if (blocks >= 512 && D <= 256) go(cl_quantize_kernel<32, 1, IN, VEC>, 32);
    else if (blocks >= 512 && D <= 512) go(cl_quantize_kernel<32, 2, IN, VEC>, 32);
    else if (blocks >= 512 && D <= 1024) go(cl_quantize_kernel<32, 4, IN, VEC>, 32);
    else if (D <= 256) go(cl_quantize_kernel<8, 1, IN, VEC>, 8);
    else if (D <= 512) go(cl_quantize_kernel<8, 2, IN, VEC>, 8);
    else if (D <= 1024) go(cl_quantize_kernel<8, 4, IN, VEC>, 8);
    else if (D <= 2048) go(cl_quantize_kernel<8, 8, IN, VEC>, 8);
    else go(cl_quantize_kernel<8, 16, IN, VEC>, 8);
}
template <typename IN>
static void cl_quantize(const void *V, int64_t n, int D, int64_t ldv, uint32_t flags, int8_t *codes, float *row_scale, hipStream_t st) {
    const bool vec = ((uintptr_t)V | (uintptr_t)(ldv * sizeof(IN))) % (4 * sizeof(IN)) == 0;
    if (vec) cl_quantize<IN, true>(V, n, D, ldv, flags, codes, row_scale, st);
    else cl_quantize<IN, false>(V, n, D, ldv, flags, codes, row_scale, st);
}

extern "C" int class_quantize_rows(const void *V, int dtype, int64_t n, int D, int64_t ldv, uint32_t flags, int8_t *codes,
                                   float *row_scale, void *stream) {
    if (!V || !codes || n < 1 || n >= (int64_t)1 << 31 || D < 1 || ldv < D) return KS_INVALID_ARG;
    if (dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32 && dtype != KS_DTYPE_INT8) return KS_INVALID_ARG;
    if (flags & ~(KS_QUANT_CLASSES | KS_QUANT_NORMALIZE) || (uintptr_t)codes % 16) return KS_INVALID_ARG;
    if ((uintptr_t)V % (dtype == KS_DTYPE_FP32 ? 4 : dtype == KS_DTYPE_BF16 ? 2 : 1)) return KS_INVALID_ARG;
    if (dtype == KS_DTYPE_INT8 ? row_scale || (flags & KS_QUANT_NORMALIZE) : !row_scale) return KS_INVALID_ARG;
    if (D > KS_MAX_INT8_D) return KS_UNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == KS_DTYPE_FP32) cl_quantize<float>(V, n, D, ldv, flags, codes, row_scale, st);
    else if (dtype == KS_DTYPE_BF16) cl_quantize<uint16_t>(V, n, D, ldv, flags, codes, row_scale, st);
    else cl_quantize<int8_t>(V, n, D, ldv, flags, codes, row_scale, st);
    KS_LAUNCH_CHECK();
    return KS_OK;
}

// ------------------------------------------------------------------------------------------------
// logits
// ------------------------------------------------------------------------------------------------
// workgroup barrier that waits for this wavefront's LDS accesses but, unlike __syncthreads(), not for loads in flight
__device__ __forceinline__ void cl_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F); // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ void cl_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void cl_store(uint16_t *p, float v) { *p = (uint16_t)ks_f2bf(v); }
// Pairs of classes pass by the caches (aux bit 1): nobody here reads a logit again, and the codes stay in them.
__device__ __forceinline__ void cl_store2(__amdgpu_buffer_rsrc_t to, uint32_t off, float v0, float v1, const float *) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(v0), __float_as_uint(v1)}, to, off, 0, 2);
}
__device__ __forceinline__ void cl_store2(__amdgpu_buffer_rsrc_t to, uint32_t off, float v0, float v1, const uint16_t *) {
    __builtin_amdgcn_raw_buffer_store_b32(ks_pack_bf2(v0, v1), to, off, 0, 2);
}
__device__ __forceinline__ void cl_store1(__amdgpu_buffer_rsrc_t to, uint32_t off, float v, const float *) {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), to, off, 0, 0);
}
__device__ __forceinline__ void cl_store1(__amdgpu_buffer_rsrc_t to, uint32_t off, float v, const uint16_t *) {
    __builtin_amdgcn_raw_buffer_store_b16((uint16_t)ks_f2bf(v), to, off, 0, 0);
}
// Logits of 32 samples from m0 on by the 64 classes from c0 on as a buffer that ends with the last class of the last sample: what lies
// behind its end (samples that do not exist, and classes: CL_NO_CLASS) the hardware leaves out, so that every row is one store on
// every way.  It ends with a whole pair, which is within the row since ldl is even here; so also where ldl < 64 the rows behind
// the last sample, from rows * ldl on, lie behind the end.  32 rows are less than 2^31 bytes (cl_logits sees to both).
template <typename OUT> __device__ __forceinline__ __amdgpu_buffer_rsrc_t cl_rows_of(OUT *out, int64_t ldl, int m0, int64_t c0, int64_t C, int B) {
    const int rows = B - m0 < 32 ? B - m0 : 32, classes = C - c0 < CL_GROUP ? (int)(C - c0) + 1 & ~1 : CL_GROUP;
    return __builtin_amdgcn_make_buffer_rsrc(out + (int64_t)m0 * ldl + c0, 0, rows > 0 ? (int)((rows - 1) * (uint32_t)(ldl * sizeof(OUT)) + classes * (uint32_t)sizeof(OUT)) : 0, 0x00020000);
}
#define CL_NO_CLASS 0x80000000u

// Scales, bias, type and store of 32 S samples from m0 on by the 64 classes from c0 on.  A lane of the result holds one column of each of
// the two blocks, which are two consecutive classes.  f: scales of the samples (LDS).  vec: pairs of classes are aligned.  ODD: the last
// of an odd number of classes, which has no pair, is stored here too (else by cl_last_class).
template <int S, bool ODD, typename OUT>
__device__ __forceinline__ void cl_finish(const cl_i32x16 (&acc)[S][2], const float *f, const float *__restrict__ ws,
                                          const float *__restrict__ bias, int64_t c0, int64_t C, int m0, int B, OUT *out, int64_t ldl, int vec) {
    const int lane = threadIdx.x & 63, half4 = 4 * (lane >> 5);
    const int64_t c = c0 + 2 * (lane & 31);
    float sw[2], b[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        sw[q] = ws[c + q < C ? c + q : C - 1];
        b[q] = bias ? bias[c + q < C ? c + q : C - 1] : 0.f;
    }
    // waited for here, once: a load left open on some way would be waited for, with all that followed it, where its register is next used
    asm volatile("" : "+v"(sw[0]), "+v"(sw[1]), "+v"(b[0]), "+v"(b[1]));
    const auto value = [&](int s, int r, int q, float4 g) __attribute__((always_inline)) {
        return fmaf((float)acc[s][q][r] * (r % 4 == 0 ? g.x : r % 4 == 1 ? g.y : r % 4 == 2 ? g.z : g.w), sw[q], b[q]);
    };
    if (vec) {
        const uint32_t row_bytes = (uint32_t)(ldl * sizeof(OUT)), off0 = c + 1 < C ? half4 * row_bytes + 2 * (lane & 31) * (uint32_t)sizeof(OUT) : CL_NO_CLASS;
        float4 f4[2][4]; // a sample block's scales are read while the one before is stored
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) f4[0][r4] = *(const float4 *)(f + half4 + r4 * 8);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (s + 1 < S)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) f4[s + 1 & 1][r4] = *(const float4 *)(f + half4 + (s + 1) * 32 + r4 * 8);
            __builtin_amdgcn_sched_barrier(0);
            const __amdgpu_buffer_rsrc_t to = cl_rows_of(out, ldl, m0 + s * 32, c0, C, B);
            uint32_t off = off0;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                cl_store2(to, off, value(s, r, 0, f4[s & 1][r / 4]), value(s, r, 1, f4[s & 1][r / 4]), (const OUT *)nullptr);
                off += r % 4 < 3 ? row_bytes : 5 * row_bytes; // the other half of the wavefront holds the four rows between
                asm volatile("" : "+v"(off));                 // one register, not sixteen that are kept from call to call
            }
        }
    }
    if (ODD && vec && (C & 1) && c0 + CL_GROUP > C) {
        const uint32_t row_bytes = (uint32_t)(ldl * sizeof(OUT)), off0 = c + 1 == C ? half4 * row_bytes + 2 * (lane & 31) * (uint32_t)sizeof(OUT) : CL_NO_CLASS;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const __amdgpu_buffer_rsrc_t to = cl_rows_of(out, ldl, m0 + s * 32, c0, C, B);
            uint32_t off = off0;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                cl_store1(to, off, value(s, r, 0, *(const float4 *)(f + half4 + s * 32 + r / 4 * 8)), (const OUT *)nullptr);
                off += r % 4 < 3 ? row_bytes : 5 * row_bytes;
                asm volatile("" : "+v"(off));
            }
        }
    }
    if (!vec) { // element by element
        int rows = B - m0 - half4;
        asm volatile("" : "+v"(rows), "+s"(ldl));
        OUT *p = out + (int64_t)(m0 + half4) * ldl + c;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float4 g = *(const float4 *)(f + half4 + s * 32 + r / 4 * 8);
                if (s * 32 + r / 4 * 8 + r % 4 < rows) {
                    if (c < C) cl_store(p, value(s, r, 0, g));
                    if (c + 1 < C) cl_store(p + 1, value(s, r, 1, g));
                }
                p += r % 4 < 3 ? ldl : 5 * ldl;
            }
    }
}

// The last of an odd number of classes, which has no pair to be stored with: the wavefronts of all workgroups take a sample each.
template <typename OUT>
__device__ __forceinline__ void cl_last_class(const int8_t *xq, const float *xs, const int8_t *wq, const float *ws, const float *bias,
                                              int64_t C, int kb, int B, float scale, OUT *out, int64_t ldl) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t wb = (C - 1) / CL_GROUP * 2; // C is odd: slot (C - 1) % 64 / 2 of the group's first block
    for (int m = blockIdx.x * waves + wave; m < B; m += gridDim.x * waves) {
        int sum = 0;
        for (int u = lane; u < 2 * kb; u += 64) { // half-pieces
            const cl_i32x4 xv = *(const cl_i32x4 *)(xq + ((int64_t)(m / 32) * kb + u / 2) * CL_PIECE + ((u & 1) * 32 + m % 32) * 16);
            const cl_i32x4 wv = *(const cl_i32x4 *)(wq + (wb * kb + u / 2) * CL_PIECE + ((u & 1) * 32 + (int)((C - 1) % CL_GROUP / 2)) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_sdot4(xv[e], wv[e], sum, false);
        }
        sum = ks_wave_sum_i(sum);
        if (lane == 0) cl_store(out + (int64_t)m * ldl + C - 1, fmaf((float)sum * (scale * xs[m]), ws[C - 1], bias ? bias[C - 1] : 0.f));
    }
}

// One wavefront: 64 classes (the two blocks of a group) by 32 S samples, codes straight from memory.  KS > 1: KS wavefronts of a
// workgroup take a part of the depth each and add their (whole) sums in LDS.  What bounds it are the codes, for few classes the way
// of one group (1 x 390,625 x 512: 31 us, 37 with codes that no cache holds, 5.4 TB/s; 64: 37 and 51; 1 x 10,000 x 128: 4.2 us).
template <int S, int KS, typename OUT>
__global__ void __launch_bounds__(CL_NT)
cl_direct_kernel(const int8_t *__restrict__ xq, const float *__restrict__ xs, const int8_t *__restrict__ wq,
                 const float *__restrict__ ws, const float *__restrict__ bias, int64_t C, int kb, int B, float scale,
                 OUT *__restrict__ out, int64_t ldl, int vec) {
    constexpr int NG = CL_NT / 64 / KS; // groups of a workgroup
    __shared__ __attribute__((aligned(16))) float s_f[32 * S];
    __shared__ int s_sum[KS > 1 ? (KS - 1) * S * 32 * 64 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % KS;
    const int sb = blockIdx.y * S, xblocks = (B + 31) / 32; // first block of samples
    if (threadIdx.x < 32 * S) s_f[threadIdx.x] = sb * 32 + (int)threadIdx.x < B ? scale * xs[sb * 32 + threadIdx.x] : 0.f;
    if (KS == 1) __syncthreads();
    const int64_t grp = (int64_t)blockIdx.x * NG + wave / KS;
    if (grp * CL_GROUP >= C) return; // KS > 1: a workgroup has one group, all its wavefronts or none
    const int8_t *wp = wq + grp * 2 * kb * CL_PIECE + lane * 16;
    const int8_t *xp[S];
#pragma unroll
    for (int s = 0; s < S; ++s) xp[s] = xq + (int64_t)min(sb + s, xblocks - 1) * kb * CL_PIECE + lane * 16;
    cl_i32x16 acc[S][2];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[s][q][r] = 0;
    const int end = kb * (part + 1) / KS;
    for (int k = kb * part / KS; k < end; ++k) {
        cl_i32x4 w[2], x[S];
#pragma unroll
        for (int q = 0; q < 2; ++q) w[q] = *(const cl_i32x4 *)(wp + ((int64_t)q * kb + k) * CL_PIECE);
#pragma unroll
        for (int s = 0; s < S; ++s) x[s] = *(const cl_i32x4 *)(xp[s] + (int64_t)k * CL_PIECE);
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int q = 0; q < 2; ++q) acc[s][q] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[s], w[q], acc[s][q], 0, 0, 0);
    }
    if (KS > 1) {
        static_assert(KS == 1 || NG == 1, "barriers");
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (part) s_sum[((part - 1) * S * 32 + s * 32 + q * 16 + r) * 64 + lane] = acc[s][q][r];
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int o = 0; o < KS - 1; ++o)
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[s][q][r] += s_sum[(o * S * 32 + s * 32 + q * 16 + r) * 64 + lane];
    }
    cl_finish<S, true>(acc, s_f, ws, bias, grp * CL_GROUP, C, sb * 32, B, out, ldl, vec);
}

// The work of a workgroup: stretches of an XCD's class groups for one sample tile each.  Workgroup i runs on XCD i % 8, and the groups are
// dealt to the XCDs in eight ranges.  Workgroups that are at the same groups at the same time share their codes in the L2, so
// the tiles of a round, at most eight, are taken by as many workgroups side by side, and the groups are divided among as many
// such sets as an XCD has room for (at least 28 of its 32 workgroups then have work).  Tiles that are not in step with each
// other read the weights from memory for each of them: 482 us instead of 320 at 1,400 x 390,625 x 512.
struct ClShare {
    int g_lo, g_n, n_sb, sb0; // the XCD's groups; tiles, those of the rounds before
    __device__ __forceinline__ ClShare(int groups, int n_sb_) {
        const int xcd = blockIdx.x & 7;
        g_lo = (int)((int64_t)groups * xcd / 8);
        g_n = (int)((int64_t)groups * (xcd + 1) / 8) - g_lo;
        n_sb = n_sb_;
        sb0 = 0;
    }
    // the next stretch: groups [first, last) of g_lo on, for tile sb (none: first >= last)
    __device__ __forceinline__ bool next(int &sb, int &first, int &last) {
        if (sb0 >= n_sb) return false;
        const int rounds = (n_sb - sb0 + 7) / 8, tiles = (n_sb - sb0 + rounds - 1) / rounds;
        const int sets = (int)(gridDim.x >> 3) / tiles, j = blockIdx.x >> 3, set = j / tiles;
        sb = sb0 + j % tiles;
        first = set < sets ? (int)((int64_t)g_n * set / sets) : 0;
        last = set < sets ? (int)((int64_t)g_n * (set + 1) / sets) : 0;
        sb0 += tiles;
        return true;
    }
};

#define CLX_KB 36 /* pieces of depth of 128 samples that lie in LDS beside their scales */
#define CLX_NT 512
// Batches of more than 64 samples, D <= 32 CLX_KB: a workgroup keeps the codes of 128 samples in LDS and its wavefronts, each on its own, go
// over groups of 64 classes: 8 matrix instructions on 2 pieces of weights, which come straight from memory a chunk of R
// k-steps ahead, also across the end of a group.  What bounds it are codes in and logits out (512 x 390,625 x 512 fp32: 169 us for 1.0 GB,
// 226 with codes that no cache holds; 256, bf16: 74 and 95), of deep rows and large batches the codes, read again for every tile of 128
// samples, and the products (codes that no cache holds: 256 x 390,625 x 768 bf16 115 us, x 1,152 152; 1,024 samples 373 and 467, which
// is 1.6 and 2.0 POP/s; fp32 525 and 615).  A wavefront that gets no group is idle: 77 x 50,021 x 333, 782 groups for 2,048 of them, 10.3 us.
template <int R, typename OUT>
__global__ void __launch_bounds__(CLX_NT, 2)
cl_resident_kernel(const int8_t *__restrict__ xq, const float *__restrict__ xs, const int8_t *__restrict__ wq,
                   const float *__restrict__ ws, const float *__restrict__ bias, int64_t C, int kb, int B, float scale,
                   OUT *__restrict__ out, int64_t ldl, int vec) {
    constexpr int NW = CLX_NT / 64;
    __shared__ __attribute__((aligned(16))) char s_x[CLX_KB * 4 * CL_PIECE];
    __shared__ __attribute__((aligned(16))) float s_f[128];
    __shared__ int s_next; // group that the next wavefront to ask gets: of two on a SIMD the older one runs ahead
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int xblocks = (B + 31) / 32, n_sb = (B + 127) / 128;
    const int chunks = (kb + R - 1) / R, last_step = (kb - (chunks - 1 > 1 ? chunks - 2 : 0) * R - R) * CL_PIECE; // kb >= R
    const int groups = (int)((C + CL_GROUP - 1) / CL_GROUP);
    ClShare share(groups, n_sb);
    const int g_lo = share.g_lo;
    int sb, first, last;
    while (share.next(sb, first, last)) {
        if (first >= last) continue;
        __syncthreads();
        // through registers: reads from LDS that a direct load may have written would wait for every load of weights in flight
        for (int p = wave; p < chunks * R * 4; p += NW) { // k-step t of sample block s at (4 t + s)
            const int blk = sb * 4 + (p & 3) < xblocks ? sb * 4 + (p & 3) : xblocks - 1, t = p >> 2;
            const int k = t < kb / R * R ? t : t - chunks * R + kb; // a last chunk that is short begins R before the end, with zeros
            cl_i32x4 v = {0, 0, 0, 0};
            if (k >= t / R * R) v = *(const cl_i32x4 *)(xq + ((int64_t)blk * kb + k) * CL_PIECE + lane * 16);
            *(cl_i32x4 *)(s_x + p * CL_PIECE + lane * 16) = v;
        }
        if (threadIdx.x < 128) s_f[threadIdx.x] = sb * 128 + (int)threadIdx.x < B ? scale * xs[sb * 128 + threadIdx.x] : 0.f;
        if (threadIdx.x == 0) s_next = first + NW;
        __syncthreads();

        int grp = first + wave;
        if (grp >= last) continue;
        cl_i32x4 w[R][2];
        cl_i32x16 acc[4][2];
        const int block_bytes = kb * CL_PIECE;
        const int8_t *p = wq + (int64_t)(g_lo + grp) * 2 * block_bytes; // chunk of the group's first block that is loaded next
#pragma unroll
        for (int kk = 0; kk < R; ++kk)
#pragma unroll
            for (int q = 0; q < 2; ++q) { // in the order in which they are used: the main loop's counted waits hold for these too
            w[kk][q] = *(const cl_i32x4 *)(p + q * block_bytes + kk * CL_PIECE + lane * 16);
            __builtin_amdgcn_sched_barrier(0);
        }
        cl_i32x4 x[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) x[s] = *(const cl_i32x4 *)(s_x + lane * 16 + s * CL_PIECE);
        while (grp < last) {
            int got = 0;
            if (lane == 0) got = atomicAdd(&s_next, 1);
            const int next = __builtin_amdgcn_readfirstlane(got), load_next = next < last ? next : grp;
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[s][q][r] = 0;
            const char *xp = s_x + lane * 16;
            for (int left = chunks; left > 0; --left, xp += R * 4 * CL_PIECE) {
                p = left == 1 ? wq + (int64_t)(g_lo + load_next) * 2 * block_bytes : left == 2 ? p + last_step : p + R * CL_PIECE;
                const int8_t *p1 = p + block_bytes;
                const char *xn = left == 1 ? s_x + lane * 16 : xp + R * 4 * CL_PIECE; // next chunk
#pragma unroll
                for (int kk = 0; kk < R; ++kk) {
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) acc[s][q] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[s], w[kk][q], acc[s][q], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                        x[s] = *(const cl_i32x4 *)((kk < R - 1 ? xp + (kk + 1) * 4 * CL_PIECE : xn) + s * CL_PIECE);
                        if (s == 3)
#pragma unroll
                            for (int q = 0; q < 2; ++q) w[kk][q] = *(const cl_i32x4 *)((q == 0 ? p : p1) + kk * CL_PIECE + lane * 16);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            cl_finish<4, false>(acc, s_f, ws, bias, (int64_t)(g_lo + grp) * CL_GROUP, C, sb * 128, B, out, ldl, vec);
            grp = next;
        }
    }
    if (vec && (C & 1)) cl_last_class(xq, xs, wq, ws, bias, C, kb, B, scale, out, ldl);
}

// Rows of up to 32 KB elements: a wavefront keeps the codes of 64 classes in registers, a workgroup those of up to 256 samples in LDS, and
// the samples go past 32 at a time: 2 KB matrix instructions a block, with the scales, conversions and stores of the block before in
// between.  (Per SIMD a matrix instruction of 32 clocks leaves room for four others; logits that are stored a row at a time do
// not hold up the loads behind them as a whole group's do.)  During a group's last block each piece of codes is replaced, when it
// has been used, by the next group's.  What bounds it are the stores, which the memory takes at 5.0 TB/s in rows of 128 or 256 bytes
// (1,024 x 390,625 bf16 at any D up to 128: 161 us), and beyond that power: D = 512 208 to 220 us (2 POP/s; codes of 0: 163), 251 to
// 265 with codes that no cache holds, fp32 318 and 386.
template <int KB, typename OUT>
__global__ void __launch_bounds__(CLX_NT, 2)
cl_steady_kernel(const int8_t *__restrict__ xq, const float *__restrict__ xs, const int8_t *__restrict__ wq,
                 const float *__restrict__ ws, const float *__restrict__ bias, int64_t C, int kb, int B, float scale,
                 OUT *__restrict__ out, int64_t ldl, int tile) { // tile: sample blocks at a time, even, at most 8
    constexpr int NW = CLX_NT / 64;
    __shared__ __attribute__((aligned(16))) char s_x[8 * KB * CL_PIECE];
    __shared__ __attribute__((aligned(16))) float s_f[256];
    __shared__ int s_next; // group that the next wavefront to ask gets: of two on a SIMD the older one runs ahead
    const uint32_t row_bytes = (uint32_t)(ldl * sizeof(OUT)); // 32 rows: less than 2^31 bytes
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half4 = 4 * (lane >> 5);
    const int xblocks = (B + 31) / 32, n_sb = (xblocks + tile - 1) / tile;
    const int groups = (int)((C + CL_GROUP - 1) / CL_GROUP);
    ClShare share(groups, n_sb);
    const int g_lo = share.g_lo;
    int sb, first, last;
    while (share.next(sb, first, last)) {
        if (first >= last) continue;
        __syncthreads();
        for (int p = wave; p < tile * KB; p += NW) { // k-step k of block i at (KB i + k), 0 beyond the depth
            const int blk = sb * tile + p / KB < xblocks ? sb * tile + p / KB : xblocks - 1, k = p % KB;
            cl_i32x4 v = {0, 0, 0, 0};
            if (k < kb) v = *(const cl_i32x4 *)(xq + ((int64_t)blk * kb + k) * CL_PIECE + lane * 16);
            *(cl_i32x4 *)(s_x + p * CL_PIECE + lane * 16) = v;
        }
        if ((int)threadIdx.x < tile * 32) {
            const int m = sb * tile * 32 + threadIdx.x;
            s_f[threadIdx.x] = m < B ? scale * xs[m] : 0.f;
        }
        if (threadIdx.x == 0) s_next = first + NW;
        __syncthreads();

        int grp = first + wave;
        if (grp >= last) continue;
        const int block_bytes = kb * CL_PIECE;
        const auto block_codes = [&](int g, int q) __attribute__((always_inline)) { // of a group's block: 0 beyond the depth
            return __builtin_amdgcn_make_buffer_rsrc((void *)(wq + ((int64_t)(g_lo + g) * 2 + q) * block_bytes), 0, block_bytes, 0x00020000);
        };
        uint32_t at[2] = {0, 0}; // of the four pieces from k - k % 4 on: one register a block, not one for every four
        const auto codes = [&](__amdgpu_buffer_rsrc_t p, int k, int q) __attribute__((always_inline)) {
            if (k % 4 == 0) {
                at[q] = lane * 16 + k * CL_PIECE;
                asm volatile("" : "+v"(at[q]));
            }
            return __builtin_bit_cast(cl_i32x4, __builtin_amdgcn_raw_buffer_load_b128(p, at[q] + k % 4 * CL_PIECE, 0, 0));
        };
        cl_i32x4 w[KB][2], x[4];
        cl_i32x16 acc[2][2];
        {
            const __amdgpu_buffer_rsrc_t p[2] = {block_codes(grp, 0), block_codes(grp, 1)};
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int q = 0; q < 2; ++q) { // in the order in which they are used: the main loop's counted waits hold for these too
                    w[k][q] = codes(p[q], k, q);
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = *(const cl_i32x4 *)(s_x + k * CL_PIECE + lane * 16);
        // the block that is finished while the next one is multiplied; none yet: a buffer of no bytes
        __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(out, 0, 0, 0x00020000);
        uint32_t off = 0;
        float sw[2] = {0.f, 0.f}, b[2] = {0.f, 0.f};
        float4 f4 = make_float4(0.f, 0.f, 0.f, 0.f), f4_next;
        const auto finish = [&](const cl_i32x16 (&a)[2], int r, const float *f) __attribute__((always_inline)) { // one row of each half
            if (r % 4 == 1 && r < 12) f4_next = *(const float4 *)(f + (r / 4 + 1) * 8);
            const float g = r % 4 == 0 ? f4.x : r % 4 == 1 ? f4.y : r % 4 == 2 ? f4.z : f4.w;
            const float v0 = fmaf((float)a[0][r] * g, sw[0], b[0]), v1 = fmaf((float)a[1][r] * g, sw[1], b[1]);
            cl_store2(to, off, v0, v1, (const OUT *)nullptr);
            off += r % 4 < 3 ? row_bytes : 5 * row_bytes;
            asm volatile("" : "+v"(off)); // one register, not sixteen that are kept for every block
            if (r % 4 == 3) f4 = f4_next;
        };
        while (grp < last) {
            int got = 0;
            if (lane == 0) got = atomicAdd(&s_next, 1);
            const int next = __builtin_amdgcn_readfirstlane(got);
            const __amdgpu_buffer_rsrc_t p_next[2] = {block_codes(next < last ? next : grp, 0), block_codes(next < last ? next : grp, 1)};
            const int64_t c0 = (int64_t)(g_lo + grp) * CL_GROUP, c = c0 + 2 * (lane & 31);
            float nsw[2], nb[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                nsw[q] = ws[c + q < C ? c + q : C - 1];
                nb[q] = bias ? bias[c + q < C ? c + q : C - 1] : 0.f;
            }
            const uint32_t off0 = c + 1 < C ? half4 * row_bytes + 2 * (lane & 31) * (uint32_t)sizeof(OUT) : CL_NO_CLASS;
            const auto block = [&](int blk, cl_i32x16 (&a)[2], const cl_i32x16 (&before)[2], auto reload) __attribute__((always_inline)) {
                const char *xp = s_x + blk * (KB * CL_PIECE) + lane * 16, *xn = reload ? s_x + lane * 16 : xp + KB * CL_PIECE;
                const float *f = s_f + (blk ? blk - 1 : tile - 1) * 32 + half4; // of the block before
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        if (k == 0) a[q] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[0], w[0][q], cl_i32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0}, 0, 0, 0);
                        else a[q] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[k & 3], w[k][q], a[q], 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    x[k & 3] = *(const cl_i32x4 *)(k + 4 < KB ? xp + (k + 4) * CL_PIECE : xn + (k + 4 - KB) * CL_PIECE);
                    if (reload)
#pragma unroll
                        for (int q = 0; q < 2; ++q) w[k][q] = codes(p_next[q], k, q);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (r * KB / 16 == k) finish(before, r, f);
                }
                to = cl_rows_of(out, ldl, (sb * tile + blk) * 32, c0, C, B);
                off = off0;
#pragma unroll
                for (int q = 0; q < 2; ++q) { sw[q] = nsw[q]; b[q] = nb[q]; }
                f4 = *(const float4 *)(s_f + blk * 32 + half4);
            };
            for (int i = 0; i + 2 < tile; i += 2) {
                block(i, acc[0], acc[1], std::false_type());
                block(i + 1, acc[1], acc[0], std::false_type());
            }
            block(tile - 2, acc[0], acc[1], std::false_type());
            block(tile - 1, acc[1], acc[0], std::true_type());
            grp = next;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) finish(acc[1], r, s_f + (tile - 1) * 32 + half4);
    }
    if (C & 1) cl_last_class(xq, xs, wq, ws, bias, C, kb, B, scale, out, ldl);
}

// Deeper rows: as in cl_resident_kernel, but the samples pass through LDS in chunks of eight k-steps, which eight wavefronts with 64
// classes each read at the same time: three buffers, a barrier a chunk.  2,048 x 131,072 x 4,096: 1,043 us = 2.11 POP/s, the matrix
// pipes 56 % busy at 1.9 GHz (codes of 0, which cost little power: 907; a bare loop of the instruction over random codes, 2.7 to 2.9 POP/s,
// would take 785).  What holds them up is the operands' way into the registers, for 64 instructions 32 KB from LDS and 20 KB through the
// caches: neither weights six k-steps ahead (1,054) nor 256 classes by 256 samples, which need 16 KB of the L2 instead of 20 (1,110),
// nor both sides in LDS and one wavefront a SIMD (1,118) were faster.
// While chunk t is multiplied, a fragment is read for the next k-step when it has been used (the last ones from chunk t + 1, which is
// there since the barrier), and chunk t + 2 is written to LDS from registers, each half of it half a chunk after it was requested.
// The chunks run on from one tile of 512 classes by 128 samples to the next.
template <typename OUT>
__global__ void __launch_bounds__(CLX_NT, 2)
cl_staged_kernel(const int8_t *__restrict__ xq, const float *__restrict__ xs, const int8_t *__restrict__ wq,
                 const float *__restrict__ ws, const float *__restrict__ bias, int64_t C, int kb, int B, float scale,
                 OUT *__restrict__ out, int64_t ldl, int vec) {
    constexpr int NW = CLX_NT / 64, R = 8, RW = 4 /* k-steps of weights ahead */, H = R / 4, CHUNK = R * 4 * CL_PIECE;
    __shared__ __attribute__((aligned(16))) char s_x[3 * CHUNK];
    __shared__ __attribute__((aligned(16))) float s_f[NW][128];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int xblocks = (B + 31) / 32, n_sb = (B + 127) / 128;
    const int chunks = (kb + R - 1) / R, last_step = (kb - (chunks - 1 > 1 ? chunks - 2 : 0) * R - R) * CL_PIECE; // kb >= R
    const int groups = (int)((C + CL_GROUP - 1) / CL_GROUP), n_ct = (groups + NW - 1) / NW;
    // workgroup i runs on XCD i % 8; an XCD has a range of the class tiles, and its workgroups take them for all samples before the
    // next ones: what 32 of them read at a time are a few class tiles and the samples
    const int xcd = blockIdx.x & 7, per_xcd = gridDim.x >> 3, j = blockIdx.x >> 3;
    const int c_lo = (int)((int64_t)n_ct * xcd / 8), c_n = (int)((int64_t)n_ct * (xcd + 1) / 8) - c_lo;
    int64_t left = (int64_t)c_n * n_sb - j; // tiles from this one on, of this and the XCD's other workgroups
    const int step_c = per_xcd / n_sb, step_s = per_xcd % n_sb; // from one of this workgroup's tiles to its next
    int ct = c_lo + j / n_sb, sb = j % n_sb;

    // samples: this wavefront moves 2 H of a chunk's 32 pieces, half of them at a time; piece 4 k + s is k-step k of sample block s
    int64_t r_left = left;
    int r_sb = sb, r_c = 0; // chunk that is requested next
    const auto request = [&](int i) __attribute__((always_inline)) {
        const int bi = r_sb * 4 + ((wave * 2 * H + i) & 3), blk = bi < xblocks ? bi : xblocks - 1;
        const int k = (r_c < chunks - 1 ? r_c * R : kb - R) + ((wave * 2 * H + i) >> 2);
        return *(const cl_i32x4 *)(xq + ((int64_t)blk * kb + k) * CL_PIECE + lane * 16);
    };
    const auto requested = [&]() __attribute__((always_inline)) { // behind the last tile: the same again, read by nobody
        if (++r_c == chunks) {
            r_c = 0;
            if (r_left > per_xcd) {
                r_left -= per_xcd;
                r_sb += step_s;
                if (r_sb >= n_sb) r_sb -= n_sb;
            }
        }
    };
    // chunk c: one that is short begins R before the end, with zeros for what the one before had
    const auto place = [&](cl_i32x4 v, int i, int c, char *to) __attribute__((always_inline)) {
        const int id = wave * 2 * H + i;
        if (c == chunks - 1 && kb - R + (id >> 2) < c * R) v = cl_i32x4{0, 0, 0, 0};
        *(cl_i32x4 *)(to + id * CL_PIECE + lane * 16) = v;
    };
    const int block_bytes = kb * CL_PIECE;
    const auto weights = [&](int tile) __attribute__((always_inline)) { // of this wavefront's classes in a tile; beyond the last group: that one
        const int g = tile * NW + wave;
        return wq + (int64_t)(g < groups ? g : groups - 1) * 2 * block_bytes;
    };
    char *b0 = s_x, *b1 = s_x + CHUNK, *b2 = s_x + 2 * CHUNK; // chunks t, t + 1, t + 2
    cl_i32x4 held[H];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < 2 * H; ++i) place(request(i), i, r_c, t ? b1 : b0);
        requested();
    }
#pragma unroll
    for (int i = 0; i < H; ++i) held[i] = request(i);
    int p_c = r_c; // its chunk
    cl_i32x4 w[RW][2], x[4];
    const int8_t *p = weights(ct);
#pragma unroll
    for (int kk = 0; kk < RW; ++kk)
#pragma unroll
        for (int q = 0; q < 2; ++q) { // in the order in which they are used: the main loop's counted waits hold for these too
            w[kk][q] = *(const cl_i32x4 *)(p + q * block_bytes + kk * CL_PIECE + lane * 16);
            __builtin_amdgcn_sched_barrier(0);
        }
    cl_barrier();
#pragma unroll
    for (int s = 0; s < 4; ++s) x[s] = *(const cl_i32x4 *)(b0 + s * CL_PIECE + lane * 16);
    for (; left > 0; left -= per_xcd) {
        int next_ct = ct + step_c, next_sb = sb + step_s;
        if (next_sb >= n_sb) { next_sb -= n_sb; ++next_ct; }
        if (left <= per_xcd) next_ct = ct;
        cl_i32x16 acc[4][2];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[s][q][r] = 0;
        for (int c = chunks; c > 0; --c) {
            const int8_t *pc = p + RW * CL_PIECE, *pc1 = pc + block_bytes;
            p = c == 1 ? weights(next_ct) : c == 2 ? p + last_step : p + R * CL_PIECE;
            const int8_t *p1 = p + block_bytes;
            cl_barrier(); // chunk t + 1 is whole, and nobody reads chunk t - 1 any more
#pragma unroll
            for (int kk = 0; kk < R; ++kk) {
                if (kk == R / 2) requested();
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int q = 0; q < 2; ++q) acc[s][q] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[s], w[kk % RW][q], acc[s][q], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    x[s] = *(const cl_i32x4 *)((kk < R - 1 ? b0 + (kk + 1) * 4 * CL_PIECE : b1) + s * CL_PIECE + lane * 16);
                    if (s == 3)
#pragma unroll
                        for (int q = 0; q < 2; ++q)
                            w[kk % RW][q] = *(const cl_i32x4 *)(kk + RW < R ? (q == 0 ? pc : pc1) + kk * CL_PIECE + lane * 16 : (q == 0 ? p : p1) + (kk + RW - R) * CL_PIECE + lane * 16);
                    if ((kk == 2 || kk == R / 2 + 2) && s < H) {
                        place(held[s], (kk == 2 ? 0 : H) + s, p_c, b2);
                        held[s] = request((kk == 2 ? H : 0) + s);
                    }
                }
            }
            p_c = r_c;
            char *const b = b0;
            b0 = b1;
            b1 = b2;
            b2 = b;
        }
        for (int i = lane; i < 128; i += 64) s_f[wave][i] = sb * 128 + i < B ? scale * xs[sb * 128 + i] : 0.f;
        const int g = ct * NW + wave;
        if (g < groups) cl_finish<4, false>(acc, s_f[wave], ws, bias, (int64_t)g * CL_GROUP, C, sb * 128, B, out, ldl, vec);
        ct = next_ct;
        sb = next_sb;
    }
    if (vec && (C & 1)) cl_last_class(xq, xs, wq, ws, bias, C, kb, B, scale, out, ldl);
}

template <typename OUT>
static void cl_logits(const int8_t *xq, const float *xs, const int8_t *wq, const float *ws, const float *bias, int64_t C, int D, int B,
                      float scale, OUT *out, int64_t ldl, hipStream_t st) {
    const int vec = ((uintptr_t)out | (uintptr_t)(ldl * sizeof(OUT))) % (2 * sizeof(OUT)) == 0 && ldl < (1 << 26) / (int64_t)sizeof(OUT), kb = (D + 31) / 32;
    const int64_t groups = ks_ceil_div(C, CL_GROUP);
    const auto direct = [&](auto kernel, int samples, int per_workgroup) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)ks_ceil_div(groups, per_workgroup), (unsigned)ks_ceil_div(B, samples)), dim3(CL_NT), 0, st, xq, xs,
                           wq, ws, bias, C, kb, B, scale, out, ldl, vec);
    };
    // vec: pairs of classes in one store; 64 MB from row to row and more, whose offsets are no 32 bits, go element by element (8 x 390,625 x 512 bf16:
    // 42 us, 41 with rows next to each other).  Pairs in rows that begin beside the 128-byte lines: 1,024 x 390,625 x 512 bf16 680 us, elements
    // 490, on the lines 260.
    // Few samples: the codes of the weights are what moves, and every wavefront reads its own.  Few wavefronts in all (a kernel of
    // 256 workgroups that keep the samples would leave most idle: 10,000 x 512, batch 256: 5.9 us, 8.0 in 128-sample tiles; 50,000
    // x 512, 128: 11.3 and 9.3; x 256: 6.8 and 8.4): the same for any batch.  Where they are deep, four wavefronts divide each group's depth (10,000 x
    // 4,096, one sample: 39 us, 13; 64: 44, 16; 50,000 x 2,048, one: 25, 20; but 64 samples, whose sums take 320 registers, only
    // where a compute unit would have a wavefront or so: 50,000 x 768: 12 us, 21).
    // Few groups of classes leave them idle too, whatever the batch: at most eight tiles of samples at a time take the groups, each with
    // 256 wavefronts (x 512, batch 82,000: C = 64 574 us, 17 by wavefronts of their own; batch 10,242: C = 1,000 81, 16; batch 1,666: C =
    // 6,000 16, 14; but C = 8,000 x 1,152, batch 1,282: 24, 25, and C = 16,000, batch 1,284: 20, 36).  Deep rows, whose groups share their
    // samples: x 2,048, batch 10,242: C = 1,000 78, 54; C = 2,000 76, 77; C = 4,000, batch 5,124: 57, 73.
    const int64_t waves = groups * ks_ceil_div(B, 64);
    const bool few_groups = groups <= (kb <= CLX_KB ? 96 : 32);
    if (B <= 32) return waves <= 1024 && kb >= 24 ? direct(cl_direct_kernel<1, 4, OUT>, 32, 1) : direct(cl_direct_kernel<1, 1, OUT>, 32, 4);
    if (B <= 64 || waves <= 1280 || few_groups || (waves <= 2048 && kb <= 8) || (kb < 4 && !vec))
        return waves <= 320 && kb >= 24 ? direct(cl_direct_kernel<2, 4, OUT>, 64, 1) : direct(cl_direct_kernel<2, 1, OUT>, 64, 4);
    // Registers hold 64 classes' codes while samples stream, or LDS holds samples while codes stream: the former is ahead for thin
    // rows (390,625 x 64, batch 1,024: 162 us, 176) and for deep ones and more than one tile of samples (x 512, batch 1,024 bf16: 219,
    // 235, and 260, 310 where no cache holds the codes, which it reads half as often; batch 256: 88, 80; fp32, more than two tiles: 512
    // samples 181, 169), if the wavefronts' last round of groups is well filled.  In between it is behind by 5 %, but where bf16 logits
    // leave codes as the larger part and the caches rarely hold them ahead by 16 % (390,625 x 256, batch 1,024: 175, 166, and 217, 259
    // from memory; 200,000 x 256, from a cache: 94, 88).
    const int xblocks = (B + 31) / 32, tiles = (xblocks + 7) / 8, tile = ((xblocks + tiles - 1) / tiles + 1) / 2 * 2;
    const int64_t sets = 32 / (tiles < 8 ? tiles : 8) * 64, rounds = ks_ceil_div(groups, sets);
    const bool thin_out = sizeof(OUT) == 2 && kb > 6 && groups * kb >= 32768; // 64 MB of codes
    if (vec && (kb < 4 || ((kb == 4 || (tiles >= (sizeof(OUT) == 2 ? 2 : 3) && kb <= 16 && (kb > 8 || thin_out))) && groups * 100 >= rounds * sets * 85)))
        hipLaunchKernelGGL((kb <= 4 ? cl_steady_kernel<4, OUT> : kb <= 12 ? cl_steady_kernel<12, OUT> : cl_steady_kernel<16, OUT>), dim3(256), dim3(CLX_NT),
                           0, st, xq, xs, wq, ws, bias, C, kb, B, scale, out, ldl, tile);
    else if (kb <= CLX_KB)
        hipLaunchKernelGGL((cl_resident_kernel<4, OUT>), dim3(256), dim3(CLX_NT), 0, st, xq, xs, wq, ws, bias, C, kb, B, scale, out, ldl, vec);
    else
        hipLaunchKernelGGL(cl_staged_kernel<OUT>, dim3(256), dim3(CLX_NT), 0, st, xq, xs, wq, ws, bias, C, kb, B, scale, out, ldl, vec);
}

extern "C" int class_logits_int8(const int8_t *x_codes, const float *x_scale, const int8_t *w_codes, const float *w_scale,
                                 const float *bias, int64_t C, int D, int B, float scale, void *logits, int dtype, int64_t ldl,
                                 void *stream) {
    if (!x_codes || !x_scale || !w_codes || !w_scale || !logits) return KS_INVALID_ARG;
    if (C < 1 || C >= (int64_t)1 << 31 || D < 1 || B < 1 || ldl < C) return KS_INVALID_ARG;
    if (dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) return KS_INVALID_ARG;
    if (((uintptr_t)x_codes | (uintptr_t)w_codes) % 16 || (uintptr_t)logits % (dtype == KS_DTYPE_FP32 ? 4 : 2)) return KS_INVALID_ARG;
    if (D > KS_MAX_INT8_D || B > KS_MAX_INT8_B) return KS_UNSUPPORTED;
    if (dtype == KS_DTYPE_FP32)
        cl_logits<float>(x_codes, x_scale, w_codes, w_scale, bias, C, D, B, scale, (float *)logits, ldl, (hipStream_t)stream);
    else
        cl_logits<uint16_t>(x_codes, x_scale, w_codes, w_scale, bias, C, D, B, scale, (uint16_t *)logits, ldl, (hipStream_t)stream);
    KS_LAUNCH_CHECK();
    return KS_OK;
}

// ------------------------------------------------------------------------------------------------
// penalties, biases, masks
// ------------------------------------------------------------------------------------------------
struct ClAdjust {
    const void *in;
    void *out;
    int64_t ldl, ldo, C, c0, Cg;
    const int64_t *seen_offsets, *bias_offsets;
    const int32_t *seen_ids, *bias_ids, *n_prompt, *mask_row;
    const float *bias_values, *repetition, *presence, *frequency;
    const uint32_t *allowed;
    int64_t seen_len, bias_len, ld_allowed;
    int B, seen_max, bias_max, n_masks, row0; // a launch takes the rows from row0 on
    int32_t *dev_status;
};

__device__ __forceinline__ float cl_load(const float *p) { return *p; }
__device__ __forceinline__ float cl_load(const uint16_t *p) { return ks_bf2f(*p); }
template <typename T> __device__ __forceinline__ T cl_minus_inf();
template <> __device__ __forceinline__ float cl_minus_inf<float>() { return __uint_as_float(0xFF800000u); }
template <> __device__ __forceinline__ uint16_t cl_minus_inf<uint16_t>() { return 0xFF80u; }

// mask of request b, -1: none
__device__ __forceinline__ int cl_mask_of(const ClAdjust &a, int b) {
    if (!a.allowed) return -1;
    const int m = a.mask_row ? a.mask_row[b] : b;
    if (m >= a.n_masks) {
        if (threadIdx.x == 0) ks_flag(a.dev_status, KS_DEV_BAD_INDEX);
        return -1;
    }
    return m;
}
// list b of a set of lists laid end to end: -> its length (0 where it is not a list), its first entry through *first
__device__ __forceinline__ int cl_list(const int64_t *offsets, int64_t len, int most, int b, int64_t *first, int32_t *dev_status) {
    if (!offsets) return 0;
    const int64_t lo = offsets[b], hi = offsets[b + 1];
    *first = lo;
    if (lo < 0 || hi < lo || hi > len || hi - lo > most) {
        if (threadIdx.x == 0) ks_flag(dev_status, KS_DEV_BAD_COUNT);
        return 0;
    }
    return (int)(hi - lo);
}
// column of an id on this node, -1 for an empty entry or another node's class
__device__ __forceinline__ int64_t cl_column(const ClAdjust &a, int32_t id, int bad) {
    if (id < 0) return -1;
    if (id >= a.Cg) {
        ks_flag(a.dev_status, bad);
        return -1;
    }
    const int64_t c = (int64_t)id - a.c0;
    return c < 0 || c >= a.C ? -1 : c;
}
// steps 1 and 2 on a logit of request b.  seen: bit 0: in the prompt, the rest: occurrences behind it; j: entry of the bias list or -1
__device__ __forceinline__ float cl_adjusted(const ClAdjust &a, int b, float z, uint32_t seen, int j, int64_t bias_first) {
    if (seen) {
        if (a.repetition) {
            const float r = a.repetition[b];
            z = z > 0.f ? z / r : z * r;
        }
        const uint32_t n = seen >> 1;
        if (n) z -= (a.frequency ? a.frequency[b] * (float)n : 0.f) + (a.presence ? a.presence[b] : 0.f);
    }
    return j >= 0 ? z + a.bias_values[bias_first + j] : z;
}
__device__ __forceinline__ bool cl_masked(const ClAdjust &a, int m, int64_t c) { // m: cl_mask_of's
    return m >= 0 && !(a.allowed[(int64_t)m * a.ld_allowed + (c >> 5)] >> (c & 31) & 1);
}

// Masks, and where COPY the logits that stay as they are; a workgroup takes a stretch of one row.  In place a vector of which some are
// masked is stored element by element, or with RMW read, changed and stored (then no other launch may change it meanwhile).
#define CLM_U(copy) ((copy) ? 2 : 4) /* vectors of a thread; copies of 256 x 390,625 fp32: 136 us, 157 with four; masks in place of bf16: 51, 47 */
template <typename T, bool COPY, bool VEC, bool RMW, int NT>
__device__ __forceinline__ void cl_mask_part(const ClAdjust &a, int b, int part) {
    constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;
    const int m = cl_mask_of(a, b);
    if (!COPY && m < 0) return;
    const uint32_t *bits = m < 0 ? nullptr : a.allowed + (int64_t)m * a.ld_allowed;
    const T *in = (const T *)a.in + b * a.ldl;
    T *out = (T *)a.out + b * a.ldo;
    const T none = cl_minus_inf<T>();
    const int64_t first = ((int64_t)part * CLM_U(COPY) * NT + threadIdx.x) * E;
#pragma unroll
    for (int u = 0; u < CLM_U(COPY); ++u) {
        const int64_t c = first + (int64_t)u * NT * E;
        if (c >= a.C) break;
        const uint32_t w = bits ? bits[c >> 5] >> (c & 31) : ~0u;
        if (E > 1 && c + E <= a.C) {
            union { uint4 q; T e[E]; } v;
            if (COPY) {
                v.q = *(const uint4 *)(in + c);
#pragma unroll
                for (int e = 0; e < E; ++e) v.e[e] = w >> e & 1 ? v.e[e] : none;
                __builtin_nontemporal_store(__builtin_bit_cast(cl_i32x4, v.q), (cl_i32x4 *)(out + c)); // 256 x 390,625 bf16: 58 us, 85 without
            } else if ((w & ((1u << E) - 1)) == 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) v.e[e] = none;
                *(uint4 *)(out + c) = v.q;
            } else if (RMW) {
                if ((~w & ((1u << E) - 1)) == 0) continue;
                v.q = *(const uint4 *)(out + c);
#pragma unroll
                for (int e = 0; e < E; ++e) v.e[e] = w >> e & 1 ? v.e[e] : none;
                *(uint4 *)(out + c) = v.q;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (!(w >> e & 1)) out[c + e] = none;
            }
        } else {
            for (int e = 0; e < E && c + e < a.C; ++e) {
                if (!(w >> e & 1)) out[c + e] = none;
                else if (COPY) out[c + e] = in[c + e];
            }
        }
    }
}

// CHECK: lists that may hold nothing are looked at here (an instance of its own: 256 x 390,625 bf16 1 us longer with the question in all)
template <typename T, bool CHECK, bool COPY, bool VEC, bool RMW>
__global__ void __launch_bounds__(CL_NT) cl_mask_kernel(ClAdjust a, int per_row) {
    const int b = a.row0 + blockIdx.x / per_row, part = blockIdx.x % per_row;
    if (CHECK && part == 0) {
        int64_t first;
        cl_list(a.seen_offsets, a.seen_len, a.seen_max, b, &first, a.dev_status);
        cl_list(a.bias_offsets, a.bias_len, a.bias_max, b, &first, a.dev_status);
    }
    cl_mask_part<T, COPY, VEC, RMW, CL_NT>(a, b, part);
}

// Lists of a request that a hash table of SLOTS classes in LDS holds (two thirds of the slots): each of them counts the class's occurrences
// and keeps the last of its biases.  The entry that takes a slot fetches the logit at once, so that it arrives while the others
// are counted, and adjusts it afterwards; nothing is read or written but the lists and the logits of their classes.
// MASKS 1, 2: the workgroups behind the requests' carry out the masks in place (1: element by element, 2: vectors): no logit
// belongs to both, so that one launch does for both.  3, 4: the same, but into another matrix: a request's workgroup copies its
// short row first.  What bounds it are the dependent accesses of one list (1 of 320 entries 4.4 us, 64 of 2,020 7.9, 256 of 6,300 13.3).
#define CLH_ENTRIES(slots) ((slots) / 3 * 2)
#define CLH_SMALL 1536
#define CLH_MID 6144
#define CLH_LARGE 12288 /* 144 KB of LDS, one workgroup on a compute unit */
template <typename T, int SLOTS, int NT, int MASKS>
__global__ void __launch_bounds__(NT) cl_hash_kernel(ClAdjust a, int requests, int per_row) {
    constexpr int K = CLH_ENTRIES(SLOTS) / NT; // entries of a thread
    static_assert(K * NT == CLH_ENTRIES(SLOTS), "");
    __shared__ uint32_t s_key[SLOTS], s_seen[SLOTS]; // column + 1, 0: free
    __shared__ int s_bias[SLOTS];
    if ((MASKS == 1 || MASKS == 2) && (int)blockIdx.x >= requests) {
        const int i = blockIdx.x - requests;
        cl_mask_part<T, false, MASKS == 2, false, NT>(a, a.row0 + i / per_row, i % per_row);
        return;
    }
    const int b = a.row0 + blockIdx.x;
    int64_t sf = 0, bf = 0;
    const int ns = cl_list(a.seen_offsets, a.seen_len, a.seen_max, b, &sf, a.dev_status);
    const int nb = cl_list(a.bias_offsets, a.bias_len, a.bias_max, b, &bf, a.dev_status);
    const int m = cl_mask_of(a, b);
    if (MASKS > 2)
        for (int part = 0; part < per_row; ++part) cl_mask_part<T, true, MASKS == 4, false, NT>(a, b, part);
    if (ns + nb == 0) return;
    const int prompt = a.n_prompt ? a.n_prompt[b] : 0;
    for (int e = threadIdx.x; e < SLOTS; e += NT) { s_key[e] = 0; s_seen[e] = 0; s_bias[e] = -1; }
    int32_t id[K];
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const int e = i * NT + threadIdx.x;
        id[i] = e < ns ? a.seen_ids[sf + e] : e < ns + nb ? a.bias_ids[bf + e - ns] : -1;
    }
    __syncthreads();
    const T *in = (const T *)a.in + b * a.ldl;
    T *out = (T *)a.out + b * a.ldo;
    int slot[K]; // where this thread's entry was the one to take it, else -1
    float z[K];
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const int e = i * NT + threadIdx.x;
        const int64_t c = cl_column(a, id[i], e < ns ? KS_DEV_BAD_LABEL : KS_DEV_BAD_INDEX);
        slot[i] = -1;
        if (c < 0) continue;
        const uint32_t key = (uint32_t)c + 1;
        uint32_t at = __umulhi(key * 0x9E3779B1u, SLOTS);
        for (;;) { // there are more slots than entries
            const uint32_t was = atomicCAS(&s_key[at], 0u, key);
            if (was == 0) {
                if (!cl_masked(a, m, c)) {
                    slot[i] = (int)at;
                    z[i] = cl_load(in + c);
                }
                break;
            }
            if (was == key) break;
            at = at + 1 == SLOTS ? 0 : at + 1;
        }
        if (e >= ns) atomicMax(&s_bias[at], e - ns);
        else if (e < prompt) atomicOr(&s_seen[at], 1u);
        else atomicAdd(&s_seen[at], 2u);
    }
    if (MASKS > 2) __builtin_amdgcn_s_waitcnt(0x0F70); // vmcnt(0): the row is copied before a logit of it changes
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (slot[i] >= 0) cl_store(out + s_key[slot[i]] - 1, cl_adjusted(a, b, z[i], s_seen[slot[i]], s_bias[slot[i]], bf));
}

// Longer lists: `parts` workgroups to a request, each with the classes whose keys, spread by an odd factor over the 32-bit numbers, lie in its
// part of them; all of them go over the whole list.  A part whose table is so full that an entry finds no slot within CLL_TRIES
// is done in several rounds, over half of the part, a quarter, and so on (different classes have different keys: that ends), and
// twice as much of it after each that held.  Its time goes into the lists, read again for every part: 256 x 131,072 bf16 with 20,000
// entries a request 138 us, one such request 22.
#define CLL_SLOTS 6144
#define CLL_TRIES 256
template <typename T>
__global__ void __launch_bounds__(1024) cl_long_kernel(ClAdjust a, int per_row, int fill) {
    __shared__ uint32_t s_key[CLL_SLOTS], s_seen[CLL_SLOTS]; // column + 1, 0: free
    __shared__ int s_bias[CLL_SLOTS];
    __shared__ int s_full;
    const int b = a.row0 + blockIdx.x / per_row, part = blockIdx.x % per_row;
    int64_t sf = 0, bf = 0;
    const int ns = cl_list(a.seen_offsets, a.seen_len, a.seen_max, b, &sf, a.dev_status);
    const int nb = cl_list(a.bias_offsets, a.bias_len, a.bias_max, b, &bf, a.dev_status);
    const int m = cl_mask_of(a, b);
    const int need = (ns + nb + 4095) / 4096, parts = need > fill ? need : fill; // at most per_row, which is for the longest list
    if (ns + nb == 0 || part >= parts) return;
    const int prompt = a.n_prompt ? a.n_prompt[b] : 0;
    const T *in = (const T *)a.in + b * a.ldl;
    T *out = (T *)a.out + b * a.ldo;
    const uint64_t end = ((uint64_t)(part + 1) << 32) / parts;
    uint64_t lo = ((uint64_t)part << 32) / parts, width = end - lo;
    while (lo < end) { // spread keys [lo, lo + width)
        if (lo + width > end) width = end - lo;
        __syncthreads();
        for (int e = threadIdx.x; e < CLL_SLOTS; e += 1024) { s_key[e] = 0; s_seen[e] = 0; s_bias[e] = -1; }
        if (threadIdx.x == 0) s_full = 0;
        __syncthreads();
        for (int e0 = threadIdx.x; e0 < ns + nb; e0 += 4 * 1024) {
            int32_t id[4]; // four loads at a time
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = e0 + i * 1024;
                id[i] = e < ns ? a.seen_ids[sf + e] : e < ns + nb ? a.bias_ids[bf + e - ns] : -1;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = e0 + i * 1024;
                const int64_t c = cl_column(a, id[i], e < ns ? KS_DEV_BAD_LABEL : KS_DEV_BAD_INDEX);
                const uint32_t key = (uint32_t)c + 1, spread = key * 0x9E3779B1u;
                if (c < 0 || (uint64_t)spread - lo >= width) continue;
                uint32_t at = __umulhi(spread * 0x85EBCA6Bu, CLL_SLOTS);
                int tries = 0;
                for (; tries < CLL_TRIES; ++tries) {
                    uint32_t was = *(volatile uint32_t *)&s_key[at]; // a read is shared by the lanes of one class, an atomic is not
                    if (was == 0) was = atomicCAS(&s_key[at], 0u, key);
                    if (was == 0 || was == key) break;
                    at = at + 1 == CLL_SLOTS ? 0 : at + 1;
                }
                if (tries == CLL_TRIES) s_full = 1;
                else if (e >= ns) atomicMax(&s_bias[at], e - ns);
                else if (e < prompt) atomicOr(&s_seen[at], 1u);
                else atomicAdd(&s_seen[at], 2u);
            }
        }
        __syncthreads();
        if (s_full) {
            width = (width + 1) / 2;
            continue;
        }
        constexpr int N = CLL_SLOTS / 1024;
        uint32_t key[N];
        float z[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { // all of them are fetched before the first one is stored
            key[i] = s_key[i * 1024 + threadIdx.x];
            if (key[i] && cl_masked(a, m, (int64_t)key[i] - 1)) key[i] = 0;
            if (key[i]) z[i] = cl_load(in + key[i] - 1);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (key[i]) cl_store(out + key[i] - 1, cl_adjusted(a, b, z[i], s_seen[i * 1024 + threadIdx.x], s_bias[i * 1024 + threadIdx.x], bf));
        lo += width;
        width *= 2;
    }
}

#define CL_MAX_GRID (1 << 21) /* workgroups of a launch: threads are counted in 32 bits */
// launch(a, rows) for stretches of rows from a.row0 on that fit into a launch, per_row workgroups each
template <class F> static void cl_rows(ClAdjust a, int per_row, F launch) {
    const int rows = per_row < CL_MAX_GRID ? CL_MAX_GRID / per_row : 1;
    for (int64_t row0 = 0; row0 < a.B; row0 += rows) { // the row behind the last stretch may be no int
        a.row0 = (int)row0;
        launch(a, (int)(rows < a.B - row0 ? rows : a.B - row0));
    }
}

template <typename T> static void cl_adjust(const ClAdjust &args, hipStream_t st) {
    const bool copy = args.in != args.out;
    const bool vec = ((uintptr_t)args.in | (uintptr_t)args.out | (uintptr_t)(args.ldl * sizeof(T)) | (uintptr_t)(args.ldo * sizeof(T))) % 16 == 0;
    const int entries = (args.seen_offsets ? args.seen_max : 0) + (args.bias_offsets ? args.bias_max : 0), E = vec ? 16 / (int)sizeof(T) : 1;
    // masks in place: together with short lists (16 x 390,625 bf16, 1,088 entries: 7.9 us, 14.2 in two launches); but from 32 MB of
    // bf16 on by themselves, reading what they change in part: a bf16 vector has eight elements, stored one by one, and reading
    // it costs less than they do (256 x 390,625, half of the classes: 49 us, 82; fp32, four elements: 112, 90)
    const bool rmw = !copy && vec && sizeof(T) == 2 && (int64_t)args.B * args.C >= 1 << 24;
    // short rows into another matrix: a workgroup each copies and changes its own, if three rounds of 1,024 threads do for the copy (1 x
    // 10,000 fp32: 5.4 us, 7.9 in two launches; x 24,000: 7.4, 8.7; x 32,000: 8.2, 8.3) and there is one for every compute unit at most
    // (2,048 x 1,000 with long lists: 38, 28)
    const bool whole = copy && entries > 0 && entries <= CLH_ENTRIES(CLH_MID) && args.B <= 256 && ks_ceil_div(args.C, (int64_t)CLM_U(true) * 1024 * E) <= 3;
    const bool fused = !copy && args.allowed && !rmw && entries > 0 && entries <= CLH_ENTRIES(CLH_MID);
    // lists that may hold nothing change no logit, but one that holds something is reported
    const bool check = entries == 0 && args.dev_status && (args.seen_offsets || args.bias_offsets);
    if ((copy || args.allowed) && !fused && !whole) {
        const int per_row = (int)ks_ceil_div(args.C, (int64_t)CLM_U(copy) * CL_NT * E);
        cl_rows(args, per_row, [&](const ClAdjust &a, int rows) {
            const auto masks = [&](auto checking, auto plain) {
                hipLaunchKernelGGL((check ? checking : plain), dim3((unsigned)per_row * (unsigned)rows), dim3(CL_NT), 0, st, a, per_row);
            };
            if (copy && vec) masks(cl_mask_kernel<T, true, true, true, false>, cl_mask_kernel<T, false, true, true, false>);
            else if (copy) masks(cl_mask_kernel<T, true, true, false, false>, cl_mask_kernel<T, false, true, false, false>);
            else if (sizeof(T) == 2 && rmw) masks(cl_mask_kernel<T, true, false, true, sizeof(T) == 2>, cl_mask_kernel<T, false, false, true, sizeof(T) == 2>);
            else if (vec) masks(cl_mask_kernel<T, true, false, true, false>, cl_mask_kernel<T, false, false, true, false>);
            else masks(cl_mask_kernel<T, true, false, false, false>, cl_mask_kernel<T, false, false, false, false>);
        });
    }
    if (entries == 0 && (!check || copy || args.allowed)) return;
    const auto hash = [&](auto kernel, int nt) {
        const int per_row = fused || whole ? (int)ks_ceil_div(args.C, (int64_t)CLM_U(whole) * nt * E) : 0;
        cl_rows(args, fused ? 1 + per_row : 1, [&](const ClAdjust &a, int rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)rows * (unsigned)(fused ? 1 + per_row : 1)), dim3(nt), 0, st, a, rows, per_row);
        });
    };
    if (entries <= CLH_ENTRIES(CLH_SMALL) && whole)
        hash(vec ? cl_hash_kernel<T, CLH_SMALL, 1024, 4> : cl_hash_kernel<T, CLH_SMALL, 1024, 3>, 1024);
    else if (entries <= CLH_ENTRIES(CLH_SMALL))
        hash(!fused ? cl_hash_kernel<T, CLH_SMALL, 256, 0> : vec ? cl_hash_kernel<T, CLH_SMALL, 256, 2> : cl_hash_kernel<T, CLH_SMALL, 256, 1>, 256);
    else if (entries <= CLH_ENTRIES(CLH_MID))
        hash(whole ? (vec ? cl_hash_kernel<T, CLH_MID, 1024, 4> : cl_hash_kernel<T, CLH_MID, 1024, 3>)
             : !fused ? cl_hash_kernel<T, CLH_MID, 1024, 0> : vec ? cl_hash_kernel<T, CLH_MID, 1024, 2> : cl_hash_kernel<T, CLH_MID, 1024, 1>, 1024);
    else if (entries <= CLH_ENTRIES(CLH_LARGE) && args.B >= 16) { // few requests leave most of the chip idle with one workgroup each
        // (131,072 classes, bf16, lists of 8,000: 16 requests 24 us, 26 in parts; 128: 33, 37; 256 of 6,000: 13, 29; one of 9,000: 30, 15)
        hash(cl_hash_kernel<T, CLH_LARGE, 1024, 0>, 1024); // the masks are set already
    } else {
        // parts of 4,096 entries on average (of 2,048: 256 lists of 20,000 202 us, 137), more where there are few requests: two
        // workgroups fit on a compute unit, and one list of 20,000 takes 26 us in 16 parts, 22 in 64
        const int fill = (int)ks_ceil_div(512, args.B) < 64 ? (int)ks_ceil_div(512, args.B) : 64, need = (int)ks_ceil_div(entries, 4096), parts = need > fill ? need : fill;
        cl_rows(args, parts, [&](const ClAdjust &a, int rows) {
            hipLaunchKernelGGL(cl_long_kernel<T>, dim3((unsigned)parts * (unsigned)rows), dim3(1024), 0, st, a, parts, fill);
        });
    }
}

extern "C" int class_logits_adjust(const void *logits, int64_t ldl, void *out, int64_t ldo, int dtype, int64_t C, int64_t c0,
                                   int64_t Cg, int B, const int64_t *seen_offsets, const int32_t *seen_ids, int64_t seen_len,
                                   int seen_max, const int32_t *n_prompt, const float *repetition, const float *presence,
                                   const float *frequency, const int64_t *bias_offsets, const int32_t *bias_ids,
                                   const float *bias_values, int64_t bias_len, int bias_max, const uint32_t *allowed,
                                   int64_t ld_allowed, int n_masks, const int32_t *mask_row, int32_t *dev_status, void *stream) {
    if (!logits || !out || B < 1 || C < 1 || c0 < 0 || Cg >= (int64_t)1 << 31 || C > Cg || c0 > Cg - C || ldl < C || ldo < C) return KS_INVALID_ARG;
    if (dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) return KS_INVALID_ARG;
    if (((uintptr_t)logits | (uintptr_t)out) % (dtype == KS_DTYPE_FP32 ? 4 : 2) || (logits == out && ldl != ldo && B > 1)) return KS_INVALID_ARG;
    if (seen_len < 0 || bias_len < 0 || seen_max < 0 || bias_max < 0 || (int64_t)seen_max + bias_max >= (int64_t)1 << 30) return KS_INVALID_ARG;
    if (seen_offsets && seen_len && !seen_ids) return KS_INVALID_ARG;
    if (bias_offsets && bias_len && (!bias_ids || !bias_values)) return KS_INVALID_ARG;
    if (allowed && (ld_allowed < (C + 31) / 32 || n_masks < 1 || (!mask_row && n_masks < B))) return KS_INVALID_ARG;
    const auto lists = [&](const int64_t *offsets, int most) { return offsets && (most || dev_status); };
    if (logits == out && !allowed && !lists(seen_offsets, seen_max) && !lists(bias_offsets, bias_max)) return KS_OK; // nothing changes or is reported
    const ClAdjust a = {logits, out, ldl, ldo, C, c0, Cg, seen_offsets, bias_offsets, seen_ids, bias_ids, n_prompt, mask_row, bias_values,
                        repetition, presence, frequency, allowed, seen_len, bias_len, ld_allowed, B, seen_max, bias_max, n_masks, 0, dev_status};
    if (dtype == KS_DTYPE_FP32) cl_adjust<float>(a, (hipStream_t)stream);
    else cl_adjust<uint16_t>(a, (hipStream_t)stream);
    KS_LAUNCH_CHECK();
    return KS_OK;
}
