// Answering with the trained layer in 4 bits (paper Section 3.1: W holds one row per class, Section 3.2: the fc forward): rows as
// microscaled 4-bit floating point in the order in which matrix instructions take them, and back; logits of a batch against every class.
#include "../../include/class_mxfp4.h"
#include "ks_common.h"
#include <type_traits>

typedef int32_t m4_i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t m4_i32x8 __attribute__((ext_vector_type(8)));

#define M4_NT 256
#define M4_PIECE 1024 /* bytes of a piece: 32 rows x 64 codes, the operand of one 32x32x64 matrix instruction, 16 bytes a lane */
#define M4_EXPS 256   /* bytes of the exponents of four pieces, a word a lane */
#define M4_GROUP 64   /* classes whose two groups of codes lie next to each other, every other class in each */

static __host__ __device__ __forceinline__ int m4_row_bytes(int kb) { return kb * M4_PIECE + (kb + 3) / 4 * M4_EXPS; } // of 32 rows of kb pieces

// ------------------------------------------------------------------------------------------------
// rows -> codes -> rows
// ------------------------------------------------------------------------------------------------
#define M4Q_DC 512                 /* elements of a row that a workgroup takes: eight pieces */
#define M4Q_HALF (32 * 16 + 16)    /* bytes of a half of a piece in LDS, and padding that spreads the halves over the banks */

// eight elements from p on, 0 from the `left`-th on
template <bool VEC> __device__ __forceinline__ void m4_load8(const float *p, int left, float (&v)[8]) {
    if (VEC && left >= 8) {
        const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
}
template <bool VEC> __device__ __forceinline__ void m4_load8(const uint16_t *p, int left, float (&v)[8]) {
    if (VEC && left >= 8) {
        const uint4 a = *(const uint4 *)p;
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? ks_bf2f(p[i]) : 0.f;
}

// A workgroup takes 32 rows (a group) and M4Q_DC elements of each; a wavefront eight of the rows, a lane eight elements, four lanes a block.
// The largest |v| as bits gives the exponent without a logarithm, v_cvt_scalef32_pk_fp4_f32 divides by the power of two and rounds (halves to
// the even code; checked at every middle and its neighbours for every exponent), and LDS turns rows into pieces, so that whole lines are stored.
// What bounds it: the rows in, the codes out; 390,625 x 512 fp32 there and back as bf16 279 us (1.41 GB at 5.05 TB/s); few rows: two launches.
template <typename IN, bool VEC>
__global__ void __launch_bounds__(M4_NT)
m4_quantize_kernel(const IN *__restrict__ V, int64_t n, int D, int64_t ldv, uint32_t flags, uint8_t *__restrict__ codes, int64_t group0) {
    __shared__ __attribute__((aligned(16))) uint8_t s_c[16 * M4Q_HALF];
    __shared__ __attribute__((aligned(16))) uint8_t s_e[2 * M4_EXPS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t group = group0 + blockIdx.x;
    const int kb = (D + 63) / 64, p0 = blockIdx.y * 8, d = blockIdx.y * M4Q_DC + lane * 8;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = wave * 8 + i;
        const int64_t row = flags & KS_MXFP4_CLASSES ? (group >> 1) * M4_GROUP + 2 * r + (group & 1) : group * 32 + r;
        const bool there = row < n && d < D;
        m4_load8<VEC>(V + (there ? row * ldv + d : 0), there ? D - d : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        int top = 0; // bits of the largest |v|: ordered as the values, NaN above infinity
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_int(v[i][j]) & 0x7FFFFFFF);
        top = max(top, KS_DPP(0, top, 0xB1, 0xf)); // quad_perm [1, 0, 3, 2]
        top = max(top, KS_DPP(0, top, 0x4E, 0xf)); // quad_perm [2, 3, 0, 1]
        const int biased = top >> 23, e = biased == 255 ? 255 : max(biased - 2, 0);
        const float unit = __int_as_float(e == 0 ? 0x00400000 : e << 23); // 2^(e - 127)
        uint32_t q = 0;
        if (biased != 255) {
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][0], v[i][1], unit, 0);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][2], v[i][3], unit, 1);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][4], v[i][5], unit, 2);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][6], v[i][7], unit, 3);
        }
        const int r = wave * 8 + i, half = lane >> 2; // half-piece of the chunk
        *(uint32_t *)(s_c + half * M4Q_HALF + r * 16 + (lane & 3) * 4) = q;
        if ((lane & 3) == 0) s_e[(half >> 3) * M4_EXPS + ((half & 1) * 32 + r) * 4 + (half >> 1 & 3)] = (uint8_t)e;
    }
    __syncthreads();
    uint8_t *const to = codes + group * m4_row_bytes(kb);
    const int pieces = min(8, kb - p0);
    for (int u = threadIdx.x; u < pieces * 64; u += M4_NT)
        *(m4_i32x4 *)(to + (int64_t)p0 * M4_PIECE + u * 16) = *(const m4_i32x4 *)(s_c + (u >> 5) * M4Q_HALF + (u & 31) * 16);
    const int words = (pieces + 3) / 4 * 64;
    for (int u = threadIdx.x; u < words; u += M4_NT)
        *(uint32_t *)(to + (int64_t)kb * M4_PIECE + p0 / 4 * M4_EXPS + u * 4) = *(const uint32_t *)(s_e + u * 4);
}

__device__ __forceinline__ void m4_store8(float *p, int left, const float (&v)[8], bool vec) {
    if (vec && left >= 8) {
        *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
        *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = v[i];
}
__device__ __forceinline__ void m4_store8(uint16_t *p, int left, const float (&v)[8], bool vec) { // the values have at most 2 bits of mantissa: the high halves
    if (vec && left >= 8) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
        *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (uint16_t)(__float_as_uint(v[i]) >> 16);
}

// The way back: whole pieces into LDS, eight elements of a row a lane out of it.
template <typename OUT>
__global__ void __launch_bounds__(M4_NT)
m4_dequantize_kernel(const uint8_t *__restrict__ codes, int64_t n, int D, uint32_t flags, OUT *__restrict__ V, int64_t ldv, int64_t group0, int vec) {
    __shared__ __attribute__((aligned(16))) uint8_t s_c[16 * M4Q_HALF];
    __shared__ __attribute__((aligned(16))) uint8_t s_e[2 * M4_EXPS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t group = group0 + blockIdx.x;
    const int kb = (D + 63) / 64, p0 = blockIdx.y * 8, d = blockIdx.y * M4Q_DC + lane * 8;
    const uint8_t *const from = codes + group * m4_row_bytes(kb);
    const int pieces = min(8, kb - p0), words = (pieces + 3) / 4 * 64;
    for (int u = threadIdx.x; u < pieces * 64; u += M4_NT)
        *(m4_i32x4 *)(s_c + (u >> 5) * M4Q_HALF + (u & 31) * 16) = *(const m4_i32x4 *)(from + (int64_t)p0 * M4_PIECE + u * 16);
    for (int u = threadIdx.x; u < words; u += M4_NT)
        *(uint32_t *)(s_e + u * 4) = *(const uint32_t *)(from + (int64_t)kb * M4_PIECE + p0 / 4 * M4_EXPS + u * 4);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = wave * 8 + i, half = lane >> 2;
        const int64_t row = flags & KS_MXFP4_CLASSES ? (group >> 1) * M4_GROUP + 2 * r + (group & 1) : group * 32 + r;
        if (row >= n || d >= D) continue;
        const uint32_t q = *(const uint32_t *)(s_c + half * M4Q_HALF + r * 16 + (lane & 3) * 4);
        const int e = s_e[(half >> 3) * M4_EXPS + ((half & 1) * 32 + r) * 4 + (half >> 1 & 3)];
        const float unit = __int_as_float(e == 0 ? 0x00400000 : e << 23);
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 w[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 3)};
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e == 255 ? __int_as_float(0x7FC00000) : w[j / 2][j % 2];
        m4_store8(V + row * ldv + d, D - d, v, vec != 0);
    }
}

extern "C" size_t class_mxfp4_bytes(int64_t n, int D, uint32_t flags) {
    if (n < 1 || n >= (int64_t)1 << 31 || D < 1 || D > KS_MAX_MXFP4_D || flags & ~KS_MXFP4_CLASSES) return 0;
    const int64_t groups = flags & KS_MXFP4_CLASSES ? ks_ceil_div(n, M4_GROUP) * 2 : ks_ceil_div(n, 32);
    return (size_t)groups * m4_row_bytes((D + 63) / 64);
}

static int m4_rows_check(const void *V, int dtype, int64_t n, int D, int64_t ldv, uint32_t flags, const uint8_t *codes) {
    if (!V || !codes || n < 1 || n >= (int64_t)1 << 31 || D < 1 || ldv < D) return KS_INVALID_ARG;
    if (dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) return KS_INVALID_ARG;
    if (flags & ~KS_MXFP4_CLASSES || (uintptr_t)codes % 16 || (uintptr_t)V % (dtype == KS_DTYPE_FP32 ? 4 : 2)) return KS_INVALID_ARG;
    return D > KS_MAX_MXFP4_D ? KS_UNSUPPORTED : KS_OK;
}
// go(first group, grid) for all groups of rows: a launch's threads are counted in 32 bits
template <typename F> static void m4_over_groups(int64_t n, int D, uint32_t flags, F go) {
    const int64_t groups = flags & KS_MXFP4_CLASSES ? ks_ceil_div(n, M4_GROUP) * 2 : ks_ceil_div(n, 32), chunks = ks_ceil_div(D, M4Q_DC);
    const int64_t most = ((int64_t)1 << 23) / chunks;
    for (int64_t g = 0; g < groups; g += most) go(g, dim3((unsigned)(groups - g < most ? groups - g : most), (unsigned)chunks));
}

extern "C" int class_quantize_mxfp4(const void *V, int dtype, int64_t n, int D, int64_t ldv, uint32_t flags, uint8_t *codes, void *stream) {
    const int rc = m4_rows_check(V, dtype, n, D, ldv, flags, codes);
    if (rc != KS_OK) return rc;
    const int64_t size = dtype == KS_DTYPE_FP32 ? 4 : 2;
    const bool vec = ((uintptr_t)V | (uintptr_t)(ldv * size)) % 16 == 0;
    m4_over_groups(n, D, flags, [&](int64_t g, dim3 grid) {
        const auto go = [&](auto kernel, auto *rows) { hipLaunchKernelGGL(kernel, grid, dim3(M4_NT), 0, (hipStream_t)stream, rows, n, D, ldv, flags, codes, g); };
        if (dtype == KS_DTYPE_FP32) go(vec ? m4_quantize_kernel<float, true> : m4_quantize_kernel<float, false>, (const float *)V);
        else go(vec ? m4_quantize_kernel<uint16_t, true> : m4_quantize_kernel<uint16_t, false>, (const uint16_t *)V);
    });
    KS_LAUNCH_CHECK();
    return KS_OK;
}

extern "C" int class_dequantize_mxfp4(const uint8_t *codes, int64_t n, int D, uint32_t flags, void *V, int dtype, int64_t ldv, void *stream) {
    const int rc = m4_rows_check(V, dtype, n, D, ldv, flags, codes);
    if (rc != KS_OK) return rc;
    const int64_t size = dtype == KS_DTYPE_FP32 ? 4 : 2;
    const int vec = ((uintptr_t)V | (uintptr_t)(ldv * size)) % 16 == 0;
    m4_over_groups(n, D, flags, [&](int64_t g, dim3 grid) {
        if (dtype == KS_DTYPE_FP32)
            hipLaunchKernelGGL(m4_dequantize_kernel<float>, grid, dim3(M4_NT), 0, (hipStream_t)stream, codes, n, D, flags, (float *)V, ldv, g, vec);
        else
            hipLaunchKernelGGL(m4_dequantize_kernel<uint16_t>, grid, dim3(M4_NT), 0, (hipStream_t)stream, codes, n, D, flags, (uint16_t *)V, ldv, g, vec);
    });
    KS_LAUNCH_CHECK();
    return KS_OK;
}

// ------------------------------------------------------------------------------------------------
// logits
// ------------------------------------------------------------------------------------------------
// 32 samples by 32 classes by 64 elements of depth, exponents in byte J of the words
template <int J> __device__ __forceinline__ f32x16_t m4_mfma(m4_i32x4 x, m4_i32x4 w, f32x16_t c, int ex, int ew) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(m4_i32x8{x[0], x[1], x[2], x[3], 0, 0, 0, 0}, m4_i32x8{w[0], w[1], w[2], w[3], 0, 0, 0, 0}, c, 4, 4,
                                                           J, ex, J, ew);
}

__device__ __forceinline__ void m4_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void m4_store(uint16_t *p, float v) { *p = (uint16_t)ks_f2bf(v); }
// Pairs of classes pass by the caches (aux bit 1): nobody here reads a logit again, and the codes stay in them.
__device__ __forceinline__ void m4_store2(__amdgpu_buffer_rsrc_t to, uint32_t off, float v0, float v1, const float *) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(v0), __float_as_uint(v1)}, to, off, 0, 2);
}
__device__ __forceinline__ void m4_store2(__amdgpu_buffer_rsrc_t to, uint32_t off, float v0, float v1, const uint16_t *) {
    __builtin_amdgcn_raw_buffer_store_b32(ks_pack_bf2(v0, v1), to, off, 0, 2);
}
// Logits of 32 samples from m0 on by the 64 classes from c0 on as a buffer that ends with the last whole pair of the last sample's
// classes: what lies behind (samples that do not exist, and classes: M4_NO_CLASS) the hardware leaves out.  ldl is even here, and 32
// rows are less than 2^31 bytes (m4_logits sees to both).
#define M4_NO_CLASS 0x80000000u
template <typename OUT> __device__ __forceinline__ __amdgpu_buffer_rsrc_t m4_rows_of(OUT *out, int64_t ldl, int m0, int64_t c0, int64_t C, int B) {
    const int rows = B - m0 < 32 ? B - m0 : 32, classes = C - c0 < M4_GROUP ? (int)(C - c0) & ~1 : M4_GROUP;
    return __builtin_amdgcn_make_buffer_rsrc(out + (int64_t)m0 * ldl + c0, 0, rows > 0 ? (int)((rows - 1) * (uint32_t)(ldl * sizeof(OUT)) + classes * (uint32_t)sizeof(OUT)) : 0, 0x00020000);
}

// Scale, bias, type and store of 32 samples from m0 on by the 64 classes from c0 on.  A lane of the result holds one column of each of the
// two groups of codes, which are two consecutive classes, and rows 8 (r / 4) + 4 (lane / 32) + r % 4.  vec: pairs of classes are aligned.
template <typename OUT>
__device__ __forceinline__ void m4_finish(const f32x16_t (&acc)[2], float scale, const float (&b)[2], int64_t c0, int64_t C, int m0, int B, OUT *out,
                                          int64_t ldl, int vec) {
    const int lane = threadIdx.x & 63, half4 = 4 * (lane >> 5);
    const int64_t c = c0 + 2 * (lane & 31);
    if (vec) {
        const uint32_t row_bytes = (uint32_t)(ldl * sizeof(OUT));
        uint32_t off = c + 1 < C ? half4 * row_bytes + 2 * (lane & 31) * (uint32_t)sizeof(OUT) : M4_NO_CLASS;
        const __amdgpu_buffer_rsrc_t to = m4_rows_of(out, ldl, m0, c0, C, B);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            m4_store2(to, off, fmaf(acc[0][r], scale, b[0]), fmaf(acc[1][r], scale, b[1]), (const OUT *)nullptr);
            off += r % 4 < 3 ? row_bytes : 5 * row_bytes; // the other half of the wavefront holds the four rows between
            asm volatile("" : "+v"(off));                 // one register, not sixteen that are kept from call to call
        }
    }
    if (!vec || c0 + M4_GROUP > C) { // element by element; of pairs only the last class that has none
        int rows = B - m0 - half4;
        asm volatile("" : "+v"(rows), "+s"(ldl));
        OUT *p = out + (int64_t)(m0 + half4) * ldl + c;
        const bool one = c < C && (!vec || c + 1 == C), two = c + 1 < C && !vec;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (r / 4 * 8 + r % 4 < rows) {
                if (one) m4_store(p, fmaf(acc[0][r], scale, b[0]));
                if (two) m4_store(p + 1, fmaf(acc[1][r], scale, b[1]));
            }
            p += r % 4 < 3 ? ldl : 5 * ldl;
            asm volatile("" : "+v"(p));
        }
    }
}
__device__ __forceinline__ void m4_bias_of(const float *__restrict__ bias, int64_t c0, int64_t C, float (&b)[2]) {
    const int64_t c = c0 + 2 * (threadIdx.x & 31);
#pragma unroll
    for (int q = 0; q < 2; ++q) b[q] = bias ? bias[c + q < C ? c + q : C - 1] : 0.f;
}

// One wavefront: 64 classes (the two groups of codes of M4_GROUP) by 32 S samples, codes straight from memory.  KS > 1: KS wavefronts of a
// workgroup take a part of the depth each and add their sums in LDS, always in the same order.
template <int S, int KS, typename OUT>
__global__ void __launch_bounds__(M4_NT)
m4_direct_kernel(const uint8_t *__restrict__ xq, const uint8_t *__restrict__ wq, const float *__restrict__ bias, int64_t C, int kb, int B, float scale,
                 OUT *__restrict__ out, int64_t ldl, int vec) {
    constexpr int NG = M4_NT / 64 / KS; // class groups of a workgroup
    __shared__ float s_sum[KS > 1 ? (KS - 1) * S * 32 * 64 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % KS;
    const int sb = blockIdx.y * S, xblocks = (B + 31) / 32; // first 32 samples
    const int64_t grp = (int64_t)blockIdx.x * NG + wave / KS;
    if (grp * M4_GROUP >= C) return; // KS > 1: a workgroup has one class group, all its wavefronts or none
    const int bytes = m4_row_bytes(kb), nq = (kb + 3) / 4;
    const uint8_t *const wp = wq + grp * 2 * bytes;
    const uint8_t *xp[S];
#pragma unroll
    for (int s = 0; s < S; ++s) xp[s] = xq + (int64_t)min(sb + s, xblocks - 1) * bytes;
    float b[2];
    m4_bias_of(bias, grp * M4_GROUP, C, b);
    f32x16_t acc[S][2];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[s][q][r] = 0.f;
    const int end = nq * (part + 1) / KS;
    for (int p4 = nq * part / KS; p4 < end; ++p4) { // four pieces at a time
        int ew[2], ex[S];
        m4_i32x4 w[4][2], x[4][S];
#pragma unroll
        for (int q = 0; q < 2; ++q) ew[q] = *(const int *)(wp + q * bytes + kb * M4_PIECE + p4 * M4_EXPS + lane * 4);
#pragma unroll
        for (int s = 0; s < S; ++s) ex[s] = *(const int *)(xp[s] + kb * M4_PIECE + p4 * M4_EXPS + lane * 4);
        const auto load = [&](int j) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 2; ++q) w[j][q] = *(const m4_i32x4 *)(wp + q * bytes + (p4 * 4 + j) * M4_PIECE + lane * 16);
#pragma unroll
            for (int s = 0; s < S; ++s) x[j][s] = *(const m4_i32x4 *)(xp[s] + (p4 * 4 + j) * M4_PIECE + lane * 16);
        };
        const auto multiply = [&](auto j) __attribute__((always_inline)) {
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int q = 0; q < 2; ++q) acc[s][q] = m4_mfma<j.value>(x[j.value][s], w[j.value][q], acc[s][q], ex[s], ew[q]);
        };
        const auto all = [&](auto n) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < n.value; ++j) load(j);
            multiply(std::integral_constant<int, 0>());
            if constexpr (n.value > 1) multiply(std::integral_constant<int, 1>());
            if constexpr (n.value > 2) multiply(std::integral_constant<int, 2>());
            if constexpr (n.value > 3) multiply(std::integral_constant<int, 3>());
        };
        const int left = kb - p4 * 4;
        if (left >= 4) all(std::integral_constant<int, 4>());
        else if (left == 3) all(std::integral_constant<int, 3>());
        else if (left == 2) all(std::integral_constant<int, 2>());
        else all(std::integral_constant<int, 1>());
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
#pragma unroll
    for (int s = 0; s < S; ++s) m4_finish(acc[s], scale, b, grp * M4_GROUP, C, (sb + s) * 32, B, out, ldl, vec);
}

// The work of a workgroup that keeps samples: stretches of an XCD's class groups for one sample tile each.  Workgroup i runs on XCD i % 8, and
// the groups are dealt to the XCDs in eight ranges; the tiles of a round, at most eight, are taken by as many workgroups side by side, which
// are at the same groups at the same time and share their codes in the L2.
struct M4Share {
    int g_lo, g_n, n_sb, sb0; // the XCD's groups; tiles, those of the rounds before
    __device__ __forceinline__ M4Share(int groups, int n_sb_) {
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

// The last of an odd number of classes, which has no pair to be stored with: the wavefronts of all workgroups take 32 samples each.
template <typename OUT>
__device__ __forceinline__ void m4_last_class(const uint8_t *xq, const uint8_t *wq, const float *bias, int64_t C, int kb, int B, float scale, OUT *out, int64_t ldl) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, bytes = m4_row_bytes(kb);
    const uint8_t *const w = wq + (C - 1) / M4_GROUP * 2 * bytes; // C is odd: slot (C - 1) % 64 / 2 of the group's first codes
    for (int sb = blockIdx.x * waves + wave; sb * 32 < B; sb += gridDim.x * waves) {
        const uint8_t *const x = xq + (int64_t)sb * bytes;
        f32x16_t acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.f;
        for (int k = 0; k < kb; ++k) {
            const int ex = *(const int *)(x + kb * M4_PIECE + k / 4 * M4_EXPS + lane * 4) >> k % 4 * 8, ew = *(const int *)(w + kb * M4_PIECE + k / 4 * M4_EXPS + lane * 4) >> k % 4 * 8;
            acc = m4_mfma<0>(*(const m4_i32x4 *)(x + k * M4_PIECE + lane * 16), *(const m4_i32x4 *)(w + k * M4_PIECE + lane * 16), acc, ex, ew);
        }
        const float b = bias ? bias[C - 1] : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int m = sb * 32 + 4 * (lane >> 5) + r / 4 * 8 + r % 4;
            if (m < B && (lane & 31) == (int)((C - 1) % M4_GROUP / 2)) m4_store(out + (int64_t)m * ldl + C - 1, fmaf(acc[r], scale, b));
        }
    }
}

#define M4X_NT 512
// Rows of up to 512 elements: a wavefront keeps the codes of 64 classes in registers, a workgroup those of up to 4,096 / KB samples in LDS, and
// the samples go past 32 at a time: 2 KB matrix instructions a block, with the stores of the block before in between.  During a group's
// last block each piece of codes is replaced, when it has been used, by the next group's.  What bounds it are the stores: 1,024 x 390,625 x 512
// bf16 200 us (0.9 GB at 4.5 TB/s), x 128 168 us; wavefronts of their own, which read the samples again for every group, take 374 and 181.
template <int KB, typename OUT>
__global__ void __launch_bounds__(M4X_NT, 2)
m4_steady_kernel(const uint8_t *__restrict__ xq, const uint8_t *__restrict__ wq, const float *__restrict__ bias, int64_t C, int kb, int B, float scale,
                 OUT *__restrict__ out, int64_t ldl, int tile) { // tile: blocks of 32 samples at a time, even, at most 128 / KB
    constexpr int NW = M4X_NT / 64, KQ = KB / 4;
    __shared__ __attribute__((aligned(16))) char s_x[128 * M4_PIECE];
    __shared__ int s_e[128 / 4 * 64];
    __shared__ int s_next; // group that the next wavefront to ask gets: of two on a SIMD the older one runs ahead
    const uint32_t row_bytes = (uint32_t)(ldl * sizeof(OUT)); // 32 rows: less than 2^31 bytes
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half4 = 4 * (lane >> 5);
    const int xblocks = (B + 31) / 32, n_sb = (xblocks + tile - 1) / tile, bytes = m4_row_bytes(kb);
    const int groups = (int)((C + M4_GROUP - 1) / M4_GROUP);
    M4Share share(groups, n_sb);
    const int g_lo = share.g_lo;
    int sb, first, last;
    while (share.next(sb, first, last)) {
        if (first >= last) continue;
        __syncthreads();
        for (int p = wave; p < tile * KB; p += NW) { // k-step k of block i at (KB i + k), 0 beyond the depth
            const int blk = sb * tile + p / KB < xblocks ? sb * tile + p / KB : xblocks - 1, k = p % KB;
            m4_i32x4 v = {0, 0, 0, 0};
            if (k < kb) v = *(const m4_i32x4 *)(xq + (int64_t)blk * bytes + k * M4_PIECE + lane * 16);
            *(m4_i32x4 *)(s_x + p * M4_PIECE + lane * 16) = v;
        }
        for (int p = wave; p < tile * KQ; p += NW) {
            const int blk = sb * tile + p / KQ < xblocks ? sb * tile + p / KQ : xblocks - 1, q = p % KQ;
            s_e[p * 64 + lane] = q * 4 < kb ? *(const int *)(xq + (int64_t)blk * bytes + kb * M4_PIECE + q * M4_EXPS + lane * 4) : 0;
        }
        if (threadIdx.x == 0) s_next = first + NW;
        __syncthreads();

        int grp = first + wave;
        if (grp >= last) continue;
        const auto group_codes = [&](int g, int q) __attribute__((always_inline)) { // of a half of a group: 0 beyond the depth
            return __builtin_amdgcn_make_buffer_rsrc((void *)(wq + ((int64_t)(g_lo + g) * 2 + q) * bytes), 0, kb * M4_PIECE, 0x00020000);
        };
        const auto group_exps = [&](int g, int q) __attribute__((always_inline)) {
            return __builtin_amdgcn_make_buffer_rsrc((void *)(wq + ((int64_t)(g_lo + g) * 2 + q) * bytes + kb * M4_PIECE), 0, (kb + 3) / 4 * M4_EXPS, 0x00020000);
        };
        const auto codes = [&](__amdgpu_buffer_rsrc_t p, int k) __attribute__((always_inline)) { // the whole offset in the register that is checked against the end
            return __builtin_bit_cast(m4_i32x4, __builtin_amdgcn_raw_buffer_load_b128(p, lane * 16 + k * M4_PIECE, 0, 0));
        };
        m4_i32x4 w[KB][2], x[4];
        int ew[KQ][2], ex[2][KQ];
        f32x16_t acc[2][2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const __amdgpu_buffer_rsrc_t p = group_codes(grp, q), e = group_exps(grp, q);
#pragma unroll
            for (int k = 0; k < KB; ++k) w[k][q] = codes(p, k);
#pragma unroll
            for (int k = 0; k < KQ; ++k) ew[k][q] = __builtin_amdgcn_raw_buffer_load_b32(e, lane * 4 + k * M4_EXPS, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = *(const m4_i32x4 *)(s_x + k * M4_PIECE + lane * 16);
#pragma unroll
        for (int k = 0; k < KQ; ++k) ex[0][k] = s_e[k * 64 + lane];
        // the block that is finished while the next one is multiplied; none yet: a buffer of no bytes
        __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(out, 0, 0, 0x00020000);
        uint32_t off = 0;
        float b[2] = {0.f, 0.f};
        const auto finish = [&](const f32x16_t (&a)[2], int r) __attribute__((always_inline)) { // one row of each half
            m4_store2(to, off, fmaf(a[0][r], scale, b[0]), fmaf(a[1][r], scale, b[1]), (const OUT *)nullptr);
            off += r % 4 < 3 ? row_bytes : 5 * row_bytes;
            asm volatile("" : "+v"(off)); // one register, not sixteen that are kept for every block
        };
        while (grp < last) {
            int got = 0;
            if (lane == 0) got = atomicAdd(&s_next, 1);
            const int next = __builtin_amdgcn_readfirstlane(got);
            const int g_next = next < last ? next : grp;
            const __amdgpu_buffer_rsrc_t p_next[2] = {group_codes(g_next, 0), group_codes(g_next, 1)}, e_next[2] = {group_exps(g_next, 0), group_exps(g_next, 1)};
            const int64_t c0 = (int64_t)(g_lo + grp) * M4_GROUP, c = c0 + 2 * (lane & 31);
            float nb[2];
            m4_bias_of(bias, c0, C, nb);
            const uint32_t off0 = c + 1 < C ? half4 * row_bytes + 2 * (lane & 31) * (uint32_t)sizeof(OUT) : M4_NO_CLASS;
            const auto block = [&](int blk, f32x16_t (&a)[2], const f32x16_t (&before)[2], const int (&e)[KQ], int (&e_after)[KQ], auto reload) __attribute__((always_inline)) {
                const int after = reload ? 0 : blk + 1;
                const char *xp = s_x + blk * (KB * M4_PIECE) + lane * 16, *xn = s_x + after * (KB * M4_PIECE) + lane * 16;
#pragma unroll
                for (int k = 0; k < KQ; ++k) e_after[k] = s_e[(after * KQ + k) * 64 + lane];
                const auto step = [&](int k4, auto j) __attribute__((always_inline)) {
                    const int k = k4 * 4 + j.value;
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        if (k == 0) a[q] = m4_mfma<0>(x[0], w[0][q], f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0}, e[0], ew[0][q]);
                        else a[q] = m4_mfma<j.value>(x[k & 3], w[k][q], a[q], e[k4], ew[k4][q]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    x[k & 3] = *(const m4_i32x4 *)(k + 4 < KB ? xp + (k + 4) * M4_PIECE : xn + (k + 4 - KB) * M4_PIECE);
                    if (reload)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            w[k][q] = codes(p_next[q], k);
                            if (j.value == 3) ew[k4][q] = __builtin_amdgcn_raw_buffer_load_b32(e_next[q], lane * 4 + k4 * M4_EXPS, 0, 0);
                        }
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (r * KB / 16 == k) finish(before, r);
                };
#pragma unroll
                for (int k4 = 0; k4 < KQ; ++k4) {
                    step(k4, std::integral_constant<int, 0>());
                    step(k4, std::integral_constant<int, 1>());
                    step(k4, std::integral_constant<int, 2>());
                    step(k4, std::integral_constant<int, 3>());
                }
                to = m4_rows_of(out, ldl, (sb * tile + blk) * 32, c0, C, B);
                off = off0;
                b[0] = nb[0];
                b[1] = nb[1];
            };
            for (int i = 0; i + 2 < tile; i += 2) {
                block(i, acc[0], acc[1], ex[0], ex[1], std::false_type());
                block(i + 1, acc[1], acc[0], ex[1], ex[0], std::false_type());
            }
            block(tile - 2, acc[0], acc[1], ex[0], ex[1], std::false_type());
            block(tile - 1, acc[1], acc[0], ex[1], ex[0], std::true_type());
            grp = next;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) finish(acc[1], r);
    }
    if (C & 1) m4_last_class(xq, wq, bias, C, kb, B, scale, out, ldl);
}

// workgroup barrier that waits for this wavefront's LDS accesses but, unlike __syncthreads(), not for loads in flight
__device__ __forceinline__ void m4_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F); // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Deeper rows: the samples pass through LDS in chunks of eight k-steps, which eight wavefronts with 64 classes each read at the same time: three
// buffers, a barrier a chunk.  While chunk t is multiplied, a fragment is read for the next k-step when it has been used (the last ones
// from chunk t + 1, which is there since the barrier), and chunk t + 2 is written to LDS from registers.  Weights come straight from memory,
// four k-steps ahead.  2,048 x 131,072 x 4,096 bf16: 650 us, 3.4 PFLOP/s (wavefronts of their own 1,320); what holds it up are the operands' ways
// into the registers, 32 KB from LDS and 18 KB through the caches for 64 matrix instructions: the matrix pipes are busy 40 % of the cycles, at 2.0 GHz
// (92 %, at 1.7 GHz and 6.1 PFLOP/s, with operands in registers).  The chunks run on from one tile of 512 classes by 128 samples to the next;
// what lies beyond the depth is loaded as 0 and multiplied (2,048 x 131,072 x 576 184 us, x 1,024 212).
template <typename OUT>
__global__ void __launch_bounds__(M4X_NT, 2)
m4_staged_kernel(const uint8_t *__restrict__ xq, const uint8_t *__restrict__ wq, const float *__restrict__ bias, int64_t C, int kb, int B, float scale,
                 OUT *__restrict__ out, int64_t ldl, int vec) {
    constexpr int NW = M4X_NT / 64, R = 8, CHUNK = R * 4 * M4_PIECE, EXPS = R / 4 * 4 * 64 /* words of a chunk's exponents */;
    __shared__ __attribute__((aligned(16))) char s_x[3 * CHUNK];
    __shared__ int s_e[3 * EXPS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int xblocks = (B + 31) / 32, n_sb = (B + 127) / 128, chunks = (kb + R - 1) / R, bytes = m4_row_bytes(kb);
    const int groups = (int)((C + M4_GROUP - 1) / M4_GROUP), n_ct = (groups + NW - 1) / NW;
    // workgroup i runs on XCD i % 8; an XCD has a range of the class tiles, and its workgroups take them for all samples before the
    // next ones: what 32 of them read at a time are a few class tiles and the samples
    const int xcd = blockIdx.x & 7, per_xcd = gridDim.x >> 3, j0 = blockIdx.x >> 3;
    const int c_lo = (int)((int64_t)n_ct * xcd / 8), c_n = (int)((int64_t)n_ct * (xcd + 1) / 8) - c_lo;
    int64_t left = (int64_t)c_n * n_sb - j0; // tiles from this one on, of this and the XCD's other workgroups
    const int step_c = per_xcd / n_sb, step_s = per_xcd % n_sb; // from one of this workgroup's tiles to its next
    int ct = c_lo + j0 / n_sb, sb = j0 % n_sb;

    // samples: this wavefront moves k-step `wave` of a chunk, for four blocks of samples, and one word of exponents
    int64_t r_left = left;
    int r_sb = sb, r_c = 0; // chunk that is requested next
    m4_i32x4 held[2];
    int held_e;
    const auto request = [&](auto h) __attribute__((always_inline)) { // a half of it
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int s = r_sb * 4 + h.value * 2 + i, blk = s < xblocks ? s : xblocks - 1;
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void *)(xq + (int64_t)blk * bytes), 0, kb * M4_PIECE, 0x00020000);
            held[i] = __builtin_bit_cast(m4_i32x4, __builtin_amdgcn_raw_buffer_load_b128(from, lane * 16 + (r_c * R + wave) * M4_PIECE, 0, 0));
        }
        if (h.value == 0) {
            const int s = r_sb * 4 + (wave & 3), blk = s < xblocks ? s : xblocks - 1;
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void *)(xq + (int64_t)blk * bytes + kb * M4_PIECE), 0, (kb + 3) / 4 * M4_EXPS, 0x00020000);
            held_e = __builtin_amdgcn_raw_buffer_load_b32(from, lane * 4 + (r_c * 2 + (wave >> 2)) * M4_EXPS, 0, 0);
        } else { // behind the last tile: the same again, read by nobody
            const bool end = ++r_c == chunks, more = end && r_left > per_xcd;
            r_c = end ? 0 : r_c;
            r_left = more ? r_left - per_xcd : r_left;
            r_sb = more ? r_sb + step_s : r_sb;
            r_sb = r_sb >= n_sb ? r_sb - n_sb : r_sb;
        }
    };
    const auto place = [&](auto h, char *to, int *to_e) __attribute__((always_inline)) { // k-step k of block s at (4 k + s)
#pragma unroll
        for (int i = 0; i < 2; ++i) *(m4_i32x4 *)(to + (wave * 4 + h.value * 2 + i) * M4_PIECE + lane * 16) = held[i];
        if (h.value == 0) to_e[wave * 64 + lane] = held_e;
    };
    const std::integral_constant<int, 0> H0;
    const std::integral_constant<int, 1> H1;
    const auto rsrc = [&](int tile, int q, bool exps) __attribute__((always_inline)) { // of this wavefront's classes in a tile; beyond the last group: that one
        const int g = tile * NW + wave;
        const uint8_t *const p = wq + ((int64_t)(g < groups ? g : groups - 1) * 2 + q) * bytes;
        return __builtin_amdgcn_make_buffer_rsrc((void *)(exps ? p + kb * M4_PIECE : p), 0, exps ? (kb + 3) / 4 * M4_EXPS : kb * M4_PIECE, 0x00020000);
    };
    char *b0 = s_x, *b1 = s_x + CHUNK, *b2 = s_x + 2 * CHUNK; // chunks t, t + 1, t + 2
    int *e0 = s_e, *e1 = s_e + EXPS, *e2 = s_e + 2 * EXPS;
    request(H0);
    place(H0, b0, e0);
    request(H1);
    place(H1, b0, e0);
    request(H0);
    place(H0, b1, e1);
    request(H1);
    place(H1, b1, e1);
    request(H0);
    m4_i32x4 w[4][2], x[4];
    int ew[2][2], ex[4]; // ew: of this and of the next four k-steps
    __amdgpu_buffer_rsrc_t wr[2] = {rsrc(ct, 0, false), rsrc(ct, 1, false)}, er[2] = {rsrc(ct, 0, true), rsrc(ct, 1, true)};
#pragma unroll
    for (int q = 0; q < 2; ++q) ew[0][q] = __builtin_amdgcn_raw_buffer_load_b32(er[q], lane * 4, 0, 0);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int q = 0; q < 2; ++q) w[kk][q] = __builtin_bit_cast(m4_i32x4, __builtin_amdgcn_raw_buffer_load_b128(wr[q], lane * 16 + kk * M4_PIECE, 0, 0));
    m4_barrier();
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        x[s] = *(const m4_i32x4 *)(b0 + s * M4_PIECE + lane * 16);
        ex[s] = e0[s * 64 + lane];
    }
    for (; left > 0; left -= per_xcd) {
        int next_ct = ct + step_c, next_sb = sb + step_s;
        if (next_sb >= n_sb) { next_sb -= n_sb; ++next_ct; }
        if (left <= per_xcd) next_ct = ct;
        f32x16_t acc[4][2];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[s][q][r] = 0.f;
        for (int c = 0; c < chunks; ++c) {
            // four k-steps on: the second half of this chunk, then the first of the next one (of the next tile)
            const int at_mid = (c * R + 4) * M4_PIECE, at_next = c + 1 < chunks ? (c + 1) * R * M4_PIECE : 0;
            // no branch for that: behind one the compiler would gather all matrix instructions before it
            const int after = c + 1 < chunks ? ct : next_ct;
            const __amdgpu_buffer_rsrc_t wn[2] = {rsrc(after, 0, false), rsrc(after, 1, false)}, en[2] = {rsrc(after, 0, true), rsrc(after, 1, true)};
            m4_barrier(); // chunk t + 1 is whole, and nobody reads chunk t - 1 any more
            const auto step = [&](auto K) __attribute__((always_inline)) {
                constexpr int kk = K.value, half = kk / 4, j = kk % 4;
                if (j == 0) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) ew[1 - half][q] = __builtin_amdgcn_raw_buffer_load_b32(half == 0 ? er[q] : en[q], lane * 4 + (half == 0 ? at_mid : at_next) / (4 * M4_PIECE) * M4_EXPS, 0, 0);
                }
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int q = 0; q < 2; ++q) acc[s][q] = m4_mfma<j>(x[s], w[j][q], acc[s][q], ex[s], ew[half][q]);
                    __builtin_amdgcn_sched_barrier(0);
                    x[s] = *(const m4_i32x4 *)((kk < R - 1 ? b0 + (kk + 1) * 4 * M4_PIECE : b1) + s * M4_PIECE + lane * 16);
                    if (j == 3) ex[s] = (half == 0 ? e0 + 4 * 64 : e1)[s * 64 + lane];
                    if (s == 3)
#pragma unroll
                        for (int q = 0; q < 2; ++q)
                            w[j][q] = __builtin_bit_cast(m4_i32x4, __builtin_amdgcn_raw_buffer_load_b128(half == 0 ? wr[q] : wn[q], lane * 16 + (half == 0 ? at_mid : at_next) + j * M4_PIECE, 0, 0));
                }
                if (kk == 2) {
                    place(H0, b2, e2);
                    request(H1);
                }
                if (kk == 6) {
                    place(H1, b2, e2);
                    request(H0);
                }
            };
            step(std::integral_constant<int, 0>());
            step(std::integral_constant<int, 1>());
            step(std::integral_constant<int, 2>());
            step(std::integral_constant<int, 3>());
            step(std::integral_constant<int, 4>());
            step(std::integral_constant<int, 5>());
            step(std::integral_constant<int, 6>());
            step(std::integral_constant<int, 7>());
#pragma unroll
            for (int q = 0; q < 2; ++q) { wr[q] = wn[q]; er[q] = en[q]; }
            char *const b = b0;
            b0 = b1; b1 = b2; b2 = b;
            int *const e = e0;
            e0 = e1; e1 = e2; e2 = e;
        }
        const int g = ct * NW + wave;
        if (g < groups) {
            float b[2];
            m4_bias_of(bias, (int64_t)g * M4_GROUP, C, b);
#pragma unroll
            for (int s = 0; s < 4; ++s) m4_finish(acc[s], scale, b, (int64_t)g * M4_GROUP, C, sb * 128 + s * 32, B, out, ldl, vec);
        }
        ct = next_ct;
        sb = next_sb;
    }
}

template <typename OUT>
static void m4_logits(const uint8_t *xq, const uint8_t *wq, const float *bias, int64_t C, int D, int B, float scale, OUT *out, int64_t ldl, hipStream_t st) {
    // vec: pairs of classes in one store; 64 MB from row to row and more, whose offsets are no 32 bits, go element by element
    const int vec = ((uintptr_t)out | (uintptr_t)(ldl * sizeof(OUT))) % (2 * sizeof(OUT)) == 0 && ldl < (1 << 26) / (int64_t)sizeof(OUT), kb = (D + 63) / 64;
    const int64_t groups = ks_ceil_div(C, M4_GROUP);
    const auto direct = [&](auto kernel, int samples, int per_workgroup) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)ks_ceil_div(groups, per_workgroup), (unsigned)ks_ceil_div(B, samples)), dim3(M4_NT), 0, st, xq, wq, bias,
                           C, kb, B, scale, out, ldl, vec);
    };
    const int64_t waves = groups * ks_ceil_div(B, 64);
    if (B <= 32) return waves <= 1024 && kb >= 16 ? direct(m4_direct_kernel<1, 4, OUT>, 32, 1) : direct(m4_direct_kernel<1, 1, OUT>, 32, 4);
    // Few samples: the codes of the weights are what moves, and every wavefront reads its own (1 x 390,625 x 512 bf16: 24 us with the features'
    // codes); where there are few wavefronts and rows are deep, four of them divide a group's depth.  Few wavefronts, or few groups of classes
    // for the 256 workgroups that keep samples, likewise, and rows that begin on an odd element, which are stored element by element.  In us, of wavefronts
    // of their own and with samples kept: 10,000 classes (157 groups), batch 1,024, x 128 8.6 and 19.6, x 512 10.5 and 15.8; 2,048 x 512 14.9 and 16.6;
    // 4,096 x 512 25.7 and 24.4; 16,000 (250 groups) 2,048 x 512 28 and 20, x 256 15.0 and 18.9; 30,000, 512 x 512 (3,752 wavefronts) 13.8 and 15.4, 1,024
    // 23.7 and 18.7; x 128, 2,048: 50,000 (782 groups) 34 and 47, 60,000 56 and 54.  Deeper rows: 10,000 x 576, 512 (1,256 wavefronts) 7.9 and 13.6, 1,024
    // 11.2 and 14.1; 131,072 x 576, 2,048 249 and 184; but 1,000 x 1,024, 8,192 11 and 25: a few tiles of 512 classes leave XCDs without work.
    if (B <= 64 || waves <= 1280 || (kb <= 8 && (!vec || groups <= 160 || waves <= 3800)) || (kb <= 2 && groups <= 800))
        return waves <= 320 && kb >= 16 ? direct(m4_direct_kernel<2, 4, OUT>, 64, 1) : direct(m4_direct_kernel<2, 1, OUT>, 64, 4);
    if (kb > 8) {
        hipLaunchKernelGGL(m4_staged_kernel<OUT>, dim3(256), dim3(M4X_NT), 0, st, xq, wq, bias, C, kb, B, scale, out, ldl, vec);
        return;
    }
    const int KB = kb <= 4 ? 4 : 8, xblocks = (B + 31) / 32, most = 128 / KB, tiles = (xblocks + most - 1) / most, tile = ((xblocks + tiles - 1) / tiles + 1) / 2 * 2;
    hipLaunchKernelGGL((KB == 4 ? m4_steady_kernel<4, OUT> : m4_steady_kernel<8, OUT>), dim3(256), dim3(M4X_NT), 0, st, xq,
                       wq, bias, C, kb, B, scale, out, ldl, tile);
}

extern "C" int class_logits_mxfp4(const uint8_t *x_codes, const uint8_t *w_codes, const float *bias, int64_t C, int D, int B, float scale,
                                  void *logits, int dtype, int64_t ldl, void *stream) {
    if (!x_codes || !w_codes || !logits) return KS_INVALID_ARG;
    if (C < 1 || C >= (int64_t)1 << 31 || D < 1 || B < 1 || ldl < C) return KS_INVALID_ARG;
    if (dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) return KS_INVALID_ARG;
    if (((uintptr_t)x_codes | (uintptr_t)w_codes) % 16 || (uintptr_t)logits % (dtype == KS_DTYPE_FP32 ? 4 : 2)) return KS_INVALID_ARG;
    if (D > KS_MAX_MXFP4_D || B > KS_MAX_MXFP4_B) return KS_UNSUPPORTED;
    if (dtype == KS_DTYPE_FP32) m4_logits<float>(x_codes, w_codes, bias, C, D, B, scale, (float *)logits, ldl, (hipStream_t)stream);
    else m4_logits<uint16_t>(x_codes, w_codes, bias, C, D, B, scale, (uint16_t *)logits, ldl, (hipStream_t)stream);
    KS_LAUNCH_CHECK();
    return KS_OK;
}
