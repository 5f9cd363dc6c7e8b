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
        }
    }
    if (!vec || c0 + M4_GROUP > C) // element by element; of pairs only the last class that has none
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int m = m0 + half4 + r / 4 * 8 + r % 4;
            OUT *const p = out + (int64_t)m * ldl + c;
            if (m < B) {
                if (c < C && (!vec || c + 1 == C)) m4_store(p, fmaf(acc[0][r], scale, b[0]));
                if (c + 1 < C && !vec) m4_store(p + 1, fmaf(acc[1][r], scale, b[1]));
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
    return waves <= 320 && kb >= 16 ? direct(m4_direct_kernel<2, 4, OUT>, 64, 1) : direct(m4_direct_kernel<2, 1, OUT>, 64, 4);
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
