// Learning from a teacher's top logits (paper Section 3.2: the softmax over the classes and its gradient, here against a distribution
// instead of a label).
//
// With l = log2(e) / T and m the row's largest logit, p_c = 2^(l (z_c - m)) / S, S the sum of those powers over the row, and
//     loss = T^2 (A + m / T + ln S),  A = sum_k q_k (ln q_k - z_k / T),
// since the q_k add up to 1: A needs neither m nor S, so that the first pass computes it beside them and the second overwrites the logits
// where that is asked for.
#include "../../include/class_distill.h"
#include "ks_common.h"

#define DS_NT 256

struct DsArgs {
    const void *logits, *t_logits;
    void *out;
    int64_t ldl, ldd, C, slice; // slice: vectors of a workgroup
    const int32_t *t_ids;
    int B, K, t_bf16, slices, parts, row0; // slices of the launch, of the first one
    float T, l, g; // g = grad_scale T / B
    float *loss, *loss_mean;
    float2 *part;  // [B, parts]: largest logit, sum of the powers relative to it
    double *a;     // [B]: A
    int32_t *dev_status;
};

template <typename T> struct DsVec; // 16 bytes
template <> struct DsVec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
    static __device__ __forceinline__ void load(const float *p, float (&v)[4]) {
        const float4 a = *(const float4 *)p;
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    }
    static __device__ __forceinline__ void store(float *p, const float (&v)[4]) { *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct DsVec<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float one(const uint16_t *p) { return ks_bf2f(*p); }
    static __device__ __forceinline__ void put(uint16_t *p, float v) { *p = (uint16_t)ks_f2bf(v); }
    static __device__ __forceinline__ void load(const uint16_t *p, float (&v)[8]) {
        const uint4 a = *(const uint4 *)p;
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float (&v)[8]) {
        *(uint4 *)p = make_uint4(ks_pack_bf2(v[0], v[1]), ks_pack_bf2(v[2], v[3]), ks_pack_bf2(v[4], v[5]), ks_pack_bf2(v[6], v[7]));
    }
};

// A workgroup's part of a row: vectors [v0, v1) of 16 bytes behind the `head` first elements (up to the first multiple of 16), the first slice
// with the head, the last with what is left of the row; in all the elements [first, last).
template <typename T, bool VEC> struct DsSlice {
    static constexpr int N = VEC ? DsVec<T>::N : 1;
    int64_t v0, v1, first, last, rest;
    int head;
    __device__ __forceinline__ DsSlice(const DsArgs &a, const T *row, int i) {
        const int beside = VEC ? (int)((0 - (uintptr_t)row) % 16 / sizeof(T)) : 0;
        head = beside < a.C ? beside : (int)a.C;
        const int64_t all = (a.C - head) / N;
        rest = head + all * N; // elements from here on are the row's last, less than a vector
        v0 = i * a.slice;
        v0 = v0 < all ? v0 : all;
        v1 = v0 + a.slice < all && i < a.slices - 1 ? v0 + a.slice : all;
        first = i == 0 ? 0 : head + v0 * N;
        last = i == a.slices - 1 ? a.C : head + v1 * N;
    }
    // f(pointer offset) for the single elements of this slice
    template <typename F> __device__ __forceinline__ void singles(const DsArgs &a, int i, F f) const {
        const int t = threadIdx.x;
        if (VEC && i == 0 && t < head) f((int64_t)t);
        if (VEC && i == a.slices - 1 && t < (int)(a.C - rest)) f(rest + t);
    }
};

// (largest, sum of 2^(l (z - largest))): NaN and +infinity stay visible, -infinity adds nothing
__device__ __forceinline__ void ds_join(float &m, float &s, float m2, float s2, float l) {
    const float top = fmaxf(m, m2), base = top > -INFINITY ? top : 0.f;
    s = s * __builtin_amdgcn_exp2f(l * (m - base)) + s2 * __builtin_amdgcn_exp2f(l * (m2 - base));
    m = top;
}

struct DsTeacher { // of a row: q_k = exp((t - top) / T) / sum; none: sum == 0
    float top, sum;
};
__device__ __forceinline__ float ds_t_logit(const DsArgs &a, int64_t at) {
    return a.t_bf16 ? ks_bf2f(((const uint16_t *)a.t_logits)[at]) : ((const float *)a.t_logits)[at];
}
__device__ __forceinline__ float ds_block_sum(float v, float *sh) { // fixed order
    v = ks_wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return sh[0] + sh[1] + sh[2] + sh[3];
}
__device__ __forceinline__ float ds_block_max(float v, float *sh) {
    v = ks_wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}
// the row's entries into LDS (ids, -1: empty, and weights), and their sum
__device__ __forceinline__ DsTeacher ds_teacher(const DsArgs &a, int row, int32_t *s_id, float *s_q, float *sh, bool report) {
    float top = -INFINITY;
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        int id = a.t_ids[(int64_t)row * a.K + k];
        if (id >= a.C) {
            if (report) ks_flag(a.dev_status, KS_DEV_BAD_LABEL);
            id = -1;
        }
        const float t = id >= 0 ? ds_t_logit(a, (int64_t)row * a.K + k) : -INFINITY;
        s_id[k] = id;
        s_q[k] = t;
        top = fmaxf(top, t);
    }
    top = ds_block_max(top, sh);
    float sum = 0.f;
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        const float t = s_q[k], q = t == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(a.l * (t - top));
        s_q[k] = q;
        sum += q;
    }
    return DsTeacher{top, ds_block_sum(sum, sh)};
}

// First pass: every slice's largest logit and sum of powers; the first slice also the row's A.
template <typename T>
__global__ void __launch_bounds__(DS_NT)
ds_stats_kernel(DsArgs a) {
    extern __shared__ int32_t s_id[];
    float *const s_q = (float *)(s_id + a.K);
    __shared__ float sh[4];
    __shared__ double shd[4];
    const int row = a.row0 + blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T *const z = (const T *)a.logits + (int64_t)row * a.ldl;
    const DsSlice<T, true> sl(a, z, blockIdx.x);
    typedef DsVec<T> V;
    constexpr int N = V::N;
    float m = -INFINITY, s = 0.f;
    for (int64_t i = sl.v0 + threadIdx.x; i < sl.v1; i += DS_NT) {
        float v[N];
        V::load(z + sl.head + i * N, v);
        float top = v[0];
#pragma unroll
        for (int j = 1; j < N; ++j) top = fmaxf(top, v[j]);
        if (top > m) { // seldom after the first ones
            s *= __builtin_amdgcn_exp2f(a.l * (m - top));
            m = top;
        }
        const float base = m > -INFINITY ? m : 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) s += __builtin_amdgcn_exp2f(a.l * (v[j] - base));
    }
    sl.singles(a, blockIdx.x, [&](int64_t c) __attribute__((always_inline)) {
        ds_join(m, s, V::one(z + c), 1.f, a.l);
    });
    const float top = ds_block_max(m, sh), base = top > -INFINITY ? top : 0.f;
    s = ds_block_sum(s * (m == base ? 1.f : __builtin_amdgcn_exp2f(a.l * (m - base))), sh);
    if (threadIdx.x == 0) a.part[(int64_t)row * a.parts + blockIdx.x] = make_float2(top, s);
    if (blockIdx.x) return;
    const DsTeacher t = ds_teacher(a, row, s_id, s_q, sh, true);
    double sum = 0.0;
    const double inv_T = 1.0 / (double)a.T, log_sum = log((double)t.sum);
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        const float q = s_q[k];
        if (s_id[k] >= 0 && q != 0.f) {
            const double log_q = ((double)ds_t_logit(a, (int64_t)row * a.K + k) - (double)t.top) * inv_T - log_sum;
            sum += (double)q / (double)t.sum * (log_q - (double)V::one(z + s_id[k]) * inv_T);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) shd[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.a[row] = shd[0] + shd[1] + shd[2] + shd[3];
}

// Second pass: the gradient of every slice, the first one also the row's loss.
template <typename T, bool VEC>
__global__ void __launch_bounds__(DS_NT)
ds_grad_kernel(DsArgs a) {
    extern __shared__ int32_t s_id[];
    float *const s_q = (float *)(s_id + a.K), *const s_grad = s_q + a.K;
    uint8_t *const s_again = (uint8_t *)(s_grad + a.K);
    __shared__ float sh[4];
    const int row = a.row0 + blockIdx.y;
    const T *const z = (const T *)a.logits + (int64_t)row * a.ldl;
    T *const out = (T *)a.out + (int64_t)row * a.ldd;
    const DsSlice<T, VEC> sl(a, z, blockIdx.x);
    typedef DsVec<T> V;
    constexpr int N = DsSlice<T, VEC>::N;
    // the row's largest logit and sum, in every workgroup in the same order
    float m = -INFINITY, s = 0.f;
    for (int i = threadIdx.x; i < a.parts; i += DS_NT) {
        const float2 p = a.part[(int64_t)row * a.parts + i];
        ds_join(m, s, p.x, p.y, a.l);
    }
    const float top = ds_block_max(m, sh), base = top > -INFINITY ? top : 0.f;
    s = ds_block_sum(s * (m == base ? 1.f : __builtin_amdgcn_exp2f(a.l * (m - base))), sh);
    const DsTeacher t = ds_teacher(a, row, s_id, s_q, sh, false);
    const bool some = t.sum != 0.f;
    // p = 2^(l (z - base)) * f; a row without a class has p = 0, one with a NaN or +infinity NaN
    const float f = !some || s == 0.f ? 0.f : top < INFINITY ? a.g / s : __int_as_float(0x7FC00000);
    if (blockIdx.x == 0 && threadIdx.x == 0)
        a.loss[row] = some ? (float)((double)a.T * (double)a.T * (a.a[row] + (s == 0.f ? 0.0 : (double)base / (double)a.T + log((double)s)))) : 0.f;
    const auto grad = [&](float v) __attribute__((always_inline)) { return f == 0.f ? 0.f : __builtin_amdgcn_exp2f(a.l * (v - base)) * f; };
    // the gradient at the named classes of this slice, before their logits may be overwritten: at a class's first entry, the others empty
    const float to_q = some ? a.g / t.sum : 0.f;
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        const int id = s_id[k];
        if (id < sl.first || id >= sl.last) continue;
        float q = 0.f;
        bool again = false;
        for (int j = 0; j < a.K; ++j)
            if (s_id[j] == id) {
                again |= j < k;
                q += s_q[j];
            }
        s_again[k] = again;
        s_grad[k] = grad(V::one(z + id)) - to_q * q;
    }
    __syncthreads();
    for (int64_t i = sl.v0 + threadIdx.x; i < sl.v1; i += DS_NT) {
        float v[N];
        if constexpr (VEC) V::load(z + sl.head + i * N, v);
        else v[0] = V::one(z + i);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = grad(v[j]);
        if constexpr (VEC) V::store(out + sl.head + i * N, v);
        else V::put(out + i, v[0]);
    }
    sl.singles(a, blockIdx.x, [&](int64_t c) __attribute__((always_inline)) { V::put(out + c, grad(V::one(z + c))); });
    // the others' stores have to be there before the named classes are stored over them
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        const int id = s_id[k];
        if (id >= sl.first && id < sl.last && !s_again[k]) V::put(out + id, s_grad[k]);
    }
}

__global__ void __launch_bounds__(DS_NT) ds_mean_kernel(const float *__restrict__ loss, int B, float *__restrict__ mean) {
    __shared__ double sh[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < B; i += DS_NT) s += (double)loss[i];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) *mean = (float)((sh[0] + sh[1] + sh[2] + sh[3]) / B);
}

#define DS_SLICE_BYTES (32 << 10)
static int ds_slices(int64_t C) { return (int)ks_ceil_div(C, DS_SLICE_BYTES / 4); } // for the smaller slices of fp32

extern "C" size_t class_distill_workspace(int64_t C, int B, int K) {
    if (C < 1 || C >= (int64_t)1 << 31 || B < 1 || K < 1 || K > KS_MAX_DISTILL_K) return 0;
    KsArena ws(nullptr);
    ws.take<float2>((size_t)B * ds_slices(C));
    ws.take<double>((size_t)B);
    return ws.off;
}

extern "C" int class_distill_fwd_bwd(const void *logits, int64_t ldl, int dtype, int64_t C, int B, const int32_t *t_ids, const void *t_logits,
                                     int t_dtype, int K, float temperature, float grad_scale, float *loss_per_sample, float *loss_mean,
                                     void *dlogits, int64_t ldd, void *ws, size_t ws_bytes, int32_t *dev_status, void *stream) {
    if (!logits || !t_ids || !t_logits || !loss_per_sample || !loss_mean || !dlogits || !ws) return KS_INVALID_ARG;
    if (C < 1 || C >= (int64_t)1 << 31 || B < 1 || K < 1 || ldl < C || ldd < C || (dlogits == logits && ldd != ldl)) return KS_INVALID_ARG;
    if ((dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) || (t_dtype != KS_DTYPE_BF16 && t_dtype != KS_DTYPE_FP32)) return KS_INVALID_ARG;
    if (!(temperature > 0.f) || temperature > 3.4028234e38f) return KS_INVALID_ARG;
    const int size = dtype == KS_DTYPE_FP32 ? 4 : 2;
    if (((uintptr_t)logits | (uintptr_t)dlogits) % size || (uintptr_t)t_logits % (t_dtype == KS_DTYPE_FP32 ? 4 : 2) || (uintptr_t)ws % 256) return KS_INVALID_ARG;
    if (((uintptr_t)t_ids | (uintptr_t)loss_per_sample | (uintptr_t)loss_mean | (uintptr_t)dev_status) % 4) return KS_INVALID_ARG;
    if (K > KS_MAX_DISTILL_K) return KS_UNSUPPORTED;
    if (ws_bytes < class_distill_workspace(C, B, K)) return KS_WORKSPACE_TOO_SMALL;
    DsArgs a;
    KsArena arena(ws);
    a.part = arena.take<float2>((size_t)B * ds_slices(C));
    a.a = arena.take<double>((size_t)B);
    a.logits = logits; a.t_logits = t_logits; a.out = dlogits;
    a.ldl = ldl; a.ldd = ldd; a.C = C; a.t_ids = t_ids; a.B = B; a.K = K; a.t_bf16 = t_dtype == KS_DTYPE_BF16;
    a.T = temperature; a.l = (float)(1.4426950408889634 / (double)temperature); a.g = (float)((double)grad_scale * (double)temperature / B);
    a.loss = loss_per_sample; a.loss_mean = loss_mean; a.dev_status = dev_status;
    // vectors are stored where rows of both matrices begin equally many bytes beside a multiple of 16
    const bool vec = ((uintptr_t)logits - (uintptr_t)dlogits) % 16 == 0 && (uint64_t)(ldl - ldd) * size % 16 == 0;
    const int n = 16 / size;
    const int64_t slice = DS_SLICE_BYTES / size; // elements
    hipStream_t st = (hipStream_t)stream;
    a.parts = (int)ks_ceil_div(ks_ceil_div(C, n), slice / n);
    for (int64_t r = 0; r < B; r += 1 << 15) { // a launch's second dimension ends at 65,535
        const unsigned rows = (unsigned)(B - r < 1 << 15 ? B - r : 1 << 15);
        a.row0 = (int)r;
        const auto go = [&](auto stats, auto grad) {
            a.slice = slice / n;
            a.slices = a.parts;
            hipLaunchKernelGGL(stats, dim3((unsigned)a.parts, rows), dim3(DS_NT), (size_t)K * 8, st, a);
            if (!vec) {
                a.slice = slice;
                a.slices = (int)ks_ceil_div(C, slice);
            }
            hipLaunchKernelGGL(grad, dim3((unsigned)a.slices, rows), dim3(DS_NT), (size_t)K * 13, st, a);
        };
        if (dtype == KS_DTYPE_FP32) go(ds_stats_kernel<float>, vec ? ds_grad_kernel<float, true> : ds_grad_kernel<float, false>);
        else go(ds_stats_kernel<uint16_t>, vec ? ds_grad_kernel<uint16_t, true> : ds_grad_kernel<uint16_t, false>);
    }
    hipLaunchKernelGGL(ds_mean_kernel, dim3(1), dim3(DS_NT), 0, st, loss_per_sample, B, loss_mean);
    KS_LAUNCH_CHECK();
    return KS_OK;
}
