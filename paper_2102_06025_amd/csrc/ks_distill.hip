// Learning from a teacher's top logits (paper Section 3.2: the softmax over the classes and its gradient, here against a distribution
// instead of a label).
//
// With l = log2(e) / T and m the row's largest logit, p_c = 2^(l (z_c - m)) / S, S the sum of those powers over the row, and
//     loss = T^2 (A + m / T + ln S),  A = sum_k q_k (ln q_k - z_k / T),
// since the q_k add up to 1: A needs neither m nor S, so that the first pass computes it beside them and the second overwrites the logits
// where that is asked for.  A and m / T are as large as the logits, whatever is left of them: what the q_k add up to has to be 1 in fp64.
#include "../../include/class_distill.h"
#include "ks_common.h"

#define DS_NT 256
#define DS_PARTS (DS_NT * DS_HELD)
#define DS_HELD 8 /* vectors of 16 bytes that a thread holds: a slice is DS_NT * DS_HELD of them */

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
    float2 *t;     // [B]: the teacher's largest logit, sum of the powers relative to it
    int32_t *dev_status;
};

template <typename T> struct DsVec; // 16 bytes
template <> struct DsVec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
    static __device__ __forceinline__ void values(uint4 a, float (&v)[4]) {
        v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    }
    static __device__ __forceinline__ uint4 packed(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct DsVec<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float one(const uint16_t *p) { return ks_bf2f(*p); }
    static __device__ __forceinline__ void put(uint16_t *p, float v) { *p = (uint16_t)ks_f2bf(v); }
    static __device__ __forceinline__ void values(uint4 a, float (&v)[8]) {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 packed(const float (&v)[8]) {
        return make_uint4(ks_pack_bf2(v[0], v[1]), ks_pack_bf2(v[2], v[3]), ks_pack_bf2(v[4], v[5]), ks_pack_bf2(v[6], v[7]));
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

// A thread's vectors of a slice, all requested at once; behind its end the last one again (one: there is at least that)
__device__ __forceinline__ void ds_hold(const void *row, int64_t v0, int64_t v1, uint4 (&held)[DS_HELD]) {
#pragma unroll
    for (int i = 0; i < DS_HELD; ++i) {
        const int64_t at = v0 + i * DS_NT + threadIdx.x;
        held[i] = ((const uint4 *)row)[at < v1 ? at : v1 - 1];
    }
}

// past the caches: nobody here reads a gradient
__device__ __forceinline__ void ds_stream(void *p, uint4 v) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, (u32x4 *)p);
}

// (largest, sum of 2^(l (z - largest))): NaN and +infinity stay visible, -infinity adds nothing
__device__ __forceinline__ void ds_join(float &m, float &s, float m2, float s2, float l) {
    const float top = fmaxf(m, m2), base = top > -INFINITY ? top : 0.f;
    s = s * __builtin_amdgcn_exp2f(l * (m - base)) + s2 * __builtin_amdgcn_exp2f(l * (m2 - base));
    m = top;
}

struct DsTeacher { // of a row: q_k = exp((t - top) / T) / sum, fp32 powers and their sum in fp64; none: sum == 0
    float top;
    double sum;
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
__device__ __forceinline__ double ds_block_sum(double v, double *sh) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
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
__device__ __forceinline__ DsTeacher ds_teacher(const DsArgs &a, int row, int32_t *s_id, float *s_q, float *sh, double *shd) {
    float top = -INFINITY;
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        int id = a.t_ids[(int64_t)row * a.K + k];
        if (id >= a.C) {
            ks_flag(a.dev_status, KS_DEV_BAD_LABEL);
            id = -1;
        }
        const float t = id >= 0 ? ds_t_logit(a, (int64_t)row * a.K + k) : -INFINITY;
        s_id[k] = id;
        s_q[k] = t;
        top = fmaxf(top, t);
    }
    top = ds_block_max(top, sh);
    double sum = 0.0;
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        const float t = s_q[k], q = t == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(a.l * (t - top));
        s_q[k] = q;
        sum += (double)q;
    }
    return DsTeacher{top, ds_block_sum(sum, shd)};
}

// First pass: every slice's largest logit and sum of powers; the first slice also the row's A.  1,024 x 390,625 bf16 144 us: HBM at 5.5 TB/s.
template <typename T>
__global__ void __launch_bounds__(DS_NT)
ds_stats_kernel(DsArgs a) {
    extern __shared__ int32_t s_id[];
    float *const s_q = (float *)(s_id + a.K);
    __shared__ float sh[4];
    __shared__ double shd[4];
    const int row = a.row0 + blockIdx.y;
    const T *const z = (const T *)a.logits + (int64_t)row * a.ldl;
    const DsSlice<T, true> sl(a, z, blockIdx.x);
    typedef DsVec<T> V;
    constexpr int N = V::N;
    float m = -INFINITY, s = 0.f;
    if (sl.v0 < sl.v1) {
        uint4 held[DS_HELD];
        ds_hold(z + sl.head, sl.v0, sl.v1, held);
#pragma unroll
        for (int i = 0; i < DS_HELD; ++i) { // a vector that is there twice changes no maximum
            float v[N];
            V::values(held[i], v);
#pragma unroll
            for (int j = 0; j < N; ++j) m = fmaxf(m, v[j]);
        }
        const float base = m > -INFINITY ? m : 0.f;
#pragma unroll
        for (int i = 0; i < DS_HELD; ++i) {
            if (sl.v0 + i * DS_NT + threadIdx.x >= sl.v1) break;
            float v[N];
            asm volatile("" : "+v"(held[i].x), "+v"(held[i].y), "+v"(held[i].z), "+v"(held[i].w)); // unpacked anew: half the registers
            V::values(held[i], v);
#pragma unroll
            for (int j = 0; j < N; ++j) s += __builtin_amdgcn_exp2f(a.l * (v[j] - base));
        }
        if (s == 0.f) m = -INFINITY; // none of them was its own
    }
    sl.singles(a, blockIdx.x, [&](int64_t c) __attribute__((always_inline)) {
        ds_join(m, s, V::one(z + c), 1.f, a.l);
    });
    const float top = ds_block_max(m, sh), base = top > -INFINITY ? top : 0.f;
    s = ds_block_sum(s * (m == base ? 1.f : __builtin_amdgcn_exp2f(a.l * (m - base))), sh);
    if (threadIdx.x == 0) a.part[(int64_t)row * a.parts + blockIdx.x] = make_float2(top, s);
    if (blockIdx.x) return;
    const DsTeacher t = ds_teacher(a, row, s_id, s_q, sh, shd);
    if (threadIdx.x == 0) a.t[row] = make_float2(t.top, (float)t.sum);
    double sum = 0.0;
    const double inv_T = 1.0 / (double)a.T, log_sum = log(t.sum);
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        const float q = s_q[k];
        if (s_id[k] >= 0 && q != 0.f) {
            const double log_q = ((double)ds_t_logit(a, (int64_t)row * a.K + k) - (double)t.top) * inv_T - log_sum;
            sum += (double)q / t.sum * (log_q - (double)V::one(z + s_id[k]) * inv_T);
        }
    }
    sum = ds_block_sum(sum, shd);
    if (threadIdx.x == 0) a.a[row] = sum;
}

__device__ __forceinline__ uint32_t ds_pad(int K) { return (uint32_t)(K + 3) & ~3u; }
// Second pass: the gradient of every slice, the first one also the row's loss.  What it has to look up is requested together with the slice's
// logits, which stay in registers: every vector (of single elements: as many as make 2,048 parts) has a chain of the classes that the teacher
// names in it, mostly none.  1,024 x 390,625 bf16, K = 128: 290 us, HBM at 5.5 TB/s (351 with the chain looked up before the logits are requested and
// the named classes stored over the others); the logits of rows in groups of 48 to 200 MB come from the last cache no faster.
template <typename T, bool VEC>
__global__ void __launch_bounds__(DS_NT)
ds_grad_kernel(DsArgs a) {
    extern __shared__ __attribute__((aligned(16))) int32_t s_id[]; // [K, up to a multiple of 4], -1: empty
    float *const s_q = (float *)(s_id + ds_pad(a.K)), *const s_sum = s_q + a.K;
    uint16_t *const s_next = (uint16_t *)(s_sum + a.K); // chains of entries + 1; only a class's first entry is in one, s_sum: what all of them come to
    __shared__ uint32_t s_chain[DS_PARTS + 1];          // the last: of the row's first and last elements, which are in no vector
    typedef DsVec<T> V;
    constexpr int N = DsSlice<T, VEC>::N, PART = V::N; // of single elements in a chain
    const int row = a.row0 + blockIdx.y, lane = threadIdx.x & 63;
    const T *const z = (const T *)a.logits + (int64_t)row * a.ldl;
    T *const out = (T *)a.out + (int64_t)row * a.ldd;
    const DsSlice<T, VEC> sl(a, z, blockIdx.x);
    uint4 held[DS_HELD];
    if (VEC && sl.v0 < sl.v1) ds_hold(z + sl.head, sl.v0, sl.v1, held);
    const float2 t = a.t[row];
    const bool some = t.y != 0.f;
    for (int i = threadIdx.x; i <= DS_PARTS; i += DS_NT) s_chain[i] = 0;
    for (int k = threadIdx.x; k < (int)ds_pad(a.K); k += DS_NT) {
        const int id = k < a.K ? a.t_ids[(int64_t)row * a.K + k] : -1;
        const float l = k < a.K ? ds_t_logit(a, (int64_t)row * a.K + k) : -INFINITY;
        const bool there = id >= 0 && id < a.C;
        s_id[k] = there ? id : -1;
        if (k < a.K) s_q[k] = !there || l == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(a.l * (l - t.x));
    }
    // the row's largest logit and sum, in every wavefront in the same order
    float m = -INFINITY, s = 0.f;
    for (int i = lane; i < a.parts; i += 64) {
        const float2 p = a.part[(int64_t)row * a.parts + i];
        ds_join(m, s, p.x, p.y, a.l);
    }
    const float top = ks_wave_max(m), base = top > -INFINITY ? top : 0.f;
    s = ks_wave_sum(s * (m == base ? 1.f : __builtin_amdgcn_exp2f(a.l * (m - base))));
    // p = 2^(l (z - base)) * f; a row without a class has p = 0, one with a NaN or +infinity NaN
    const float f = !some || s == 0.f ? 0.f : top < INFINITY ? a.g / s : __int_as_float(0x7FC00000), to_q = some ? a.g / t.y : 0.f;
    const auto grad = [&](float v) __attribute__((always_inline)) { return f == 0.f ? 0.f : __builtin_amdgcn_exp2f(a.l * (v - base)) * f; };
    __syncthreads();
    const int64_t from = sl.head + sl.v0 * N; // of the first vector
    for (int k = threadIdx.x; k < a.K; k += DS_NT) {
        const int id = s_id[k];
        if (id < sl.first || id >= sl.last) continue;
        float q = 0.f;
        int before = k;
#pragma unroll 4
        for (int j = 0; j < a.K; j += 4) {
            const int4 other = *(const int4 *)(s_id + j);
            if (other.x == id) { q += s_q[j]; before = j < before ? j : before; }
            if (other.y == id) { q += s_q[j + 1]; before = j + 1 < before ? j + 1 : before; }
            if (other.z == id) { q += s_q[j + 2]; before = j + 2 < before ? j + 2 : before; }
            if (other.w == id) { q += s_q[j + 3]; before = j + 3 < before ? j + 3 : before; }
        }
        if (before < k) continue;
        s_sum[k] = q * to_q;
        const int64_t at = (id - from) / N;
        const int part = id >= from && at < sl.v1 - sl.v0 ? (int)(VEC ? at : at / PART) : DS_PARTS;
        s_next[k] = (uint16_t)atomicExch(&s_chain[part], k + 1);
    }
    __syncthreads();
    // what the teacher takes off at N classes from c on
    const auto named = [&](uint32_t chain, int64_t c, auto &v) __attribute__((always_inline)) {
        constexpr int M = sizeof(v) / sizeof(v[0]);
        while (chain) {
            const int64_t at = s_id[chain - 1] - c;
            const float q = s_sum[chain - 1];
#pragma unroll
            for (int j = 0; j < M; ++j) v[j] -= at == j ? q : 0.f;
            chain = s_next[chain - 1];
        }
    };
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < DS_HELD; ++i) {
            const int at = i * DS_NT + threadIdx.x;
            if (sl.v0 + at >= sl.v1) break;
            float v[N];
            V::values(held[i], v);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = grad(v[j]);
            named(s_chain[at], from + (int64_t)at * N, v);
            ds_stream(out + from + (int64_t)at * N, V::packed(v));
        }
    } else
        for (int at = threadIdx.x; sl.v0 + at < sl.v1; at += DS_NT) {
            float v[1] = {grad(V::one(z + sl.v0 + at))};
            named(s_chain[at / PART], sl.v0 + at, v);
            V::put(out + sl.v0 + at, v[0]);
        }
    sl.singles(a, blockIdx.x, [&](int64_t c) __attribute__((always_inline)) {
        float v[1] = {grad(V::one(z + c))};
        named(s_chain[DS_PARTS], c, v);
        V::put(out + c, v[0]);
    });
    if (blockIdx.x == 0 && threadIdx.x == 0)
        a.loss[row] = some ? (float)((double)a.T * (double)a.T * (a.a[row] + (s == 0.f ? 0.0 : (double)base / (double)a.T + log((double)s)))) : 0.f;
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

#define DS_SLICE_BYTES (DS_NT * DS_HELD * 16)
static int ds_slices(int64_t C) { return (int)ks_ceil_div(C, DS_SLICE_BYTES / 4); } // for the smaller slices of fp32

extern "C" size_t class_distill_workspace(int64_t C, int B, int K) {
    if (C < 1 || C >= (int64_t)1 << 31 || B < 1 || K < 1 || K > KS_MAX_DISTILL_K) return 0;
    KsArena ws(nullptr);
    ws.take<float2>((size_t)B * ds_slices(C));
    ws.take<double>((size_t)B);
    ws.take<float2>((size_t)B);
    return ws.off;
}

extern "C" int class_distill_fwd_bwd(const void *logits, int64_t ldl, int dtype, int64_t C, int B, const int32_t *t_ids, const void *t_logits,
                                     int t_dtype, int K, float temperature, float grad_scale, float *loss_per_sample, float *loss_mean,
                                     void *dlogits, int64_t ldd, void *ws, size_t ws_bytes, int32_t *dev_status, void *stream) {
    if (!logits || !t_ids || !t_logits || !loss_per_sample || !loss_mean || !dlogits || !ws) return KS_INVALID_ARG;
    if (C < 1 || C >= (int64_t)1 << 31 || B < 1 || K < 1 || ldl < C || ldd < C || (dlogits == logits && ldd != ldl)) return KS_INVALID_ARG;
    if ((dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) || (t_dtype != KS_DTYPE_BF16 && t_dtype != KS_DTYPE_FP32)) return KS_INVALID_ARG;
    if (!(temperature >= 1e-30f && temperature <= 1e30f)) return KS_INVALID_ARG; // log2(e) / T is an ordinary fp32 number
    const int size = dtype == KS_DTYPE_FP32 ? 4 : 2;
    if (((uintptr_t)logits | (uintptr_t)dlogits) % size || (uintptr_t)t_logits % (t_dtype == KS_DTYPE_FP32 ? 4 : 2) || (uintptr_t)ws % 256) return KS_INVALID_ARG;
    if (((uintptr_t)t_ids | (uintptr_t)loss_per_sample | (uintptr_t)loss_mean | (uintptr_t)dev_status) % 4) return KS_INVALID_ARG;
    if (K > KS_MAX_DISTILL_K) return KS_UNSUPPORTED;
    if (ws_bytes < class_distill_workspace(C, B, K)) return KS_WORKSPACE_TOO_SMALL;
    DsArgs a;
    KsArena arena(ws);
    a.part = arena.take<float2>((size_t)B * ds_slices(C));
    a.a = arena.take<double>((size_t)B);
    a.t = arena.take<float2>((size_t)B);
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
            hipLaunchKernelGGL(grad, dim3((unsigned)a.slices, rows), dim3(DS_NT), (size_t)K * 14 + 16, st, a);
        };
        if (dtype == KS_DTYPE_FP32) go(ds_stats_kernel<float>, vec ? ds_grad_kernel<float, true> : ds_grad_kernel<float, false>);
        else go(ds_stats_kernel<uint16_t>, vec ? ds_grad_kernel<uint16_t, true> : ds_grad_kernel<uint16_t, false>);
    }
    hipLaunchKernelGGL(ds_mean_kernel, dim3(1), dim3(DS_NT), 0, st, loss_per_sample, B, loss_mean);
    KS_LAUNCH_CHECK();
    return KS_OK;
}
