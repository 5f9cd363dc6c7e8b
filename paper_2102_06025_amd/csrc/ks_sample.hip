// Drawing one class per request from its row of the logits (paper Section 3.2: the softmax over the classes): temperature, top-k, top-p and
// min-p, by given random numbers.
//
// The first launch reads the logits once, all compute units sharing the rows: the largest logit of every segment of 512 classes, and where it
// is needed the segment's weight.  The second has a workgroup per row, which learns from the segments which of them can hold a kept class
// and reads only those: with k classes to keep, the segments down to the k-th largest of their maxima hold them all; with a share p of
// the weight, segments that hold less than that do not.  A flat distribution, of which most is kept, leaves all segments: the same
// steps over the whole row.
#include "../../include/class_sample.h"
#include "ks_common.h"

#define SP_NT 1024
#define SP_WAVES (SP_NT / 64)
#define SP_CHUNK 512     /* classes that a wavefront takes at a time: eight consecutive ones a lane */
#define SP_SEGS 4096     /* most segments of a row */
#define SP_BINS 2048     /* of the weights: 32 to a factor of two */
#define SP_PER_BINADE 32
#define SP_CAND 4096     /* classes of one bin that are put in order in LDS */
#define SP_NO_BIN (1 << 20)
#define SP_PER (SP_SEGS / SP_NT) /* most segments of a thread */

// of one type: min() and max() of the runtime's headers go through double for 64-bit numbers
template <typename T> static __device__ __forceinline__ T sp_min(T a, T b) { return b < a ? b : a; }
template <typename T> static __device__ __forceinline__ T sp_max(T a, T b) { return a < b ? b : a; }

struct SpArgs {
    const void *logits;
    int64_t ldl, C, seg; // classes of a segment, a multiple of SP_CHUNK
    int nseg, bits, row0;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    float *seg_max;  // [B, nseg]
    double *seg_sum; // [B, nseg]: sum of exp((z - seg_max) / T)
    int32_t *ids;
    float *logprob;
};

// what a row asks for
struct SpRule {
    double c;            // weight of z: 2^(c (z - z_max))
    int64_t k;           // 0: all
    double p;
    float m;
    bool greedy, use_k, use_p, use_m, sums; // sums: the segments' weights are needed
    __device__ __forceinline__ SpRule(const SpArgs &a, int row) {
        const float t = a.temperature ? a.temperature[row] : 1.f;
        greedy = !(t > 0.f);
        c = greedy ? 0.0 : 1.4426950408889634 / (double)t;
        k = a.top_k ? a.top_k[row] : 0;
        const float pp = a.top_p ? a.top_p[row] : 1.f, mm = a.min_p ? a.min_p[row] : 0.f;
        p = fmaxf(pp, 0.f);
        use_k = k > 0 && k < a.C;
        use_p = pp < 1.f;
        use_m = mm > 0.f;
        m = fminf(mm, 1.f);
        sums = !greedy && !use_k && (use_p || !use_m);
    }
};

// 2^t for t >= -200, by 2^rint(t) and the series of exp around 0: the first term left out is less than 1e-17
__device__ __forceinline__ double sp_exp2(double t) {
    const double n = rint(t), x = (t - n) * 0.6931471805599453;
    double s = 1.0 / 6227020800.0;
    s = __builtin_fma(s, x, 1.0 / 479001600.0);
    s = __builtin_fma(s, x, 1.0 / 39916800.0);
    s = __builtin_fma(s, x, 1.0 / 3628800.0);
    s = __builtin_fma(s, x, 1.0 / 362880.0);
    s = __builtin_fma(s, x, 1.0 / 40320.0);
    s = __builtin_fma(s, x, 1.0 / 5040.0);
    s = __builtin_fma(s, x, 1.0 / 720.0);
    s = __builtin_fma(s, x, 1.0 / 120.0);
    s = __builtin_fma(s, x, 1.0 / 24.0);
    s = __builtin_fma(s, x, 1.0 / 6.0);
    s = __builtin_fma(s, x, 0.5);
    s = __builtin_fma(s, x, 1.0);
    s = __builtin_fma(s, x, 1.0);
    return __hiloint2double(__double2hiint(s) + ((int)n << 20), __double2loint(s));
}
// log2 of the weight of z relative to that of ref, -200 for less: infinities of either sign, and 0 times them, end there
__device__ __forceinline__ double sp_log2w(float z, float ref, double c) {
    return z == ref ? 0.0 : fmax(((double)z - (double)ref) * c, -200.0);
}
// weight as a whole number of 2^-bits: less than 2^49, rounded by the addition of 2^52
__device__ __forceinline__ uint64_t sp_weight(float z, float top, double c, int bits) {
    const double w = sp_exp2(sp_log2w(z, top, c) + bits) + 4503599627370496.0;
    return (uint64_t)__double_as_longlong(w) & 0xFFFFFFFFFFFFFull;
}
// number of a weight's bin, which grows as z falls: the fp32 operations keep the order of the z
__device__ __forceinline__ int sp_bin(float z, float top, float c32) {
    if (z == top) return 0;
    if (!(z > -INFINITY)) return SP_NO_BIN;
    return (int)fminf((top - z) * c32, (float)SP_NO_BIN);
}
// place in the order as one number, lower first: z falling, then id rising
__device__ __forceinline__ uint64_t sp_place(float z, uint32_t id) {
    const uint32_t b = __float_as_uint(z), up = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (uint64_t)~up << 32 | id;
}
__device__ __forceinline__ float sp_place_z(uint64_t place) {
    const uint32_t up = ~(uint32_t)(place >> 32);
    return __uint_as_float(up & 0x80000000u ? up ^ 0x80000000u : ~up);
}

// eight consecutive logits from class e on; -infinity beyond C and for NaN, no negative 0
__device__ __forceinline__ void sp_load(const float *row, bool vec, int64_t e, int64_t C, float (&v)[8]) {
    if (vec && e + 8 <= C) {
        const float4 a = *(const float4 *)(row + e), b = *(const float4 *)(row + e + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e + i < C ? row[e + i] : -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] == v[i] ? v[i] + 0.f : -INFINITY;
}
__device__ __forceinline__ void sp_load(const uint16_t *row, bool vec, int64_t e, int64_t C, float (&v)[8]) {
    if (vec && e + 8 <= C) {
        const uint4 a = *(const uint4 *)(row + e);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e + i < C ? ks_bf2f(row[e + i]) : -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] == v[i] ? v[i] + 0.f : -INFINITY;
}
template <typename T> __device__ __forceinline__ const T *sp_row(const SpArgs &a, int row, bool &vec) {
    const T *p = (const T *)a.logits + (int64_t)row * a.ldl;
    vec = (uintptr_t)p % 16 == 0;
    return p;
}
__device__ __forceinline__ double sp_wave_sum(double v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// A wavefront per segment.
template <typename T>
__global__ void __launch_bounds__(256)
sp_segments_kernel(SpArgs a) {
    const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = a.row0 + blockIdx.y;
    if (s >= a.nseg) return;
    const SpRule rule(a, row);
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    const int64_t first = s * a.seg, last = sp_min(first + a.seg, a.C);
    float top = -INFINITY;
    float v[8];
    for (int64_t e = first; e < last; e += SP_CHUNK) {
        sp_load(z, vec, e + lane * 8, a.C, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i]);
    }
    top = ks_wave_max(top);
    double sum = 0.0;
    if (rule.sums && top > -INFINITY)
        for (int64_t e = first; e < last; e += SP_CHUNK) {
            if (a.seg > SP_CHUNK) sp_load(z, vec, e + lane * 8, a.C, v); // else they are there
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += sp_exp2(sp_log2w(v[i], top, rule.c));
        }
    sum = sp_wave_sum(sum);
    if (lane == 0) {
        a.seg_max[(int64_t)row * a.nseg + s] = top;
        if (rule.sums) a.seg_sum[(int64_t)row * a.nseg + s] = sum;
    }
}

// inclusive sum over the wavefront
__device__ __forceinline__ uint64_t sp_wave_scan(uint64_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_up((unsigned long long)v, d);
        if (lane >= d) v += o;
    }
    return v;
}

struct SpShared {
    uint32_t n[SP_BINS];   // of the bins: classes (at first: segments), and their weight
    uint64_t w[SP_BINS];
    union {
        uint64_t cand[SP_CAND]; // places of the classes of one bin
        struct {
            uint32_t n[SP_BINS];
            uint64_t w[SP_BINS];
        } sub;                  // parts of a bin that has too many
    };
    uint64_t seg_w[SP_SEGS]; // kept weight of the listed segments
    int32_t list[SP_SEGS];
    uint64_t wave_w[SP_WAVES + 1], wave_v[SP_WAVES + 1];
    uint32_t wave_n[SP_WAVES + 1];
    uint64_t found_w, found_place;
    uint32_t found_n, fill;
    int found, n_list;
};

// exclusive sums over the workgroup of a weight and a number a thread, and their totals
__device__ __forceinline__ void sp_scan(SpShared &sh, uint64_t w, uint32_t n, uint64_t &w0, uint32_t &n0, uint64_t &w_all, uint32_t &n_all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t wi = sp_wave_scan(w);
    const uint32_t ni = (uint32_t)ks_wave_iscan((int)n);
    __syncthreads();
    if (lane == 63) { sh.wave_w[wave] = wi; sh.wave_n[wave] = ni; }
    __syncthreads();
    w0 = wi - w; n0 = ni - n; w_all = 0; n_all = 0;
#pragma unroll
    for (int i = 0; i < SP_WAVES; ++i) {
        if (i < wave) { w0 += sh.wave_w[i]; n0 += sh.wave_n[i]; }
        w_all += sh.wave_w[i];
        n_all += sh.wave_n[i];
    }
}
__device__ __forceinline__ float sp_block_max(SpShared &sh, float v) {
    v = ks_wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.wave_n[threadIdx.x >> 6] = __float_as_uint(v);
    __syncthreads();
    v = __uint_as_float(sh.wave_n[0]);
#pragma unroll
    for (int i = 1; i < SP_WAVES; ++i) v = fmaxf(v, __uint_as_float(sh.wave_n[i]));
    return v;
}
__device__ __forceinline__ void sp_clear(uint32_t *n, uint64_t *w) {
    __syncthreads();
    for (int i = threadIdx.x; i < SP_BINS; i += SP_NT) { n[i] = 0; w[i] = 0; }
    __syncthreads();
}
// The first bin at which the running number (by_n) or weight reaches `target` >= 1: found (-1: none does), and what lies before it;
// the totals.
__device__ __forceinline__ void sp_find(SpShared &sh, const uint32_t *n, const uint64_t *w, bool by_n, uint64_t target, uint64_t &w_all, uint32_t &n_all) {
    __syncthreads();
    if (threadIdx.x == 0) sh.found = -1;
    constexpr int EACH = SP_BINS / SP_NT;
    const int b = threadIdx.x * EACH;
    uint64_t w0, w_mine = 0;
    uint32_t n0, n_mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) { w_mine += w[b + i]; n_mine += n[b + i]; }
    sp_scan(sh, w_mine, n_mine, w0, n0, w_all, n_all);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint64_t before = by_n ? n0 : w0, size = by_n ? n[b + i] : w[b + i];
        if (before < target && target <= before + size) { sh.found = b + i; sh.found_n = n0; sh.found_w = w0; }
        n0 += n[b + i];
        w0 += w[b + i];
    }
    __syncthreads();
}

// f(z, id) for the eight classes a lane of all listed segments
template <typename T, typename F> __device__ __forceinline__ void sp_over_list(const SpArgs &a, const T *z, bool vec, const SpShared &sh, F f) {
    const int lane = threadIdx.x & 63;
    for (int i = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < sh.n_list; i += SP_WAVES) {
        const int64_t first = sh.list[i] * a.seg, last = sp_min(first + a.seg, a.C);
        for (int64_t e = first; e < last; e += SP_CHUNK) {
            float v[8];
            sp_load(z, vec, e + lane * 8, a.C, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) f(v[j], (uint32_t)(e + lane * 8 + j));
        }
    }
}

// Of the listed classes of bin `bin`, which are sh.n[bin]: the place of the one at which the running number or weight reaches `target`, in
// the order; `weight`: their weight up to it.  Too many for LDS (a bin of equal logits) are cut into parts of equal ranges of places first.
template <typename T>
__device__ uint64_t sp_refine(const SpArgs &a, const T *z, bool vec, SpShared &sh, float top, double c, float c32, int bin, bool by_n, uint64_t target,
                              uint64_t &weight) {
    uint64_t lo = 0, hi = ~0ull, before = 0;
    uint32_t n = sh.n[bin];
    while (n > SP_CAND) {
        uint64_t least = ~0ull, most = 0;
        sp_over_list(a, z, vec, sh, [&](float v, uint32_t id) __attribute__((always_inline)) {
            if (sp_bin(v, top, c32) != bin) return;
            const uint64_t place = sp_place(v, id);
            if (place < lo || place > hi) return;
            least = sp_min(least, place);
            most = sp_max(most, place);
        });
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            least = sp_min(least, (uint64_t)__shfl_xor((unsigned long long)least, d));
            most = sp_max(most, (uint64_t)__shfl_xor((unsigned long long)most, d));
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) { sh.wave_w[threadIdx.x >> 6] = least; sh.wave_v[threadIdx.x >> 6] = most; }
        __syncthreads();
        for (int i = 0; i < SP_WAVES; ++i) { least = sp_min(least, sh.wave_w[i]); most = sp_max(most, sh.wave_v[i]); }
        int shift = 0;
        while ((most - least) >> shift >= SP_BINS) ++shift;
        sp_clear(sh.sub.n, sh.sub.w);
        sp_over_list(a, z, vec, sh, [&](float v, uint32_t id) __attribute__((always_inline)) {
            if (sp_bin(v, top, c32) != bin) return;
            const uint64_t place = sp_place(v, id);
            if (place < least || place > most) return;
            const int part = (int)((place - least) >> shift);
            atomicAdd(&sh.sub.n[part], 1u);
            atomicAdd((unsigned long long *)&sh.sub.w[part], (unsigned long long)sp_weight(v, top, c, a.bits));
        });
        uint64_t w_all;
        uint32_t n_all;
        sp_find(sh, sh.sub.n, sh.sub.w, by_n, target, w_all, n_all);
        const int part = sh.found; // there is one: the target lies within the bin
        lo = least + ((uint64_t)part << shift);
        hi = sp_min(most, lo + (((uint64_t)1 << shift) - 1));
        n = sh.sub.n[part];
        target -= by_n ? sh.found_n : sh.found_w;
        before += sh.found_w;
    }
    __syncthreads();
    if (threadIdx.x == 0) { sh.fill = 0; sh.found_place = 0; sh.found_w = 0; }
    int size = 64;
    while (size < (int)n) size <<= 1;
    for (int i = n + threadIdx.x; i < size; i += SP_NT) sh.cand[i] = ~0ull;
    __syncthreads();
    sp_over_list(a, z, vec, sh, [&](float v, uint32_t id) __attribute__((always_inline)) {
        if (sp_bin(v, top, c32) != bin) return;
        const uint64_t place = sp_place(v, id);
        if (place >= lo && place <= hi) {
            const uint32_t at = atomicAdd(&sh.fill, 1u);
            if (at < n) sh.cand[at] = place;
        }
    });
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1) // bitonic sort
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int i = threadIdx.x; i < size / 2; i += SP_NT) {
                const int x = i / j * 2 * j + i % j, y = x + j;
                const uint64_t p = sh.cand[x], q = sh.cand[y];
                if ((p > q) == ((x & k) == 0)) { sh.cand[x] = q; sh.cand[y] = p; }
            }
            __syncthreads();
        }
    // SP_CAND / SP_NT consecutive candidates a thread
    constexpr int EACH = SP_CAND / SP_NT;
    uint64_t w[EACH], mine = 0, w0, w_all;
    uint32_t unused, unused_all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = threadIdx.x * EACH + i;
        w[i] = at < (int)n ? sp_weight(sp_place_z(sh.cand[at]), top, c, a.bits) : 0;
        mine += w[i];
    }
    sp_scan(sh, mine, 0, w0, unused, w_all, unused_all);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = threadIdx.x * EACH + i;
        if (at < (int)n && (by_n ? at + 1 == (int)target : w0 < target && target <= w0 + w[i])) {
            sh.found_place = sh.cand[at];
            sh.found_w = w0 + w[i];
        }
        w0 += w[i];
    }
    __syncthreads();
    weight = before + sh.found_w;
    return sh.found_place;
}

// One wavefront: of the classes of segment s that are kept, the one at which the running weight exceeds `target`; if rounding left less
// weight than that the last that is kept.  -> its id and logit
template <typename T>
__device__ void sp_pick(const SpArgs &a, const T *z, bool vec, int s, uint64_t target, float top, double c, uint64_t cut, uint64_t floor_w, int &id, float &logit) {
    const int lane = threadIdx.x & 63;
    const int64_t first = s * a.seg, last = sp_min(first + a.seg, a.C);
    id = -1;
    logit = -INFINITY;
    for (int64_t e = first; e < last; e += SP_CHUNK) {
        float v[8];
        uint64_t w[8], mine = 0;
        sp_load(z, vec, e + lane * 8, a.C, v);
        int my_last = -1;
        float my_z = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = v[i] > -INFINITY ? sp_weight(v[i], top, c, a.bits) : 0;
            const bool kept = v[i] > -INFINITY && sp_place(v[i], (uint32_t)(e + lane * 8 + i)) <= cut && w[i] >= floor_w;
            if (kept) { my_last = (int)(e + lane * 8 + i); my_z = v[i]; }
            else w[i] = 0;
            mine += w[i];
        }
        const uint64_t upto = sp_wave_scan(mine), all = __shfl((unsigned long long)upto, 63);
        const uint64_t here = __ballot(my_last >= 0);
        if (target < all) {
            uint64_t run = upto - mine;
            int got = -1;
            float got_z = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (got < 0 && run <= target && target < run + w[i]) { got = (int)(e + lane * 8 + i); got_z = v[i]; }
                run += w[i];
            }
            const uint64_t who = __ballot(got >= 0);
            const int l = __ffsll((unsigned long long)who) - 1;
            id = __shfl(got, l);
            logit = __shfl(got_z, l);
            return;
        }
        target -= all;
        if (here) {
            const int l = 63 - __clzll((long long)here);
            id = __shfl(my_last, l);
            logit = __shfl(my_z, l);
        }
    }
}

// A workgroup per row.
template <typename T>
__global__ void __launch_bounds__(SP_NT)
sp_draw_kernel(SpArgs a) {
    __shared__ SpShared sh;
    const int row = a.row0 + blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const SpRule rule(a, row);
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    const float *const seg_max = a.seg_max + (int64_t)row * a.nseg;
    const double *const seg_sum = a.seg_sum + (int64_t)row * a.nseg;
    // up to SP_PER consecutive segments a thread
    const int per = (a.nseg + SP_NT - 1) / SP_NT;
    float my_max[SP_PER];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < SP_PER; ++i) {
        const int s = threadIdx.x * per + i;
        my_max[i] = i < per && s < a.nseg ? seg_max[s] : -INFINITY;
        top = fmaxf(top, my_max[i]);
    }
    top = sp_block_max(sh, top);
    if (!(top > -INFINITY)) {
        if (threadIdx.x == 0) {
            a.ids[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        return;
    }
    const double c = rule.c;
    const float c32 = (float)(c * SP_PER_BINADE);
    const int limit = (a.bits + 1) * SP_PER_BINADE; // from this bin on weights are 0
    const auto seg_mass = [&](int i) __attribute__((always_inline)) -> uint64_t {
        const int s = threadIdx.x * per + i;
        return my_max[i] > -INFINITY ? (uint64_t)(seg_sum[s] * sp_exp2(sp_log2w(my_max[i], top, c) + a.bits) + 0.5) : 0;
    };

    uint64_t cut = ~0ull, floor_w = 0, all_w = 0;
    uint32_t unused_n, unused_all;
    uint64_t my_w[SP_PER] = {}, w0;
    const bool plain = !rule.greedy && !rule.use_k && !rule.use_p && !rule.use_m;
    if (rule.greedy) { // the first class with the largest logit: the only one that is kept
        if (threadIdx.x == 0) { sh.fill = 0x7FFFFFFF; sh.n_list = 1; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SP_PER; ++i)
            if (my_max[i] == top) atomicMin(&sh.fill, (uint32_t)(threadIdx.x * per + i));
        __syncthreads();
        if (wave == 0) {
            const int64_t first = (int64_t)sh.fill * a.seg, last = sp_min(first + a.seg, a.C);
            for (int64_t e = first; e < last; e += SP_CHUNK) {
                float v[8];
                sp_load(z, vec, e + lane * 8, a.C, v);
                int got = -1;
#pragma unroll
                for (int i = 7; i >= 0; --i)
                    if (v[i] == top) got = (int)(e + lane * 8 + i);
                const uint64_t who = __ballot(got >= 0);
                if (who) {
                    const int id = __shfl(got, __ffsll((unsigned long long)who) - 1);
                    if (lane == 0) {
                        a.ids[row] = id;
                        if (a.logprob) a.logprob[row] = 0.f;
                    }
                    break;
                }
            }
        }
        return;
    }
    if (plain) { // all classes: the segments' weights say where to look
#pragma unroll
        for (int i = 0; i < SP_PER; ++i) my_w[i] = seg_mass(i);
    } else {
        // 1  down to which bin segments and classes have to be looked at
        const int bin_m = rule.use_m ? (int)fminf(-log2f(rule.m) * SP_PER_BINADE + 2.f, (float)(limit - 1)) : limit - 1;
        int b0 = bin_m;
        uint64_t target_p = 0;
        if (rule.use_k || rule.use_p) {
            sp_clear(sh.n, sh.w);
            uint64_t mine = 0;
#pragma unroll
            for (int i = 0; i < SP_PER; ++i) {
                const int b = sp_bin(my_max[i], top, c32);
                if (b >= limit) continue;
                atomicAdd(&sh.n[b], 1u);
                if (!rule.use_k) {
                    const uint64_t w = seg_mass(i);
                    mine += w;
                    atomicAdd((unsigned long long *)&sh.w[b], (unsigned long long)w);
                }
            }
            uint64_t w_all;
            uint32_t n_all;
            if (!rule.use_k) {
                sp_scan(sh, mine, 0, w0, unused_n, w_all, unused_all);
                target_p = sp_max((uint64_t)ceil(rule.p * (double)w_all), (uint64_t)1);
            }
            sp_find(sh, sh.n, sh.w, rule.use_k, rule.use_k ? (uint64_t)rule.k : target_p, w_all, n_all);
            const int found = sh.found < 0 ? limit - 1 : sh.found;
            b0 = rule.use_k ? (rule.use_p ? found : sp_min(found, bin_m)) : sp_min(found + SP_PER_BINADE, bin_m);
        }
        // 2  numbers and weights of the bins down to there; more of them while a share of the weight is not reached
        uint64_t w_all;
        uint32_t n_all;
        for (;;) {
            int mine = 0;
            bool in[SP_PER];
#pragma unroll
            for (int i = 0; i < SP_PER; ++i) {
                in[i] = sp_bin(my_max[i], top, c32) <= b0;
                mine += in[i];
            }
            uint32_t at, n_list;
            sp_scan(sh, 0, (uint32_t)mine, w0, at, w_all, n_list);
#pragma unroll
            for (int i = 0; i < SP_PER; ++i)
                if (in[i]) sh.list[at++] = threadIdx.x * per + i;
            if (threadIdx.x == 0) sh.n_list = (int)n_list;
            sp_clear(sh.n, sh.w);
            if (!rule.use_k && !rule.use_p) break; // min-p alone
            sp_over_list(a, z, vec, sh, [&](float v, uint32_t) __attribute__((always_inline)) {
                const int b = sp_bin(v, top, c32);
                if (b > b0) return;
                atomicAdd(&sh.n[b], 1u);
                atomicAdd((unsigned long long *)&sh.w[b], (unsigned long long)sp_weight(v, top, c, a.bits));
            });
            if (rule.use_k) break;
            sp_find(sh, sh.n, sh.w, false, target_p, w_all, n_all);
            if (sh.found >= 0 || b0 >= bin_m) break;
            b0 = (int)n_list * 2 > a.nseg ? bin_m : sp_min(b0 + 2 * SP_PER_BINADE, bin_m);
        }
        // 3  the last class that top-k, then top-p keeps
        if (rule.use_k) {
            sp_find(sh, sh.n, sh.w, true, (uint64_t)rule.k, w_all, n_all);
            if (sh.found >= 0) {
                const uint64_t before = sh.found_w;
                uint64_t w;
                cut = sp_refine(a, z, vec, sh, top, c, c32, sh.found, true, (uint64_t)rule.k - sh.found_n, w);
                w_all = before + w;
            }
            target_p = sp_max((uint64_t)ceil(rule.p * (double)w_all), (uint64_t)1);
        }
        if (rule.use_p) {
            uint64_t all;
            sp_find(sh, sh.n, sh.w, false, target_p, all, n_all);
            if (sh.found >= 0) {
                uint64_t w;
                cut = sp_min(cut, sp_refine(a, z, vec, sh, top, c, c32, sh.found, false, target_p - sh.found_w, w));
            }
        }
        if (rule.use_m) floor_w = sp_max((uint64_t)ceil((double)rule.m * (double)(1ull << a.bits)), (uint64_t)1);
        // 4  what is kept of each listed segment
        __syncthreads();
        for (int i = wave; i < sh.n_list; i += SP_WAVES) {
            const int64_t first = sh.list[i] * a.seg, last = sp_min(first + a.seg, a.C);
            uint64_t sum = 0;
            for (int64_t e = first; e < last; e += SP_CHUNK) {
                float v[8];
                sp_load(z, vec, e + lane * 8, a.C, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (sp_bin(v[j], top, c32) > b0 || sp_place(v[j], (uint32_t)(e + lane * 8 + j)) > cut) continue;
                    const uint64_t w = sp_weight(v[j], top, c, a.bits);
                    if (w >= floor_w) sum += w;
                }
            }
            sum = sp_wave_scan(sum);
            if (lane == 63) sh.seg_w[i] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SP_PER; ++i)
            if (threadIdx.x * SP_PER + i < sh.n_list) my_w[i] = sh.seg_w[threadIdx.x * SP_PER + i];
    }
    // the segment, then the class, at which the running weight exceeds u times all of it
    uint64_t mine = 0;
#pragma unroll
    for (int i = 0; i < SP_PER; ++i) mine += my_w[i];
    sp_scan(sh, mine, 0, w0, unused_n, all_w, unused_all);
    const double share = fmax((double)a.u[row], 0.0) * (double)all_w;
    const uint64_t target = share >= (double)all_w ? all_w - 1 : sp_min((uint64_t)share, all_w - 1);
#pragma unroll
    for (int i = 0; i < SP_PER; ++i) {
        if (w0 <= target && target < w0 + my_w[i]) {
            sh.found = plain ? threadIdx.x * per + i : sh.list[threadIdx.x * SP_PER + i];
            sh.found_w = target - w0;
        }
        w0 += my_w[i];
    }
    __syncthreads();
    if (wave == 0) {
        int id;
        float logit;
        sp_pick(a, z, vec, sh.found, sh.found_w, top, c, cut, floor_w, id, logit);
        if (lane == 0) {
            a.ids[row] = id;
            if (a.logprob) // log of 2^(c (z - top)) / (all_w 2^-bits)
                a.logprob[row] = (float)((sp_log2w(logit, top, c) - (log2((double)all_w) - a.bits)) * 0.6931471805599453);
        }
    }
}

static bool sp_sizes(int64_t C, int B, int64_t &seg, int &nseg, int &bits) {
    if (C < 1 || C >= (int64_t)1 << 31 || B < 1) return false;
    seg = SP_CHUNK;
    while (ks_ceil_div(C, seg) > SP_SEGS) seg *= 2;
    nseg = (int)ks_ceil_div(C, seg);
    int lg = 0;
    while (((int64_t)1 << lg) < C) ++lg;
    bits = 62 - lg < 48 ? 62 - lg : 48;
    return true;
}

extern "C" size_t class_sample_workspace(int64_t C, int B) {
    int64_t seg;
    int nseg, bits;
    if (!sp_sizes(C, B, seg, nseg, bits)) return 0;
    KsArena ws(nullptr);
    ws.take<float>((size_t)B * nseg);
    ws.take<double>((size_t)B * nseg);
    return ws.off;
}

extern "C" int class_sample(const void *logits, int64_t ldl, int dtype, int64_t C, int B, const float *u, const float *temperature,
                            const int32_t *top_k, const float *top_p, const float *min_p, int32_t *ids, float *logprob, void *ws,
                            size_t ws_bytes, void *stream) {
    SpArgs a;
    if (!logits || !u || !ids || !ws || ldl < C || !sp_sizes(C, B, a.seg, a.nseg, a.bits)) return KS_INVALID_ARG;
    if (dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) return KS_INVALID_ARG;
    if ((uintptr_t)logits % (dtype == KS_DTYPE_FP32 ? 4 : 2) || (uintptr_t)ws % 256) return KS_INVALID_ARG;
    if (((uintptr_t)u | (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)ids | (uintptr_t)logprob) % 4) return KS_INVALID_ARG;
    if (ws_bytes < class_sample_workspace(C, B)) return KS_WORKSPACE_TOO_SMALL;
    KsArena arena(ws);
    a.seg_max = arena.take<float>((size_t)B * a.nseg);
    a.seg_sum = arena.take<double>((size_t)B * a.nseg);
    a.logits = logits; a.ldl = ldl; a.C = C;
    a.u = u; a.temperature = temperature; a.top_p = top_p; a.min_p = min_p; a.top_k = top_k;
    a.ids = ids; a.logprob = logprob;
    for (int64_t r = 0; r < B; r += 1 << 15) { // a launch's second dimension ends at 65,535
        const unsigned rows = (unsigned)(B - r < 1 << 15 ? B - r : 1 << 15);
        a.row0 = (int)r;
        const dim3 grid((unsigned)((a.nseg + 3) / 4), rows);
        if (dtype == KS_DTYPE_FP32) {
            hipLaunchKernelGGL(sp_segments_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, a);
            hipLaunchKernelGGL(sp_draw_kernel<float>, dim3(rows), dim3(SP_NT), 0, (hipStream_t)stream, a);
        } else {
            hipLaunchKernelGGL(sp_segments_kernel<uint16_t>, grid, dim3(256), 0, (hipStream_t)stream, a);
            hipLaunchKernelGGL(sp_draw_kernel<uint16_t>, dim3(rows), dim3(SP_NT), 0, (hipStream_t)stream, a);
        }
    }
    KS_LAUNCH_CHECK();
    return KS_OK;
}
