// Drawing one class per request from its row of the logits (paper Section 3.2: the softmax over the classes): temperature, top-k, top-p and
// min-p, by given random numbers.
//
// The first launch reads the logits once, all compute units sharing the rows: the largest logit of every granule of 8 to 512 classes (at most
// 4,096 granules a row), and where it is needed the granule's weight.  The second has a workgroup per row, which learns from the granules
// which of them can hold a kept class and reads only those: with k classes to keep, the granules down to the k-th largest of their maxima
// hold them all; with a share p of the weight, granules that hold less than that do not.  What may be kept is put in order in LDS.  Rows of
// which more is kept than LDS holds (a flat distribution) are left to a third launch.
#include "../../include/class_sample.h"
#include "ks_common.h"

#define SP_NT 512  /* threads of a row: with 256 1 x 10,000 fp32, k = 50 takes 2 us less, 256 x 390,625 bf16, k = 500 20 more */
#define SP_NT2 1024 /* where much is kept */
#define SP_CHUNK 512     /* classes that a wavefront takes at a time: eight consecutive ones a lane */
#define SP_GRANULES 4096 /* most granules of a row */
#define SP_BINS 2048     /* of the weights: 32 to a factor of two */
#define SP_PER_BINADE 32
#define SP_CAND 4096     /* classes that are put in order in LDS */
#define SP_NO_BIN (1 << 20)

// of one type: min() and max() of the runtime's headers go through double for 64-bit numbers
template <typename T> static __device__ __forceinline__ T sp_min(T a, T b) { return b < a ? b : a; }
template <typename T> static __device__ __forceinline__ T sp_max(T a, T b) { return a < b ? b : a; }

struct SpRow;
struct SpArgs {
    const void *logits;
    int64_t ldl, C, gran; // classes of a granule: 8 << lg, beyond 512 a multiple of that
    int lg, gshift, ngr, bits, row0; // gran = 1 << gshift
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    float *g_max;  // [B, ngr]
    double *g_sum; // [B, ngr]: sum of exp((z - g_max) / T)
    int32_t *many; // [B]: the row is left to the third launch
    int64_t most;  // classes that a row's workgroup looks at itself
    int64_t span;  // classes of a workgroup that counts
    // where all compute units share such a row:
    SpRow *rows;        // [B], NULL: they do not
    float *row_top;     // [B]
    uint32_t *bins_n;   // [B, SP_BINS]: classes, and their weight
    uint64_t *bins_w;
    uint64_t *pool, *pool_used, pool_size; // places of classes of the bins in which top-k and top-p end, of all rows
    int32_t *ids;
    float *logprob;
};

// a row that all compute units share
struct SpRow {
    int b0, bin_k, p_first, p_last, sure; // bins: the last to look at; of top-k (-1: none); of top-p; those before `sure` are kept (but for min-p)
    uint32_t k_rest, n_cand, fill, done;
    uint64_t target_p, w_all, before_k, before_p; // weight of all (or up to bin_k: before_k), before p_first
    uint64_t cand0;                               // of its candidates in the pool
};
// what a row asks for
struct SpRule {
    double c;            // weight of z: 2^(c (z - z_max))
    int64_t k;           // 0: all
    double p;
    float m;
    bool greedy, use_k, use_p, use_m, sums; // sums: the granules' weights are needed
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

// 2^t for -200 <= t < 900: the addition of 1.5 * 2^52 leaves the nearest whole number in the low bits; of the rest (at most a half) the series
// of 2^f = exp(f ln 2), whose first term left out is less than 1e-17
#define SP_LN2 0.69314718055994530942
static constexpr double sp_term(int k) { return k == 0 ? 1.0 : sp_term(k - 1) * SP_LN2 / k; }
__device__ __forceinline__ double sp_exp2(double t) {
    const double whole = t + 6755399441055744.0, f = t - (whole - 6755399441055744.0);
    constexpr double c1 = sp_term(1), c2 = sp_term(2), c3 = sp_term(3), c4 = sp_term(4), c5 = sp_term(5), c6 = sp_term(6), c7 = sp_term(7),
                     c8 = sp_term(8), c9 = sp_term(9), c10 = sp_term(10), c11 = sp_term(11), c12 = sp_term(12), c13 = sp_term(13);
    double s = c13;
    s = __builtin_fma(s, f, c12);
    s = __builtin_fma(s, f, c11);
    s = __builtin_fma(s, f, c10);
    s = __builtin_fma(s, f, c9);
    s = __builtin_fma(s, f, c8);
    s = __builtin_fma(s, f, c7);
    s = __builtin_fma(s, f, c6);
    s = __builtin_fma(s, f, c5);
    s = __builtin_fma(s, f, c4);
    s = __builtin_fma(s, f, c3);
    s = __builtin_fma(s, f, c2);
    s = __builtin_fma(s, f, c1);
    s = __builtin_fma(s, f, 1.0);
    return __hiloint2double(__double2hiint(s) + (__double2loint(whole) << 20), __double2loint(s));
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
// Number of a weight's bin, which grows as z falls: the fp32 operations keep the order of the z.  A difference beyond fp32 (which weighs
// something at a temperature of 1e37 or more) and a c32 beyond it end at its largest number: a bin that is too low has its class looked at,
// and the class's weight decides.
#define SP_MOST 3.402823466e38f
__device__ __forceinline__ int sp_bin(float z, float top, float c32) {
    if (z == top) return 0;
    if (!(z > -INFINITY)) return SP_NO_BIN;
    return (int)fminf(fminf(top - z, SP_MOST) * c32, (float)SP_NO_BIN);
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
// op over groups of 2^LG lanes, in all of them
template <int CTRL> __device__ __forceinline__ float sp_move(float v) { return KS_DPP_F(v, v, CTRL, 0xf); }
template <int CTRL> __device__ __forceinline__ double sp_move(double v) {
    const int lo = __double2loint(v), hi = __double2hiint(v);
    return __hiloint2double(KS_DPP(hi, hi, CTRL, 0xf), KS_DPP(lo, lo, CTRL, 0xf));
}
template <int LG, typename V, typename OP> __device__ __forceinline__ V sp_lanes(V v, OP op) {
    if (LG > 0) v = op(v, sp_move<0xB1>(v));  // quad_perm [1, 0, 3, 2]
    if (LG > 1) v = op(v, sp_move<0x4E>(v));  // quad_perm [2, 3, 0, 1]
    if (LG > 2) v = op(v, sp_move<0x141>(v)); // row_half_mirror
    if (LG > 3) v = op(v, sp_move<0x140>(v)); // row_mirror
    if (LG > 4) v = op(v, (V)__shfl_xor(v, 16));
    if (LG > 5) v = op(v, (V)__shfl_xor(v, 32));
    return v;
}

// A wavefront per 512 classes, or per granule of more.  256 x 390,625 bf16: 47 to 52 us (200 MB at 3.8 to 4.3 TB/s), 72 where a third of the rows needs the
// granules' weights: fp64 powers.
template <int LG, typename T>
__global__ void __launch_bounds__(256)
sp_granules_kernel(SpArgs a) {
    const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = a.row0 + blockIdx.y;
    if (a.rows && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.pool_used = 0;
    const int64_t span = LG < 6 ? SP_CHUNK : a.gran, first = wave * span, last = sp_min(first + span, a.C);
    if (first >= a.C) return;
    const SpRule rule(a, row);
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    float top = -INFINITY;
    float v[8];
    for (int64_t e = first; e < last; e += SP_CHUNK) {
        sp_load(z, vec, e + lane * 8, a.C, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i]);
    }
    top = sp_lanes<LG>(top, [](float x, float y) __attribute__((always_inline)) { return fmaxf(x, y); });
    const int64_t g = LG < 6 ? (first >> (LG + 3)) + (lane >> LG) : wave;
    const bool writes = (lane & ((1 << LG) - 1)) == 0 && g < a.ngr;
    if (writes) a.g_max[(int64_t)row * a.ngr + g] = top;
    if (!rule.sums) return;
    double sum = 0.0;
    if (top > -INFINITY)
        for (int64_t e = first; e < last; e += SP_CHUNK) {
            if (LG == 6 && a.gran > SP_CHUNK) sp_load(z, vec, e + lane * 8, a.C, v); // else they are there
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += sp_exp2(sp_log2w(v[i], top, rule.c));
        }
    sum = sp_lanes<LG>(sum, [](double x, double y) __attribute__((always_inline)) { return x + y; });
    if (writes) a.g_sum[(int64_t)row * a.ngr + g] = sum;
}

// inclusive sum over the wavefront, as ks_wave_iscan
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t sp_moved(uint64_t v) {
    return (uint64_t)(uint32_t)KS_DPP(0, (int)(v >> 32), CTRL, ROWS) << 32 | (uint32_t)KS_DPP(0, (int)(uint32_t)v, CTRL, ROWS);
}
__device__ __forceinline__ uint64_t sp_wave_scan(uint64_t v) {
    v += sp_moved<0x111, 0xf>(v);
    v += sp_moved<0x112, 0xf>(v);
    v += sp_moved<0x114, 0xf>(v);
    v += sp_moved<0x118, 0xf>(v);
    v += sp_moved<0x142, 0xa>(v);
    v += sp_moved<0x143, 0xc>(v);
    return v;
}

struct SpScan {
    uint64_t w[16], v[16]; // of wavefronts
    uint32_t n[16];
    uint64_t found_w;
    uint32_t found_n;
    int found;
};

// exclusive sums over the workgroup of a weight and a number a thread, and their totals
template <int NT> __device__ __forceinline__ void sp_scan(SpScan &sh, uint64_t w, uint32_t n, uint64_t &w0, uint32_t &n0, uint64_t &w_all, uint32_t &n_all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t wi = sp_wave_scan(w);
    const uint32_t ni = (uint32_t)ks_wave_iscan((int)n);
    __syncthreads();
    if (lane == 63) { sh.w[wave] = wi; sh.n[wave] = ni; }
    __syncthreads();
    w0 = wi - w; n0 = ni - n; w_all = 0; n_all = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
        if (i < wave) { w0 += sh.w[i]; n0 += sh.n[i]; }
        w_all += sh.w[i];
        n_all += sh.n[i];
    }
}
template <int NT> __device__ __forceinline__ uint64_t sp_total(SpScan &sh, uint64_t w) {
    uint64_t w0, w_all;
    uint32_t n0, n_all;
    sp_scan<NT>(sh, w, 0, w0, n0, w_all, n_all);
    return w_all;
}
template <int NT> __device__ __forceinline__ float sp_block_max(SpScan &sh, float v) {
    v = ks_wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.n[threadIdx.x >> 6] = __float_as_uint(v);
    __syncthreads();
    v = __uint_as_float(sh.n[0]);
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v = fmaxf(v, __uint_as_float(sh.n[i]));
    return v;
}
template <int NT> __device__ __forceinline__ void sp_clear(uint32_t *n, uint64_t *w) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SP_BINS / NT; ++i) { n[i * NT + threadIdx.x] = 0; w[i * NT + threadIdx.x] = 0; }
    __syncthreads();
}
// The first bin at which the running number (by_n) or weight reaches `target` >= 1: found (-1: none does), and what lies before it;
// the totals.
template <int NT>
__device__ __forceinline__ void sp_find(SpScan &sh, const uint32_t *n, const uint64_t *w, bool by_n, uint64_t target, uint64_t &w_all, uint32_t &n_all) {
    __syncthreads();
    if (threadIdx.x == 0) sh.found = -1;
    constexpr int EACH = SP_BINS / NT;
    const int b = threadIdx.x * EACH;
    uint64_t w0, w_mine = 0;
    uint32_t n0, n_mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) { w_mine += w[b + i]; n_mine += n[b + i]; }
    sp_scan<NT>(sh, w_mine, n_mine, w0, n0, w_all, n_all);
    const uint64_t before = by_n ? n0 : w0, mine = by_n ? n_mine : w_mine;
    if (before < target && target <= before + mine) // one thread
        for (int i = 0;; ++i) {
            if (target <= (by_n ? n0 + n[b + i] : w0 + w[b + i])) {
                sh.found = b + i;
                sh.found_n = n0;
                sh.found_w = w0;
                break;
            }
            n0 += n[b + i];
            w0 += w[b + i];
        }
    __syncthreads();
}

// Weight of granule g of a row, whose largest logit is `z`: the rounded sum, and none where no class of it has a weight (many that are less than
// half of 2^-bits each would add up to one that belongs to nobody)
__device__ __forceinline__ uint64_t sp_mass(const SpArgs &a, int row, int g, float z, float top, double c) {
    if (!(z > -INFINITY)) return 0;
    const uint64_t most = sp_weight(z, top, c, a.bits);
    return most ? sp_max((uint64_t)(a.g_sum[(int64_t)row * a.ngr + g] * sp_exp2(sp_log2w(z, top, c) + a.bits) + 0.5), most) : 0;
}
__device__ __forceinline__ float sp_c32(const SpRule &rule) { return fminf((float)(rule.c * SP_PER_BINADE), SP_MOST); }
// from this bin on weights are 0: half of 2^-bits lies at the end of bin (bits + 1) * SP_PER_BINADE - 1, and bins are found with roundings
__device__ __forceinline__ int sp_limit(const SpArgs &a) { return (a.bits + 1) * SP_PER_BINADE + 1; }
__device__ __forceinline__ uint64_t sp_floor(const SpArgs &a, const SpRule &rule) { // least weight that is kept
    return rule.use_m ? sp_max((uint64_t)ceil((double)rule.m * (double)((uint64_t)1 << a.bits)), (uint64_t)1) : 1;
}
// last bin with weights of m or more: whole ones, which half of 2^-bits less is rounded up to
__device__ __forceinline__ int sp_bin_m(const SpArgs &a, const SpRule &rule) {
    return rule.use_m ? (int)fminf(((float)a.bits - log2f((float)sp_floor(a, rule) - 0.5f)) * SP_PER_BINADE + 2.f, (float)(sp_limit(a) - 1)) : sp_limit(a) - 1;
}
__device__ __forceinline__ uint64_t sp_share(double p, uint64_t w) { return sp_max((uint64_t)ceil(p * (double)w), (uint64_t)1); } // the weight that is p of w
__device__ __forceinline__ uint64_t sp_target(const SpArgs &a, int row, uint64_t w) { // the running weight that the drawn class exceeds: u of w
    const double share = fmax((double)a.u[row], 0.0) * (double)w;
    return share >= (double)w ? w - 1 : sp_min((uint64_t)share, w - 1);
}
__device__ __forceinline__ void sp_result(const SpArgs &a, int row, int id, float z, float top, double c, uint64_t w) {
    a.ids[row] = id;
    if (a.logprob) a.logprob[row] = (float)((sp_log2w(z, top, c) - (log2((double)w) - a.bits)) * 0.6931471805599453); // log of 2^(c (z - top)) / (w 2^-bits)
}

// One wavefront: of the classes [first, last) that are kept (weights of floor_w >= 1 or more), the one at which the running weight exceeds `target`;
// if there is less weight than that the last that is kept.  -> its id and logit
template <typename T>
__device__ __forceinline__ void sp_pick(const SpArgs &a, const T *z, bool vec, int64_t first, int64_t last, uint64_t target, float top, double c, uint64_t cut,
                                        uint64_t floor_w, int &id, float &logit) {
    const int lane = threadIdx.x & 63;
    id = -1;
    logit = -INFINITY;
    for (int64_t e = first; e < last; e += SP_CHUNK) {
        float v[8];
        uint64_t w[8], mine = 0;
        sp_load(z, vec, e + lane * 8, last, v);
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
            const int l = __ffsll((unsigned long long)__ballot(got >= 0)) - 1;
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
// the first class of [first, last) with logit `top`
template <typename T> __device__ __forceinline__ int sp_first(const SpArgs &a, const T *z, bool vec, int64_t first, int64_t last, float top) {
    const int lane = threadIdx.x & 63;
    for (int64_t e = first; e < last; e += SP_CHUNK) {
        float v[8];
        sp_load(z, vec, e + lane * 8, last, v);
        int got = -1;
#pragma unroll
        for (int i = 7; i >= 0; --i)
            if (v[i] == top) got = (int)(e + lane * 8 + i);
        const uint64_t who = __ballot(got >= 0);
        if (who) return __shfl(got, __ffsll((unsigned long long)who) - 1);
    }
    return -1;
}

// f(z, id) for eight classes a thread of the n listed granules; all lanes of a wavefront call it together
template <int NT, typename T, typename F>
__device__ __forceinline__ void sp_over_list(const SpArgs &a, const T *z, bool vec, const int32_t *list, int n, F f) {
    if (a.gran <= SP_CHUNK) {
        const int lanes = 1 << a.lg, at_once = NT >> a.lg, sub = threadIdx.x & (lanes - 1), own = threadIdx.x >> a.lg;
        const auto at = [&](int i) __attribute__((always_inline)) { return i < n ? list[i] * a.gran + sub * 8 : a.C; };
        for (int i0 = 0; i0 < n; i0 += at_once) {
            const int64_t e = at(i0 + own);
            float v[8];
            sp_load(z, vec, e, a.C, v);
            f(v, (uint32_t)e);
        }
    } else {
        const int lane = threadIdx.x & 63;
        for (int i = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < n; i += NT / 64) {
            const int64_t first = list[i] * a.gran, last = sp_min(first + a.gran, a.C);
            for (int64_t e = first + lane * 8; e - lane * 8 < last; e += SP_CHUNK) {
                float v[8];
                sp_load(z, vec, e, a.C, v);
                f(v, (uint32_t)e);
            }
        }
    }
}

// p[0 .. size) into ascending order (bitonic), size a power of two, at least 64.  A wavefront's 64 pairs lie within 128 numbers where they are at
// most 64 apart: only wider steps, and the first one after them, wait for the other wavefronts.
template <int NT> __device__ __forceinline__ void sp_sort(uint64_t *p, int size) {
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            if (j >= 64) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (int i = threadIdx.x; i < size / 2; i += NT) {
                const int x = ((i & ~(j - 1)) << 1) | (i & (j - 1)), y = x + j;
                const uint64_t u = p[x], v = p[y];
                if ((u > v) == ((x & k) == 0)) { p[x] = v; p[y] = u; }
            }
        }
    __syncthreads();
}

struct SpOrder {
    uint32_t n[SP_BINS];   // of buckets
    int32_t slot[SP_CAND]; // of a place in its bucket
    unsigned long long lo, hi;
    uint32_t most;
};
// p[0 .. n) into ascending order: into buckets of equal ranges, then by counting inside them; with many in one bucket (equal logits) as above.
// tmp: as long as p, p up to the next power of two.
template <int NT> __device__ __forceinline__ void sp_order(uint64_t *p, uint64_t *tmp, int n, SpOrder &o, SpScan &sh) {
    constexpr int EACH = SP_BINS / NT;
    __syncthreads();
    if (threadIdx.x == 0) { o.lo = ~0ull; o.hi = 0; o.most = 0; }
#pragma unroll
    for (int i = 0; i < EACH; ++i) o.n[i * NT + threadIdx.x] = 0;
    uint64_t lo = ~(uint64_t)0, hi = 0;
    for (int i = threadIdx.x; i < n; i += NT) {
        lo = sp_min(lo, p[i]);
        hi = sp_max(hi, p[i]);
    }
    __syncthreads();
    if (lo <= hi) {
        atomicMin(&o.lo, (unsigned long long)lo);
        atomicMax(&o.hi, (unsigned long long)hi);
    }
    __syncthreads();
    lo = o.lo;
    const uint64_t span = o.hi - lo;
    const int top = 63 - __clzll((long long)(span | 1)), shift = top < 11 ? 0 : top - 10; // span >> shift < 2^11
    for (int i = threadIdx.x; i < n; i += NT) o.slot[i] = (int)atomicAdd(&o.n[(p[i] - lo) >> shift], 1u);
    __syncthreads();
    uint32_t mine = 0, most = 0, before, all;
    uint64_t w0, w_all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        mine += o.n[threadIdx.x * EACH + i];
        most = sp_max(most, o.n[threadIdx.x * EACH + i]);
    }
    if (most > 64) atomicMax(&o.most, most);
    sp_scan<NT>(sh, 0, mine, w0, before, w_all, all);
    if (o.most > 512) {
        int size = 64;
        while (size < n) size <<= 1;
        for (int i = n + threadIdx.x; i < size; i += NT) p[i] = ~(uint64_t)0;
        __syncthreads();
        sp_sort<NT>(p, size);
        return;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint32_t k = o.n[threadIdx.x * EACH + i];
        o.n[threadIdx.x * EACH + i] = before;
        before += k;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) tmp[o.n[(p[i] - lo) >> shift] + o.slot[i]] = p[i];
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t place = tmp[i];
        const int b = (int)((place - lo) >> shift), first = (int)o.n[b], last = b + 1 < SP_BINS ? (int)o.n[b + 1] : n;
        int at = first;
        for (int j = first; j < last; ++j) at += tmp[j] < place;
        p[at] = place;
    }
    __syncthreads();
}

__device__ __forceinline__ void sp_share_row(const SpArgs &a, int row, float top, int b0, uint64_t target_p);
// What bounds it is the way through its short steps: 1 x 10,000 fp32, k = 50 13 us; 256 x 390,625 bf16, k = 500 44 to 47.
struct SpShared {
    SpScan scan;
    float top[SP_GRANULES]; // of the granules
    uint32_t n[SP_BINS];    // of the bins: granules, and their weight; then of ranges of ids
    uint64_t w[SP_BINS];
    uint64_t cand[SP_CAND]; // places of classes that may be kept
    union {
        int32_t list[SP_GRANULES]; // granules
        uint64_t cand_w[SP_CAND];  // the candidates' weights, 0 for those that are not kept
    };
    union {
        int32_t member[SP_CAND]; // candidates of one range of ids
        SpOrder order;
    };
    uint32_t fill;
};

// A workgroup per row.
template <typename T>
__global__ void __launch_bounds__(SP_NT)
sp_draw_kernel(SpArgs a) {
    __shared__ SpShared sh;
    constexpr int NT = SP_NT;
    const int row = a.row0 + blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const SpRule rule(a, row);
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    float top = -INFINITY;
    for (int i = threadIdx.x; i < a.ngr; i += NT) {
        const float t = a.g_max[(int64_t)row * a.ngr + i];
        sh.top[i] = t;
        top = fmaxf(top, t);
    }
    top = sp_block_max<NT>(sh.scan, top);
    if (threadIdx.x == 0) a.many[row] = 0;
    if (!(top > -INFINITY)) {
        if (threadIdx.x == 0) {
            a.ids[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        return;
    }
    const double c = rule.c;
    uint64_t w0, w_all;
    uint32_t n0, n_all;
    // consecutive granules of a thread
    const int per = (a.ngr + NT - 1) / NT, g0 = sp_min((int)threadIdx.x * per, a.ngr), g1 = sp_min(g0 + per, a.ngr);
    const auto mass = [&](int g) __attribute__((always_inline)) { return sp_mass(a, row, g, sh.top[g], top, c); };
    if (rule.greedy) { // the first class with the largest logit: the only one that is kept
        if (threadIdx.x == 0) sh.fill = 0x7FFFFFFF;
        __syncthreads();
        for (int g = g1 - 1; g >= g0; --g)
            if (sh.top[g] == top) atomicMin(&sh.fill, (uint32_t)g);
        __syncthreads();
        if (wave == 0) {
            const int64_t first = sh.fill * a.gran;
            const int id = sp_first(a, z, vec, first, sp_min(first + a.gran, a.C), top);
            if (lane == 0) {
                a.ids[row] = id;
                if (a.logprob) a.logprob[row] = 0.f;
            }
        }
        return;
    }
    if (!rule.use_k && !rule.use_p && !rule.use_m) { // all classes: the granules' weights say where to look
        uint64_t sum = 0;
        for (int g = g0; g < g1; ++g) sum += mass(g);
        sp_scan<NT>(sh.scan, sum, 0, w0, n0, w_all, n_all);
        const uint64_t target = sp_target(a, row, w_all);
        if (w0 <= target && target < w0 + sum) // one thread
            for (int g = g0; g < g1; ++g) {
                const uint64_t w = mass(g);
                if (target < w0 + w) { sh.scan.found = g; sh.scan.found_w = target - w0; break; }
                w0 += w;
            }
        __syncthreads();
        if (wave == 0) {
            int id;
            float logit;
            // from the granule on: its classes' own weights may come to less than its rounded sum, what is left of the target goes on to the next ones
            sp_pick(a, z, vec, sh.scan.found * a.gran, a.C, sh.scan.found_w, top, c, ~(uint64_t)0, sp_floor(a, rule), id, logit);
            if (lane == 0) sp_result(a, row, id, logit, top, c, w_all);
        }
        return;
    }
    // 1  down to which bin granules and classes have to be looked at
    const float c32 = sp_c32(rule);
    const int limit = sp_limit(a), bin_m = sp_bin_m(a, rule);
    int b0 = bin_m;
    uint64_t target_p = 0;
    if (rule.use_k || rule.use_p) {
        sp_clear<NT>(sh.n, sh.w);
        uint64_t sum = 0;
        for (int g = g0; g < g1; ++g) {
            const int b = sp_bin(sh.top[g], top, c32);
            if (b >= limit) continue;
            atomicAdd(&sh.n[b], 1u);
            if (!rule.use_k) {
                const uint64_t w = mass(g);
                sum += w;
                atomicAdd((unsigned long long *)&sh.w[b], (unsigned long long)w);
            }
        }
        if (!rule.use_k) target_p = sp_share(rule.p, sp_total<NT>(sh.scan, sum));
        sp_find<NT>(sh.scan, sh.n, sh.w, rule.use_k, rule.use_k ? (uint64_t)rule.k : target_p, w_all, n_all);
        const int found = sh.scan.found < 0 ? limit - 1 : sh.scan.found;
        // A share is looked for half a binade beyond where the granules' own weights reach it, and then two binades on at a time (256 x 390,625 bf16, spread 4,
        // p = 0.9: 416 us; from the granules' bin on 433, two binades beyond it 425; 16 x 30,000 fp32 81, 76 and 54, and by one binade at a time 73)
        b0 = rule.use_k ? (rule.use_p ? found : sp_min(found, bin_m)) : sp_min(found + SP_PER_BINADE / 2, bin_m);
    }
    // 2  the classes down to there in order, and their running weight; more of them while a share of the weight is not reached
    int n, c0, c1; // consecutive candidates of a thread
    for (;;) {
        uint32_t listed = 0;
        for (int g = g0; g < g1; ++g) listed += sp_bin(sh.top[g], top, c32) <= b0;
        sp_scan<NT>(sh.scan, 0, listed, w0, n0, w_all, n_all);
        // Rows that list more than a span of classes are shared.  With top-k four of them: candidates are found by one read, what it costs to share
        // them is more (256 x 390,625 bf16, k = 500: 101 us, with two spans 177, with one 225; 64 rows, k = 3,000: 124 with one to eight, 297 with sixteen)
        if (n_all > SP_CAND || (rule.use_k && rule.k > SP_CAND) || n_all * a.gran > (rule.use_k ? 4 * a.most : a.most)) n = SP_CAND + 1; // a class of each granule is in
        else {
            if (threadIdx.x == 0) sh.fill = 0;
            for (int g = g0; g < g1; ++g)
                if (sp_bin(sh.top[g], top, c32) <= b0) sh.list[n0++] = g;
            __syncthreads();
            sp_over_list<NT>(a, z, vec, sh.list, (int)n_all, [&](const float (&v)[8], uint32_t id) __attribute__((always_inline)) {
                float best = v[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) best = fmaxf(best, v[i]);
                if (sp_bin(best, top, c32) > b0) return;
                uint32_t in = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) in |= (uint32_t)(sp_bin(v[i], top, c32) <= b0) << i;
                uint32_t at = atomicAdd(&sh.fill, (uint32_t)__popc(in));
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (in >> i & 1) {
                        if (at < SP_CAND) sh.cand[at] = sp_place(v[i], id + i);
                        ++at;
                    }
            });
            __syncthreads();
            n = (int)sh.fill;
        }
        if (n > SP_CAND) { // more than LDS holds
            if (threadIdx.x == 0) a.many[row] = 1;
            if (a.rows) sp_share_row(a, row, top, rule.use_k ? b0 : bin_m, target_p);
            return;
        }
        if (n <= NT) { // a candidate's place in the order is the number of those before it; several threads count for one where there are few
            const int lg = n <= 64 ? 6 : n <= 128 ? 7 : n <= 256 ? 8 : 9, each = threadIdx.x & ((1 << lg) - 1), parts = NT >> lg, part = threadIdx.x >> lg;
            const uint64_t place = each < n ? sh.cand[each] : 0;
            uint32_t before = 0;
#pragma unroll 4
            for (int j = part; j < n; j += parts) before += sh.cand[j] < place;
            sh.member[threadIdx.x] = 0;
            __syncthreads();
            if (each < n) atomicAdd(&sh.member[each], (int)before);
            __syncthreads();
            if (part == 0 && each < n) sh.cand[sh.member[each]] = place;
        } else sp_order<NT>(sh.cand, sh.cand_w, n, sh.order, sh.scan);
        __syncthreads();
        const int each = (n + NT - 1) / NT;
        c0 = sp_min((int)threadIdx.x * each, n);
        c1 = sp_min(c0 + each, n);
        uint64_t sum = 0;
        for (int i = c0; i < c1; ++i) {
            const uint64_t w = sp_weight(sp_place_z(sh.cand[i]), top, c, a.bits);
            sh.cand_w[i] = w;
            sum += w;
        }
        sp_scan<NT>(sh.scan, sum, 0, w0, n0, w_all, n_all);
        if (!rule.use_p || rule.use_k || w_all >= target_p || b0 >= bin_m) break;
        b0 = sp_min(b0 + 2 * SP_PER_BINADE, bin_m);
    }
    // 3  how many of them top-k, then top-p and min-p keep, and their weight
    int keep = rule.use_k && rule.k < n ? (int)rule.k : n;
    if (rule.use_p) {
        if (rule.use_k && keep < n) { // the share is one of the weight that top-k keeps
            if (c0 < keep && keep <= c1) {
                uint64_t run = w0;
                for (int i = c0; i < keep; ++i) run += sh.cand_w[i];
                sh.scan.found_w = run;
            }
            __syncthreads();
            w_all = sh.scan.found_w;
        }
        if (rule.use_k) target_p = sp_share(rule.p, w_all);
        if (threadIdx.x == 0) sh.scan.found = n;
        __syncthreads();
        uint64_t run = w0;
        for (int i = c0; i < c1; ++i) {
            const uint64_t w = sh.cand_w[i];
            if (run < target_p && target_p <= run + w) sh.scan.found = i + 1;
            run += w;
        }
        __syncthreads();
        keep = sp_min(keep, sh.scan.found);
    }
    const uint64_t floor_w = sp_floor(a, rule);
    uint64_t kept = 0;
    for (int i = c0; i < c1; ++i) {
        const uint64_t w = sh.cand_w[i];
        if (i >= keep || w < floor_w) sh.cand_w[i] = 0;
        else kept += w;
    }
    w_all = sp_total<NT>(sh.scan, kept);
    uint64_t target = sp_target(a, row, w_all);
    // 4  by id: the class at which the running weight exceeds the target, among few in number, or of a range of ids
    int members = n;
    if (n > NT) {
        int shift = 0;
        while ((a.C - 1) >> shift >= SP_BINS) ++shift;
        sp_clear<NT>(sh.n, sh.w);
        for (int i = c0; i < c1; ++i)
            if (sh.cand_w[i]) atomicAdd((unsigned long long *)&sh.w[(uint32_t)sh.cand[i] >> shift], (unsigned long long)sh.cand_w[i]);
        uint64_t unused;
        sp_find<NT>(sh.scan, sh.n, sh.w, false, target + 1, unused, n_all);
        target -= sh.scan.found_w;
        const uint32_t range = (uint32_t)sh.scan.found;
        if (threadIdx.x == 0) sh.fill = 0;
        __syncthreads();
        for (int i = c0; i < c1; ++i)
            if (sh.cand_w[i] && (uint32_t)sh.cand[i] >> shift == range) sh.member[atomicAdd(&sh.fill, 1u)] = i;
        __syncthreads();
        members = (int)sh.fill;
    }
    for (int i = threadIdx.x; i < members; i += NT) {
        const int at = n > NT ? sh.member[i] : i;
        const uint64_t place = sh.cand[at], w = sh.cand_w[at];
        uint64_t before = 0;
        if (n > NT)
            for (int j = 0; j < members; ++j) before += (uint32_t)sh.cand[sh.member[j]] < (uint32_t)place ? sh.cand_w[sh.member[j]] : 0;
        else
#pragma unroll 4
            for (int j = 0; j < keep; ++j) before += (uint32_t)sh.cand[j] < (uint32_t)place ? sh.cand_w[j] : 0;
        if (before <= target && target < before + w) sp_result(a, row, (int)(uint32_t)place, sp_place_z(place), top, c, w_all);
    }
}

// ------------------------------------------------------------------------------------------------
// rows of which more may be kept than LDS holds
// ------------------------------------------------------------------------------------------------
// granules of a workgroup's threads, SP_PER consecutive ones each
#define SP_PER (SP_GRANULES / SP_NT2)
struct SpMine {
    float top[SP_PER], row_top;
    int first, n; // of the thread
    __device__ __forceinline__ SpMine(const SpArgs &a, int row, SpScan &sh) {
        const int per = (a.ngr + SP_NT2 - 1) / SP_NT2;
        first = threadIdx.x * per;
        n = sp_max(0, sp_min(per, a.ngr - first));
        row_top = -INFINITY;
#pragma unroll
        for (int i = 0; i < SP_PER; ++i) {
            top[i] = i < n ? a.g_max[(int64_t)row * a.ngr + first + i] : -INFINITY;
            row_top = fmaxf(row_top, top[i]);
        }
        row_top = sp_block_max<SP_NT2>(sh, row_top);
    }
    __device__ __forceinline__ uint64_t mass(const SpArgs &a, int row, const SpRule &rule, int i) const { return i < n ? sp_mass(a, row, first + i, top[i], row_top, rule.c) : 0; }
};
// the granules whose largest logit lies in bin b0 or before, in order: list, and how many
__device__ __forceinline__ int sp_list(const SpMine &mine, SpScan &sh, float c32, int b0, int32_t *list) {
    bool in[SP_PER];
    int n = 0;
#pragma unroll
    for (int i = 0; i < SP_PER; ++i) {
        in[i] = sp_bin(mine.top[i], mine.row_top, c32) <= b0;
        n += in[i];
    }
    uint64_t w0, w_all;
    uint32_t at, all;
    sp_scan<SP_NT2>(sh, 0, (uint32_t)n, w0, at, w_all, all);
#pragma unroll
    for (int i = 0; i < SP_PER; ++i)
        if (in[i]) list[at++] = mine.first + i;
    __syncthreads();
    return (int)all;
}

struct SpMany {
    SpScan scan;
    uint32_t n[SP_BINS];   // of the bins: classes (at first: granules), and their weight
    uint64_t w[SP_BINS];
    union {
        uint64_t cand[SP_GRANULES]; // places of the classes of one bin
        struct {
            uint32_t n[SP_BINS];
            uint64_t w[SP_BINS];
        } sub;                      // parts of a bin that has too many
    };
    uint64_t g_w[SP_GRANULES]; // kept weight of the listed granules
    int32_t list[SP_GRANULES];
    int n_list;
    uint32_t fill;
    uint64_t place;
};
#define SP_MANY_CAND SP_GRANULES

// Of the listed classes of bin `bin`, which are sh.n[bin]: the place of the one at which the running number or weight reaches `target`, in
// the order; `weight`: their weight up to it.  Too many for LDS (a bin of equal logits) are cut into parts of equal ranges of places first.
template <typename T>
__device__ __forceinline__ uint64_t sp_refine(const SpArgs &a, const T *z, bool vec, SpMany &sh, float top, double c, float c32, int bin, bool by_n, uint64_t target,
                                           uint64_t &weight) {
    uint64_t lo = 0, hi = ~(uint64_t)0, before = 0;
    uint32_t n = sh.n[bin];
    while (n > SP_MANY_CAND) {
        uint64_t least = ~(uint64_t)0, most = 0;
        sp_over_list<SP_NT2>(a, z, vec, sh.list, sh.n_list, [&](const float (&v)[8], uint32_t id) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t place = sp_place(v[i], id + i);
                if (sp_bin(v[i], top, c32) != bin || place < lo || place > hi) continue;
                least = sp_min(least, place);
                most = sp_max(most, place);
            }
        });
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            least = sp_min(least, (uint64_t)__shfl_xor((unsigned long long)least, d));
            most = sp_max(most, (uint64_t)__shfl_xor((unsigned long long)most, d));
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) { sh.scan.w[threadIdx.x >> 6] = least; sh.scan.v[threadIdx.x >> 6] = most; }
        __syncthreads();
        for (int i = 0; i < (SP_NT2 / 64); ++i) { least = sp_min(least, sh.scan.w[i]); most = sp_max(most, sh.scan.v[i]); }
        int shift = 0;
        while ((most - least) >> shift >= SP_BINS) ++shift;
        sp_clear<SP_NT2>(sh.sub.n, sh.sub.w);
        sp_over_list<SP_NT2>(a, z, vec, sh.list, sh.n_list, [&](const float (&v)[8], uint32_t id) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t place = sp_place(v[i], id + i);
                if (sp_bin(v[i], top, c32) != bin || place < least || place > most) continue;
                const int part = (int)((place - least) >> shift);
                atomicAdd(&sh.sub.n[part], 1u);
                atomicAdd((unsigned long long *)&sh.sub.w[part], (unsigned long long)sp_weight(v[i], top, c, a.bits));
            }
        });
        uint64_t w_all;
        uint32_t n_all;
        sp_find<SP_NT2>(sh.scan, sh.sub.n, sh.sub.w, by_n, target, w_all, n_all);
        const int part = sh.scan.found; // there is one: the target lies within the bin
        lo = least + ((uint64_t)part << shift);
        hi = sp_min(most, lo + (((uint64_t)1 << shift) - 1));
        n = sh.sub.n[part];
        target -= by_n ? sh.scan.found_n : sh.scan.found_w;
        before += sh.scan.found_w;
    }
    __syncthreads();
    if (threadIdx.x == 0) { sh.fill = 0; sh.place = 0; sh.scan.found_w = 0; }
    int size = 64;
    while (size < (int)n) size <<= 1;
    for (int i = n + threadIdx.x; i < size; i += SP_NT2) sh.cand[i] = ~(uint64_t)0;
    __syncthreads();
    sp_over_list<SP_NT2>(a, z, vec, sh.list, sh.n_list, [&](const float (&v)[8], uint32_t id) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint64_t place = sp_place(v[i], id + i);
            if (sp_bin(v[i], top, c32) != bin || place < lo || place > hi) continue;
            const uint32_t at = atomicAdd(&sh.fill, 1u);
            if (at < n) sh.cand[at] = place;
        }
    });
    __syncthreads();
    sp_sort<SP_NT2>(sh.cand, size);
    constexpr int EACH = SP_MANY_CAND / SP_NT2;
    uint64_t w[EACH], mine = 0, w0, w_all;
    uint32_t unused, unused_all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = threadIdx.x * EACH + i;
        w[i] = at < (int)n ? sp_weight(sp_place_z(sh.cand[at]), top, c, a.bits) : 0;
        mine += w[i];
    }
    sp_scan<SP_NT2>(sh.scan, mine, 0, w0, unused, w_all, unused_all);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = threadIdx.x * EACH + i;
        if (at < (int)n && (by_n ? at + 1 == (int)target : w0 < target && target <= w0 + w[i])) {
            sh.place = sh.cand[at];
            sh.scan.found_w = w0 + w[i];
        }
        w0 += w[i];
    }
    __syncthreads();
    weight = before + sh.scan.found_w;
    return sh.place;
}

// The class of a row that all compute units shared: the classes of the bins in which top-k and top-p end in order, what they add to their granules.
struct SpFinal {
    SpScan scan;
    uint64_t cand[SP_CAND], cand_w[SP_CAND], g_w[SP_GRANULES];
    SpOrder order;
};
template <typename T> __device__ __forceinline__ void sp_final(const SpArgs &a, int row, SpFinal &sh) {
    constexpr int NT = SP_NT2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const SpRule rule(a, row);
    const SpRow &st = a.rows[row];
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    const float top = a.row_top[row], c32 = sp_c32(rule);
    const double c = rule.c;
    const int bin_k = st.bin_k, p_first = st.p_first, p_last = st.p_last;
    const uint64_t floor_w = sp_floor(a, rule), *const g_w = (const uint64_t *)a.g_sum + (int64_t)row * a.ngr;
    const uint32_t n = st.n_cand;
    for (int g = threadIdx.x; g < a.ngr; g += NT) sh.g_w[g] = g_w[g];
    for (int i = threadIdx.x; i < (int)n; i += NT) sh.cand[i] = a.pool[st.cand0 + i];
    if (n) sp_order<NT>(sh.cand, sh.cand_w, n, sh.order, sh.scan);
    const int each = (n + NT - 1) / NT, c0 = sp_min((int)threadIdx.x * each, (int)n), c1 = sp_min(c0 + each, (int)n);
    // the last class that top-k, then top-p keeps
    uint64_t cut = ~(uint64_t)0, w0, all, target = st.target_p, sum = 0;
    uint32_t n0, n_all, in_k = 0;
    for (int i = c0; i < c1; ++i) {
        const float v = sp_place_z(sh.cand[i]);
        sh.cand_w[i] = sp_weight(v, top, c, a.bits);
        in_k += sp_bin(v, top, c32) == bin_k;
    }
    if (bin_k >= 0) {
        for (int i = c0; i < c1; ++i)
            if (sp_bin(sp_place_z(sh.cand[i]), top, c32) == bin_k) sum += sh.cand_w[i];
        sp_scan<NT>(sh.scan, sum, in_k, w0, n0, all, n_all);
        if (n0 < st.k_rest && st.k_rest <= n0 + in_k) // one thread
            for (int i = c0; i < c1; ++i)
                if (sp_bin(sp_place_z(sh.cand[i]), top, c32) == bin_k) {
                    ++n0;
                    w0 += sh.cand_w[i];
                    if (n0 == st.k_rest) {
                        sh.scan.found_w = w0;
                        sh.scan.found = i;
                    }
                }
        __syncthreads();
        cut = sh.cand[sh.scan.found];
        target = sp_share(rule.p, st.before_k + sh.scan.found_w);
    } else if (rule.use_k) target = sp_share(rule.p, st.w_all);
    if (p_first < SP_NO_BIN) {
        sum = 0;
        for (int i = c0; i < c1; ++i) {
            const int b = sp_bin(sp_place_z(sh.cand[i]), top, c32);
            if (b >= p_first && b <= p_last) sum += sh.cand_w[i];
        }
        sp_scan<NT>(sh.scan, sum, 0, w0, n0, all, n_all);
        w0 += st.before_p;
        if (threadIdx.x == 0) sh.scan.found = -1;
        __syncthreads();
        for (int i = c0; i < c1; ++i) {
            const int b = sp_bin(sp_place_z(sh.cand[i]), top, c32);
            if (b < p_first || b > p_last) continue;
            if (w0 < target && target <= w0 + sh.cand_w[i]) sh.scan.found = i;
            w0 += sh.cand_w[i];
        }
        __syncthreads();
        if (sh.scan.found >= 0) cut = sp_min(cut, sh.cand[sh.scan.found]);
    }
    __syncthreads();
    for (int i = c0; i < c1; ++i) {
        const uint64_t place = sh.cand[i], w = sh.cand_w[i];
        if (place <= cut && w >= floor_w) atomicAdd((unsigned long long *)&sh.g_w[(uint32_t)place >> a.gshift], (unsigned long long)w);
    }
    __syncthreads();
    const int per = (a.ngr + NT - 1) / NT, g0 = sp_min((int)threadIdx.x * per, a.ngr), g1 = sp_min(g0 + per, a.ngr);
    sum = 0;
    for (int g = g0; g < g1; ++g) sum += sh.g_w[g];
    sp_scan<NT>(sh.scan, sum, 0, w0, n0, all, n_all);
    target = sp_target(a, row, all);
    if (w0 <= target && target < w0 + sum) // one thread
        for (int g = g0; g < g1; ++g) {
            if (target < w0 + sh.g_w[g]) { sh.scan.found = g; sh.scan.found_w = target - w0; break; }
            w0 += sh.g_w[g];
        }
    __syncthreads();
    if (wave == 0) {
        int id;
        float logit;
        const int64_t from = sh.scan.found * a.gran;
        sp_pick(a, z, vec, from, sp_min(from + a.gran, a.C), sh.scan.found_w, top, c, cut, floor_w, id, logit);
        if (lane == 0) sp_result(a, row, id, logit, top, c, all);
    }
}

// A workgroup per row: numbers and weights of the bins, the bin in which top-k or top-p ends in order, what is kept of every granule, the class.
template <typename T>
__global__ void __launch_bounds__(SP_NT2)
sp_many_kernel(SpArgs a) {
    __shared__ union U {
        SpMany many;
        SpFinal final;
        __device__ U() {}
    } u;
    const int row = a.row0 + blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), state = a.many[row];
    if (state == 3) sp_final<T>(a, row, u.final);
    if (state != (a.rows ? 2 : 1)) return;
    SpMany &sh = u.many;
    const SpRule rule(a, row);
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    const SpMine mine(a, row, sh.scan);
    const float top = mine.row_top;
    const double c = rule.c;
    const float c32 = sp_c32(rule);
    const int limit = sp_limit(a);
    int b0 = sp_bin_m(a, rule);
    uint64_t w0, w_all, target_p = 0;
    uint32_t n0, n_all;
    if (rule.use_k) {
        sp_clear<SP_NT2>(sh.n, sh.w);
#pragma unroll
        for (int i = 0; i < SP_PER; ++i) {
            const int b = sp_bin(mine.top[i], top, c32);
            if (b < limit) atomicAdd(&sh.n[b], 1u);
        }
        sp_find<SP_NT2>(sh.scan, sh.n, sh.w, true, (uint64_t)rule.k, w_all, n_all);
        const int found = sh.scan.found < 0 ? limit - 1 : sh.scan.found;
        b0 = rule.use_p ? found : sp_min(found, b0);
    } else if (rule.use_p && a.rows) target_p = a.rows[row].target_p;
    else if (rule.use_p) {
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < SP_PER; ++i) sum += mine.mass(a, row, rule, i);
        sp_scan<SP_NT2>(sh.scan, sum, 0, w0, n0, w_all, n_all);
        target_p = sp_share(rule.p, w_all);
    }
    const int n_list = sp_list(mine, sh.scan, c32, b0, sh.list);
    if (threadIdx.x == 0) sh.n_list = n_list;
    sp_clear<SP_NT2>(sh.n, sh.w);
    uint64_t cut = ~(uint64_t)0;
    if (rule.use_k || rule.use_p) {
        sp_over_list<SP_NT2>(a, z, vec, sh.list, n_list, [&](const float (&v)[8], uint32_t) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int b = sp_bin(v[i], top, c32);
                if (b > b0) continue;
                atomicAdd(&sh.n[b], 1u);
                atomicAdd((unsigned long long *)&sh.w[b], (unsigned long long)sp_weight(v[i], top, c, a.bits));
            }
        });
        if (rule.use_k) {
            sp_find<SP_NT2>(sh.scan, sh.n, sh.w, true, (uint64_t)rule.k, w_all, n_all);
            if (sh.scan.found >= 0) {
                const uint64_t before = sh.scan.found_w;
                uint64_t w;
                cut = sp_refine(a, z, vec, sh, top, c, c32, sh.scan.found, true, (uint64_t)rule.k - sh.scan.found_n, w);
                w_all = before + w;
            }
            target_p = sp_share(rule.p, w_all);
        }
        if (rule.use_p) {
            uint64_t all;
            sp_find<SP_NT2>(sh.scan, sh.n, sh.w, false, target_p, all, n_all);
            if (sh.scan.found >= 0) {
                uint64_t w;
                cut = sp_min(cut, sp_refine(a, z, vec, sh, top, c, c32, sh.scan.found, false, target_p - sh.scan.found_w, w));
            }
        }
    }
    const uint64_t floor_w = sp_floor(a, rule);
    for (int i = threadIdx.x; i < n_list; i += SP_NT2) sh.g_w[i] = 0;
    __syncthreads();
    const int at_once = SP_NT2 >> a.lg;
    int turn = 0; // which of its granules a thread is at
    sp_over_list<SP_NT2>(a, z, vec, sh.list, n_list, [&](const float (&v)[8], uint32_t id) __attribute__((always_inline)) {
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (sp_bin(v[i], top, c32) > b0 || sp_place(v[i], id + i) > cut) continue;
            const uint64_t w = sp_weight(v[i], top, c, a.bits);
            if (w >= floor_w) sum += w;
        }
        int at;
        if (a.gran <= SP_CHUNK) {
            at = turn * at_once + (threadIdx.x >> a.lg);
            ++turn;
        } else {
            at = wave + turn * (SP_NT2 / 64);
            if ((int64_t)(id - lane * 8) + SP_CHUNK >= sp_min((sh.list[at] + (int64_t)1) * a.gran, a.C)) ++turn;
        }
        if (sum) atomicAdd((unsigned long long *)&sh.g_w[at], (unsigned long long)sum);
    });
    __syncthreads();
    uint64_t w[SP_PER], sum = 0;
#pragma unroll
    for (int i = 0; i < SP_PER; ++i) {
        w[i] = threadIdx.x * SP_PER + i < n_list ? sh.g_w[threadIdx.x * SP_PER + i] : 0;
        sum += w[i];
    }
    sp_scan<SP_NT2>(sh.scan, sum, 0, w0, n0, w_all, n_all);
    const uint64_t target = sp_target(a, row, w_all);
#pragma unroll
    for (int i = 0; i < SP_PER; ++i) {
        if (w0 <= target && target < w0 + w[i]) { sh.scan.found = sh.list[threadIdx.x * SP_PER + i]; sh.scan.found_w = target - w0; }
        w0 += w[i];
    }
    __syncthreads();
    if (wave == 0) {
        int id;
        float logit;
        const int64_t first = sh.scan.found * a.gran;
        sp_pick(a, z, vec, first, sp_min(first + a.gran, a.C), sh.scan.found_w, top, c, cut, floor_w, id, logit);
        if (lane == 0) sp_result(a, row, id, logit, top, c, w_all);
    }
}

// ------------------------------------------------------------------------------------------------
// such rows of many classes: all compute units share them
// ------------------------------------------------------------------------------------------------
// Two launches before the one above.  In the first the workgroups of a row count its bins; the one that is done last knows in which bin top-k ends,
// and between which bins top-p does (the weight that top-k keeps is known but for a part of its own bin).  In the second they write what
// lies before those bins, which is kept, granule by granule, and the places of the classes inside them, which the last launch puts in order.
#define SP_SPAN 32768
// what the two launches start from; all threads of the row's workgroup
__device__ __forceinline__ void sp_share_row(const SpArgs &a, int row, float top, int b0, uint64_t target_p) {
    for (int i = threadIdx.x; i < SP_BINS; i += blockDim.x) {
        a.bins_n[(int64_t)row * SP_BINS + i] = 0;
        a.bins_w[(int64_t)row * SP_BINS + i] = 0;
    }
    if (a.gran > SP_CHUNK) // granules' kept weights are added up there (the granules' own are no longer needed)
        for (int i = threadIdx.x; i < a.ngr; i += blockDim.x) ((uint64_t *)a.g_sum)[(int64_t)row * a.ngr + i] = 0;
    if (threadIdx.x == 0) {
        SpRow &st = a.rows[row];
        st.b0 = b0;
        st.target_p = target_p;
        st.fill = st.done = 0;
        a.row_top[row] = top;
    }
}

template <typename V> __device__ __forceinline__ V sp_read(const V *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// The workgroup that calls this last of `all` ones finds what the others have added and stored: all of it by atomic operations at the device's
// scope, which have been done (a wavefront's own are waited for here) before `done` is counted up.  A fence would also write back the
// whole L2, for each workgroup: 256 x 390,625 bf16 took 550 us in either launch.
__device__ __forceinline__ bool sp_last(uint32_t *done, int all, uint32_t &sh) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (threadIdx.x == 0) sh = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return sh == (uint32_t)all - 1;
}

struct SpCount {
    SpScan scan;
    uint32_t n[SP_BINS];
    uint64_t w[SP_BINS];
    uint32_t done;
};
template <typename T>
__global__ void __launch_bounds__(SP_NT2)
sp_count_kernel(SpArgs a) {
    constexpr int NT = SP_NT2;
    __shared__ SpCount sh;
    const int row = a.row0 + blockIdx.y;
    if (a.many[row] != 1) return;
    const SpRule rule(a, row);
    SpRow &st = a.rows[row];
    uint32_t *const g_n = a.bins_n + (int64_t)row * SP_BINS;
    uint64_t *const g_w = a.bins_w + (int64_t)row * SP_BINS;
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    const float top = a.row_top[row], c32 = sp_c32(rule);
    const double c = rule.c;
    const int b0 = st.b0;
    sp_clear<NT>(sh.n, sh.w);
    const int64_t first = blockIdx.x * a.span, last = sp_min(first + a.span, a.C);
    for (int64_t e = first + threadIdx.x * 8; e < last; e += NT * 8) {
        if (!(sp_bin(a.g_max[(int64_t)row * a.ngr + (e >> a.gshift)], top, c32) <= b0)) continue;
        float v[8];
        sp_load(z, vec, e, last, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int b = sp_bin(v[i], top, c32);
            if (b > b0) continue;
            atomicAdd(&sh.n[b], 1u);
            atomicAdd((unsigned long long *)&sh.w[b], (unsigned long long)sp_weight(v[i], top, c, a.bits));
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SP_BINS / NT; ++i) {
        const int b = i * NT + threadIdx.x;
        if (sh.n[b]) {
            atomicAdd(&g_n[b], sh.n[b]);
            atomicAdd((unsigned long long *)&g_w[b], (unsigned long long)sh.w[b]);
        }
    }
    if (!sp_last(&st.done, gridDim.x, sh.done)) return;
#pragma unroll
    for (int i = 0; i < SP_BINS / NT; ++i) {
        const int b = i * NT + threadIdx.x;
        sh.n[b] = sp_read(&g_n[b]);
        sh.w[b] = sp_read(&g_w[b]);
    }
    uint64_t w_all, target = st.target_p, before_k = 0, before_p = 0, unused;
    uint32_t n_all, k_rest = 0;
    int bin_k = -1, p_first = SP_NO_BIN + 1, p_last = -1;
    uint64_t most;
    if (rule.use_k) {
        sp_find<NT>(sh.scan, sh.n, sh.w, true, (uint64_t)rule.k, w_all, n_all);
        bin_k = sh.scan.found;
        most = w_all;
        if (bin_k >= 0) {
            before_k = sh.scan.found_w;
            k_rest = (uint32_t)(rule.k - sh.scan.found_n);
            w_all = before_k;
            most = before_k + sh.w[bin_k];
        }
    } else most = w_all = 0;
    if (rule.use_p) {
        sp_find<NT>(sh.scan, sh.n, sh.w, false, rule.use_k ? sp_share(rule.p, w_all) : target, unused, n_all);
        if (sh.scan.found >= 0) { // else top-p ends behind what min-p keeps
            p_first = p_last = sh.scan.found;
            before_p = sh.scan.found_w;
            if (bin_k >= 0) {
                sp_find<NT>(sh.scan, sh.n, sh.w, false, sp_share(rule.p, most), unused, n_all);
                p_last = sh.scan.found;
            }
        }
    }
    __syncthreads();
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < SP_BINS / NT; ++i) {
        const int b = i * NT + threadIdx.x;
        if (b == bin_k || (b >= p_first && b <= p_last)) mine += sh.n[b];
    }
    uint64_t w0;
    uint32_t n0, n_cand;
    sp_scan<NT>(sh.scan, 0, mine, w0, n0, unused, n_cand);
    if (threadIdx.x == 0) {
        st.bin_k = bin_k;
        st.p_first = p_first;
        st.p_last = p_last;
        st.sure = sp_min(p_first, bin_k >= 0 ? bin_k : b0 + 1);
        st.k_rest = k_rest;
        st.n_cand = n_cand;
        st.w_all = w_all;
        st.before_k = before_k;
        st.before_p = before_p;
        uint64_t at = 0;
        if (n_cand <= SP_CAND) at = atomicAdd((unsigned long long *)a.pool_used, (unsigned long long)n_cand);
        st.cand0 = at;
        a.many[row] = n_cand <= SP_CAND && at + n_cand <= a.pool_size ? 3 : 2; // 2: a bin of equal logits, one workgroup's work
    }
}

#define SP_NT3 512
#define SP_SPAN3 8192 /* classes of a workgroup */
struct SpKeep {
    uint64_t cand[SP_CAND];
    uint32_t fill, at;
};
template <typename T>
__global__ void __launch_bounds__(SP_NT3)
sp_keep_kernel(SpArgs a) {
    constexpr int NT = SP_NT3;
    __shared__ SpKeep sh;
    const int row = a.row0 + blockIdx.y, lane = threadIdx.x & 63;
    if (a.many[row] != 3) return;
    const SpRule rule(a, row);
    SpRow &st = a.rows[row];
    bool vec;
    const T *const z = sp_row<T>(a, row, vec);
    const float top = a.row_top[row], c32 = sp_c32(rule);
    const double c = rule.c;
    const int b0 = st.b0, bin_k = st.bin_k, p_first = st.p_first, p_last = st.p_last, sure = st.sure;
    const uint64_t floor_w = sp_floor(a, rule), cand0 = st.cand0;
    const uint32_t n = st.n_cand;
    uint64_t *const g_w = (uint64_t *)a.g_sum + (int64_t)row * a.ngr;
    const int64_t first = (int64_t)blockIdx.x * SP_SPAN3, last = sp_min(first + SP_SPAN3, a.C);
    if (threadIdx.x == 0) sh.fill = 0;
    __syncthreads();
    for (int64_t e0 = first; e0 < last; e0 += NT * 8) {
        const int64_t e = e0 + threadIdx.x * 8;
        uint64_t sum = 0;
        if (e < last && sp_bin(a.g_max[(int64_t)row * a.ngr + (e >> a.gshift)], top, c32) <= b0) {
            float v[8];
            sp_load(z, vec, e, last, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int b = sp_bin(v[i], top, c32);
                if (b < sure && b <= b0) {
                    const uint64_t w = sp_weight(v[i], top, c, a.bits);
                    if (w >= floor_w) sum += w;
                } else if (b == bin_k || (b >= p_first && b <= p_last)) {
                    const uint32_t at = atomicAdd(&sh.fill, 1u);
                    if (at < SP_CAND) sh.cand[at] = sp_place(v[i], (uint32_t)(e + i)); // the row has no more than that
                }
            }
        }
        if (a.gran <= SP_CHUNK) {
            for (int d = 1; d < 1 << a.lg; d <<= 1) sum += __shfl_xor((unsigned long long)sum, d);
            if ((lane & ((1 << a.lg) - 1)) == 0 && e < last) g_w[e >> a.gshift] = sum;
        } else {
            sum = sp_wave_scan(sum);
            if (lane == 63 && e - lane * 8 < last) { // several wavefronts, in any order
                const int64_t g = (e - lane * 8) >> a.gshift;
                atomicAdd((unsigned long long *)&g_w[g], (unsigned long long)sum);
            }
        }
    }
    __syncthreads();
    const uint32_t here = sp_min(sh.fill, (uint32_t)SP_CAND);
    if (threadIdx.x == 0 && here) sh.at = atomicAdd(&st.fill, here);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < here; i += NT)
        if (sh.at + i < n) a.pool[cand0 + sh.at + i] = sh.cand[i];
}

static bool sp_sizes(int64_t C, int B, SpArgs &a) {
    if (C < 1 || C >= (int64_t)1 << 31 || B < 1) return false;
    a.C = C;
    a.gran = 8;
    while (ks_ceil_div(C, a.gran) > SP_GRANULES) a.gran *= 2;
    a.ngr = (int)ks_ceil_div(C, a.gran);
    a.gshift = 3;
    while ((int64_t)1 << a.gshift < a.gran) ++a.gshift;
    a.lg = 0;
    while (a.lg < 6 && 8 << a.lg < a.gran) ++a.lg;
    int lg = 0;
    while (((int64_t)1 << lg) < C) ++lg;
    a.bits = 62 - lg < 48 ? 62 - lg : 48;
    return true;
}
// From this many classes on, rows that keep much are shared by all compute units (16 x 100,000 fp32, p = 0.98: 87 us, 234 with a workgroup a row;
// 300 x 40,000: 150 and 238, x 20,000: 145 and 153); two launches more, together 3.5 us where no row needs them
#define SP_SHARED_C 32768
static void sp_places(KsArena &ws, int B, SpArgs &a) {
    a.g_max = ws.take<float>((size_t)B * a.ngr);
    a.g_sum = ws.take<double>((size_t)B * a.ngr);
    a.many = ws.take<int32_t>((size_t)B);
    a.rows = nullptr;
    a.most = (int64_t)1 << 40;
    if (a.C < SP_SHARED_C) return;
    a.most = SP_SPAN;
    a.span = B * ks_ceil_div(a.C, SP_SPAN) < 512 ? SP_SPAN / 4 : SP_SPAN; // few rows: more workgroups; many: fewer bins to add up
    a.rows = ws.take<SpRow>((size_t)B);
    a.row_top = ws.take<float>((size_t)B);
    a.bins_n = ws.take<uint32_t>((size_t)B * SP_BINS);
    a.bins_w = ws.take<uint64_t>((size_t)B * SP_BINS);
    a.pool_size = (uint64_t)(B < 256 ? B : 256) * SP_CAND;
    a.pool = ws.take<uint64_t>((size_t)a.pool_size);
    a.pool_used = ws.take<uint64_t>(1);
}

extern "C" size_t class_sample_workspace(int64_t C, int B) {
    SpArgs a;
    if (!sp_sizes(C, B, a)) return 0;
    KsArena ws(nullptr);
    sp_places(ws, B, a);
    return ws.off;
}

template <typename T> static void sp_sample(SpArgs &a, int B, hipStream_t st) {
    for (int64_t r = 0; r < B; r += 1 << 15) { // a launch's second dimension ends at 65,535
        const unsigned rows = (unsigned)(B - r < 1 << 15 ? B - r : 1 << 15);
        a.row0 = (int)r;
        const int64_t waves = a.gran < SP_CHUNK ? ks_ceil_div(a.C, SP_CHUNK) : a.ngr;
        const dim3 grid((unsigned)ks_ceil_div(waves, 4), rows);
        const auto granules = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
        switch (a.lg) {
        case 0: granules(sp_granules_kernel<0, T>); break;
        case 1: granules(sp_granules_kernel<1, T>); break;
        case 2: granules(sp_granules_kernel<2, T>); break;
        case 3: granules(sp_granules_kernel<3, T>); break;
        case 4: granules(sp_granules_kernel<4, T>); break;
        case 5: granules(sp_granules_kernel<5, T>); break;
        default: granules(sp_granules_kernel<6, T>);
        }
        hipLaunchKernelGGL(sp_draw_kernel<T>, dim3(rows), dim3(SP_NT), 0, st, a);
        if (a.rows) {
            hipLaunchKernelGGL(sp_count_kernel<T>, dim3((unsigned)ks_ceil_div(a.C, a.span), rows), dim3(SP_NT2), 0, st, a);
            hipLaunchKernelGGL(sp_keep_kernel<T>, dim3((unsigned)ks_ceil_div(a.C, SP_SPAN3), rows), dim3(SP_NT3), 0, st, a);
        }
        if (a.C > SP_CAND) hipLaunchKernelGGL(sp_many_kernel<T>, dim3(rows), dim3(SP_NT2), 0, st, a); // else LDS holds all
    }
}

extern "C" int class_sample(const void *logits, int64_t ldl, int dtype, int64_t C, int B, const float *u, const float *temperature,
                            const int32_t *top_k, const float *top_p, const float *min_p, int32_t *ids, float *logprob, void *ws,
                            size_t ws_bytes, void *stream) {
    SpArgs a;
    if (!logits || !u || !ids || !ws || ldl < C || !sp_sizes(C, B, a)) return KS_INVALID_ARG;
    if (dtype != KS_DTYPE_BF16 && dtype != KS_DTYPE_FP32) return KS_INVALID_ARG;
    if ((uintptr_t)logits % (dtype == KS_DTYPE_FP32 ? 4 : 2) || (uintptr_t)ws % 256) return KS_INVALID_ARG;
    if (((uintptr_t)u | (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)ids | (uintptr_t)logprob) % 4) return KS_INVALID_ARG;
    if (ws_bytes < class_sample_workspace(C, B)) return KS_WORKSPACE_TOO_SMALL;
    KsArena arena(ws);
    sp_places(arena, B, a);
    a.logits = logits; a.ldl = ldl;
    a.u = u; a.temperature = temperature; a.top_p = top_p; a.min_p = min_p; a.top_k = top_k;
    a.ids = ids; a.logprob = logprob;
    if (dtype == KS_DTYPE_FP32) sp_sample<float>(a, B, (hipStream_t)stream);
    else sp_sample<uint16_t>(a, B, (hipStream_t)stream);
    KS_LAUNCH_CHECK();
    return KS_OK;
}
