// Log probabilities of given tokens with entropy and top alternatives, in one pass over the logits.
//
// In powers of two, against a whole number c near max x * log2(e): y = x log2(e) - c (one rounding), S = sum 2^y, T = sum 2^y y;
// log p(i) = ln2 (y_i - log2 S), entropy = ln2 (log2 S - T / S). Every thread keeps its own (c, S, T) in fp32 and rescales when its
// maximum grows (a power of two, exact; once per slice, whose maximum is known before its exponentials); parts are joined in a fixed
// order. Two elements at a time (fma.f32x2): 4.5 instructions each, of which one is the exponential (16 per clock and SM).
//
// The top n: the first slice of a CTA's part of a row gives a list of its n best (value, id) keys (collect). Later slices push
// what reaches the list's n-th best into shared memory without meeting; after slices 2, 4, 8 ... the list is made anew
// from both by counting. A thread finds its candidates by the maxima of its 16-byte vectors and reads those vectors again.
//
// Slices are as in verify.cu: a launch has up to two CTAs per SM, each takes a contiguous range of slices and publishes a part
// for every row that it meets; the CTA that completes a row joins the row's parts and writes its outputs.
#include "logprobs.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace fmtp {

namespace {

constexpr uint32_t kDevBadToken = 0x1u, kDevAllNan = 0x10u;
constexpr int kLpThreads = 256, kLpCtasPerSm = 2, kLpWarps = kLpThreads / 32;
constexpr int kLpCap = kLpMaxTop * 64;               // candidates of a slice: n threads' elements at most
constexpr float kLpLow = -2097152.f;                 // lower values count as this in the sums: as nothing, but for rows that finish() adds up anew
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLpMaxRef = 4194304.f, kLpMinRef = -3000000.f;        // references c outside: likewise

// Key of a value: larger value, larger key; minus infinity and NaN have the same, the smallest (1).
__device__ __forceinline__ uint32_t lp_order(float v) { return v > -INFINITY ? float_order_key(v + 0.0f) : 1u; }       // + 0: -0 and +0 are one value
__device__ __forceinline__ float lp_value(uint32_t k) { return k <= 1u ? -INFINITY : __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k); }

template <bool F32> struct Elem;
template <> struct Elem<false> {
    typedef bf16_t T;
    static constexpr int N = 8;                      // elements of a 16-byte vector
    static constexpr uint32_t NONE = 0xff80ff80u;    // minus infinity
    static __device__ __forceinline__ float at(const uint4 &v, int i) {
        const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return (i & 1) ? bf16hi_f32(w) : bf16lo_f32(w);
    }
    static __device__ __forceinline__ float one(const T *p) { return bf16bits_f32(*p); }
    // NaN, minus infinity and what is below it become kLpLow
    static __device__ __forceinline__ void clean(uint4 &v) {
        constexpr uint32_t low = 0xca00ca00u;
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.x) : "r"(low));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.y) : "r"(low));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.z) : "r"(low));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.w) : "r"(low));
    }
    static __device__ __forceinline__ float vec_max(const uint4 &v) {        // of a cleaned vector
        uint32_t a, b;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
        return fmaxf(bf16lo_f32(a), bf16hi_f32(a));
    }
};
template <> struct Elem<true> {
    typedef float T;
    static constexpr int N = 4;
    static constexpr uint32_t NONE = 0xff800000u;
    static __device__ __forceinline__ float at(const uint4 &v, int i) { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
    static __device__ __forceinline__ float one(const T *p) { return *p; }
    static __device__ __forceinline__ void clean(uint4 &v) {
        constexpr float low = kLpLow;
        v.x = __float_as_uint(fmaxf(__uint_as_float(v.x), low)); v.y = __float_as_uint(fmaxf(__uint_as_float(v.y), low));
        v.z = __float_as_uint(fmaxf(__uint_as_float(v.z), low)); v.w = __float_as_uint(fmaxf(__uint_as_float(v.w), low));
    }
    static __device__ __forceinline__ float vec_max(const uint4 &v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
};

struct LpArgs {
    LpCall c;
    int spr;                                         // slices per row
    long long n_items;                               // slices of all rows
};

struct LpShared {
    unsigned long long cand[kLpCap], list[kLpMaxTop], next[kLpMaxTop], best[kLpThreads];
    float red[3][kLpWarps];
    uint32_t warp_bound[kLpWarps];
    int n_cand, n_list, last;
    unsigned long long bound;
};

__device__ __forceinline__ void push(LpShared &sh, unsigned long long key) {
    const int at = atomicAdd(&sh.n_cand, 1);
    if (at < kLpCap) sh.cand[at] = key;
}

// The n best of the candidates and of the list become the list, best first; no candidates are left. Every thread calls it, with all
// candidates visible.
__device__ __forceinline__ void rank(LpShared &sh, int n) {
    const int tid = threadIdx.x, nc = min(sh.n_cand, kLpCap), nl = sh.n_list, all = nc + nl;
    for (int i = tid; i < all; i += kLpThreads) {    // keys differ: an entry's place is the number of larger ones
        const unsigned long long key = i < nc ? sh.cand[i] : sh.list[i - nc];
        int above = 0;
#pragma unroll 4
        for (int u = 0; u < nc; ++u) above += sh.cand[u] > key;
#pragma unroll 4
        for (int u = 0; u < nl; ++u) above += sh.list[u] > key;
        if (above < n) sh.next[above] = key;
    }
    __syncthreads();
    const int nn = min(all, n);
    if (tid < nn) sh.list[tid] = sh.next[tid];
    if (tid == 0) { sh.n_list = nn; sh.n_cand = 0; }
    __syncthreads();
}

// Takes up to n best of the threads' elements and of the list into the list, whatever the elements are. each(bound, f) hands f the
// thread's elements as (value, id) keys, all whose order key is `bound` or more at least; the order key of the thread's largest value
// is `top` at most and `sure` at least (0: it has no element). Every thread calls it, with no candidates left over.
template <typename Each>
__device__ __forceinline__ void collect(LpShared &sh, int n, uint32_t top, uint32_t sure, Each each) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned long long floor_key = sh.n_list == n ? sh.list[n - 1] : 0ull;             // an element has to be above this
    const bool may = top != 0u && top >= (uint32_t)(floor_key >> 32), whole = __all_sync(0xffffffffu, may);
    const int cnt = __syncthreads_count(may);
    if (cnt == 0) return;
    // Lower bound of the n-th best: of the f warps all of whose lanes may have something, the smallest of their ceil(n / f)-th
    // largest maxima: n threads at least hold a value as large
    uint32_t bound = 0u;
    if (cnt > n) {
        const int full = __syncthreads_count(whole) / 32;
        if (full > 0) {
            const int rounds = (n + full - 1) / full;
            uint32_t k = may ? sure : 0u, b = 0xffffffffu;
            if (whole)
                for (int r = 0; r < rounds; ++r) {
                    b = __reduce_max_sync(0xffffffffu, k);
                    const uint32_t who = __ballot_sync(0xffffffffu, k == b);
                    if (lane == __ffs(who) - 1) k = 0u;
                }
            if (lane == 0) sh.warp_bound[warp] = b;
            __syncthreads();
            bound = sh.warp_bound[0];
#pragma unroll
            for (int w = 1; w < kLpWarps; ++w) bound = min(bound, sh.warp_bound[w]);
        }
    }
    if (may && top >= bound)
        each(bound, [&](unsigned long long key) { if ((uint32_t)(key >> 32) >= bound && key > floor_key) push(sh, key); });
    __syncthreads();
    if (sh.n_cand > kLpCap) {
        // Too many equal values (or no warp to take a bound from): the exact n-th best of the threads' own best keys bounds the
        // candidates to the elements of n threads
        __syncthreads();
        unsigned long long mine = 0ull;
        if (may) each(0u, [&](unsigned long long key) { mine = key > mine ? key : mine; });
        sh.best[tid] = mine;
        if (tid == 0) { sh.n_cand = 0; sh.bound = 0ull; }
        __syncthreads();
        int above = 0;
        for (int u = 0; u < kLpThreads; ++u) above += sh.best[u] > mine;
        if (mine != 0ull && above == n - 1) sh.bound = mine;
        __syncthreads();
        const unsigned long long lo = sh.bound;
        if (mine != 0ull && mine >= lo)
            each((uint32_t)(lo >> 32), [&](unsigned long long key) { if (key >= lo && key > floor_key) push(sh, key); });
        __syncthreads();
    }
    rank(sh, n);
}

// Sum over the block in a fixed order, and maximum; every thread gets them.
__device__ __forceinline__ float lp_sum(float v, float *red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kLpWarps; ++w) t += red[w];
    return t;
}
__device__ __forceinline__ float lp_max(float v, float *red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = red[0];
#pragma unroll
    for (int w = 1; w < kLpWarps; ++w) t = fmaxf(t, red[w]);
    return t;
}

__device__ __forceinline__ float lp_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 values at a time.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(f32x2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <bool F32, int NV>
__global__ void __launch_bounds__(kLpThreads, kLpCtasPerSm) logprobs_kernel(const __grid_constant__ LpArgs a) {
    chain_release();
    chain_wait();
    typedef Elem<F32> El;
    typedef typename El::T T;
    constexpr int EV = El::N, SLICE = kLpThreads * NV * EV;
    __shared__ LpShared sh;
    const LpCall &c = a.c;
    const int tid = threadIdx.x, V = c.V, n = c.top;
    const T *logits = static_cast<const T *>(c.logits);
    const long long G = gridDim.x, N = a.n_items;
    const long long i0 = (long long)blockIdx.x * N / G, i1 = ((long long)blockIdx.x + 1) * N / G;

    // Slice s of a row starts s * SLICE elements behind the 16-byte boundary at or below the row; a vector that lies across one of
    // the row's ends is put together from single elements, minus infinity for what is outside
    auto row_ptr = [&](int row) -> const T * { return logits + (long long)row * c.ld; };
    auto first_of = [&](int row, int slice) -> int {          // the thread's first element in a slice
        return slice * SLICE + tid * EV - (int)((reinterpret_cast<uintptr_t>(row_ptr(row)) & 15u) / sizeof(T));
    };
    auto load_vec = [&](const T *p, int e) -> uint4 {
        if (e >= 0 && e + EV <= V) return ldnc128(p + e);
        uint32_t w[4] = {El::NONE, El::NONE, El::NONE, El::NONE};
        if (e + EV > 0 && e < V) {
#pragma unroll
            for (int q = 0; q < EV; ++q)
                if ((unsigned)(e + q) < (unsigned)V) {
                    if constexpr (F32) w[q] = __float_as_uint(p[e + q]);
                    else w[q >> 1] = (q & 1) ? (w[q >> 1] & 0xffffu) | ((uint32_t)p[e + q] << 16) : (w[q >> 1] & 0xffff0000u) | p[e + q];
                }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    };
    auto load = [&](int row, int slice, uint4 (&v)[NV]) {
        const T *p = row_ptr(row);
        const int e0 = first_of(row, slice);
        if (__all_sync(0xffffffffu, e0 >= 0 && e0 + (NV - 1) * kLpThreads * EV + EV <= V)) {
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = ldnc128(p + e0 + j * kLpThreads * EV);
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = load_vec(p, e0 + j * kLpThreads * EV);
        }
    };
    // the elements of the thread's vectors in `mask` (read once more) whose order key is `bound` or more
    auto scan = [&](int row, int slice, uint32_t mask, uint32_t bound, auto f) {
        const T *p = row_ptr(row);
        const int e0 = first_of(row, slice);
        while (mask) {
            const int j = __ffs(mask) - 1, e = e0 + j * kLpThreads * EV;
            mask &= mask - 1;
            const uint4 v = load_vec(p, e);
#pragma unroll
            for (int q = 0; q < EV; ++q) {
                const float x = El::at(v, q);
                const uint32_t k = lp_order(x);
                if (k >= bound && (unsigned)(e + q) < (unsigned)V) f(((unsigned long long)k << 32) | (0xffffffffu - (uint32_t)(e + q)));
            }
        }
    };
    // which of the vectors hold a value whose order key is `bound` or more, or might (all of them where that is hard to tell)
    auto vectors = [&](const uint4 (&v)[NV], uint32_t bound) -> uint32_t {
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            uint4 x = v[j];
            El::clean(x);
            mask |= (lp_order(El::vec_max(x)) >= bound ? 1u : 0u) << j;
        }
        return mask;
    };
    // collect() on a slice in registers
    auto collect_slice = [&](int row, int slice, const uint4 (&v)[NV]) {
        float bm = kLpLow;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            uint4 x = v[j];
            El::clean(x);
            bm = fmaxf(bm, El::vec_max(x));
        }
        const bool some = first_of(row, slice) < V;          // (a row's first vector may begin before the row)
        collect(sh, n, some ? lp_order(bm) : 0u, !some ? 0u : bm > kLpLow ? lp_order(bm) : 1u,
                [&](uint32_t bound, auto f) { scan(row, slice, vectors(v, bound), bound, f); });
    };

    uint4 cur[NV], nxt[NV];
    int row = (int)(i0 / a.spr), slice = (int)(i0 - (long long)row * a.spr);
    if (i0 < i1) load(row, slice, cur);
    float ref = -1e30f;                              // the thread's part of the current row
    f32x2 S2 = 0ull, T2 = 0ull;
    int k = 0, slice0 = slice;                       // slices of the row so far, the first one
    float tau = 0.f;                                 // the list's n-th best value once there is one
    if (tid == 0) { sh.n_list = 0; sh.n_cand = 0; }
    __syncthreads();
    for (long long item = i0; item < i1; ++item) {
        int nrow = row, nslice = slice + 1;
        if (nslice == a.spr) { nslice = 0; ++nrow; }
        if (item + 1 < i1) load(nrow, nslice, nxt);  // the next slice's loads go out before this one's values are used
        const bool ends = nrow != row || item + 1 == i1;
        ++k;
        // ---- sums
        uint32_t hits = 0;
        {
            uint4 x[NV];
            float bm = kLpLow;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                x[j] = cur[j];
                El::clean(x[j]);
                const float vm = El::vec_max(x[j]);
                hits |= (vm >= tau ? 1u : 0u) << j;
                bm = fmaxf(bm, vm);
            }
            const float want = rintf(bm * kLog2e);
            if (want > ref) {
                const float d = ref - want, f = lp_exp2(d);
                float s0, s1, t0, t1;
                unpair(S2, s0, s1);
                unpair(T2, t0, t1);
                T2 = pair(f * fmaf(s0, d, t0), f * fmaf(s1, d, t1));
                S2 = pair(f * s0, f * s1);
                ref = want;
            }
            const f32x2 L2 = pair(kLog2e, kLog2e), R2 = pair(-ref, -ref);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int q = 0; q < EV; q += 2) {
                    const f32x2 y = fma2(pair(El::at(x[j], q), El::at(x[j], q + 1)), L2, R2);
                    float y0, y1;
                    unpair(y, y0, y1);
                    const f32x2 e = pair(lp_exp2(y0), lp_exp2(y1));
                    S2 = add2(S2, e);
                    T2 = fma2(e, y, T2);
                }
        }
        // ---- top candidates (of the values as they are)
        if (n > 0) {
            if (k == 1) collect_slice(row, slice, cur);
            else if (hits) scan(row, slice, hits, sh.n_list == n ? (uint32_t)(sh.list[n - 1] >> 32) : 0u, [&](unsigned long long key) { push(sh, key); });
            if (k > 1 && ((k & (k - 1)) == 0 || ends)) {
                __syncthreads();
                if (sh.n_cand <= kLpCap) rank(sh, n);
                else {                               // every slice beats the ones before by far: over again, slice by slice
                    __syncthreads();
                    if (tid == 0) { sh.n_cand = 0; sh.n_list = 0; }
                    __syncthreads();
                    for (int q = slice0; q <= slice; ++q) {
                        load(row, q, cur);
                        collect_slice(row, q, cur);
                    }
                }
            }
            // a list that is not full (a part shorter than n) takes everything
            if ((k & (k - 1)) == 0) tau = sh.n_list == n ? lp_value((uint32_t)(sh.list[n - 1] >> 32)) : -INFINITY;
        }
        if (ends) {
            // ---- this CTA's part of the row is done
            const long long r0 = (long long)row * a.spr;
            const int c_first = (int)(((r0 + 1) * G - 1) / N), c_last = (int)(((r0 + a.spr) * G - 1) / N), parts = c_last - c_first + 1;
            float R = lp_max(ref, sh.red[0]);
            float Sr, Tr;
            {
                const float d = ref - R, f = lp_exp2(d);
                float s0, s1, t0, t1;
                unpair(S2, s0, s1);
                unpair(T2, t0, t1);
                Tr = lp_sum(f * fmaf(s0 + s1, d, t0 + t1), sh.red[1]);
                Sr = lp_sum(f * (s0 + s1), sh.red[2]);
            }
            bool finish = parts == 1;
            if (!finish) {
                LpPart *p = c.parts + row + blockIdx.x;
                if (tid == 0) { p->m = R; p->s = Sr; p->t = Tr; }
                if (tid < n) p->top[tid] = tid < sh.n_list ? sh.list[tid] : 0ull;
                __threadfence();
                __syncthreads();
                if (tid == 0) {
                    sh.last = atomicAdd(c.counters + row, 1u) == (uint32_t)(parts - 1);
                    if (sh.last) c.counters[row] = 0u;
                    sh.n_list = 0;
                }
                __syncthreads();
                finish = sh.last;
                if (finish) {
                    __threadfence();
                    const LpPart *p0 = c.parts + row + c_first;
                    float mm = -1e30f;
                    for (int i = tid; i < parts; i += kLpThreads) mm = fmaxf(mm, ldcg_f32(&p0[i].m));
                    R = lp_max(mm, sh.red[0]);
                    float s = 0.f, t = 0.f;
                    for (int i = tid; i < parts; i += kLpThreads) {
                        const float ps = ldcg_f32(&p0[i].s), pt = ldcg_f32(&p0[i].t), d = ldcg_f32(&p0[i].m) - R, f = lp_exp2(d);
                        s += f * ps;
                        t += f * fmaf(ps, d, pt);
                    }
                    Sr = lp_sum(s, sh.red[1]);
                    Tr = lp_sum(t, sh.red[2]);
                    if (n > 0) {
                        const int keys = parts * n;
                        uint32_t top = 0u;
                        for (int i = tid; i < keys; i += kLpThreads) top = max(top, (uint32_t)(ldcg_u64(&p0[i / n].top[i % n]) >> 32));
                        collect(sh, n, top, top, [&](uint32_t bound, auto f) {
                            for (int i = tid; i < keys; i += kLpThreads) {
                                const unsigned long long key = ldcg_u64(&p0[i / n].top[i % n]);
                                if (key && (uint32_t)(key >> 32) >= bound) f(key);
                            }
                        });
                    }
                }
            }
            if (finish) {
                const T *p = row_ptr(row);
                // Rows whose maximum is too far from zero for the sums above (or infinite) are added up anew, against the maximum itself
                const bool far = !(R > kLpMinRef && R < kLpMaxRef);
                bool nothing = false;
                float M = 0.f;
                if (far) {
                    float mx = -INFINITY;
                    for (int i = tid; i < V; i += kLpThreads) mx = fmaxf(mx, El::one(p + i));
                    M = lp_max(mx, sh.red[0]);
                    nothing = M == -INFINITY;
                    float s = 0.f, t = 0.f;
                    for (int i = tid; i < V; i += kLpThreads) {
                        const float x = El::one(p + i), y = (x - M) * kLog2e;
                        if (x == M) s += 1.f;
                        else if (y > -200.f) { s += lp_exp2(y); t = fmaf(lp_exp2(y), y, t); }
                    }
                    Sr = lp_sum(s, sh.red[1]);
                    Tr = lp_sum(t, sh.red[2]);
                }
                const float lgS = log2f(Sr);
                auto logprob = [&](float x) -> float {
                    if (nothing || !(x > -INFINITY)) return -INFINITY;
                    if (far) return (x == M ? 0.f : x - M) - kLn2 * lgS;
                    return x < kLpLow ? x - kLn2 * (R + lgS) : kLn2 * (fmaf(x, kLog2e, -R) - lgS);
                };
                if (tid == 0) {
                    if (nothing) atomicOr(c.status, kDevAllNan);
                    if (c.out_logprob) {
                        int tok = c.tokens[row];
                        if ((unsigned)tok >= (unsigned)V) { atomicOr(c.status, kDevBadToken); tok = 0; }
                        c.out_logprob[row] = logprob(El::one(p + tok));
                    }
                    if (c.out_entropy) c.out_entropy[row] = nothing ? 0.f : fmaxf(kLn2 * (lgS - Tr / Sr), 0.f);
                }
                if (tid < n) {                       // (V >= n: the list is full)
                    const unsigned long long key = sh.list[tid];
                    const size_t o = (size_t)row * n + tid;
                    if (c.out_ids) c.out_ids[o] = (int32_t)argmax_key_id(key);
                    if (c.out_tops) c.out_tops[o] = logprob(lp_value((uint32_t)(key >> 32)));
                }
            }
            __syncthreads();
            if (tid == 0) { sh.n_list = 0; sh.n_cand = 0; }
            __syncthreads();
            ref = -1e30f;
            S2 = T2 = 0ull;
            k = 0;
            slice0 = nslice;
            tau = 0.f;
        }
        row = nrow;
        slice = nslice;
#pragma unroll
        for (int j = 0; j < NV; ++j) cur[j] = nxt[j];
    }
}

}  // namespace

int logprobs_slots(int n_sm) { return kLpMaxRows + n_sm * kLpCtasPerSm + 1; }

int logprobs_launch(const LpCall &c, cudaStream_t st) {
    LpArgs a{};
    a.c = c;
    const int ev = c.f32 ? 4 : 8;
    const long long ctas = (long long)c.n_sm * kLpCtasPerSm;
    auto per_row = [&](int nv) { const int e = kLpThreads * nv * ev; return (int)(((long long)c.V + ev - 1 + e - 1) / e); };   // a row may start ev - 1 elements after a boundary
    int nv = 8;
    while (nv > 1 && (long long)c.rows * per_row(nv) < ctas) nv >>= 1;
    a.spr = per_row(nv);
    a.n_items = (long long)c.rows * a.spr;
    const int grid = (int)(a.n_items < ctas ? a.n_items : ctas);
    void (*kern)(LpArgs);
    if (c.f32) kern = nv == 8 ? logprobs_kernel<true, 8> : nv == 4 ? logprobs_kernel<true, 4> : nv == 2 ? logprobs_kernel<true, 2> : logprobs_kernel<true, 1>;
    else kern = nv == 8 ? logprobs_kernel<false, 8> : nv == 4 ? logprobs_kernel<false, 4> : nv == 2 ? logprobs_kernel<false, 2> : logprobs_kernel<false, 1>;
    return (int)launch_chained(kern, dim3(grid), dim3(kLpThreads), 0, st, a);
}

}  // namespace fmtp
