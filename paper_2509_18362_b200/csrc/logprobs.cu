// Log probabilities of given tokens with entropy and top alternatives, in one pass over the logits.
//
// With m = max x, S = sum e^(x - m), T = sum e^(x - m) (x - m): log p(i) = (x_i - m) - ln S, entropy = ln S - T / S. Every thread
// keeps its own running (m, S, T) in fp32, rescaled when its maximum grows (once per slice, the slice's maximum is known before
// its exponentials); parts are joined in a fixed order.
//
// The top n: a CTA keeps the n best (value, id) keys of its part so far. A slice can only matter where a thread's maximum reaches
// the n-th best, which after the first slices is rare, so the usual cost is one comparison per thread and slice. Where it happens
// the threads that can contribute push their elements above a lower bound of the slice's own n-th best (see collect), and
// the list is ranked by counting.
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
constexpr float kLpFar = 1e30f;                      // beyond: see finish

// Key of a value: larger value, larger key; minus infinity and NaN have the same, the smallest (1).
__device__ __forceinline__ uint32_t lp_order(float v) { return v > -INFINITY ? float_order_key(v + 0.0f) : 1u; }       // + 0: -0 and +0 are one value
__device__ __forceinline__ float lp_value(uint32_t k) { return k <= 1u ? -INFINITY : __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ unsigned long long lp_key(float v, int id) { return ((unsigned long long)lp_order(v) << 32) | (0xffffffffu - (uint32_t)id); }

template <bool F32> struct Elem;
template <> struct Elem<false> {
    typedef bf16_t T;
    static constexpr int N = 8;                      // elements of a 16-byte vector
    static constexpr uint32_t NONE = 0xff80ff80u;    // minus infinity
    static constexpr float LOWEST = -3.3895313892515355e38f;
    static __device__ __forceinline__ float at(const uint4 &v, int i) {
        const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return (i & 1) ? bf16hi_f32(w) : bf16lo_f32(w);
    }
    static __device__ __forceinline__ float one(const T *p) { return bf16bits_f32(*p); }
    // NaN and minus infinity become the type's lowest number
    static __device__ __forceinline__ void clean(uint4 &v) {
        constexpr uint32_t low = 0xff7fff7fu;
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
    static constexpr float LOWEST = -3.4028234663852886e38f;
    static __device__ __forceinline__ float at(const uint4 &v, int i) { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
    static __device__ __forceinline__ float one(const T *p) { return *p; }
    static __device__ __forceinline__ void clean(uint4 &v) {
        constexpr float low = LOWEST;
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

// Takes up to n best of the threads' elements and of the list into the list. The threads' elements are what each(f) hands to f as
// (value, id) keys; the order key of the thread's largest value is `top` at most and `sure` at least (0: it has no element). Every
// thread calls it.
template <typename Each>
__device__ __forceinline__ void collect(LpShared &sh, int n, uint32_t top, uint32_t sure, Each each) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned long long floor_key = sh.n_list == n ? sh.list[n - 1] : 0ull;             // an element has to be above this
    const bool may = top != 0u && top >= (uint32_t)(floor_key >> 32);
    const int cnt = __syncthreads_count(may);
    if (cnt == 0) return;
    // Lower bound of the n-th best: of the f warps all of whose lanes may have something, the smallest of their ceil(n / f)-th
    // largest maxima: n threads at least hold a value as large
    uint32_t bound = 0u;
    if (cnt > n) {
        const int full = __syncthreads_count(__all_sync(0xffffffffu, may)) / 32;
        if (full > 0) {
            const int rounds = (n + full - 1) / full;
            uint32_t k = may ? sure : 0u, b = 0xffffffffu;
            if (__all_sync(0xffffffffu, may))
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
    if (tid == 0) sh.n_cand = 0;
    __syncthreads();
    if (may && top >= bound)
        each([&](unsigned long long key) {
            if ((uint32_t)(key >> 32) >= bound && key > floor_key) {
                const int at = atomicAdd(&sh.n_cand, 1);
                if (at < kLpCap) sh.cand[at] = key;
            }
        });
    __syncthreads();
    if (sh.n_cand > kLpCap) {
        // Too many equal values (or one warp with nothing near): the exact n-th best of the threads' own best keys bounds the
        // candidates to the elements of n threads
        unsigned long long mine = 0ull;
        if (may) each([&](unsigned long long key) { mine = key > mine ? key : mine; });
        sh.best[tid] = mine;
        if (tid == 0) { sh.n_cand = 0; sh.bound = 0ull; }
        __syncthreads();
        int above = 0;
        for (int u = 0; u < kLpThreads; ++u) above += sh.best[u] > mine;
        if (mine != 0ull && above == n - 1) sh.bound = mine;
        __syncthreads();
        const unsigned long long lo = sh.bound;
        if (mine != 0ull && mine >= lo)
            each([&](unsigned long long key) {
                if (key >= lo && key > floor_key) {
                    const int at = atomicAdd(&sh.n_cand, 1);
                    if (at < kLpCap) sh.cand[at] = key;
                }
            });
        __syncthreads();
    }
    const int nc = min(sh.n_cand, kLpCap), nl = sh.n_list, all = nc + nl;
    for (int i = tid; i < all; i += kLpThreads) {    // keys differ: an entry's place is the number of larger ones
        const unsigned long long key = i < nc ? sh.cand[i] : sh.list[i - nc];
        int above = 0;
        for (int u = 0; u < nc; ++u) above += sh.cand[u] > key;
        for (int u = 0; u < nl; ++u) above += sh.list[u] > key;
        if (above < n) sh.next[above] = key;
    }
    __syncthreads();
    const int nn = min(all, n);
    if (tid < nn) sh.list[tid] = sh.next[tid];
    if (tid == 0) sh.n_list = nn;
    __syncthreads();
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

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float lp_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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
    auto offset_of = [&](const T *p) -> int { return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T)); };
    auto load = [&](int row, int slice, uint4 (&v)[NV]) {
        const T *p = row_ptr(row);
        const int off = offset_of(p);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = slice * SLICE + (j * kLpThreads + tid) * EV - off;      // the vector's first element
            if (e >= 0 && e + EV <= V) v[j] = ldnc128(p + e);
            else {
                uint32_t w[4] = {El::NONE, El::NONE, El::NONE, El::NONE};
                if (e + EV > 0 && e < V) {
#pragma unroll
                    for (int q = 0; q < EV; ++q)
                        if ((unsigned)(e + q) < (unsigned)V) {
                            if constexpr (F32) w[q] = __float_as_uint(p[e + q]);
                            else w[q >> 1] = (q & 1) ? (w[q >> 1] & 0xffffu) | ((uint32_t)p[e + q] << 16) : (w[q >> 1] & 0xffff0000u) | p[e + q];
                        }
                }
                v[j] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    };

    uint4 cur[NV], nxt[NV];
    int row = (int)(i0 / a.spr), slice = (int)(i0 - (long long)row * a.spr);
    if (i0 < i1) load(row, slice, cur);
    float m = -INFINITY, S = 0.f, Tt = 0.f;          // the thread's part of the current row
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    for (long long item = i0; item < i1; ++item) {
        int nrow = row, nslice = slice + 1;
        if (nslice == a.spr) { nslice = 0; ++nrow; }
        if (item + 1 < i1) load(nrow, nslice, nxt);  // the next slice's loads go out before this one's values are used
        // ---- sums
        float bm = -INFINITY;
        {
            uint4 x[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                x[j] = cur[j];
                El::clean(x[j]);
                bm = fmaxf(bm, El::vec_max(x[j]));
            }
            if (bm > m) {
                const float d = m - bm, f = lp_exp2(d * kLog2e);                  // (0 for the first slice)
                Tt = f > 0.f ? f * (Tt + S * d) : 0.f;
                S *= f;
                m = bm;
            }
            float s0 = 0.f, s1 = 0.f, t0 = 0.f, t1 = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int q = 0; q < EV; q += 2) {
                    const float d0 = El::at(x[j], q) - m, d1 = El::at(x[j], q + 1) - m;
                    const float e0 = lp_exp2(d0 * kLog2e), e1 = lp_exp2(d1 * kLog2e);
                    s0 += e0; s1 += e1;
                    t0 = fmaf(e0, d0, t0); t1 = fmaf(e1, d1, t1);
                }
            S += s0 + s1;
            Tt += t0 + t1;
        }
        // ---- top candidates (of the values as they are: minus infinity is below the lowest number)
        if (n > 0) {
            const int first = slice * SLICE + tid * EV - offset_of(row_ptr(row));
            const bool some = first < V;             // (a row's first vector may begin before the row)
            collect(sh, n, some ? lp_order(bm) : 0u, !some ? 0u : bm > El::LOWEST ? lp_order(bm) : 1u, [&](auto f) {
#pragma unroll 1
                for (int j = 0; j < NV; ++j) {
                    uint4 v = cur[0];
#pragma unroll
                    for (int u = 1; u < NV; ++u) if (u == j) v = cur[u];
#pragma unroll
                    for (int q = 0; q < EV; ++q) {
                        const int id = first + j * kLpThreads * EV + q;
                        if ((unsigned)id < (unsigned)V) f(lp_key(El::at(v, q), id));
                    }
                }
            });
        }
        if (nrow != row || item + 1 == i1) {
            // ---- this CTA's part of the row is done
            const long long r0 = (long long)row * a.spr;
            const int c_first = (int)(((r0 + 1) * G - 1) / N), c_last = (int)(((r0 + a.spr) * G - 1) / N), parts = c_last - c_first + 1;
            float M = lp_max(m, sh.red[0]);
            const float f = m > -INFINITY ? lp_exp2((m - M) * kLog2e) : 0.f;
            const float dm = m - M;
            float Tr = lp_sum(S > 0.f && f > 0.f ? f * (Tt + S * dm) : 0.f, sh.red[1]);
            float Sr = lp_sum(S > 0.f ? f * S : 0.f, sh.red[2]);
            bool finish = parts == 1;
            if (!finish) {
                LpPart *p = c.parts + row + blockIdx.x;
                if (tid == 0) { p->m = M; p->s = Sr; p->t = Tr; }
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
                    float mm = -INFINITY;
                    for (int i = tid; i < parts; i += kLpThreads) mm = fmaxf(mm, ldcg_f32(&p0[i].m));
                    M = lp_max(mm, sh.red[0]);
                    float s = 0.f, t = 0.f;
                    for (int i = tid; i < parts; i += kLpThreads) {
                        const float pm = ldcg_f32(&p0[i].m), ps = ldcg_f32(&p0[i].s), pt = ldcg_f32(&p0[i].t);
                        const float d = pm - M, e = pm > -INFINITY ? lp_exp2(d * kLog2e) : 0.f;
                        s += e * ps;
                        t += e > 0.f ? e * (pt + ps * d) : 0.f;
                    }
                    Sr = lp_sum(s, sh.red[1]);
                    Tr = lp_sum(t, sh.red[2]);
                    if (n > 0) {
                        const int keys = parts * n;
                        uint32_t top = 0u;
                        for (int i = tid; i < keys; i += kLpThreads) top = max(top, (uint32_t)(ldcg_u64(&p0[i / n].top[i % n]) >> 32));
                        collect(sh, n, top, top, [&](auto f2) {
                            for (int i = tid; i < keys; i += kLpThreads) {
                                const unsigned long long key = ldcg_u64(&p0[i / n].top[i % n]);
                                if (key) f2(key);
                            }
                        });
                    }
                }
            }
            if (finish) {
                const T *p = row_ptr(row);
                // Far from zero two different values are so far apart that only the largest count; there a sum of its own, which also
                // tells the type's lowest number from minus infinity and takes an infinite maximum
                bool nothing = false;
                if (!(fabsf(M) < kLpFar)) {
                    float mx = -INFINITY;
                    for (int i = tid; i < V; i += kLpThreads) mx = fmaxf(mx, El::one(p + i));
                    M = lp_max(mx, sh.red[0]);
                    int cnt = 0;
                    for (int i = tid; i < V; i += kLpThreads) cnt += El::one(p + i) == M;
                    Sr = lp_sum((float)cnt, sh.red[1]);
                    Tr = 0.f;
                    nothing = M == -INFINITY;
                }
                const float lnS = logf(Sr);
                auto logprob = [&](float x) -> float { return nothing || !(x > -INFINITY) ? -INFINITY : x == M ? -lnS : (x - M) - lnS; };
                if (tid == 0) {
                    if (nothing) atomicOr(c.status, kDevAllNan);
                    if (c.out_logprob) {
                        int tok = c.tokens[row];
                        if ((unsigned)tok >= (unsigned)V) { atomicOr(c.status, kDevBadToken); tok = 0; }
                        c.out_logprob[row] = logprob(El::one(p + tok));
                    }
                    if (c.out_entropy) c.out_entropy[row] = nothing ? 0.f : fmaxf(lnS - Tr / Sr, 0.f);
                }
                if (tid < n) {                       // (V >= n: the list is full)
                    const unsigned long long key = sh.list[tid];
                    const size_t o = (size_t)row * n + tid;
                    if (c.out_ids) c.out_ids[o] = (int32_t)argmax_key_id(key);
                    if (c.out_tops) c.out_tops[o] = logprob(lp_value((uint32_t)(key >> 32)));
                }
            }
            __syncthreads();
            if (tid == 0) sh.n_list = 0;
            __syncthreads();
            m = -INFINITY; S = 0.f; Tt = 0.f;
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
