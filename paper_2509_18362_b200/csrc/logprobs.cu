// Log probabilities of given tokens with entropy and top alternatives, in one pass over the logits.
//
// In powers of two, against a whole number c near max x * log2(e): y = x log2(e) - c (one rounding), S = sum 2^y, T = sum 2^y y;
// log p(i) = ln2 (y_i - log2 S), entropy = ln2 (log2 S - T / S). Every thread keeps its own (c, S, T) in fp32 and rescales when its
// maximum grows (a power of two, exact; once per slice, whose maximum is known before its exponentials); parts are joined in a fixed
// order.
//
// The top n: the pass itself only keeps every strip's maximum (a strip: what one thread has of a row in a CTA's part of it, or one
// warp where parts are short). The CTA that completes a row finds a lower bound of the n-th best value from the maxima, which leaves
// a few more than n strips, and reads those again (from L2): their elements that reach the bound are ranked by counting. Where
// equal values leave too many strips, only the strips above the bound are read, and the bound's own ids are looked for from the
// row's beginning.
//
// Slices are as in verify.cu: a launch has up to four CTAs per SM, each takes a contiguous range of slices and publishes a part
// for every row that it meets; the CTA that completes a row joins the row's parts and writes its outputs.
#include "logprobs.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace fmtp {

namespace {

constexpr uint32_t kDevBadToken = 0x1u, kDevAllNan = 0x10u;
constexpr int kLpThreads = kLpStrips, kLpCtasPerSm = 4, kLpWarps = kLpThreads / 32;
constexpr int kLpCap = kLpMaxTop * 64;               // candidates that are ranked at once
constexpr int kLpStripCap = 256;                     // strips that are read again
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
    static __device__ __forceinline__ float vec_max(const uint4 &v) {        // (NaN only if nothing else)
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
    int warp_strips;                                 // strips are warps' (else threads'): parts are short and many
    long long n_items;                               // slices of all rows
};

struct LpShared {
    unsigned long long cand[kLpCap], list[kLpMaxTop], next[kLpMaxTop], best[kLpThreads], bound64;
    float red[3][kLpWarps];
    uint32_t warp_bound[kLpWarps], strip_key[kLpStripCap], bound;
    int strip[kLpStripCap];
    int n_cand, n_list, n_strip, last;
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

// Lower bound of the n-th largest of the threads' keys (0: none), n <= 32: the smallest, over the warps, of a warp's ceil(n / 8)-th
// largest key. Every thread calls it.
__device__ __forceinline__ uint32_t nth_bound(LpShared &sh, int n, uint32_t k) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t b = 0;
    for (int r = (n + kLpWarps - 1) / kLpWarps; r > 0; --r) {
        b = __reduce_max_sync(0xffffffffu, k);
        const uint32_t who = __ballot_sync(0xffffffffu, k == b);
        if (lane == __ffs(who) - 1) k = 0u;
    }
    if (lane == 0) sh.warp_bound[warp] = b;
    __syncthreads();
    b = sh.warp_bound[0];
#pragma unroll
    for (int w = 1; w < kLpWarps; ++w) b = min(b, sh.warp_bound[w]);
    return b;
}

// Takes the n best of a slice's elements and of the list into the list, whatever they are: the exact n-th best of the threads' best
// keys leaves n threads, whose elements are candidates. each(f) hands f the thread's elements as (value, id) keys.
template <typename Each>
__device__ __forceinline__ void collect(LpShared &sh, int n, Each each) {
    const int tid = threadIdx.x;
    unsigned long long mine = 0ull;
    each([&](unsigned long long key) { mine = key > mine ? key : mine; });
    sh.best[tid] = mine;
    if (tid == 0) { sh.n_cand = 0; sh.bound64 = 0ull; }
    __syncthreads();
    int above = 0;
    for (int u = 0; u < kLpThreads; ++u) above += sh.best[u] > mine;
    if (mine != 0ull && above == n - 1) sh.bound64 = mine;
    __syncthreads();
    const unsigned long long lo = sh.bound64;
    if (mine != 0ull && mine >= lo) each([&](unsigned long long key) { if (key >= lo) push(sh, key); });
    __syncthreads();
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
    // hands f the elements of the vector at element e as (value, id) keys
    auto keys_of = [&](const T *p, int e, auto f) {
        const uint4 v = load_vec(p, e);
#pragma unroll
        for (int q = 0; q < EV; ++q)
            if ((unsigned)(e + q) < (unsigned)V) f(((unsigned long long)lp_order(El::at(v, q)) << 32) | (0xffffffffu - (uint32_t)(e + q)));
    };
    const bool by_warp = a.warp_strips != 0;

    uint4 cur[NV];
    int row = (int)(i0 / a.spr), slice = (int)(i0 - (long long)row * a.spr);
    float ref = -1e30f, S0 = 0.f, S1 = 0.f, T0 = 0.f, T1 = 0.f;          // the thread's part of the current row
    float top = -INFINITY;                           // its largest value
    for (long long item = i0; item < i1; ++item) {
        load(row, slice, cur);
        int nrow = row, nslice = slice + 1;
        if (nslice == a.spr) { nslice = 0; ++nrow; }
        // ---- sums
        float bm = kLpLow;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            top = fmaxf(top, El::vec_max(cur[j]));
            El::clean(cur[j]);
        }
        bm = fmaxf(bm, top);
        const float want = rintf(bm * kLog2e);
        if (want > ref) {
            const float d = ref - want, f = lp_exp2(d);
            T0 = f * fmaf(S0, d, T0); T1 = f * fmaf(S1, d, T1);
            S0 *= f; S1 *= f;
            ref = want;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int q = 0; q < EV; q += 2) {
                const float y0 = fmaf(El::at(cur[j], q), kLog2e, -ref), y1 = fmaf(El::at(cur[j], q + 1), kLog2e, -ref);
                const float e0 = lp_exp2(y0), e1 = lp_exp2(y1);
                S0 += e0; S1 += e1;
                T0 = fmaf(e0, y0, T0); T1 = fmaf(e1, y1, T1);
            }
        if (nrow != row || item + 1 == i1) {
            // ---- this CTA's part of the row is done
            const long long r0 = (long long)row * a.spr;
            const int c_first = (int)(((r0 + 1) * G - 1) / N), c_last = (int)(((r0 + a.spr) * G - 1) / N), parts = c_last - c_first + 1;
            const size_t slot0 = (size_t)row + c_first;
            if (n > 0) {
                uint32_t k = lp_order(top);
                uint32_t *strips = c.strips + ((size_t)row + blockIdx.x) * kLpStrips;
                if (by_warp) {
                    k = __reduce_max_sync(0xffffffffu, k);
                    if ((tid & 31) == 0) strips[tid >> 5] = k;
                } else strips[tid] = k;
            }
            float R = lp_max(ref, sh.red[0]);
            const float dr = ref - R, fr = lp_exp2(dr);
            float Tr = lp_sum(fr * fmaf(S0 + S1, dr, T0 + T1), sh.red[1]);
            float Sr = lp_sum(fr * (S0 + S1), sh.red[2]);
            bool finish = parts == 1;
            if (!finish) {
                LpPart *p = c.parts + row + blockIdx.x;
                if (tid == 0) { p->m = R; p->s = Sr; p->t = Tr; }
                __threadfence();
                __syncthreads();
                if (tid == 0) {
                    sh.last = atomicAdd(c.counters + row, 1u) == (uint32_t)(parts - 1);
                    if (sh.last) c.counters[row] = 0u;
                }
                __syncthreads();
                finish = sh.last;
                if (finish) {
                    __threadfence();
                    const LpPart *p0 = c.parts + slot0;
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
                }
            }
            if (finish) {
                const T *p = row_ptr(row);
                const int off = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
                if (n > 0) {
                    __syncthreads();                 // (a row of one part: its strips are written)
                    // strips of the row, numbered part by part
                    const int PER = by_warp ? kLpWarps : kLpThreads;
                    const int n_strips = parts * PER;
                    auto strip_key = [&](int i) -> uint32_t { return ldcg_u32(c.strips + (slot0 + i / PER) * kLpStrips + i % PER); };
                    uint32_t mx = 0;
                    for (int i = tid; i < n_strips; i += kLpThreads) mx = max(mx, strip_key(i));
                    if (tid == 0) { sh.n_strip = 0; sh.n_cand = 0; sh.n_list = 0; sh.bound = 0; }
                    uint32_t bound = nth_bound(sh, n, mx);
                    auto take = [&](uint32_t lo) {   // the strips that reach lo
                        for (int i = tid; i < n_strips; i += kLpThreads) {
                            const uint32_t k = strip_key(i);
                            if (k >= lo) {
                                const int at = atomicAdd(&sh.n_strip, 1);
                                if (at < kLpStripCap) { sh.strip[at] = i; sh.strip_key[at] = k; }
                            }
                        }
                        __syncthreads();
                    };
                    take(bound);
                    int ns = sh.n_strip;
                    bool ties = ns > kLpStripCap;    // too many strips hold the bound itself
                    if (!ties) {
                        // the n-th largest of their maxima is a closer bound
                        int above = 0, same = 0;
                        const uint32_t k = tid < ns ? sh.strip_key[tid] : 0u;
                        if (tid < ns)
                            for (int u = 0; u < ns; ++u) { above += sh.strip_key[u] > k; same += sh.strip_key[u] == k; }
                        if (tid < ns && above < n && above + same >= n) sh.bound = k;
                        __syncthreads();
                        bound = max(bound, sh.bound);
                    } else {
                        __syncthreads();
                        if (tid == 0) sh.n_strip = 0;
                        __syncthreads();
                        take(bound + 1u);
                        ns = sh.n_strip;
                    }
                    if (ns <= kLpStripCap) {
                        const uint32_t lo = ties ? bound + 1u : bound;
                        const int most = (int)((N + G - 1) / G);                 // slices of a part at most
                        const int vecs = (most < a.spr ? most : a.spr) * NV * (by_warp ? 32 : 1);
                        for (int i = tid; i < ns * vecs; i += kLpThreads) {
                            const int q = i / vecs, s = sh.strip[q];
                            int v = i - q * vecs, t = s % PER;
                            if (sh.strip_key[q] < lo) continue;
                            if (by_warp) { t = t * 32 + (v & 31); v >>= 5; }
                            const long long part = c_first + s / PER;
                            const long long from = part * N / G - r0, to = (part + 1) * N / G - r0;
                            const int sl = (int)(from > 0 ? from : 0) + v / NV;
                            if (sl >= to || sl >= a.spr) continue;
                            keys_of(p, sl * SLICE + ((v % NV) * kLpThreads + t) * EV - off, [&](unsigned long long key) { if ((uint32_t)(key >> 32) >= lo) push(sh, key); });
                        }
                        __syncthreads();
                        if (ties) {
                            // the bound's own ids, from the row's beginning, until the list is full
                            const int have = sh.n_cand;
                            int width = 32;          // vectors of a step: few at first, they are dense or there would not be so many strips
                            for (int e = -off; e < V; e += width * EV, width = min(2 * width, kLpThreads)) {
                                __syncthreads();
                                if (have >= n || sh.n_cand >= n) break;
                                __syncthreads();
                                if (tid < width) keys_of(p, e + tid * EV, [&](unsigned long long key) { if ((uint32_t)(key >> 32) == bound) push(sh, key); });
                            }
                            __syncthreads();
                        }
                    }
                    if (ns > kLpStripCap || sh.n_cand > kLpCap) {
                        // hardly ever: slice by slice, whatever the elements are
                        __syncthreads();
                        for (int e = -off; e < V; e += SLICE)
                            collect(sh, n, [&](auto f) {
#pragma unroll 1
                                for (int j = 0; j < NV; ++j) keys_of(p, e + (j * kLpThreads + tid) * EV, f);
                            });
                    } else rank(sh, n);
                }
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
                __syncthreads();
            }
            ref = -1e30f;
            S0 = S1 = T0 = T1 = 0.f;
            top = -INFINITY;
        }
        row = nrow;
        slice = nslice;
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
    // a few hundred strips per row are enough to leave little to read again, and few enough for one CTA to look through
    const long long per_part = (a.n_items + grid - 1) / grid;
    a.warp_strips = (a.spr + per_part - 1) / per_part >= 32;
    void (*kern)(LpArgs);
    if (c.f32) kern = nv == 8 ? logprobs_kernel<true, 8> : nv == 4 ? logprobs_kernel<true, 4> : nv == 2 ? logprobs_kernel<true, 2> : logprobs_kernel<true, 1>;
    else kern = nv == 8 ? logprobs_kernel<false, 8> : nv == 4 ? logprobs_kernel<false, 4> : nv == 2 ? logprobs_kernel<false, 2> : logprobs_kernel<false, 1>;
    return (int)launch_chained(kern, dim3(grid), dim3(kLpThreads), 0, st, a);
}

}  // namespace fmtp
