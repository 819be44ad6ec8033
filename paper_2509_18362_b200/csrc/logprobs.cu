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
// A row is cut into equal parts, as many as give every resident CTA one; the CTA that completes a row joins the row's parts and
// writes its outputs.
//
// What bounds it (B200): the pass is bound by instructions, 13 for an element (its power of two, two sums, the strips' maxima) at 1.5 per cycle and SM, not by
// bytes: 256 rows of 152 064 bf16 with 20 alternatives 35.6 us, 2.2 TB/s (a third of the measured copy rate). Few rows are bound by
// latency, the pass's and the completing CTA's: four such rows 10.0 us, 75 rows of 32 001 fp32 10.8 us. The 256 rows took 48 us with lists
// of candidates kept along the way and parts of whole slices, 88 with one element at a time.
#include "logprobs.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace fmtp {

namespace {

constexpr uint32_t kDevBadToken = 0x1u, kDevAllNan = 0x10u;
constexpr int kLpThreads = kLpStrips, kLpCtasPerSm = 4, kLpWarps = kLpThreads / 32;
constexpr int kLpCap = kLpMaxTop * 33;               // candidates that are ranked at once: a list and 32 threads' elements of a slice
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
    int spr, parts;                                  // slices and parts of a row: part i has slices [i * spr / parts, (i + 1) * spr / parts)
    int warp_strips;                                 // strips are warps' (else threads'): parts are short and many
};

struct LpSum { float m, s, t; };                     // with y = x log2(e) - m: sum of 2^y, sum of 2^y y

struct LpShared {
    unsigned long long cand[kLpCap], list[kLpMaxTop], next[kLpMaxTop], best[kLpThreads], bound64;
    LpSum sum[2][kLpWarps];
    float red[kLpWarps];
    uint32_t warp_bound[kLpWarps], strip_key[kLpStripCap], bound;
    int strip[kLpStripCap];
    int n_cand, n_list, n_strip, last;
};

__device__ __forceinline__ void push(LpShared &sh, unsigned long long key) {
    const int at = atomicAdd(&sh.n_cand, 1);
    if (at < kLpCap) sh.cand[at] = key;
}

// Hands f(place, key) the n best of `count` keys that differ, each in one thread: a key's place is the number of larger ones.
template <typename F>
__device__ __forceinline__ void rank(const unsigned long long *keys, int count, int n, F f) {
    for (int i = threadIdx.x; i < count; i += kLpThreads) {
        const unsigned long long key = keys[i];
        int above = 0;
#pragma unroll 8
        for (int u = 0; u < count; ++u) above += keys[u] > key;
        if (above < n) f(above, key);
    }
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
    const int nc = sh.n_cand, nl = sh.n_list;        // nc <= n threads' elements <= kLpCap - kLpMaxTop
    __syncthreads();
    if (tid < nl) sh.cand[nc + tid] = sh.list[tid];
    __syncthreads();
    rank(sh.cand, nc + nl, n, [&](int at, unsigned long long key) { sh.next[at] = key; });
    __syncthreads();
    const int nn = min(nc + nl, n);
    if (tid < nn) sh.list[tid] = sh.next[tid];
    if (tid == 0) sh.n_list = nn;
    __syncthreads();
}

__device__ __forceinline__ float lp_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// b relative to the larger reference m (a difference of whole numbers, a power of two).
__device__ __forceinline__ void lp_shift(LpSum &b, float m) {
    const float d = b.m - m, f = lp_exp2(d);
    b.t = f * fmaf(b.s, d, b.t);
    b.s *= f;
    b.m = m;
}
// The block's sums, in a fixed order; every thread gets them. One barrier; `buf` is not used again before another one.
__device__ __forceinline__ LpSum lp_block(LpSum v, LpSum *buf) {
    float m = v.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    lp_shift(v, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(0xffffffffu, v.s, o);
        v.t += __shfl_xor_sync(0xffffffffu, v.t, o);
    }
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int w = 1; w < kLpWarps; ++w) m = fmaxf(w == 1 ? v.m : m, buf[w].m);
    lp_shift(v, m);
#pragma unroll
    for (int w = 1; w < kLpWarps; ++w) {
        LpSum x = buf[w];
        lp_shift(x, m);
        v.s += x.s;
        v.t += x.t;
    }
    return v;
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

template <bool F32, int NV>
__global__ void __launch_bounds__(kLpThreads, kLpCtasPerSm) logprobs_kernel(const __grid_constant__ LpArgs a) {
    chain_release();
    chain_wait();
    typedef Elem<F32> El;
    typedef typename El::T T;
    constexpr int EV = El::N, SLICE = kLpThreads * NV * EV;
    constexpr int KEPT = 8;                          // strips per thread whose keys stay in registers
    __shared__ LpShared sh;
    const LpCall &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, V = c.V, n = c.top;
    const T *logits = static_cast<const T *>(c.logits);
    const int row = blockIdx.y, part = blockIdx.x, parts = a.parts;
    auto first_slice = [&](int i) -> int { return (int)((long long)i * a.spr / parts); };
    const T *p = logits + (long long)row * c.ld;
    const int off = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));

    // Slice s of a row starts s * SLICE elements behind the 16-byte boundary at or below the row; a vector that lies across one of
    // the row's ends is put together from single elements, minus infinity for what is outside
    auto load_vec = [&](int e) -> uint4 {
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
    auto load = [&](int slice, uint4 (&v)[NV]) {
        const int e0 = slice * SLICE + tid * EV - off;
        if (__all_sync(0xffffffffu, e0 >= 0 && e0 + (NV - 1) * kLpThreads * EV + EV <= V)) {
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = ldnc128(p + e0 + j * kLpThreads * EV);
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = load_vec(e0 + j * kLpThreads * EV);
        }
    };
    // hands f the elements of a vector, the first of them e, as (value, id) keys
    auto keys_of = [&](const uint4 &v, int e, auto f) {
#pragma unroll
        for (int q = 0; q < EV; ++q)
            if ((unsigned)(e + q) < (unsigned)V) f(((unsigned long long)lp_order(El::at(v, q)) << 32) | (0xffffffffu - (uint32_t)(e + q)));
    };

    // the given token, for the CTA that completes the row
    float xt = 0.f;
    bool bad_token = false;
    if (tid == 0 && c.out_logprob) {
        int tok = c.tokens[row];
        bad_token = (unsigned)tok >= (unsigned)V;
        xt = El::one(p + (bad_token ? 0 : tok));
    }
    uint4 cur[NV], nxt[NV];
    const int slice0 = first_slice(part), slice1 = first_slice(part + 1);
    load(slice0, cur);
    float ref = -1e30f, S0 = 0.f, S1 = 0.f, T0 = 0.f, T1 = 0.f;
    float top = -INFINITY;                           // the thread's largest value
    for (int slice = slice0; slice < slice1; ++slice) {
        if (slice + 1 < slice1) load(slice + 1, nxt);        // the next slice's loads go out before this one's values are used
        // ---- sums
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            top = fmaxf(top, El::vec_max(cur[j]));
            El::clean(cur[j]);
        }
        const float want = rintf(fmaxf(top, kLpLow) * kLog2e);
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
#pragma unroll
        for (int j = 0; j < NV; ++j) cur[j] = nxt[j];
    }
    // ---- this CTA's part of the row is done
    if (n > 0) {
        uint32_t k = lp_order(top);
        uint32_t *strips = c.strips + ((size_t)row * parts + part) * kLpStrips;
        if (a.warp_strips) {
            k = __reduce_max_sync(0xffffffffu, k);
            if (lane == 0) strips[warp] = k;
        } else strips[tid] = k;
    }
    LpSum sum = lp_block(LpSum{ref, S0 + S1, T0 + T1}, sh.sum[0]);
    bool finish = parts == 1;
    if (!finish) {
        if (tid == 0) *reinterpret_cast<float4 *>(c.parts + (size_t)row * parts + part) = make_float4(sum.m, sum.s, sum.t, 0.f);
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            sh.last = atomicAdd(c.counters + row, 1u) == (uint32_t)(parts - 1);
            if (sh.last) c.counters[row] = 0u;
        }
    }
    if (tid == 0) { sh.n_strip = 0; sh.n_cand = 0; sh.n_list = 0; sh.bound = 0; }
    __syncthreads();
    if (!finish) finish = sh.last;
    if (!finish) return;
    {
        if (parts > 1) __threadfence();
        // parts and strips' maxima are asked for at once
        const size_t slot0 = (size_t)row * parts;
        const int per = a.warp_strips ? kLpWarps : kLpThreads, shift = a.warp_strips ? 3 : 8, n_strips = n > 0 ? parts * per : 0;
        auto strip_at = [&](int i) -> const uint32_t * { return c.strips + (slot0 + (i >> shift)) * kLpStrips + (i & (per - 1)); };
        uint32_t kept[KEPT], mx = 0;
#pragma unroll
        for (int u = 0; u < KEPT; ++u) kept[u] = tid + u * kLpThreads < n_strips ? ldcg_u32(strip_at(tid + u * kLpThreads)) : 0u;
        if (parts > 1) {
            LpSum v{-1e30f, 0.f, 0.f};
            for (int i = tid; i < parts; i += kLpThreads) {
                const uint4 u = ldcg128(c.parts + slot0 + i);
                LpSum x{__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z)};
                const float m = fmaxf(v.m, x.m);
                lp_shift(v, m);
                lp_shift(x, m);
                v.s += x.s;
                v.t += x.t;
            }
            sum = lp_block(v, sh.sum[1]);
        }
        // Rows whose maximum is too far from zero for the sums above (or infinite) are added up anew, against the maximum itself
        const bool far = !(sum.m > kLpMinRef && sum.m < kLpMaxRef);
        bool nothing = false;
        float M = 0.f;
        if (far) {
            float v = -INFINITY;
            for (int i = tid; i < V; i += kLpThreads) v = fmaxf(v, El::one(p + i));
            M = lp_max(v, sh.red);
            nothing = M == -INFINITY;
            LpSum x{0.f, 0.f, 0.f};
            for (int i = tid; i < V; i += kLpThreads) {
                const float e = El::one(p + i), y = (e - M) * kLog2e;
                if (e == M) x.s += 1.f;
                else if (y > -200.f) { x.s += lp_exp2(y); x.t = fmaf(lp_exp2(y), y, x.t); }
            }
            __syncthreads();
            sum = lp_block(x, sh.sum[1]);
        }
        const float lgS = log2f(sum.s), R = sum.m;
        auto logprob = [&](float x) -> float {
            if (nothing || !(x > -INFINITY)) return -INFINITY;
            if (far) return (x == M ? 0.f : x - M) - kLn2 * lgS;
            return x < kLpLow ? x - kLn2 * (R + lgS) : kLn2 * (fmaf(x, kLog2e, -R) - lgS);
        };
        auto put = [&](int at, unsigned long long key) {
            const size_t o = (size_t)row * n + at;
            if (c.out_ids) c.out_ids[o] = (int32_t)argmax_key_id(key);
            if (c.out_tops) c.out_tops[o] = logprob(lp_value((uint32_t)(key >> 32)));
        };
        if (tid == 0) {
            if (nothing) atomicOr(c.status, kDevAllNan);
            if (bad_token) atomicOr(c.status, kDevBadToken);
            if (c.out_logprob) c.out_logprob[row] = logprob(xt);
            if (c.out_entropy) c.out_entropy[row] = nothing ? 0.f : fmaxf(kLn2 * (lgS - sum.t / sum.s), 0.f);
        }
        if (n > 0) {
#pragma unroll
            for (int u = 0; u < KEPT; ++u) mx = max(mx, kept[u]);
            for (int i = tid + KEPT * kLpThreads; i < n_strips; i += kLpThreads) mx = max(mx, ldcg_u32(strip_at(i)));
            // Lower bound of the n-th best value: the smallest, over the warps, of a warp's ceil(n / 8)-th largest of its lanes' maxima
            {
                uint32_t k = mx, b = 0;
                for (int r = (n + kLpWarps - 1) / kLpWarps; r > 0; --r) {
                    b = __reduce_max_sync(0xffffffffu, k);
                    const uint32_t who = __ballot_sync(0xffffffffu, k == b);
                    if (lane == __ffs(who) - 1) k = 0u;
                }
                if (lane == 0) sh.warp_bound[warp] = b;
            }
            __syncthreads();
            uint32_t bound = sh.warp_bound[0];
#pragma unroll
            for (int w = 1; w < kLpWarps; ++w) bound = min(bound, sh.warp_bound[w]);
            auto take = [&](uint32_t lo) {   // the strips that reach lo
                auto one = [&](int i, uint32_t k) {
                    const int at = atomicAdd(&sh.n_strip, 1);
                    if (at < kLpStripCap) { sh.strip[at] = i; sh.strip_key[at] = k; }
                };
#pragma unroll
                for (int u = 0; u < KEPT; ++u)
                    if (kept[u] >= lo && tid + u * kLpThreads < n_strips) one(tid + u * kLpThreads, kept[u]);
                for (int i = tid + KEPT * kLpThreads; i < n_strips; i += kLpThreads) {
                    const uint32_t k = ldcg_u32(strip_at(i));
                    if (k >= lo) one(i, k);
                }
                __syncthreads();
            };
            take(bound);
            int ns = sh.n_strip;
            const bool ties = ns > kLpStripCap;          // too many strips hold the bound itself
            if (!ties) {
                // the n-th largest of their maxima is a closer bound
                if (tid < ns) {
                    const uint32_t k = sh.strip_key[tid];
                    int above = 0, same = 0;
#pragma unroll 8
                    for (int u = 0; u < ns; ++u) { above += sh.strip_key[u] > k; same += sh.strip_key[u] == k; }
                    if (above < n && above + same >= n) sh.bound = k;
                }
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
                auto take_vec = [&](const uint4 &v, int e) { if (lp_order(El::vec_max(v)) >= lo) keys_of(v, e, [&](unsigned long long key) { if ((uint32_t)(key >> 32) >= lo) push(sh, key); }); };
                // A strip's vectors: NV for each slice of its part, times 32 if it is a warp's. A group of 8 lanes takes a strip, four
                // vectors at a time
                for (int q = tid >> 3; q < ns; q += kLpThreads / 8) {
                    if (sh.strip_key[q] < lo) continue;
                    const int s = sh.strip[q], col = s & (per - 1);
                    const int s0 = first_slice(s >> shift), s1 = first_slice((s >> shift) + 1);
                    const int count = (s1 - s0) * NV << (a.warp_strips ? 5 : 0);
                    auto elem = [&](int v) -> int {
                        int t = col;
                        if (a.warp_strips) { t = col * 32 + (v & 31); v >>= 5; }
                        return (s0 + v / NV) * SLICE + ((v % NV) * kLpThreads + t) * EV - off;
                    };
                    for (int v = tid & 7; v < count; v += 32) {
                        uint4 x[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (v + 8 * u < count) x[u] = load_vec(elem(v + 8 * u));
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (v + 8 * u < count) take_vec(x[u], elem(v + 8 * u));
                    }
                }
                __syncthreads();
                if (ties) {
                    // the bound's own ids, from the row's beginning, until there are n keys
                    const int have = sh.n_cand;
                    int width = 32;          // vectors of a step: few at first, they are dense or there would not be so many strips
                    for (int e = -off; e < V; e += width * EV, width = min(2 * width, kLpThreads)) {
                        __syncthreads();
                        if (have >= n || sh.n_cand >= n) break;
                        __syncthreads();
                        if (tid < width) keys_of(load_vec(e + tid * EV), e + tid * EV, [&](unsigned long long key) { if ((uint32_t)(key >> 32) == bound) push(sh, key); });
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
                        for (int j = 0; j < NV; ++j) {
                            const int at = e + (j * kLpThreads + tid) * EV;
                            keys_of(load_vec(at), at, f);
                        }
                    });
                if (tid < n) put(tid, sh.list[tid]);     // (V >= n: the list is full)
            } else rank(sh.cand, sh.n_cand, n, put);
        }
    }
}

}  // namespace

int logprobs_slots(int n_sm) { return kLpMaxRows + n_sm * kLpCtasPerSm; }

int logprobs_launch(const LpCall &c, cudaStream_t st) {
    LpArgs a{};
    a.c = c;
    const int ev = c.f32 ? 4 : 8, ctas = c.n_sm * kLpCtasPerSm;
    auto per_row = [&](int nv) { const int e = kLpThreads * nv * ev; return (int)(((long long)c.V + ev - 1 + e - 1) / e); };   // a row may start ev - 1 elements after a boundary
    // as many parts as give every resident CTA one, and the slice length that leaves the longest part the shortest
    const int want = c.rows < ctas ? ctas / c.rows : 1;
    int nv = 4;
    long long least = -1;
    for (int v = 4; v > 0; v >>= 1) {
        const int spr = per_row(v), parts = want < spr ? want : spr;
        const long long cost = (long long)((spr + parts - 1) / parts) * v;
        if (least < 0 || cost < least) { least = cost; nv = v; }
    }
    a.spr = per_row(nv);
    a.parts = want < a.spr ? want : a.spr;
    // a few hundred strips per row are enough to leave little to read again, and few enough for one CTA to look through
    a.warp_strips = a.parts >= 32;
    void (*kern)(LpArgs);
    if (c.f32) kern = nv == 4 ? logprobs_kernel<true, 4> : nv == 2 ? logprobs_kernel<true, 2> : logprobs_kernel<true, 1>;
    else kern = nv == 4 ? logprobs_kernel<false, 4> : nv == 2 ? logprobs_kernel<false, 2> : logprobs_kernel<false, 1>;
    return (int)launch_chained(kern, dim3(a.parts, c.rows), dim3(kLpThreads), 0, st, a);
}

}  // namespace fmtp
