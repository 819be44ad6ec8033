// Operators over a paged K/V cache held in 8 bits: see kv8.cuh.
#include "kv8.cuh"
#include "batched.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace fmtp {

namespace {

constexpr uint32_t kDevBadPage = 0x2u, kDevBadPos = 0x4u, kDevTimeout8 = 0x8u;
constexpr int kMaxLen = 1 << 30;      // a longer committed length is the caller's error: flagged like any position without a slot

__device__ __forceinline__ int kv8_len(const Kv8Ptrs &kv, int b) { return min(max(kv.seq_lens[b], 0), kMaxLen); }
__device__ __forceinline__ int kv8_rows(const int32_t *n_new, int b, int M) { return n_new ? min(max(n_new[b], 0), M) : M; }
// Quotient by the page size: a shift for powers of two (shift >= 0).
__device__ __forceinline__ int page_of(int pos, int page, int shift) { return shift >= 0 ? pos >> shift : pos / page; }
int shift_of(int page) {
    for (int s = 0; s < 31; ++s) if (page == (1 << s)) return s;
    return -1;
}

// ---- e4m3 (4 significant bits, largest number 448, smallest 2^-9, NaN but no infinity)
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {          // nearest, halves to even; beyond +-448: +-448
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint16_t v) {               // exact
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(v));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_e4m3x2(uint32_t v) {               // as to_e4m3x2
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
__device__ __forceinline__ void f16x2_f32(uint32_t h, float &a, float &b) {
    asm("{.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(a), "=f"(b) : "r"(h));
}
__device__ __forceinline__ void e4m3x4_f32(uint32_t w, float (&x)[4]) {
    f16x2_f32(e4m3x2_f16x2((uint16_t)(w & 0xffffu)), x[0], x[1]);
    f16x2_f32(e4m3x2_f16x2((uint16_t)(w >> 16)), x[2], x[3]);
}
__device__ __forceinline__ uint32_t to_e4m3x4(const float (&x)[4], float f) {
    return to_e4m3x2(x[0] * f, x[1] * f) | (to_e4m3x2(x[2] * f, x[3] * f) << 16);
}
// Largest finite magnitude of eight bf16 values as bf16 bits (infinities and NaN do not count), joined to `m` (two lanes).
__device__ __forceinline__ uint32_t finite_max(uint32_t m, uint32_t w) {
    const uint32_t a = w & 0x7fff7fffu;
    return __vmaxu2(m, a & ~__vcmpgeu2(a, 0x7f807f80u));
}
// Smallest power of two s >= 2^-120 with amax <= 448 s, from amax's bf16 bits: amax = 1.f * 2^E, 448 = 1.75 * 2^8.
constexpr int kMinScaleExp = -120;
__device__ __forceinline__ float scale_for(uint32_t amax_bits) {
    int e = (int)(amax_bits >> 7) - 127 - 8 + ((amax_bits & 0x7fu) > 0x60u ? 1 : 0);
    e = max(e, kMinScaleExp);
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// ---- append: a warp quantises the new tokens of one block of one sequence and KV head (K and V are separate warps). Positions
// [first, end) of the block are new, those before `first` committed. The new scale covers the new tokens and is never below the
// committed tokens' one; where it grows, these are rounded once more (a shift of the exponent, exact but for subnormal codes).
// What lies behind `end` (rejected drafts, nothing) is left and does not count.
// A block's new rows have to be seen before its scale is known: up to 16 of them are read once, into registers (eight times 16 bytes per
// lane at dh = 128), the largest value is found by shuffles and the codes leave as 8-byte stores. Bound by the copy rate where there is much to do (16
// prompts of up to 4096 tokens, 4 x 128: 23.4 us, 4.3 TB/s; rows requested before the block table's entry: 25.4 us before), by the
// launch where there is little.
struct Append8Args {
    int Hkv, page, shift, max_ctx, B, M, nb;         // nb: blocks that M rows can touch
    const bf16_t *k, *v;
    long long ld;
    const int32_t *n_new;
    Kv8Ptrs kv;
    uint32_t *status;
};
constexpr int kAppendWarps = 4;

template <int DH>
__global__ void __launch_bounds__(kAppendWarps * 32, 8) kv8_append_kernel(const Append8Args a) {
    chain_release();
    chain_wait();
    constexpr int LPR = DH / 8;                      // lanes per row: eight values each
    constexpr int RPI = 32 / LPR;                    // rows per step of the warp
    constexpr int NT = 16 / RPI;                     // steps of a 16-token tile
    const int lane = threadIdx.x & 31, piece = lane % LPR, sub = lane / LPR;
    const long long w = (long long)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
    const int head2 = (int)(w % (2 * a.Hkv));        // key heads, then value heads
    const long long t = w / (2 * a.Hkv);
    const int i = (int)(t % a.nb), b = (int)(t / a.nb);
    if (b >= a.B) return;
    const int L = kv8_len(a.kv, b), n = kv8_rows(a.n_new, b, a.M);
    if (n == 0) return;                              // sits out: neither its table nor the scale of its last block is touched
    const int max_tokens = min((int)min((long long)a.kv.max_pages * a.page, (long long)kMaxLen), a.max_ctx);
    const int blk = page_of(L, a.page, a.shift) + i;
    const int at = blk * a.page;                     // position of the block's first token
    if (at >= L + n) return;
    const int first = max(L, at);
    int end = min(L + n, at + a.page);
    if (end > max_tokens) {                          // positions without a slot: flagged, not written
        if (lane == 0) atomicOr(a.status, kDevBadPos);
        end = max_tokens;
        if (first >= end) return;
    }
    const bool is_v = head2 >= a.Hkv;
    const int kvh = is_v ? head2 - a.Hkv : head2;
    const bf16_t *src = (is_v ? a.v : a.k) + ((long long)b * a.M - L) * a.ld + (long long)kvh * DH + piece * 8;      // + position * ld
    uint4 x[NT];
    auto load = [&](int p0) {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const int p = p0 + u * RPI + sub;
            x[u] = p < end ? *reinterpret_cast<const uint4 *>(src + p * a.ld) : make_uint4(0, 0, 0, 0);
        }
    };
    uint32_t m = 0;
    auto largest = [&]() {
#pragma unroll
        for (int u = 0; u < NT; ++u) m = finite_max(finite_max(finite_max(finite_max(m, x[u].x), x[u].y), x[u].z), x[u].w);
    };
    load(first);                                     // (on their way while the block is looked up)
    const int page = a.kv.block_table[(size_t)b * a.kv.max_pages + blk];
    if ((unsigned)page >= (unsigned)a.kv.num_pages) {          // not written either
        if (lane == 0) atomicOr(a.status, kDevBadPage);
        return;
    }
    const size_t slot = (size_t)page * a.Hkv + kvh;
    uint8_t *dst = (is_v ? a.kv.v_pages : a.kv.k_pages) + slot * a.page * DH + piece * 8;
    float *scale = (is_v ? a.kv.v_scales : a.kv.k_scales) + slot;
    const float s_old = first > at ? *scale : 0.f;
    largest();
    for (int p0 = first + 16; p0 < end; p0 += 16) {  // (blocks longer than 16 tokens)
        load(p0);
        largest();
    }
    m = max(m & 0xffffu, m >> 16);
    m = __reduce_max_sync(0xffffffffu, m);
    float s = scale_for(m);
    if (first > at) {
        if (s_old >= s) s = s_old;
        else {
            const float f = s_old / s;               // (a scale that is not a positive number makes the committed codes zeros or NaN)
            for (int p = at + sub; p < first; p += RPI) {
                uint2 *c = reinterpret_cast<uint2 *>(dst + (size_t)(p - at) * DH);
                uint2 v = *c;
                float y[4];
                e4m3x4_f32(v.x, y);
                v.x = to_e4m3x4(y, f);
                e4m3x4_f32(v.y, y);
                v.y = to_e4m3x4(y, f);
                *c = v;
            }
        }
    }
    if (lane == 0) *scale = s;
    const float inv = 1.0f / s;                      // exact for a power of two
    for (int p0 = first; p0 < end; p0 += 16) {
        if (end - first > 16) load(p0);
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const int p = p0 + u * RPI + sub;
            if (p >= end) continue;
            const float y[4] = {bf16lo_f32(x[u].x), bf16hi_f32(x[u].x), bf16lo_f32(x[u].y), bf16hi_f32(x[u].y)};
            const float z[4] = {bf16lo_f32(x[u].z), bf16hi_f32(x[u].z), bf16lo_f32(x[u].w), bf16hi_f32(x[u].w)};
            *reinterpret_cast<uint2 *>(dst + (size_t)(p - at) * DH) = make_uint2(to_e4m3x4(y, inv), to_e4m3x4(z, inv));
        }
    }
}

// ---- reading back: a warp takes 16 tokens of one sequence and KV head, 16 codes per lane and step, all requested before the first is
// converted. Bound by the copy rate: 32 ragged caches of 8 x 128 (286 MB of codes, twice that written) 155 us, 85% of it.
struct Read8Args {
    int Hkv, page, shift, max_ctx, B, max_n, tiles;
    const int32_t *start, *count;
    Kv8Ptrs kv;
    bf16_t *out_k, *out_v;
    uint32_t *status;
};
constexpr int kReadWarps = 4;

__device__ __forceinline__ uint4 dequant8(uint32_t a, uint32_t b, float s) {
    float x[4], y[4];
    e4m3x4_f32(a, x);
    e4m3x4_f32(b, y);
    uint4 r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.x) : "f"(x[1] * s), "f"(x[0] * s));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.y) : "f"(x[3] * s), "f"(x[2] * s));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.z) : "f"(y[1] * s), "f"(y[0] * s));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w) : "f"(y[3] * s), "f"(y[2] * s));
    return r;
}

template <int DH>
__global__ void __launch_bounds__(kReadWarps * 32) kv8_read_kernel(const Read8Args a) {
    chain_release();
    chain_wait();
    constexpr int LPR = DH / 16, RPI = 32 / LPR, NT = 16 / RPI;
    const int lane = threadIdx.x & 31, piece = lane % LPR, sub = lane / LPR;
    const long long w = (long long)blockIdx.x * kReadWarps + (threadIdx.x >> 5);
    const int kvh = (int)(w % a.Hkv);
    const long long t = w / a.Hkv;
    const int tile = (int)(t % a.tiles), b = (int)(t / a.tiles);
    if (b >= a.B) return;
    const int max_tokens = min((int)min((long long)a.kv.max_pages * a.page, (long long)kMaxLen), a.max_ctx);
    const int s0 = a.start ? min(max(a.start[b], 0), kMaxLen) : 0;
    int n = a.count ? max(a.count[b], 0) : max(kv8_len(a.kv, b) - s0, 0);
    n = min(n, a.max_n);
    if (n > max(max_tokens - s0, 0)) {
        if (lane == 0 && tile == 0) atomicOr(a.status, kDevBadPos);
        n = max(max_tokens - s0, 0);
    }
    const int i0 = tile * 16;
    if (i0 >= n) return;
    size_t row[NT];
    float sk[NT], sv[NT];
    uint4 ck[NT], cv[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const int pos = s0 + min(i0 + u * RPI + sub, n - 1), blk = page_of(pos, a.page, a.shift);
        int page = a.kv.block_table[(size_t)b * a.kv.max_pages + blk];
        if ((unsigned)page >= (unsigned)a.kv.num_pages) { atomicOr(a.status, kDevBadPage); page = 0; }
        const size_t slot = (size_t)page * a.Hkv + kvh;
        sk[u] = a.kv.k_scales[slot];
        sv[u] = a.kv.v_scales[slot];
        row[u] = slot * a.page + (pos - blk * a.page);
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        ck[u] = ldnc128(a.kv.k_pages + row[u] * DH + piece * 16);
        cv[u] = ldnc128(a.kv.v_pages + row[u] * DH + piece * 16);
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const int i = i0 + u * RPI + sub;
        if (i >= n) continue;
        const size_t o = (((size_t)b * a.max_n + i) * a.Hkv + kvh) * DH + piece * 16;
        *reinterpret_cast<uint4 *>(a.out_k + o) = dequant8(ck[u].x, ck[u].y, sk[u]);
        *reinterpret_cast<uint4 *>(a.out_k + o + 8) = dequant8(ck[u].z, ck[u].w, sk[u]);
        *reinterpret_cast<uint4 *>(a.out_v + o) = dequant8(cv[u].x, cv[u].y, sv[u]);
        *reinterpret_cast<uint4 *>(a.out_v + o + 8) = dequant8(cv[u].z, cv[u].w, sv[u]);
    }
}

// ---- attention. Two kernels and a join. kv8_attn_kernel, here: the (row, query head) pairs that share a KV head of a sequence are dealt to tiles of
// eight; a work item is one chunk of a sequence's context for one KV head and a set of RW * WR tiles. A CTA of four warps walks a
// contiguous range of items. Its WT = 4 / WR groups of WR warps take the chunk's 32-token stages in turn, each with a ring of its own, and meet at
// the chunk's end, where their results are joined in shared memory; a group's warps take RW tiles each, which share the
// conversions. (A warp for an item kept the SMs busy for three quarters of the time: an item of 256 tokens took it 25 us.)
//
// What bounds it (B200): instructions. A stage of one tile is about 730 of them, 128 conversions and 32 products among them, at 1.7 per cycle and
// SM with 12 warps; the bytes alone would take two thirds of the time. 64 contexts of 512 to 8192 tokens, 28/4 heads of 128, one row each: 71 us, 4.2
// TB/s of codes and scales (65% of the measured copy rate); two contexts of 50 000 to 60 000 tokens, 32/8 heads: 51 us, 4.4 TB/s; 64 contexts of 4096, 16/16
// heads of 64: 118 us, 4.5 TB/s. Short calls are latency: 2048 tokens of one sequence 12 us in two launches.
//
// Both products run on mma.sync.m16n8k16 with f16 operands (sm_100a has no mma.sync on e4m3: the assembler emulates it with fifteen
// instructions each). K and V are the A operand, 16 tokens or 16 dims, so that eight pairs fill the n side: S^T = K Q^T, O^T = V^T
// P^T. An e4m3 code is exact in f16, a bf16 query (over a power of two, eight bits) as well. A word of K is four dims of a token, and the contraction takes them in the order in which a
// lane holds them. V's transposed 16-bit ldmatrix gives dims 2u, 2u + 1 of two tokens in a word, which a byte permutation sorts;
// movmatrix turns a tile of probabilities from the first product's layout into the second one's.
//
// Scores are scaled by the token's K scale. What is multiplied with V's codes is a weight, a probability times the token's V scale, and weights have a reference of
// their own for every pair: f16 holds them right over 2^31 only, and where the scales differ, the largest weight need not be the largest
// probability's. A weight is rounded to 2^-11 of itself or 2^-27 of the pair's largest so far at least; a pair's references depend on what it sees alone.
// The reference of the exponentials is the maximum of a group's first stage and is moved only when a score lies 2^5 above it, so most
// stages need neither the maximum over all lanes nor a rescaling (partial results carry their reference). As long as all scales are within 2^3 of the first
// token's, the weights' reference is the probabilities' times that scale, and a weight costs a product. (The 64 contexts above: 68.7 us with one reference for all
// pairs, the largest scale that anyone met, which could leave a row nothing; 73.3 with an exponential for each weight whose scale is not the first one's.)
// A stage of the ring is 32 tokens of K and V with their scales, copied by the warps that read them (16-byte cp.async, any page
// size).
struct Attn8Args {
    int Hq, Hkv, gq, page, shift, max_ctx, slots, B, M;       // slots: chunks of a context that `part` has room for
    int tiles16;                                     // blocks are whole 16-token tiles
    const bf16_t *q;
    long long ldq;
    const int32_t *n_new;
    Kv8Ptrs kv;
    float *part;
    bf16_t *out, *xop;
    int ld_xop;
    uint32_t *status;
    unsigned long long wait_limit_ns;                // kv8_tile_kernel: a wait gives up after this long
    int extra_arrivals;                              // self-test: a K stage expects copies that are never made
};

constexpr int kA8Warps = 4, kA8Threads = kA8Warps * 32;
constexpr int kA8Blk = 32;                           // tokens of a stage
constexpr float kP8Log2 = 6.f;                       // probabilities relative to the reference are held times 2^6: f16 reaches down to 2^-24,
constexpr float kW8Max = 15.f, kW8Min = 2.f;          // the largest weight so far is kept between 2^2 and 2^15
constexpr float kNear8 = 8.f;                        // V scales within this factor of the reference leave weights and probabilities one reference,
constexpr float kP8Max = 11.f;                       // which is moved when a probability comes out above 2^11 (times eight: below 2^15)
constexpr float kBig8 = 0x1p-26f, kBig8Log2 = 26.f;   // partial results of scales above 1 are kept times 2^-26, with a reference 2^26 higher: their sums
                                                     // (up to 2^15 for each token) of large values stay numbers
constexpr float kQ8 = 32.f;                          // queries below 448 * 32

// Tokens of a chunk: a function of the sequence's committed length and of the call's rows per sequence, never of the batch. Short
// enough for a context to keep many CTAs busy, long enough for the partial results (dh + 4 fp32 words for each pair and chunk,
// 512 bytes against 256 bytes of K/V per token at dh = 128) to stay a small part of the traffic: up to `few` chunks until a chunk is
// 2^base long, up to `most` chunks of that and more tokens beyond.
// (few = 8 / 16 for 33 to 128 pairs, one set of tiles: 112 pairs of 1 x 4000 tokens 26.3 / 20.7 us, of 4 x 4000 29.3 / 23.8; for 448: 29.6 / 23.1 and
// 58.4 / 67.3, the sets fill the SMs and each chunk's result costs.)
struct Chunk8 { int first, few, base, most; };       // first and base: powers of two
__host__ __device__ __forceinline__ Chunk8 chunk8_rule(int pairs) {
    return pairs <= 8 ? Chunk8{7, 16, 9, 128} : pairs <= 32 ? Chunk8{7, 16, 9, 64} : pairs <= 128 ? Chunk8{8, 16, 9, 32} : Chunk8{8, 8, 9, 32};
}
__host__ __device__ __forceinline__ int chunk8(int n_ctx, int pairs) {      // log2
    const Chunk8 r = chunk8_rule(pairs);
    int c = r.first;
    while (c < r.base && n_ctx > r.few << c) ++c;
    while (((n_ctx - 1) >> c) >= r.most) ++c;
    return c;
}

// Words from one partial result to the next: dh weighted values, their reference and sum, and two that keep 16 bytes' alignment.
__host__ __device__ constexpr int part8_ld(int dh) { return dh + 4; }
constexpr int kList8Words = 6 * kBatchRows + 2;       // see List8

template <int DH, int RW, int WR>
struct Attn8Smem {
    static_assert(WR == 1 || WR == 2, "a CTA has four groups or two");
    static constexpr int WT = kA8Warps / WR;                                 // groups of a CTA
    static constexpr int CTAS = (DH == 128 ? 3 : 4) - (RW - 1);              // resident per SM
    static constexpr int S = (DH == 128 && RW == 1 ? 8 : 12) / WT;           // stages
    static constexpr int KV = kA8Blk * DH;                                   // bytes of a stage's K (or V) codes
    static constexpr int STAGE = 2 * KV + 2 * kA8Blk * 4;
    static constexpr int O_ML = WT * S * STAGE;                              // [4 warps][8 pairs] maximum, sum
    static constexpr int O_LAST = O_ML + kA8Warps * 8 * 8;                   // [WT] the stage that a group read last
    static constexpr int O_TAB = O_LAST + kA8Warps * 4;
    static constexpr int TOTAL = O_TAB + kList8Words * 4;
};

// (Warp-wide instructions are volatile: the compiler may move an asm statement without side effects into a branch that uses its result,
// and all lanes have to execute them at once, which the .aligned forms do not see to. So a __syncwarp() stands between them and whatever
// the lanes could have come through apart: a wait, a copy's conditions, a branch that is the same for all lanes but does not look it.)
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3lo_f16x2(uint32_t w) { return e4m3x2_f16x2((uint16_t)(w & 0xffffu)); }
__device__ __forceinline__ uint32_t e4m3hi_f16x2(uint32_t w) { return e4m3x2_f16x2((uint16_t)(w >> 16)); }
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float lds32f(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float exp2_approx(float x) {      // 2^x; results below the normal range are zero, as is 2^-inf
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {         // NaN if one is
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// How far (log2) the references of a pair's probabilities and weights move in a stage whose largest exponents are ym and zm: a reference above which
// something lies too far, or which is not there yet, to 2^6 below the largest. The weights' moves along with the probabilities' (so that
// equal scales keep both the same) unless the largest weight would leave its range; then it stays or goes its own way.
struct Moved8 { float p, w; };
__device__ __forceinline__ Moved8 move8(float ym, float zm, bool first, float most) {
    Moved8 mv;
    mv.p = (first || ym > most) && ym > -INFINITY ? ym - kP8Log2 : 0.f;
    const float z = zm - mv.p;
    mv.w = z <= kW8Max && (z >= kW8Min || (mv.p == 0.f && !first)) ? mv.p : (first || zm > kW8Max) && zm > -INFINITY ? zm - kP8Log2 : 0.f;
    return mv;
}
// Byte position of 16-byte piece c of token row t: the eight rows an ldmatrix phase reads lie in different banks.
template <int DH>
__device__ __forceinline__ uint32_t piece_at(int t, int c) {
    return (uint32_t)(t * DH + ((DH == 128 ? (c ^ (t & 7)) : (c ^ ((t >> 1) & 3))) << 4));
}

// Meeting of a group's warps. Not the aligned form of the barrier, which the compiler does not know to need all lanes of a warp.
template <int WR>
__device__ __forceinline__ void group_sync(int wt) {
    __syncwarp();
    if constexpr (WR > 1) asm volatile("barrier.sync %0, %1;" ::"r"(1 + wt), "n"(WR * 32) : "memory");
    __syncwarp();
}

// A place in the list of items: sequences, their KV heads, tile sets, chunks (the chunks of one context follow each other).
struct Item8 {
    int seq, kvh, set, chunk;
    int t0, t1;                                      // the chunk's tokens [t0, t1): never empty, the sequence's last row sees them all
};

// The list itself. An item has PAIRS pairs; it costs EACH and one for every STRIDE tokens, the
// first of a context FRESH more.
template <int PAIRS, int STRIDE, int EACH, int FRESH>
struct List8 {
    int *prefix, *pcost;                             // [B + 1] items before a sequence, and their cost
    int *tpos, *tval, *tchk, *tnum;                  // position of a sequence's row 0, its rows that count, tokens of its chunks (log2), chunks | sets << 16
    int B, Hkv, max_tokens;

    __device__ __forceinline__ List8(const Attn8Args &a, void *mem) {
        prefix = static_cast<int *>(mem);
        pcost = prefix + kBatchRows + 1;
        tpos = pcost + kBatchRows + 1;
        tval = tpos + kBatchRows;
        tchk = tval + kBatchRows;
        tnum = tchk + kBatchRows;
        B = a.B;
        Hkv = a.Hkv;
        max_tokens = min((int)min((long long)a.kv.max_pages * a.page, (long long)kMaxLen), a.max_ctx);
    }
    __device__ __forceinline__ int row_ctx(int pos0, int m) const { return min(pos0 + m, max_tokens - 1) + 1; }     // positions that row m sees
    __device__ __forceinline__ void build(const Attn8Args &a, int lane) {      // one warp, two sequences per lane
        int cnt[2], cost[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int s = 2 * lane + u;
            cnt[u] = cost[u] = 0;
            if (s < a.B) {
                const int len = kv8_len(a.kv, s), nv = kv8_rows(a.n_new, s, a.M);
                const int c = chunk8(row_ctx(len, a.M - 1), a.M * a.gq);
                tpos[s] = len; tval[s] = nv; tchk[s] = c;
                tnum[s] = 0;
                if (nv > 0) {
                    const int n = row_ctx(len, nv - 1), chunks = ((n - 1) >> c) + 1, sets = (nv * a.gq + PAIRS - 1) / PAIRS;
                    tnum[s] = chunks | (sets << 16);
                    cnt[u] = chunks * a.Hkv * sets;
                    cost[u] = (FRESH + chunks * EACH + (n + STRIDE - 1) / STRIDE) * a.Hkv * sets;
                    if (len + nv > max_tokens && blockIdx.x == 0) atomicOr(a.status, kDevBadPos);
                }
            }
        }
        int incl = cnt[0] + cnt[1], icost = cost[0] + cost[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, incl, o), tc = __shfl_up_sync(0xffffffffu, icost, o);
            if (lane >= o) { incl += t; icost += tc; }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int s = 2 * lane + u;
            if (s < a.B) {
                prefix[s + 1] = u ? incl : incl - cnt[1];
                pcost[s + 1] = u ? icost : icost - cost[1];
            }
        }
        if (lane == 0) prefix[0] = pcost[0] = 0;
    }
    // CTAs' shares of the list have the same cost up to an item: CTA i of n begins with the first item that starts at or behind its share
    __device__ __forceinline__ int begin_of(int i, int n) const {
        const int n_cost = pcost[B], each = n_cost / n, x = i * each + i * (n_cost - each * n) / n;      // i * n_cost / n
        if (x >= n_cost) return prefix[B];
        int s = 0;
        while (pcost[s + 1] <= x) ++s;
        const int rem = x - pcost[s], chunks = tnum[s] & 0xffff;
        const int cost = (pcost[s + 1] - pcost[s]) / (Hkv * (tnum[s] >> 16)), ctx = rem / cost, one = (1 << tchk[s]) / STRIDE + EACH;
        const int in = rem - ctx * cost;             // (item k > 0 starts at FRESH + k * one)
        return prefix[s] + ctx * chunks + (in == 0 ? 0 : min(max((in - FRESH + one - 1) / one, 1), chunks));
    }
    __device__ __forceinline__ void bounds(Item8 &it) const {
        const int c = tchk[it.seq];
        it.t0 = it.chunk << c;
        it.t1 = min(it.t0 + (1 << c), row_ctx(tpos[it.seq], tval[it.seq] - 1));
    }
    __device__ __forceinline__ void at(Item8 &it, int i) const {
        int s = 0;
        while (prefix[s + 1] <= i) ++s;
        const int rem = i - prefix[s], chunks = tnum[s] & 0xffff, sets = tnum[s] >> 16, t = rem / chunks;
        it.seq = s;
        it.chunk = rem - t * chunks;
        it.kvh = t / sets;
        it.set = t - it.kvh * sets;
        bounds(it);
    }
    __device__ __forceinline__ bool next(Item8 &it) const {          // whether the queries change (there is another item)
        bool fresh = false;
        if (++it.chunk == (tnum[it.seq] & 0xffff)) {
            it.chunk = 0;
            fresh = true;
            if (++it.set == tnum[it.seq] >> 16) {
                it.set = 0;
                if (++it.kvh == Hkv) {
                    it.kvh = 0;
                    do ++it.seq; while (prefix[it.seq + 1] == prefix[it.seq]);
                }
            }
        }
        bounds(it);
        return fresh;
    }
};

template <int DH, int RW, int WR>
__global__ void __launch_bounds__(kA8Threads, Attn8Smem<DH, RW, WR>::CTAS) kv8_attn_kernel(const __grid_constant__ Attn8Args a) {
    chain_wait();
    using Lay = Attn8Smem<DH, RW, WR>;
    constexpr int WT = Lay::WT, S = Lay::S, KS = DH / 32, ND = DH / 16, TILES = RW * WR;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wr = warp % WR, wt = warp / WR;
    const int gq = a.gq;
    constexpr int STRIDE = WT * kA8Blk;              // tokens from one stage of a group to its next
    List8<8 * TILES, STRIDE, 1, 0> list(a, smem + Lay::O_TAB);
    if (warp == 0) list.build(a, lane);
    __syncwarp();
    __syncthreads();
    const int i_begin = list.begin_of((int)blockIdx.x, (int)gridDim.x), i_end = list.begin_of((int)blockIdx.x + 1, (int)gridDim.x);
    if (i_begin >= i_end) return;                    // (an exit releases the successor as well)

    // ---- copying. Block-table entries are read a segment ahead (a read queues behind the copies that are on their way, which takes
    // longer than a stage): lane i holds the page of the segment's i-th block. A segment is part of one item: stages whose tokens lie in
    // 32 blocks
    const uint64_t policy = l2_evict_first();
    unsigned char *ring = smem + (size_t)wt * S * Lay::STAGE;
    struct Segment { int tok, end, t1, blk, kvh, page; };     // next stage's first token; behind the last one; end of what is seen; first block
    Segment cur{}, nxt{};
    Item8 li{};
    int litem = i_begin, ltok = 0, cslot = 0;
    auto load_segment = [&](Segment &g) {
        while (litem < i_end && ltok >= li.t1) {     // (an item may be too short for this group)
            if (++litem < i_end) {
                list.next(li);
                ltok = li.t0 + wt * kA8Blk;
            }
        }
        if (litem >= i_end) { g.tok = g.end = 0; return; }
        g.tok = ltok;
        g.t1 = li.t1;
        g.kvh = li.kvh;
        g.blk = page_of(ltok, a.page, a.shift);
        // stages whose tokens lie in the 32 blocks (the first one does) and in the chunk
        const long long room = ((long long)g.blk + 32) * a.page - ltok - kA8Blk;
        g.end = ltok + min((int)min(room / STRIDE, 1ll << 20) + 1, (li.t1 - ltok + STRIDE - 1) / STRIDE) * STRIDE;
        const int blk = min(g.blk + lane, page_of(li.t1 - 1, a.page, a.shift));
        g.page = a.kv.block_table[(size_t)li.seq * a.kv.max_pages + blk];
        ltok = g.end;
    };
    auto copy_stage = [&]() {
        if (cur.tok < cur.end) {
            const int pos = min(cur.tok + lane, cur.t1 - 1), blk = page_of(pos, a.page, a.shift);      // lane: a token of the stage
            int page = __shfl_sync(0xffffffffu, cur.page, blk - cur.blk);
            if ((unsigned)page >= (unsigned)a.kv.num_pages) { atomicOr(a.status, kDevBadPage); page = 0; }
            const uint32_t sb = smem_u32(ring + (size_t)cslot * Lay::STAGE);
            const uint32_t slot = (uint32_t)page * (uint32_t)a.Hkv + (uint32_t)cur.kvh;
            const uint32_t row = slot * (uint32_t)a.page + (uint32_t)(pos - blk * a.page);
            constexpr int LPR = DH / 16, RPI = 32 / LPR;         // lanes per token, tokens per step of a warp
            const int piece = lane % LPR, sub = lane / LPR;
            if (a.tiles16 && cur.tok + kA8Blk <= cur.t1) {
                // whole tiles of 16 tokens, which lie together: two addresses for K and two for V
                const size_t at0 = (size_t)__shfl_sync(0xffffffffu, row, 0) * DH + lane * 16 + wr * 512, at1 = (size_t)__shfl_sync(0xffffffffu, row, 16) * DH + lane * 16 + wr * 512;
                const uint32_t d0 = sb + piece_at<DH>(wr * RPI + sub, piece);
#pragma unroll
                for (int u = 0; u < kA8Blk / RPI / WR; ++u) {
                    constexpr int TILE = 16 * DH;
                    const int byte = u * WR * 512;               // 32 lanes x 16 bytes for each of the group's warps
                    // (at dh = 128 every other step of four tokens has the pieces' third bit the other way round)
                    const uint32_t d = (DH == 128 && (u * WR & 1) ? d0 ^ 64u : d0) + byte;
                    const size_t at = (byte < TILE ? at0 : at1) + byte % TILE;
                    cp_async16_full_hint<0>(d, a.kv.k_pages + at, policy);
                    cp_async16_full_hint<0>(d + Lay::KV, a.kv.v_pages + at, policy);
                }
            } else {
#pragma unroll
                for (int u = 0; u < kA8Blk / RPI / WR; ++u) {
                    const int t = (u * WR + wr) * RPI + sub;
                    const size_t off = (size_t)__shfl_sync(0xffffffffu, row, t) * DH + piece * 16;
                    const uint32_t d = sb + piece_at<DH>(t, piece), n = cur.tok + t < cur.t1 ? 16u : 0u;      // zeros beyond what is seen
                    cp_async16_off_hint<0>(d, a.kv.k_pages + off, n, policy);
                    cp_async16_off_hint<0>(d + Lay::KV, a.kv.v_pages + off, n, policy);
                }
            }
            if (wr == 0) {                           // (beyond what is seen: the last token's scales, so that the stage's need not differ)
                cp_async4(sb + 2 * Lay::KV + lane * 4, a.kv.k_scales + slot);
                cp_async4(sb + 2 * Lay::KV + kA8Blk * 4 + lane * 4, a.kv.v_scales + slot);
            }
            if (++cslot == S) cslot = 0;
            cur.tok += STRIDE;
            if (cur.tok >= cur.end) {
                cur = nxt;
                load_segment(nxt);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    list.at(li, i_begin);
    Item8 it = li;
    ltok = li.t0 + wt * kA8Blk;
    load_segment(cur);
    load_segment(nxt);
#pragma unroll 1
    for (int s = 0; s < S - 1; ++s) copy_stage();

    // ---- computing
    const int g = lane >> 2, kq = (lane & 3) * 2;    // of a tile's pairs, a lane has kq and kq + 1; as a B operand's column, g
    const float sm_scale = (1.0f / sqrtf((float)DH)) * 1.4426950408889634f;
    // ldmatrix rows: K: tokens 0-7 and 8-15 of one piece, then of the next; V: four groups of eight tokens of one piece
    const int ktok = lane & 15, kpc = lane >> 4;
    uint32_t qb[RW][2 * KS][2];
    float fs[RW][2];                                     // a query element times a key code times the K scale -> log2 units
    int pn[RW][2], prow[RW][2];                              // positions that a pair sees, its row (no such pair: any, the sequence's number of rows)
    size_t pout[RW][2];                                  // where its partial results go
    bool fresh = true;
    int slot = 0, last_slot = 0, nv = 0;
    for (int item = i_begin; item < i_end; ++item) {
        if (fresh) {                                 // the queries stay in registers while the items are chunks of one context
            nv = list.tval[it.seq];
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const int pair0 = ((it.set * WR + wr) * RW + r) * 8;
                auto pair_at = [&](int pair, int &m, int &row, int &head) -> bool {
                    const bool there = pair < nv * gq;
                    m = there ? pair / gq : 0;
                    row = it.seq * a.M + m;
                    head = it.kvh * gq + (there ? pair - m * gq : 0);
                    return there;
                };
                int m, row, head;
                pair_at(pair0 + g, m, row, head);
                const bf16_t *qp = a.q + (long long)row * a.ldq + (long long)head * DH;
                uint2 x[2 * KS];
                uint32_t am = 0;
#pragma unroll
                for (int j = 0; j < 2 * KS; ++j) {
                    x[j] = *reinterpret_cast<const uint2 *>(qp + j * 16 + kq * 2);
                    am = finite_max(finite_max(am, x[j].x), x[j].y);
                }
                am = max(am & 0xffffu, am >> 16);
                am = max(am, __shfl_xor_sync(0xffffffffu, am, 1));
                am = max(am, __shfl_xor_sync(0xffffffffu, am, 2));
                const float qs = scale_for(am), inv = kQ8 / qs;
#pragma unroll
                for (int j = 0; j < 2 * KS; ++j) {       // (a query that is not finite becomes NaN)
                    float y[4] = {bf16lo_f32(x[j].x), bf16hi_f32(x[j].x), bf16lo_f32(x[j].y), bf16hi_f32(x[j].y)};
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = fabsf(y[i]) < INFINITY ? y[i] * inv : __uint_as_float(0x7fffffffu);
                    qb[r][j][0] = pack_f16x2(y[0], y[1]);
                    qb[r][j][1] = pack_f16x2(y[2], y[3]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    fs[r][e] = __shfl_sync(0xffffffffu, qs, (kq + e) * 4) * (sm_scale / kQ8);
                    const bool there = pair_at(pair0 + kq + e, m, row, head);
                    prow[r][e] = there ? m : nv;
                    pn[r][e] = there ? list.row_ctx(list.tpos[it.seq], m) : kMaxLen;
                    pout[r][e] = ((size_t)row * a.Hq + head) * a.slots * part8_ld(DH);
                }
            }
        }
        float mo[RW][2], l_run[RW][2], o[RW][ND][4];         // a score's exponent: fma(score, fs, mo)
        float sv_ref = 1.f, sv_inv = 1.f, vo[RW][2];        // weights (see above) are held times 2^vo / sv_ref
        bool level = true;                           // all vo are zero
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            mo[r][0] = mo[r][1] = kP8Log2;
            l_run[r][0] = l_run[r][1] = vo[r][0] = vo[r][1] = 0.f;
#pragma unroll
            for (int i = 0; i < ND; ++i) o[r][i][0] = o[r][i][1] = o[r][i][2] = o[r][i][3] = 0.f;
        }
        const int tb0 = it.t0 + wt * kA8Blk;
#pragma unroll 1
        for (int tb = tb0; tb < it.t1; tb += STRIDE) {
            asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
            group_sync<WR>(wt);
            copy_stage();                            // into the stage that was read last
            __syncwarp();
            const uint32_t sb = smem_u32(ring + (size_t)slot * Lay::STAGE);
            last_slot = slot;
            if (++slot == S) slot = 0;
            // ---- scores: tokens 16 h + g, 16 h + 8 + g of pairs kq, kq + 1
            float y[RW][2][4];
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) y[r][h][0] = y[r][h][1] = y[r][h][2] = y[r][h][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {        // 32 dims
                uint32_t kf[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) ldsm4(sb + piece_at<DH>(h * 16 + ktok, 2 * ks + kpc), kf[h]);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t a0 = e4m3lo_f16x2(kf[h][2 * u]), a1 = e4m3lo_f16x2(kf[h][2 * u + 1]);
                        const uint32_t a2 = e4m3hi_f16x2(kf[h][2 * u]), a3 = e4m3hi_f16x2(kf[h][2 * u + 1]);
#pragma unroll
                        for (int r = 0; r < RW; ++r) mma_f16(y[r][h], a0, a1, a2, a3, qb[r][2 * ks + u][0], qb[r][2 * ks + u][1]);
                    }
            }
            // ---- exponents; V scales of the lane's tokens
            float sv[2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t at = sb + 2 * Lay::KV + (h * 16 + u * 8 + g) * 4;
                    const float sk = lds32f(at);
                    sv[h][u] = lds32f(at + kA8Blk * 4);
#pragma unroll
                    for (int r = 0; r < RW; ++r) {
                        y[r][h][2 * u] = fmaf(y[r][h][2 * u] * sk, fs[r][0], mo[r][0]);
                        y[r][h][2 * u + 1] = fmaf(y[r][h][2 * u + 1] * sk, fs[r][1], mo[r][1]);
                    }
                }
            int least = kMaxLen;                     // what the pair that sees least sees
#pragma unroll
            for (int r = 0; r < RW; ++r) least = min(least, min(pn[r][0], pn[r][1]));
            const bool edge = __any_sync(0xffffffffu, least - tb < kA8Blk);
            if (edge) {
#pragma unroll
                for (int r = 0; r < RW; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (tb + h * 16 + (i >> 1) * 8 + g >= pn[r][i & 1]) y[r][h][i] = -INFINITY;
            }
            __syncwarp();
            const bool first = tb == tb0;
            if (first) {                             // the group's first token: whoever sees any of its tokens sees this one
                sv_ref = __shfl_sync(0xffffffffu, sv[0][0], 0);
                if (!(sv_ref >= 0x1p-120f && sv_ref <= 0x1p120f)) sv_ref = 1.f;          // (one whose inverse need not be right: weights go their own way)
                sv_inv = __fdividef(1.0f, sv_ref);
            }
            float ym[RW][2], most = -INFINITY;
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    ym[r][e] = fmaxf(fmaxf(y[r][0][e], y[r][0][2 + e]), fmaxf(y[r][1][e], y[r][1][2 + e]));
                    most = fmaxf(most, ym[r][e]);
                }
            const float s0 = min_nan(min_nan(sv[0][0], sv[0][1]), min_nan(sv[1][0], sv[1][1])), s1 = fmaxf(fmaxf(sv[0][0], sv[0][1]), fmaxf(sv[1][0], sv[1][1]));
            uint32_t pb[RW][2][2];
            if (__all_sync(0xffffffffu, level && s0 * kNear8 >= sv_ref && s1 <= sv_ref * kNear8)) {
                if (first || __any_sync(0xffffffffu, most > kP8Max)) {
                    // new references: the stage's maximum where it is the first or far above (the weights' move along)
#pragma unroll
                    for (int r = 0; r < RW; ++r) {
                        float corr[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
#pragma unroll
                            for (int x = 4; x < 32; x <<= 1) ym[r][e] = fmaxf(ym[r][e], __shfl_xor_sync(0xffffffffu, ym[r][e], x));
                            const float d = (first || ym[r][e] > kP8Max) && ym[r][e] > -INFINITY ? ym[r][e] - kP8Log2 : 0.f;
                            mo[r][e] -= d;
#pragma unroll
                            for (int h = 0; h < 2; ++h) { y[r][h][e] -= d; y[r][h][2 + e] -= d; }
                            corr[e] = first ? 1.f : exp2_approx(-d);
                            l_run[r][e] *= corr[e];
                        }
                        if (!first) {
#pragma unroll
                            for (int i = 0; i < ND; ++i) { o[r][i][0] *= corr[0]; o[r][i][1] *= corr[1]; o[r][i][2] *= corr[0]; o[r][i][3] *= corr[1]; }
                        }
                    }
                }
                __syncwarp();
                // ---- probabilities and, as f16, weights
                const bool scaled = !__all_sync(0xffffffffu, s0 == sv_ref && s1 == sv_ref);
#pragma unroll
                for (int r = 0; r < RW; ++r) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[r][h][i] = exp2_approx(y[r][h][i]);
                    l_run[r][0] += (y[r][0][0] + y[r][0][2]) + (y[r][1][0] + y[r][1][2]);
                    l_run[r][1] += (y[r][0][1] + y[r][0][3]) + (y[r][1][1] + y[r][1][3]);
                    if (scaled) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const float f = sv[h][u] * sv_inv;
                                y[r][h][2 * u] *= f;
                                y[r][h][2 * u + 1] *= f;
                            }
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < 2; ++u) pb[r][h][u] = pack_f16x2(y[r][h][2 * u], y[r][h][2 * u + 1]);
                }
            } else {
                // the same with weights that have references of their own
                const float sv_log2 = __log2f(sv_ref);
                float lf[2][2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        lf[h][u] = __log2f(sv[h][u]) - sv_log2;
                        if (lf[h][u] < -300.f) lf[h][u] = -300.f;        // a scale of zero
                    }
                bool zero = true;
#pragma unroll
                for (int r = 0; r < RW; ++r) {
                    float corr[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float z = fmaxf(fmaxf(y[r][0][e] + lf[0][0], y[r][0][2 + e] + lf[0][1]), fmaxf(y[r][1][e] + lf[1][0], y[r][1][2 + e] + lf[1][1]));
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) {
                            ym[r][e] = fmaxf(ym[r][e], __shfl_xor_sync(0xffffffffu, ym[r][e], x));
                            z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, x));
                        }
                        const Moved8 mv = move8(ym[r][e], z + vo[r][e], first, kP8Max);
                        mo[r][e] -= mv.p;
                        vo[r][e] += mv.p - mv.w;
                        zero = zero && vo[r][e] == 0.f;
                        l_run[r][e] *= first ? 1.f : exp2_approx(-mv.p);
                        corr[e] = first ? 1.f : exp2_approx(-mv.w);
                        float sum[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const float x = y[r][h][2 * u + e] - mv.p, f = sv[h][u] * sv_inv, p = exp2_approx(x);
                                sum[h] = u ? sum[h] + p : p;
                                // (what a pair gets does not depend on which of the two ways its stage takes)
                                const float w = vo[r][e] == 0.f && f >= 1.0f / kNear8 && f <= kNear8 ? p * f : exp2_approx(x + (lf[h][u] + vo[r][e]));
                                y[r][h][2 * u + e] = x == -INFINITY ? 0.f : w;
                            }
                        l_run[r][e] += sum[0] + sum[1];
                    }
                    if (!first) {
#pragma unroll
                        for (int i = 0; i < ND; ++i) { o[r][i][0] *= corr[0]; o[r][i][1] *= corr[1]; o[r][i][2] *= corr[0]; o[r][i][3] *= corr[1]; }
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < 2; ++u) pb[r][h][u] = pack_f16x2(y[r][h][2 * u], y[r][h][2 * u + 1]);
                }
                level = __all_sync(0xffffffffu, zero);
            }
            __syncwarp();
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int u = 0; u < 2; ++u) pb[r][h][u] = movmatrix_trans(pb[r][h][u]);
            // ---- weighted values: dims 16 c + 2 g, 16 c + 2 g + 1 of pairs kq, kq + 1. In a stage that some row does not see whole, what
            // it does not see is a later row's value and need not be a number: there a value that is no number counts as 0 in the
            // products, and is put in afterwards where it is seen
            uint32_t bad = 0;
#pragma unroll
            for (int c = 0; c < ND; ++c) {
                uint32_t v[4];
                ldsm4_trans(sb + Lay::KV + piece_at<DH>(lane, c), v);
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t nan = __vcmpeq4(v[i] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                        v[i] &= ~nan;
                        bad |= nan;
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t w0 = __byte_perm(v[2 * h], 0, 0x3120), w1 = __byte_perm(v[2 * h + 1], 0, 0x3120);       // tokens 8 more
                    const uint32_t a0 = e4m3lo_f16x2(w0), a1 = e4m3hi_f16x2(w0), a2 = e4m3lo_f16x2(w1), a3 = e4m3hi_f16x2(w1);
#pragma unroll
                    for (int r = 0; r < RW; ++r) mma_f16(o[r][c], a0, a1, a2, a3, pb[r][h][0], pb[r][h][1]);
                }
            }
            if (edge && __any_sync(0xffffffffu, bad != 0u)) {
#pragma unroll
                for (int c = 0; c < ND; ++c)
#pragma unroll 1
                    for (int t = 0; t < kA8Blk; ++t) {
                        uint16_t w;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(sb + Lay::KV + piece_at<DH>(t, c) + (uint32_t)g * 2) : "memory");
                        const bool n0 = (w & 0x7fu) == 0x7fu, n1 = (w & 0x7f00u) == 0x7f00u;
#pragma unroll
                        for (int r = 0; r < RW; ++r)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const bool seen = tb + t < pn[r][e];
                                o[r][c][e] += seen && n0 ? NAN : 0.f;
                                o[r][c][2 + e] += seen && n1 ? NAN : 0.f;
                            }
                    }
            }
            __syncwarp();
        }
        // ---- the chunk's partial result: o and the sum relative to the reference, the reference (log2 units; what a group does not
        // see of the chunk from its first stage on, it does not see at all)
        const int groups = min(WT, (it.t1 - it.t0 + kA8Blk - 1) / kA8Blk);       // the others had none of the chunk's stages
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            float m_ref[2], back[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float lb = (vo[r][e] == 0.f ? 0.f : __log2f(sv_ref)) - vo[r][e];
                const bool large = vo[r][e] == 0.f ? sv_ref > 1.f : lb > 0.f;
                back[e] = vo[r][e] == 0.f ? (large ? sv_ref * kBig8 : sv_ref) : exp2f(large ? lb - kBig8Log2 : lb);
                m_ref[e] = pn[r][e] > tb0 ? kP8Log2 - mo[r][e] + (large ? kBig8Log2 : 0.f) : -INFINITY;
                if (large) l_run[r][e] *= kBig8;
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l_run[r][e] += __shfl_xor_sync(0xffffffffu, l_run[r][e], x);
            }
            if (groups == 1) {
                if (wt == 0) {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (prow[r][e] < nv && pn[r][e] > it.t0) {             // such a pair, and it sees something of the chunk
                            float *out = a.part + pout[r][e] + (size_t)it.chunk * part8_ld(DH);
#pragma unroll
                            for (int c = 0; c < ND; ++c) *reinterpret_cast<float2 *>(out + c * 16 + g * 2) = make_float2(o[r][c][e] * back[e], o[r][c][2 + e] * back[e]);
                            if (g == 0) *reinterpret_cast<float2 *>(out + DH) = make_float2(m_ref[e], l_run[r][e]);
                        }
                }
            } else {
                // Each warp leaves a tile's result in the stage that its group read last (free until the group's next copy), and the tile's warps add
                // them up in the groups' order, 8 / WT pairs each
                constexpr int LD = DH + 4;               // (rows of pairs start in different banks)
                static_assert(8 * LD * 4 * WR <= Lay::STAGE, "a tile of each warp fits the stage");
                float2 *ml = reinterpret_cast<float2 *>(smem + Lay::O_ML);
                int *last = reinterpret_cast<int *>(smem + Lay::O_LAST);
                if (r == 0) group_sync<WR>(wt);          // all readers of the stage are done
                if (wt < groups) {
                    float *mine = reinterpret_cast<float *>(ring + (size_t)last_slot * Lay::STAGE) + wr * 8 * LD;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int c = 0; c < ND; ++c) *reinterpret_cast<float2 *>(mine + (kq + e) * LD + c * 16 + g * 2) = make_float2(o[r][c][e] * back[e], o[r][c][2 + e] * back[e]);
                        if (g == 0) ml[warp * 8 + kq + e] = make_float2(m_ref[e], l_run[r][e]);
                    }
                    if (lane == 0 && wr == 0) last[wt] = last_slot;
                }
                __syncthreads();
                constexpr int LPP = DH / 4, PPW = 8 / WT;            // lanes per pair (four dims each), pairs per warp
#pragma unroll 1
                for (int q0 = 0; q0 < PPW; q0 += 32 / LPP) {
                    const int q = wt * PPW + q0 + lane / LPP, d = lane % LPP * 4, pair = ((it.set * WR + wr) * RW + r) * 8 + q;
                    float mm = -INFINITY;
#pragma unroll
                    for (int x = 0; x < WT; ++x)
                        if (x < groups) mm = fmaxf(mm, ml[(x * WR + wr) * 8 + q].x);
                    const float mu = mm == -INFINITY ? 0.f : mm;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    float l = 0.f;
#pragma unroll
                    for (int x = 0; x < WT; ++x) {
                        if (x >= groups) continue;
                        const float2 z = ml[(x * WR + wr) * 8 + q];
                        const float f = exp2_approx(z.x - mu);
                        const float4 v = *reinterpret_cast<const float4 *>(smem + (size_t)(x * S + last[x]) * Lay::STAGE + ((wr * 8 + q) * LD + d) * 4);
                        acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
                        l += z.y * f;
                    }
                    const int m = pair / gq;
                    if (pair < nv * gq && list.row_ctx(list.tpos[it.seq], m) > it.t0) {
                        float *out = a.part + (((size_t)(it.seq * a.M + m) * a.Hq + it.kvh * gq + (pair - m * gq)) * a.slots + it.chunk) * part8_ld(DH);
                        *reinterpret_cast<float2 *>(out + d) = make_float2(acc.x, acc.y);
                        *reinterpret_cast<float2 *>(out + d + 2) = make_float2(acc.z, acc.w);
                        if (d == 0) *reinterpret_cast<float2 *>(out + DH) = make_float2(mm, l);
                    }
                }
                __syncthreads();
            }
        }
        __syncwarp();
        if (item + 1 < i_end) fresh = list.next(it);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    chain_release();
}

// ---- attention of many pairs per KV head (dh = 128): a set is 128 pairs, the rows of a tcgen05 tile, and an item a chunk of a context
// for one KV head and a set; blocks of 64 tokens. Scores: K's codes are an e4m3 operand as they lie in the cache, a query
// is two (its nearest e4m3 and the rest's: 8 bits, a bf16's own, down to 2^-9 of the row's largest element; below that it is off by up to 2^-17 of the
// largest), both against the same K tile. Values: f16 operands, the codes converted on the way into shared memory, the weights (probability times V scale)
// rounded as in kv8_attn_kernel, with a reference of each row's own; V's tile is token-major, which is the product's MN-major operand.
// Warps 0-3 are the softmax, a thread a row (its scores are 64 columns of the thread's TMEM lane): the row's maximum and sum need no exchange.
// Warps 4-7 bring K (cp.async) and V (through registers), both two blocks ahead; one thread of warp 8 issues the products:
// block n + 1's scores before block n's values, which wait for its probabilities. Two CTAs per SM: one's softmax runs beside the other's
// products. What bounds it (B200): issue and latency of softmax and conversions, 5 200 warp instructions per block at 1.8 per cycle and SM (a
// block's exponentials alone are 512 cycles of an SM, its products 256), and the ends: 4 us of set-up and first loads, 5 us of
// queries, 3 us for each chunk's result. Four contexts of 3500 to 4200 tokens, 64 rows each, 28/4 heads: 61.6 us with the join (7 us); held scores
// (64 registers, spilt) 109 us, page look-ups one block ahead 84 us. Without the search for a maximum (block's exponentials first, again where one
// does not fit f16) wide scores took 70 instead of 66 us.
constexpr int kT8Pairs = 128, kT8Blk = 64, kT8Threads = 288, kT8Copiers = 128, kT8KStages = 3;
struct Tile8Block {                                  // per V buffer, written beside its values
    float sk[4], sv_log2[4];                         // of the block's 16-token tiles
    uint32_t bad[4];                                 // values that are no number were left out (see kv8_attn_kernel); of each copy warp
};
struct Tile8Smem {
    static constexpr int TILE = 128 * 128, K = kT8Blk * 128, V = kT8Blk * 256;
    static constexpr int O_K = 2 * TILE, O_V = O_K + kT8KStages * K, O_P = O_V + 2 * V, O_BLK = O_P + TILE;
    static constexpr int O_BAR = O_BLK + 2 * (int)sizeof(Tile8Block);        // a multiple of eight
    static constexpr int N_BAR = 2 * kT8KStages + 2 + 2 + 2 + 3;
    static constexpr int O_WORDS = O_BAR + N_BAR * 8;                        // TMEM address, abort
    static constexpr int O_LIST = O_WORDS + 8;
    static constexpr int TOTAL = O_LIST + kList8Words * 4;
};
static_assert(sizeof(Tile8Block) % 16 == 0 && offsetof(Tile8Block, sv_log2) == 16 && 2 * (Tile8Smem::TOTAL + 1024) <= 228 * 1024, "two CTAs per SM");

// Waits until the limit or, unless the wait is for what is under way for sure (`always`), until another wait of the CTA has given up.
__device__ __forceinline__ bool tile8_wait(volatile uint32_t *abort_flag, uint64_t *bar, uint32_t parity, unsigned long long limit_ns, bool always = false) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_timer_ns();
    uint32_t polls = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++polls & 63u) == 0) {
            if (*abort_flag && !always) return false;
            if (global_timer_ns() - t0 > limit_ns) {
                *abort_flag = 1u;
                return false;
            }
        }
    }
    return true;
}

__global__ void __launch_bounds__(kT8Threads, 2) kv8_tile_kernel(const __grid_constant__ Attn8Args a) {
    using Lay = Tile8Smem;
    constexpr int DH = 128;
    constexpr uint32_t kFull = 0xffffffffu;
    extern __shared__ __align__(1024) unsigned char smem_t[];
    unsigned char *const smem = smem_t;
    uint64_t *kfull = reinterpret_cast<uint64_t *>(smem + Lay::O_BAR), *kempty = kfull + kT8KStages;
    uint64_t *vfull = kempty + kT8KStages, *vempty = vfull + 2, *sfull = vempty + 2;         // vempty: the block's values are added up
    uint64_t *pready = sfull + 2, *qready = pready + 1, *drain = qready + 1;
    volatile uint32_t *words = reinterpret_cast<volatile uint32_t *>(smem + Lay::O_WORDS), *abort_flag = words + 1;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    List8<kT8Pairs, kT8Blk, 2, 3> list(a, smem + Lay::O_LIST);
    if (tid == 32) {
        for (int i = 0; i < kT8KStages; ++i) { mbar_init(&kfull[i], kT8Copiers + a.extra_arrivals); mbar_init(&kempty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&vfull[i], kT8Copiers); mbar_init(&vempty[i], 1); mbar_init(&sfull[i], 1); }
        mbar_init(pready, 128);
        mbar_init(qready, 128);
        mbar_init(drain, 1);
        words[1] = (smem_u32(smem) & 1023u) != 0u;   // swizzled tiles need the alignment: nothing runs without it
        mbar_fence_init();
    }
    if (warp == 8) {
        tmem_alloc(const_cast<uint32_t *>(words), 256);
        tmem_relinquish();
        tc_fence_before_sync();
    }
    chain_wait();
    if (warp == 0) list.build(a, lane);
    __syncwarp();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = words[0], tmem_o = tmem + 128;       // two blocks' scores, 64 columns each; 128 columns of weighted values
    const int gq = a.gq;
    const int i_begin = list.begin_of((int)blockIdx.x, (int)gridDim.x), i_end = *abort_flag ? i_begin : list.begin_of((int)blockIdx.x + 1, (int)gridDim.x);
    const uint32_t base = smem_u32(smem);

    if (warp < 4) {
        // ================= softmax
        const uint32_t lane_addr = (uint32_t)(warp * 32) << 16, sw = (uint32_t)(tid & 7), p_row = base + Lay::O_P + (uint32_t)tid * 128;
        const float sm_scale = (1.0f / sqrtf((float)DH)) * 1.4426950408889634f;
        Item8 it{};
        if (i_begin < i_end) list.at(it, i_begin);
        bool fresh = true, ok = true;
        int n = 0, pn = kMaxLen;
        uint32_t prow = kFull;                       // the row's place among the partial results, divided by a.slots; kFull: no such pair
        float fs = 0.f;
        for (int item = i_begin; item < i_end && ok; ++item) {
            if (fresh) {
                // queries, two rows at a time, eight dims per lane (the last block's scores are there, so the old ones have been read)
                const int nv = list.tval[it.seq], pair = it.set * kT8Pairs + tid;
                const bool there = pair < nv * gq;
                const int m = there ? pair / gq : 0, row = it.seq * a.M + m, head = it.kvh * gq + (there ? pair - m * gq : 0);
                pn = there ? list.row_ctx(list.tpos[it.seq], m) : kMaxLen;
                prow = there ? (uint32_t)(row * a.Hq + head) : kFull;
                const int piece = lane & 15, half = lane >> 4;
                float qs = 1.f;
                uint4 x[2], ahead[2];
#pragma unroll 1
                for (int r0 = -4; r0 < 32; r0 += 4) {          // the next four rows are on their way
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int from = min(r0 + 4 + 2 * i + half, 31), qrow = __shfl_sync(kFull, row, from), qhead = __shfl_sync(kFull, head, from);
                        ahead[i] = *reinterpret_cast<const uint4 *>(a.q + (long long)qrow * a.ldq + qhead * DH + piece * 8);      // (no such pair: the first one's)
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (r0 < 0) break;
                        const int r = warp * 32 + r0 + 2 * i + half;
                        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                        uint32_t am = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
                        am = max(am & 0xffffu, am >> 16);
#pragma unroll
                        for (int o = 1; o < 16; o <<= 1) am = max(am, __shfl_xor_sync(kFull, am, o));
                        const float rs = scale_for(am), other = __shfl_sync(kFull, rs, (lane & 1) * 16);
                        if ((lane >> 1) == (r0 >> 1) + i) qs = other;
                        // the power of two's inverse; a row that is not finite is NaN
                        const float inv = am < 0x7f80u ? __uint_as_float(0x7f000000u - __float_as_uint(rs)) : __uint_as_float(0x7fffffffu);
                        uint32_t hi[2], lo[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t y0 = pack_f16x2(bf16lo_f32(w[2 * h]) * inv, bf16hi_f32(w[2 * h]) * inv);       // (below 448: exact, but for what is below 2^-14)
                            const uint32_t y1 = pack_f16x2(bf16lo_f32(w[2 * h + 1]) * inv, bf16hi_f32(w[2 * h + 1]) * inv);
                            const uint32_t h0 = f16x2_e4m3x2(y0), h1 = f16x2_e4m3x2(y1);
                            hi[h] = h0 | (h1 << 16);
                            lo[h] = f16x2_e4m3x2(sub_f16x2(y0, e4m3x2_f16x2((uint16_t)h0))) | (f16x2_e4m3x2(sub_f16x2(y1, e4m3x2_f16x2((uint16_t)h1))) << 16);
                        }
                        unsigned char *at = smem + r * 128 + (((piece >> 1) ^ (r & 7)) << 4) + (piece & 1) * 8;
                        *reinterpret_cast<uint2 *>(at) = make_uint2(hi[0], hi[1]);
                        *reinterpret_cast<uint2 *>(at + Lay::TILE) = make_uint2(lo[0], lo[1]);
                    }
                    x[0] = ahead[0];
                    x[1] = ahead[1];
                }
                fs = qs * sm_scale;
                fence_proxy_async();
                mbar_arrive(qready);
            }
            float mo = kP8Log2, l_run = 0.f, vo = 0.f;           // weights are held times 2^vo
            uint32_t bad = 0;
#pragma unroll 1
            for (int tb = it.t0; tb < it.t1; tb += kT8Blk, ++n) {
                const int b = n & 1;
                const uint32_t ph = (uint32_t)(n >> 1) & 1u, tmem_s = tmem + lane_addr + (uint32_t)(b * kT8Blk);
                ok = tile8_wait(abort_flag, &vfull[b], ph, a.wait_limit_ns) && tile8_wait(abort_flag, &sfull[b], ph, a.wait_limit_ns);
                if (__any_sync(kFull, !ok)) { ok = false; break; }
                __syncwarp();
                tc_fence_after_sync();
                const Tile8Block *blk = reinterpret_cast<const Tile8Block *>(smem + Lay::O_BLK) + b;
                const float4 sk4 = *reinterpret_cast<const float4 *>(blk->sk);
                float4 sl4 = *reinterpret_cast<const float4 *>(blk->sv_log2);
                const bool first = tb == it.t0;
                if (first) vo = -sl4.x;              // (the chunk's first tile, which every row sees that sees any of it)
                const uint4 bd = *reinterpret_cast<const uint4 *>(blk->bad);
                bad |= bd.x | bd.y | bd.z | bd.w;
                // a code product times c is a score in log2 units (c > 0: nothing seen, -inf, stays that)
                const float c[4] = {fmaxf(sk4.x * fs, 1e-37f), fmaxf(sk4.y * fs, 1e-37f), fmaxf(sk4.z * fs, 1e-37f), fmaxf(sk4.w * fs, 1e-37f)};
                const int vis = pn - tb;
                if (__any_sync(kFull, vis < kT8Blk)) {
#pragma unroll 1
                    for (int j0 = 0; j0 < kT8Blk; j0 += 16) {
                        uint32_t x[16];
                        tmem_ld16_issue(tmem_s + (uint32_t)j0, x);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) if (j0 + j >= vis) x[j] = 0xff800000u;
                        tmem_st16(tmem_s + (uint32_t)j0, x);
                    }
                    tmem_st_wait();
                }
                __syncwarp();
                // ---- the largest score (the scores are read from tensor memory twice: 64 of them would not fit the registers)
                float ym = -INFINITY, zm = -INFINITY;
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[32];
                    tmem_ld32_issue(tmem_s + (uint32_t)(h * 32), x);
                    const float ch[2] = {h ? c[2] : c[0], h ? c[3] : c[1]}, lh[2] = {h ? sl4.z : sl4.x, h ? sl4.w : sl4.y};
                    tmem_ld_wait();
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        float m4[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) m4[j] = fmaxf(fmaxf(__uint_as_float(x[g * 16 + j]), __uint_as_float(x[g * 16 + 4 + j])),
                                                                  fmaxf(__uint_as_float(x[g * 16 + 8 + j]), __uint_as_float(x[g * 16 + 12 + j])));
                        const float yg = fmaf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), ch[g], mo);
                        ym = fmaxf(ym, yg);
                        zm = fmaxf(zm, yg + (lh[g] + vo));
                    }
                }
                const Moved8 mv = move8(ym, zm, first, kW8Max);
                mo -= mv.p;
                vo += mv.p - mv.w;
                const float corr = first ? 1.f : exp2_approx(-mv.w);
                l_run *= first ? 1.f : exp2_approx(-mv.p);
                // ---- the block before has been added up: its probabilities may be overwritten, what it left can be scaled
                if (n > 0) {
                    ok = tile8_wait(abort_flag, &vempty[b ^ 1], (uint32_t)((n - 1) >> 1) & 1u, a.wait_limit_ns);
                    if (__any_sync(kFull, !ok)) { ok = false; break; }
                    tc_fence_after_sync();
                }
                __syncwarp();
                if (!first && __any_sync(kFull, corr != 1.f)) {
#pragma unroll 1
                    for (int o0 = 0; o0 < DH; o0 += 16) {
                        uint32_t o[16];
                        tmem_ld16_issue(tmem_o + lane_addr + (uint32_t)o0, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
                        tmem_st16(tmem_o + lane_addr + (uint32_t)o0, o);
                    }
                    tmem_st_wait();
                }
                __syncwarp();
                // ---- weights as f16: a tile's V scale is in the exponent, and taken out of its sum again (a weight 2^-60 of its probability
                // counts as that: it is nothing beside the largest)
                sl4 = *reinterpret_cast<const float4 *>(blk->sv_log2);
                const float t[4] = {fmaxf(sl4.x + vo, -60.f), fmaxf(sl4.y + vo, -60.f), fmaxf(sl4.z + vo, -60.f), fmaxf(sl4.w + vo, -60.f)};
                const float e[4] = {mo + t[0], mo + t[1], mo + t[2], mo + t[3]}, f[4] = {exp2_approx(-t[0]), exp2_approx(-t[1]), exp2_approx(-t[2]), exp2_approx(-t[3])};
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[32];
                    tmem_ld32_issue(tmem_s + (uint32_t)(h * 32), x);
                    const float ch[2] = {h ? c[2] : c[0], h ? c[3] : c[1]}, eh[2] = {h ? e[2] : e[0], h ? e[3] : e[1]}, fh[2] = {h ? f[2] : f[0], h ? f[3] : f[1]};
                    tmem_ld_wait();
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        float sum = 0.f;
#pragma unroll
                        for (int q = 2 * g; q < 2 * g + 2; ++q) {
                            float p[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) p[i] = exp2_approx(fmaf(__uint_as_float(x[q * 8 + i]), ch[g], eh[g]));
                            sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                            sts128(p_row + (((uint32_t)(h * 4 + q) ^ sw) << 4), pack_f16x2(p[0], p[1]), pack_f16x2(p[2], p[3]), pack_f16x2(p[4], p[5]), pack_f16x2(p[6], p[7]));
                        }
                        l_run = fmaf(sum, fh[g], l_run);
                    }
                }
                fence_proxy_async();
                tc_fence_before_sync();
                mbar_arrive(pready);
            }
            if (!ok) break;
            // ---- the chunk's partial result, as kv8_attn_kernel leaves it; a warp writes four rows at a time
            ok = tile8_wait(abort_flag, &vempty[(n - 1) & 1], (uint32_t)((n - 1) >> 1) & 1u, a.wait_limit_ns);
            if (__any_sync(kFull, !ok)) break;
            tc_fence_after_sync();
            const uint32_t out_row = prow != kFull && pn > it.t0 ? prow * (uint32_t)a.slots + (uint32_t)it.chunk : kFull;
            float *mine = a.part + (size_t)out_row * part8_ld(DH);
            const bool large = vo < 0.f;
            const float back = exp2f(large ? -vo - kBig8Log2 : -vo);
            if (out_row != kFull)
                *reinterpret_cast<float2 *>(mine + DH) = make_float2(kP8Log2 - mo + (large ? kBig8Log2 : 0.f), large ? l_run * kBig8 : l_run);
            uint32_t to[8];                          // rows of the four that a warp writes at a time
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = __shfl_sync(kFull, out_row, 4 * i + (lane >> 3));
            __syncwarp();
#pragma unroll 1
            for (int c0 = 0; c0 < DH; c0 += 32) {
                uint32_t o[32];
                tmem_ld32_issue(tmem_o + lane_addr + (uint32_t)c0, o);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * back);
#pragma unroll
                for (int c = 0; c < 8; ++c) sts128(p_row + (((uint32_t)c ^ sw) << 4), o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 4 * i + (lane >> 3), c = lane & 7;
                    const float4 v = *reinterpret_cast<const float4 *>(smem + Lay::O_P + (warp * 32 + r) * 128 + ((c ^ (r & 7)) << 4));
                    if (to[i] != kFull) *reinterpret_cast<float4 *>(a.part + (size_t)to[i] * part8_ld(DH) + c0 + c * 4) = v;
                }
                __syncwarp();
            }
            if (bad) {                               // values that are no number, where the row sees them
                __syncwarp();
                for (int t = max(it.t0, list.row_ctx(list.tpos[it.seq], 0)); out_row != kFull && t < min(it.t1, pn); ++t) {
                    const int blk = page_of(t, a.page, a.shift), pg = a.kv.block_table[(size_t)it.seq * a.kv.max_pages + blk];
                    if ((unsigned)pg >= (unsigned)a.kv.num_pages) continue;
                    const uint8_t *code = a.kv.v_pages + (((size_t)pg * a.Hkv + it.kvh) * a.page + (t - blk * a.page)) * DH;
                    for (int i = 0; i < DH; ++i) if ((code[i] & 0x7f) == 0x7f) mine[i] = NAN;
                }
                __syncwarp();
            }
            tc_fence_before_sync();
            if (item + 1 < i_end) fresh = list.next(it);
        }
    } else if (warp < 8) {
        // ================= copies: thread = a 16-byte piece of tokens trow + 16 u. (Eight lanes hold four pieces of two tokens: their f16 values,
        // two pieces of a row of 64 dims, lie in all banks.)
        const int piece = (lane & 3) | (lane >> 1 & 4), trow = (warp - 4) * 4 + (lane >> 2 & 1) + (lane >> 3 & 2);
        struct Block { int tok, t1, kvh, edge, pg, off; };     // first token (-1: none), the chunk's end, tokens that every row sees; 16-token tile `lane & 3`: page, place in it
        Item8 w{};
        int witem = i_begin, wtok = 0;
        if (i_begin < i_end) { list.at(w, i_begin); wtok = w.t0; }
        auto walk = [&](Block &x) {
            x.tok = -1;
            if (witem >= i_end) return;
            x.tok = wtok; x.t1 = w.t1; x.kvh = w.kvh;
            x.edge = list.row_ctx(list.tpos[w.seq], 0) - wtok;
            const int tile = min(wtok + (lane & 3) * 16, (w.t1 - 1) & ~15), blk = page_of(tile, a.page, a.shift);
            x.off = tile - blk * a.page;
            x.pg = a.kv.block_table[(size_t)w.seq * a.kv.max_pages + blk];
            wtok += kT8Blk;
            if (wtok >= w.t1 && ++witem < i_end) { list.next(w); wtok = w.t0; }
        };
        const uint64_t policy = l2_evict_first();
        struct Values { uint4 v[4]; float scale; int edge; bool there; };       // scale: lanes 0-3 of warp 4: K's of a tile, 4-7: V's
        int ks = 0;
        uint32_t kph = 0;
        const uint32_t k_at = base + Lay::O_K + piece_at<DH>(trow, piece);
        const size_t from = (size_t)trow * DH + piece * 16;
        auto fetch = [&](const Block &x, Values &y) -> bool {          // K into the ring, V into registers
            y.there = x.tok >= 0;
            y.edge = x.edge;
            if (!y.there) return true;
            if (__any_sync(kFull, !tile8_wait(abort_flag, &kempty[ks], kph ^ 1u, a.wait_limit_ns))) return false;
            int pg = x.pg;
            if ((unsigned)pg >= (unsigned)a.kv.num_pages) { atomicOr(a.status, kDevBadPage); pg = 0; }
            const uint32_t slot = (uint32_t)pg * (uint32_t)a.Hkv + (uint32_t)x.kvh, row = slot * (uint32_t)a.page + (uint32_t)x.off;
            if (warp == 4 && lane < 8) y.scale = (lane < 4 ? a.kv.k_scales : a.kv.v_scales)[slot];
            const uint32_t dst = k_at + (uint32_t)(ks * Lay::K);
            const int left = x.t1 - x.tok - trow;                      // (zeros beyond the chunk's end)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const size_t at = (size_t)__shfl_sync(kFull, row, u) * DH + from;
                cp_async16_off_hint<0>(dst + (uint32_t)(u * 16 * DH), a.kv.k_pages + at, u * 16 < left ? 16u : 0u, policy);
                y.v[u] = make_uint4(0, 0, 0, 0);
                if (u * 16 < left) y.v[u] = *reinterpret_cast<const uint4 *>(a.kv.v_pages + at);
            }
            cp_async_arrive(&kfull[ks]);
            if (++ks == kT8KStages) { ks = 0; kph ^= 1u; }
            return true;
        };
        int n = 0;
        const uint32_t v_at = base + Lay::O_V + (uint32_t)(piece >> 2) * (Lay::V / 2) + (uint32_t)trow * 128;
        const uint32_t v0 = v_at + ((uint32_t)((2 * (piece & 3)) ^ (trow & 7)) << 4), v1 = v_at + ((uint32_t)((2 * (piece & 3) + 1) ^ (trow & 7)) << 4);
        auto convert = [&](Values &y) -> bool {
            const int b = n & 1;
            if (__any_sync(kFull, !tile8_wait(abort_flag, &vempty[b], ((uint32_t)(n >> 1) & 1u) ^ 1u, a.wait_limit_ns))) return false;
            Tile8Block *blk = reinterpret_cast<Tile8Block *>(smem + Lay::O_BLK) + b;
            bool bad = false;
            if (y.edge < kT8Blk) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    uint32_t c[4] = {y.v[u].x, y.v[u].y, y.v[u].z, y.v[u].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t nan = trow + 16 * u >= y.edge ? __vcmpeq4(c[i] & 0x7f7f7f7fu, 0x7f7f7f7fu) : 0u;
                        c[i] &= ~nan;
                        bad = bad || nan != 0u;
                    }
                    y.v[u] = make_uint4(c[0], c[1], c[2], c[3]);
                }
                bad = __any_sync(kFull, bad);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t o = (uint32_t)(b * Lay::V + u * 16 * 128);
                sts128(v0 + o, e4m3lo_f16x2(y.v[u].x), e4m3hi_f16x2(y.v[u].x), e4m3lo_f16x2(y.v[u].y), e4m3hi_f16x2(y.v[u].y));
                sts128(v1 + o, e4m3lo_f16x2(y.v[u].z), e4m3hi_f16x2(y.v[u].z), e4m3lo_f16x2(y.v[u].w), e4m3hi_f16x2(y.v[u].w));
            }
            if (warp == 4 && lane < 8) {
                if (lane < 4) blk->sk[lane] = y.scale;
                else blk->sv_log2[lane - 4] = fmaxf(__log2f(y.scale), -300.f);       // (a scale of zero)
            }
            if (lane == 0) blk->bad[warp - 4] = bad ? 1u : 0u;
            fence_proxy_async();
            mbar_arrive(&vfull[b]);
            ++n;
            return true;
        };
        // two blocks are on their way, and the pages of a third
        Block next;
        Values y0, y1;
        walk(next);
        bool ok = fetch(next, y0);
        walk(next);
        ok = ok && fetch(next, y1);
        walk(next);
        while (ok && y0.there) {
            if (!(ok = convert(y0) && fetch(next, y0))) break;
            walk(next);
            if (!y1.there) break;
            if (!(ok = convert(y1) && fetch(next, y1))) break;
            walk(next);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        // ================= products: one thread
        if (lane == 0 && i_begin < i_end) {
            constexpr uint32_t kIdS = (1u << 4) | ((uint32_t)(kT8Blk >> 3) << 17) | (8u << 24);                     // e4m3, both K-major
            constexpr uint32_t kIdO = (1u << 4) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | (8u << 24);            // f16, B MN-major
            const uint32_t qd = umma_desc_lo(base), kd = umma_desc_lo(base + Lay::O_K), pd = umma_desc_lo(base + Lay::O_P);
            // V: two atoms of 64 dims V / 2 apart, groups of eight tokens 1024 bytes apart
            const uint32_t vd = ((base + Lay::O_V) >> 4) | ((uint32_t)(Lay::V / 2 >> 4) << 16);
            int ks = 0;
            uint32_t kph = 0, qph = 0;
            auto scores = [&](int n, bool fresh) -> bool {
                if (fresh) {
                    if (!tile8_wait(abort_flag, qready, qph, a.wait_limit_ns)) return false;
                    qph ^= 1u;
                }
                if (!tile8_wait(abort_flag, &kfull[ks], kph, a.wait_limit_ns)) return false;
                fence_proxy_async();                 // the copies' shared-memory writes, before the tensor core reads them
                tc_fence_after_sync();
                const uint32_t d = tmem + (uint32_t)((n & 1) * kT8Blk), k = kd + (uint32_t)(ks * (Lay::K >> 4));
#pragma unroll
                for (int j = 0; j < 8; ++j) umma_f8(d, qd + (uint32_t)((j >> 2) * (Lay::TILE >> 4) + (j & 3) * 2), k + (uint32_t)((j & 3) * 2), kIdS, j > 0);
                umma_commit(&sfull[n & 1]);
                umma_commit(&kempty[ks]);
                if (++ks == kT8KStages) { ks = 0; kph ^= 1u; }
                return true;
            };
            Item8 it{};
            list.at(it, i_begin);
            int item = i_begin, tok = it.t0, n = 0;
            bool ok = scores(0, true), first = true;
            while (ok) {
                // the block behind this one
                bool more = true, fresh = false, first_next = false;
                tok += kT8Blk;
                if (tok >= it.t1) {
                    more = ++item < i_end;
                    if (more) {
                        fresh = list.next(it);
                        tok = it.t0;
                        first_next = true;
                    }
                }
                if (more && !fresh && !(ok = scores(n + 1, false))) break;
                if (!(ok = tile8_wait(abort_flag, pready, (uint32_t)n & 1u, a.wait_limit_ns) && tile8_wait(abort_flag, &vfull[n & 1], (uint32_t)(n >> 1) & 1u, a.wait_limit_ns))) break;
                tc_fence_after_sync();
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    umma_bf16(tmem_o, pd + (uint32_t)(j * 2), vd + (uint32_t)((n & 1) * (Lay::V >> 4) + j * (2048 >> 4)), kIdO, !(first && j == 0));
                umma_commit(&vempty[n & 1]);
                if (!more) break;
                if (fresh) ok = scores(n + 1, true);         // (the new queries wait for this block's values)
                first = first_next;
                ++n;
            }
            // every product issued above is done once this arrival lands: waited for whatever has given up, before tensor memory is
            // freed and the tiles' shared memory left
            umma_commit(drain);
            tile8_wait(abort_flag, drain, 0, a.wait_limit_ns, true);
        }
        __syncwarp();
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 256);
    }
    if (tid == 0 && *abort_flag) atomicOr(a.status, kDevTimeout8);
    chain_release();
}

// ---- a row's chunks joined in ascending order. A warp for a (query head, row), DH / 32 dims per lane; its lanes hold the weights of
// 32 chunks, and a batch of the chunks' values is requested before they are known. WARPS > 1: the warps of a block take the 32s in turn and are joined in
// their order (contexts that may be long: few rows of many chunks).
template <int DH, int WARPS>
__global__ void __launch_bounds__(128) kv8_merge_kernel(const Attn8Args a) {
    chain_release();
    chain_wait();
    constexpr int stride = part8_ld(DH), D = DH / 32, G = 16, RESULTS = 4 / WARPS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, share = warp % WARPS;
    const int at = (int)blockIdx.x * RESULTS + warp / WARPS, r = at / a.Hq, head = at - r * a.Hq;
    const int seq = r / a.M, m = r - seq * a.M;
    if (seq >= a.B || m >= kv8_rows(a.n_new, seq, a.M)) return;      // padding: left as it was (a block's warps agree where they meet)
    const int max_tokens = min((int)min((long long)a.kv.max_pages * a.page, (long long)kMaxLen), a.max_ctx);
    const int len = kv8_len(a.kv, seq);
    const int n = min(len + m, max_tokens - 1) + 1, c = chunk8(min(len + a.M - 1, max_tokens - 1) + 1, a.M * a.gq);
    const int chunks = ((n - 1) >> c) + 1;
    const float *base = a.part + (size_t)at * a.slots * stride;
    float mu = -INFINITY, l = 0.f, acc[D] = {};
    for (int c0 = share * 32; c0 < chunks; c0 += 32 * WARPS) {
        const int i = c0 + lane;
        const float2 ml = i < chunks ? *reinterpret_cast<const float2 *>(base + (size_t)i * stride + DH) : make_float2(-INFINITY, 0.f);
        float v[G][D];
        auto load = [&](int g0) {
#pragma unroll
            for (int u = 0; u < G; ++u) {
                const float *p = base + (size_t)min(c0 + g0 + u, chunks - 1) * stride + lane * D;
                if constexpr (D == 4) { const float4 x = *reinterpret_cast<const float4 *>(p); v[u][0] = x.x; v[u][1] = x.y; v[u][2] = x.z; v[u][3] = x.w; }
                else { const float2 x = *reinterpret_cast<const float2 *>(p); v[u][0] = x.x; v[u][1] = x.y; }
            }
        };
        load(0);
        float mx = fmaxf(mu, ml.x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float ref = mx == -INFINITY ? 0.f : mx, old = exp2f(mu - ref), w = i < chunks ? exp2f(ml.x - ref) : 0.f;
        mu = mx;
        float lw = ml.y * w;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lw += __shfl_xor_sync(0xffffffffu, lw, o);
        l = l * old + lw;
#pragma unroll
        for (int d = 0; d < D; ++d) acc[d] *= old;
#pragma unroll 1
        for (int g0 = 0; g0 < 32 && c0 + g0 < chunks; g0 += G) {
            if (g0) load(g0);
#pragma unroll
            for (int u = 0; u < G; ++u) {
                const float wu = __shfl_sync(0xffffffffu, w, g0 + u);
                if (c0 + g0 + u < chunks) {
#pragma unroll
                    for (int d = 0; d < D; ++d) acc[d] += v[u][d] * wu;
                }
            }
        }
    }
    if constexpr (WARPS > 1) {
        __shared__ float sm[WARPS][DH + 2];
        const int used = min(WARPS, (chunks + 31) / 32);
        if (used > 1) {
#pragma unroll
            for (int d = 0; d < D; ++d) sm[share][lane * D + d] = acc[d];
            if (lane == 0) { sm[share][DH] = mu; sm[share][DH + 1] = l; }
            __syncthreads();
            if (share) return;
            for (int x = 1; x < used; ++x) mu = fmaxf(mu, sm[x][DH]);
            const float ref = mu == -INFINITY ? 0.f : mu;
            l = 0.f;
#pragma unroll
            for (int d = 0; d < D; ++d) acc[d] = 0.f;
            for (int x = 0; x < used; ++x) {
                const float w = exp2f(sm[x][DH] - ref);
                l += sm[x][DH + 1] * w;
#pragma unroll
                for (int d = 0; d < D; ++d) acc[d] += sm[x][lane * D + d] * w;
            }
        } else if (share) return;
    }
#pragma unroll
    for (int d = 0; d < D; ++d) {
        const float o = acc[d] / l;
        if (a.xop) {
            uint16_t hi, lo;
            split_bf16(o, hi, lo);
            a.xop[(size_t)(2 * r) * a.ld_xop + head * DH + lane * D + d] = hi;
            a.xop[(size_t)(2 * r + 1) * a.ld_xop + head * DH + lane * D + d] = lo;
        } else {
            a.out[((size_t)r * a.Hq + head) * DH + lane * D + d] = f32_bf16bits(o);
        }
    }
}

template <int DH>
int attn8_launch(void (*kern)(const Attn8Args), int ctas, int threads, int smem, const Attn8Args &a, int rows, bool *raised, cudaStream_t st) {
    cudaError_t e = cudaSuccess;
    if (!*raised) {                                  // once per context (every context sets the same limit)
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        *raised = e == cudaSuccess;
    }
    if (e == cudaSuccess) e = launch_chained(kern, dim3(ctas), dim3(threads), (size_t)smem, st, a);
    // (by what the context's max_ctx allows, not by the call's lengths, which the host does not know: room for more than 32 chunks has a result's
    // warps share them)
    if (e == cudaSuccess) e = a.slots > 32 ? launch_chained(kv8_merge_kernel<DH, 4>, dim3(a.Hq * rows), dim3(128), 0, st, a)
                                           : launch_chained(kv8_merge_kernel<DH, 1>, dim3((a.Hq * rows + 3) / 4), dim3(128), 0, st, a);
    return (int)e;
}
template <int DH, int RW, int WR>
int attn8_warps(const Attn8Args &a, int rows, int n_sm, bool *raised, cudaStream_t st) {
    using Lay = Attn8Smem<DH, RW, WR>;
    return attn8_launch<DH>(kv8_attn_kernel<DH, RW, WR>, Lay::CTAS * n_sm, kA8Threads, Lay::TOTAL, a, rows, raised, st);
}

// One tile of pairs: four groups of one warp; up to four: two groups of two, a set for every two tiles. More: tiles of 128 pairs on tcgen05 where
// a 16-token tile has one scale (dh = 128), else two groups of two warps with two tiles each. By the pairs alone, not by the batch or its contexts, so that what a sequence
// gives does not depend on what it is called with, though that is not the faster form everywhere. Measured, us, 28/4 heads of 128, chunks as they are (tcgen05 / the other form): 28
// pairs of 1 x 4000 tokens 19.4 / 15.4, of 17 x up to 4100 49.6 / 50.3, of 48 x 2000 89.0 / 101.5; 35 pairs of 1 x 4000 19.5 / 19.2, of 16 x 1000 22.4 /
// 34.8; 84 pairs of 4 x 4000 22.1 / 44.2; 448 pairs of 1 x 4000 29.6 / 47.2, of 4 x 4000 58.5 / 141.8. Without tcgen05, 16/2 heads, 4 x 4000 tokens: 128 pairs, heads of 64,
// 25.3, of 128 in blocks of 24 tokens 32.2; 512 pairs, heads of 64, 52.1.
template <int DH>
int attn8_pick(const Attn8Args &a, int rows, int n_sm, bool *raised, cudaStream_t st) {
    const int pairs = a.M * a.gq;
    if (pairs <= 8) return attn8_warps<DH, 1, 1>(a, rows, n_sm, raised, st);
    if (pairs <= 32) return attn8_warps<DH, 1, 2>(a, rows, n_sm, raised + 1, st);
    if (DH == 128 && a.tiles16) return attn8_launch<DH>(kv8_tile_kernel, 2 * n_sm, kT8Threads, Tile8Smem::TOTAL, a, rows, raised + 3, st);
    return attn8_warps<DH, 2, 2>(a, rows, n_sm, raised + 2, st);
}

}  // namespace

int kv8_append(const Kv8Shape &sh, const bf16_t *k, const bf16_t *v, long long ld, const Kv8Ptrs &kv, int B, int M, const int32_t *n_new,
               uint32_t *status, cudaStream_t st, long long *launches) {
    Append8Args a{};
    a.Hkv = sh.Hkv; a.page = sh.page; a.shift = shift_of(sh.page); a.max_ctx = sh.max_ctx; a.B = B; a.M = M;
    a.nb = (M + sh.page - 2) / sh.page + 1;
    a.k = k; a.v = v; a.ld = ld; a.n_new = n_new; a.kv = kv; a.status = status;
    const long long warps = (long long)B * a.nb * 2 * sh.Hkv, blocks = (warps + kAppendWarps - 1) / kAppendWarps;
    if (blocks > 0x7fffffffll) return (int)cudaErrorInvalidConfiguration;
    ++*launches;
    auto kern = sh.dh == 128 ? kv8_append_kernel<128> : kv8_append_kernel<64>;
    return (int)launch_chained(kern, dim3((unsigned)blocks), dim3(kAppendWarps * 32), 0, st, a);
}

int kv8_read(const Kv8Shape &sh, const Kv8Ptrs &kv, int B, int max_n, const int32_t *start, const int32_t *count, bf16_t *out_k, bf16_t *out_v,
             uint32_t *status, cudaStream_t st, long long *launches) {
    Read8Args a{};
    a.Hkv = sh.Hkv; a.page = sh.page; a.shift = shift_of(sh.page); a.max_ctx = sh.max_ctx; a.B = B; a.max_n = max_n;
    const long long slots = (long long)kv.max_pages * sh.page, most = slots < sh.max_ctx ? slots : sh.max_ctx;       // no sequence has more to read
    a.tiles = (int)(((max_n < most ? max_n : most) + 15) / 16); a.start = start; a.count = count; a.kv = kv; a.out_k = out_k; a.out_v = out_v; a.status = status;
    const long long warps = (long long)B * a.tiles * sh.Hkv, blocks = (warps + kReadWarps - 1) / kReadWarps;
    if (blocks > 0x7fffffffll) return (int)cudaErrorInvalidConfiguration;
    ++*launches;
    auto kern = sh.dh == 128 ? kv8_read_kernel<128> : kv8_read_kernel<64>;
    return (int)launch_chained(kern, dim3((unsigned)blocks), dim3(kReadWarps * 32), 0, st, a);
}

int kv8_attention_slots(const Kv8Shape &sh, int M) {
    // the largest number of chunks of any context up to max_ctx
    const Chunk8 r = chunk8_rule(M * (sh.Hq / sh.Hkv));
    auto up = [](int n, int c) { return ((n - 1) >> c) + 1; };
    const int few = up(sh.max_ctx, r.first) < r.few ? up(sh.max_ctx, r.first) : r.few, most = up(sh.max_ctx, r.base) < r.most ? up(sh.max_ctx, r.base) : r.most;
    return few > most ? few : most;
}

int kv8_attention_sequences(const Kv8Shape &sh, int M) {
    // a list's costs (see List8) are added up in 31 bits: the sets and strides of attn8_pick's forms, at max_ctx
    const int pairs = M * (sh.Hq / sh.Hkv), set = pairs <= 8 ? 8 : pairs <= 32 ? 16 : sh.dh == 128 && sh.page % 16 == 0 ? kT8Pairs : 32, stride = pairs <= 8 ? 4 * kA8Blk : 2 * kA8Blk;
    const long long cost = (3 + 2ll * kv8_attention_slots(sh, M) + (sh.max_ctx + stride - 1) / stride) * sh.Hkv * ((pairs + set - 1) / set);
    const long long fit = 0x7fffffffll / cost;
    return fit < kBatchRows ? (int)fit : kBatchRows;
}

int kv8_attention(const Kv8AttnCall &c, cudaStream_t st, long long *launches) {
    Attn8Args a{};
    a.Hq = c.sh.Hq; a.Hkv = c.sh.Hkv; a.gq = c.sh.Hq / c.sh.Hkv; a.page = c.sh.page; a.shift = shift_of(c.sh.page); a.max_ctx = c.sh.max_ctx;
    a.slots = kv8_attention_slots(c.sh, c.M); a.tiles16 = c.sh.page % 16 == 0; a.B = c.B; a.M = c.M; a.q = c.q; a.ldq = c.ldq; a.n_new = c.n_new; a.kv = c.kv; a.part = c.part;
    a.out = c.out; a.xop = c.xop; a.ld_xop = c.ld_xop; a.status = c.status;
    a.wait_limit_ns = c.wait_limit_ns; a.extra_arrivals = c.extra_arrivals;
    *launches += 2;
    return c.sh.dh == 128 ? attn8_pick<128>(a, c.B * c.M, c.n_sm, c.raised, st) : attn8_pick<64>(a, c.B * c.M, c.n_sm, c.raised, st);
}

}  // namespace fmtp
