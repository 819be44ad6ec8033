// Operators over a paged K/V cache held in 8 bits (e4m3 codes, one fp32 scale for each block of tokens and KV head; a block is a
// page): quantising rows into it, reading it back, attention over it. Used by the entry points of api.cu and by the batched
// target step.
#pragma once
#include "mega.cuh"

namespace fmtp {

struct Kv8Ptrs {
    uint8_t *k_pages, *v_pages;           // [num_pages][Hkv][page][dh]
    float *k_scales, *v_scales;           // [num_pages][Hkv]
    const int32_t *block_table, *seq_lens;
    int num_pages, max_pages;
};

struct Kv8Shape {
    int Hq, Hkv, dh, page, max_ctx;
};

// Rows m < n_new[b] (NULL: all M) of every sequence become positions L_b + m of the cache.
int kv8_append(const Kv8Shape &sh, const bf16_t *k, const bf16_t *v, long long ld, const Kv8Ptrs &kv, int B, int M, const int32_t *n_new,
               uint32_t *status, cudaStream_t st, long long *launches);

// Positions start[b] .. start[b] + count[b] - 1 (NULL: 0, and what is committed from there on), at most max_n of them.
int kv8_read(const Kv8Shape &sh, const Kv8Ptrs &kv, int B, int max_n, const int32_t *start, const int32_t *count, bf16_t *out_k, bf16_t *out_v,
             uint32_t *status, cudaStream_t st, long long *launches);

struct Kv8AttnCall {
    Kv8Shape sh;
    Kv8Ptrs kv;
    const bf16_t *q;                      // row r = b * M + m at q + r * ldq: [Hq][dh]
    long long ldq;
    int B, M;                             // B <= 64 sequences, M <= 64 rows of each
    const int32_t *n_new;                 // as above
    float *part;                          // [rows][Hq][kv8_attention_slots][dh + 4] partial results of a context's chunks
    bf16_t *out;                          // [rows][Hq][dh], or
    bf16_t *xop;                          // the next GEMM's operand: rows 2r (high parts) and 2r + 1 (low parts), ld_xop apart
    int ld_xop;
    uint32_t *status;
    int n_sm;
    unsigned long long wait_limit_ns;     // every wait inside the kernels gives up after this long
    int extra_arrivals;                   // self-test: see fmtp_selftest_inject_wait_timeout
    bool *raised;                         // [4] the context's: kernels whose shared-memory limit has been raised
};
int kv8_attention_slots(const Kv8Shape &sh, int M);
int kv8_attention_sequences(const Kv8Shape &sh, int M);       // that a launch takes, 0 to 64
int kv8_attention(const Kv8AttnCall &c, cudaStream_t st, long long *launches);

}  // namespace fmtp
