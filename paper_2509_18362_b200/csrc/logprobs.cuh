// Log probabilities of given tokens, entropy and top alternatives of rows of logits: see include/fastmtp.h.
#pragma once
#include "mega.cuh"

namespace fmtp {

constexpr int kLpMaxRows = 4096;
constexpr int kLpMaxTop = 32;
constexpr int kLpStrips = 256;                       // maxima of a part (see logprobs.cu)

// What a CTA knows of its part of a row.
struct LpPart {
    float m, s, t, pad;                              // with y = x log2(e) - m: sum of 2^y, sum of 2^y y
};

struct LpCall {
    const void *logits;                              // [rows][ld], bf16 or fp32
    int f32;
    long long ld;
    const int32_t *tokens;                           // [rows] or NULL
    int rows, V, top;
    float *out_logprob, *out_entropy;                // [rows] or NULL
    int32_t *out_ids;                                // [rows][top]
    float *out_tops;                                 // [rows][top]
    LpPart *parts;                                   // [logprobs_slots(n_sm)]
    uint32_t *strips;                                // [logprobs_slots(n_sm)][kLpStrips]
    uint32_t *counters;                              // [kLpMaxRows], zero between calls
    uint32_t *status;
    int n_sm;
};

int logprobs_slots(int n_sm);
int logprobs_launch(const LpCall &c, cudaStream_t st);

}  // namespace fmtp
