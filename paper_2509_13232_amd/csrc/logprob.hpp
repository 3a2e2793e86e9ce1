// Log-probs of given tokens with entropy and top alternatives, and their gradient: what the logits-in and the head forms share.
#pragma once

#include "pg_common.hpp"

namespace spo {

// Entries of exponent zero weigh nothing in an entropy, however far below the maximum they lie: z - max is kept above this
// (in binary logarithms), so that a logit of -inf adds an exact zero and not 0 * -inf.
constexpr float kLowest2 = -1024.0f;
constexpr float kLn2 = 0.6931471805599453f;

// Running (maximum m, sum s of 2^x, sum u of x 2^x) with x = (z - m) log2(e), joined with another one.
__device__ __forceinline__ void score_join(float &m, float &s, float &u, float om, float os, float ou) {
    const float nm = fmaxf(m, om);
    const float d = fmaxf((m - nm) * kLog2e, kLowest2), od = fmaxf((om - nm) * kLog2e, kLowest2);
    const float f = __builtin_amdgcn_exp2f(d), of = __builtin_amdgcn_exp2f(od);
    u = f * fmaf(d, s, u) + of * fmaf(od, os, ou);
    s = f * s + of * os;
    m = nm;
}

// entropy = lse - sum p z = ln s - ln2 u / s
__device__ __forceinline__ float score_entropy(float s, float u) { return logf(s) - kLn2 * (u / s); }

int head_logprob_fwd_workspace(const spo_logprob_desc *d, size_t *bytes);
int head_logprob_fwd(const spo_logprob_desc *d, float *logp, float *lse, float *entropy, void *ws, size_t ws_bytes, hipStream_t s);
int head_logprob_bwd_workspace(const spo_logprob_desc *d, int64_t chunk_tokens, size_t *bytes);
int head_logprob_bwd(const spo_logprob_desc *d, const float *lse, const float *entropy, const float *d_logp, const float *d_entropy,
                     void *d_hidden, int d_hidden_dtype, void *d_W, int d_W_dtype, int accumulate_dW, int64_t chunk_tokens, void *ws,
                     size_t ws_bytes, hipStream_t s);

}  // namespace spo
