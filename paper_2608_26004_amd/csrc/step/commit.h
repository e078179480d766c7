// Committed tokens: one wave per request, one lane per token of the step (K + 1
// of at most 64), so the cut behind the first stop token is one ballot.  A few
// hundred bytes a request; the launch bounds it (2.3 us for 8 requests of 3 tokens, 3.2 for
// 512 of 9 with 5 stop tokens).

#ifndef ASYMSPEC_STEP_COMMIT_H_
#define ASYMSPEC_STEP_COMMIT_H_

#include "row.h"

namespace asym_step {

constexpr int kCommitThreads = 256;
constexpr int kCommitPer = kCommitThreads / 64;     // requests of a workgroup

struct CommitArgs {
  const int32_t* accept_len;
  const int32_t* next_token;
  const int32_t* draft_tokens;
  int64_t draft_stride;
  int32_t* history;
  const int32_t* lengths;
  const int32_t* finished;
  const int32_t* stop_tokens;
  const int32_t* max_lengths;
  int32_t* lengths_out;
  int32_t* finished_out;
  int32_t* tokens_out;
  int32_t* counts_out;
  int max_history, n_stop, B, K;
};

__global__ __launch_bounds__(kCommitThreads) void commit_kernel(CommitArgs A) {
  const int b = (int)blockIdx.x * kCommitPer + ((int)threadIdx.x >> 6), i = (int)threadIdx.x & 63;
  if (b >= A.B) return;
  const int acc = A.accept_len[b], len = A.lengths[b];
  const bool done = A.finished && A.finished[b] != 0;
  const bool valid = acc >= 0 && acc <= A.K;
  const int limit = A.max_lengths ? min(max(A.max_lengths[b], 0), A.max_history) : A.max_history;
  int tok = A.next_token[b];
  if (i < acc && i < A.K) tok = A.draft_tokens[b * A.draft_stride + i];
  int n = valid && !done && len >= 0 ? min(acc + 1, max(limit - len, 0)) : 0;
  bool stop = false;
  for (int k = 0; k < A.n_stop; ++k) stop = stop || tok == A.stop_tokens[k];
  const unsigned long long hits = __ballot(stop && i < n);
  if (hits != 0ull) n = __ffsll(hits);
  if (i < n) A.history[(size_t)b * A.max_history + len + i] = tok;
  if (i <= A.K) A.tokens_out[(size_t)b * (A.K + 1) + i] = i < n ? tok : -1;
  if (i == 0) {
    A.lengths_out[b] = len + n;
    A.finished_out[b] = done || hits != 0ull || (valid && len + n >= limit) ? 1 : 0;
    A.counts_out[b] = n;
  }
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_COMMIT_H_
