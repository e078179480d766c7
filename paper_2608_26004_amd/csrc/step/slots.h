// Block tables and slot maps.  Which blocks a request gets depends on what all
// requests before it need, so every workgroup first scans the requests (a few
// words each, at most 4096 of them) into LDS and then does its share of the
// work, which is one list after another of independent entries: new table
// entries, entries given back, slots.  An entry finds its request by a binary
// search of the scanned sums, so a step of many requests with a token each and
// a prompt of 10^5 tokens spread over the chip alike, in one launch and with no
// workgroup waiting for another: the state a call reads (counts, the ring's
// front) is not what it writes.
//
// A launch and three dependent loads (requests, tables or ring, entries) behind two scans
// bound it: 3.3 us for 8 requests, 5.1 for 512 of 9 tokens each, 5.3 for 64 prompts of 200000
// tokens in all (6.6 and 6.7 with scans of 64 bits over shuffles and a thread's requests
// loaded one behind the other).

#ifndef ASYMSPEC_STEP_SLOTS_H_
#define ASYMSPEC_STEP_SLOTS_H_

#include "row.h"

namespace asym_step {

constexpr int kSlotsThreads = 256;

struct SlotsArgs {
  const int32_t* lengths;
  const int32_t* new_tokens;
  const int32_t* release;
  int32_t* table;
  const int32_t* n_blocks;
  int32_t* ring;
  const int32_t* state;
  int64_t* slots;
  int32_t* starts;
  int32_t* short_out;
  int32_t* n_blocks_out;
  int32_t* state_out;
  int max_blocks, ring_size, block_size, B, width, total;
};

// What a request has and needs.  Lengths and new tokens are below 2^31 each, so
// positions fit 32 bits without a sign.
struct SlotsReq {
  uint32_t need;          // blocks
  int held, fresh;        // blocks held; new tokens
};
STEP_DEV SlotsReq slots_req(const SlotsArgs& A, int given, int len, int held, int release) {
  int n = max(given, 0);
  if (A.width > 0) n = min(n, A.width);
  const uint32_t end = (uint32_t)max(len, 0) + (uint32_t)n, bs = (uint32_t)A.block_size, full = end / bs;
  SlotsReq q;
  q.fresh = release != 0 ? 0 : n;
  q.need = release != 0 ? 0u : full + (end != full * bs ? 1u : 0u);
  q.held = min(max(held, 0), A.max_blocks);
  return q;
}

// Sums below 2^32, or 2^32 - 1.
STEP_DEV uint32_t slots_add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
template <int CTRL, int ROWMASK = 0xF>
STEP_DEV uint32_t slots_dpp(uint32_t x) {     // 0 where a lane has no source
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWMASK, 0xF, false);
}
// Exclusive sums of N values over the workgroup's threads, in their order.
template <int N>
STEP_DEV void slots_scan(uint32_t (&v)[N], uint32_t (*lds)[3]) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  uint32_t up[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    uint32_t x = v[k];
    x = slots_add(x, slots_dpp<0x111>(x));
    x = slots_add(x, slots_dpp<0x112>(x));
    x = slots_add(x, slots_dpp<0x114>(x));
    x = slots_add(x, slots_dpp<0x118>(x));
    x = slots_add(x, slots_dpp<0x142, 0xA>(x));
    up[k] = slots_add(x, slots_dpp<0x143, 0xC>(x));
    v[k] = slots_dpp<0x138>(up[k]);
  }
  __syncthreads();
  if (lane == 63) {
#pragma unroll
    for (int k = 0; k < N; ++k) lds[wave][k] = up[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
#pragma unroll
    for (int w = 0; w < kSlotsThreads / 64; ++w) v[k] = slots_add(v[k], w < wave ? lds[w][k] : 0u);
  }
}

// The request whose run [from[b], from[b + 1]) holds i (from[0] <= i < from[B]).
STEP_DEV int slots_find(const int* from, int B, int i) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (from[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kSlotsThreads) void slots_kernel(SlotsArgs A) {
  extern __shared__ int slots_lds[];
  __shared__ uint32_t sums[kSlotsThreads / 64][3];
  const int tid = (int)threadIdx.x, B = A.B, N = A.ring_size;
  int* taken = slots_lds;                   // [B + 1] blocks taken ahead of a request
  int* given = slots_lds + B + 1;           // [B + 1] blocks given back ahead of it
  int* start = slots_lds + 2 * (B + 1);     // [B + 1] new tokens ahead of it
  int* delta = slots_lds + 3 * (B + 1);     // [B] blocks needed beyond those held; kShort
  constexpr int kShort = (int)0x80000000;
  const int count = min(max(A.state[1], 0), N);
  int head = A.state[0] % N;
  if (head < 0) head += N;

  // each thread scans a run of requests: what all ask for decides who is short,
  // and what the others take and give is scanned again.  Blocks are below 2^31
  // (B * max_blocks), new tokens may add up to more.
  const int per = (B + kSlotsThreads - 1) / kSlotsThreads;
  const int lo = min(B, tid * per), hi = min(B, lo + per);
  uint32_t ask[1] = {0u};
  constexpr int kAhead = 4;             // requests whose values are on their way together
  for (int b0 = lo; b0 < hi; b0 += kAhead) {
    int len[kAhead], held[kAhead], given[kAhead], release[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int b = min(b0 + u, hi - 1);
      len[u] = A.lengths[b];
      held[u] = A.n_blocks[b];
      given[u] = A.width;
      release[u] = 0;
    }
    if (A.new_tokens) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) given[u] = A.new_tokens[min(b0 + u, hi - 1)];
    }
    if (A.release) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) release[u] = A.release[min(b0 + u, hi - 1)];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (b0 + u < hi) {
        const SlotsReq q = slots_req(A, given[u], len[u], held[u], release[u]);
        const int d = q.need <= (uint32_t)A.max_blocks ? (int)q.need - q.held : kShort;
        delta[b0 + u] = d;
        start[b0 + u] = q.fresh;
        if (d > 0) ask[0] += (uint32_t)d;
      }
    }
  }
  slots_scan(ask, sums);
  uint32_t asked = ask[0], v[3] = {0u, 0u, 0u};
  for (int b = lo; b < hi; ++b) {
    const int d = delta[b];
    if (d > 0) {
      asked += (uint32_t)d;
      if (asked > (uint32_t)count) delta[b] = kShort;
      else v[0] += (uint32_t)d;
    } else if (d != kShort) {
      v[1] += (uint32_t)-d;
    }
    v[2] = slots_add(v[2], (uint32_t)start[b]);
  }
  slots_scan(v, sums);
  auto most = [](uint32_t x) { return (int)min(x, 0x7FFFFFFFu); };
  for (int b = lo; b < hi; ++b) {
    const int d = delta[b], fresh = start[b];
    taken[b] = (int)v[0];
    given[b] = (int)v[1];
    start[b] = most(v[2]);
    if (d > 0) v[0] += (uint32_t)d;
    else if (d != kShort) v[1] += (uint32_t)-d;
    v[2] = slots_add(v[2], (uint32_t)fresh);
  }
  if (lo < hi && hi == B) {
    taken[B] = (int)v[0];
    given[B] = (int)v[1];
    start[B] = most(v[2]);
  }
  __syncthreads();

  auto ring_at = [&](int i) {         // i < 2 N entries behind the ring's front
    const uint32_t at = (uint32_t)head + (uint32_t)i;
    return A.ring + (at >= (uint32_t)N ? at - (uint32_t)N : at);
  };
  auto held_of = [&](int b) { return min(max(A.n_blocks[b], 0), A.max_blocks); };
  const int first = (int)blockIdx.x * kSlotsThreads + tid, step = (int)gridDim.x * kSlotsThreads;

  // the lists one behind the other, so that a thread has few entries of any
  const int places = A.width > 0 ? B * A.width : A.total, n_taken = taken[B], n_given = given[B];
  const int64_t all = (int64_t)places + n_taken + n_given;
  for (int64_t i = first; i < all; i += step) {
    if (i < places) {
      const int b = A.width > 0 ? (int)((uint32_t)i / (uint32_t)A.width) : slots_find(start, B, (int)i);
      const int j = A.width > 0 ? (int)i - b * A.width : (int)i - start[b];
      int64_t slot = -1;
      if (j < start[b + 1] - start[b] && delta[b] != kShort) {
        const uint32_t p = (uint32_t)max(A.lengths[b], 0) + (uint32_t)j, bs = (uint32_t)A.block_size;
        const int k = (int)(p / bs), held = held_of(b);
        const int id = k < held ? A.table[(size_t)b * A.max_blocks + k] : *ring_at(taken[b] + (k - held));
        slot = (int64_t)id * A.block_size + (p - (uint32_t)k * bs);
      }
      A.slots[i] = slot;
    } else if (i < (int64_t)places + n_taken) {
      const int q = (int)(i - places), b = slots_find(taken, B, q);
      A.table[(size_t)b * A.max_blocks + held_of(b) + (q - taken[b])] = *ring_at(q);
    } else {
      const int q = (int)(i - places - n_taken), b = slots_find(given, B, q);
      int32_t* e = A.table + (size_t)b * A.max_blocks + held_of(b) + delta[b] + (q - given[b]);
      if (q < N - count) *ring_at(count + q) = *e;
      *e = -1;
    }
  }
  for (int b = first; b < B; b += step) {
    const bool is_short = delta[b] == kShort;
    A.short_out[b] = is_short ? 1 : 0;
    A.n_blocks_out[b] = held_of(b) + (is_short ? 0 : delta[b]);
  }
  if (A.starts)
    for (int b = first; b <= B; b += step) A.starts[b] = start[b];
  if (first == 0) {
    const int64_t back = min((int64_t)n_given, (int64_t)N - count);
    A.state_out[0] = (int)(((int64_t)head + n_taken) % N);
    A.state_out[1] = (int)((int64_t)count - n_taken + back);
  }
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_SLOTS_H_
