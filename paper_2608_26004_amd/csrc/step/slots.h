// Block tables and slot maps.  Which blocks a request gets depends on what all
// requests before it need, so every workgroup first scans the requests (a few
// words each, at most 4096 of them) into LDS and then does its share of the
// work, which is one list after another of independent entries: new table
// entries, entries given back, slots.  An entry finds its request by a binary
// search of the scanned sums, so a step of many requests with a token each and
// a prompt of 10^5 tokens spread over the chip alike, in one launch and with no
// workgroup waiting for another: the state a call reads (counts, the ring's
// front) is not what it writes.

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
STEP_DEV SlotsReq slots_req(const SlotsArgs& A, int b) {
  const int given = A.new_tokens ? A.new_tokens[b] : A.width, len = A.lengths[b], held = A.n_blocks[b];
  const bool gone = A.release && A.release[b] != 0;
  int n = max(given, 0);
  if (A.width > 0) n = min(n, A.width);
  const uint32_t end = (uint32_t)max(len, 0) + (uint32_t)n, bs = (uint32_t)A.block_size, full = end / bs;
  SlotsReq q;
  q.fresh = gone ? 0 : n;
  q.need = gone ? 0u : full + (end != full * bs ? 1u : 0u);
  q.held = min(max(held, 0), A.max_blocks);
  return q;
}

// Exclusive sums of three values over the workgroup's threads, in their order.
STEP_DEV void slots_scan(int64_t (&v)[3], int64_t (*lds)[3]) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  int64_t up[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) up[k] = v[k];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int64_t o = __shfl_up(up[k], off, 64);
      if (lane >= off) up[k] += o;
    }
  }
  __syncthreads();
  if (lane == 63) {
#pragma unroll
    for (int k = 0; k < 3; ++k) lds[wave][k] = up[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    for (int w = 0; w < wave; ++w) up[k] += lds[w][k];
    v[k] = up[k] - v[k];
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
  __shared__ int64_t sums[kSlotsThreads / 64][3];
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
  // and what the others take and give is scanned again
  const int per = (B + kSlotsThreads - 1) / kSlotsThreads;
  const int lo = min(B, tid * per), hi = min(B, lo + per);
  int64_t v[3] = {0, 0, 0};
  for (int b = lo; b < hi; ++b) {
    const SlotsReq q = slots_req(A, b);
    delta[b] = q.need <= (uint32_t)A.max_blocks ? (int)q.need - q.held : kShort;
    start[b] = q.fresh;
    if (delta[b] > 0) v[0] += delta[b];
  }
  slots_scan(v, sums);
  int64_t asked = v[0];
  v[0] = v[1] = v[2] = 0;
  for (int b = lo; b < hi; ++b) {
    const int d = delta[b];
    if (d > 0) {
      asked += d;
      if (asked > count) delta[b] = kShort;
      else v[0] += d;
    } else if (d != kShort) {
      v[1] -= d;
    }
    v[2] += start[b];
  }
  slots_scan(v, sums);
  for (int b = lo; b < hi; ++b) {
    const int d = delta[b], fresh = start[b];
    taken[b] = (int)v[0];
    given[b] = (int)v[1];
    start[b] = (int)min(v[2], (int64_t)0x7FFFFFFF);
    if (d > 0) v[0] += d;
    else if (d != kShort) v[1] -= d;
    v[2] += fresh;
  }
  if (lo < hi && hi == B) {
    taken[B] = (int)v[0];
    given[B] = (int)v[1];
    start[B] = (int)min(v[2], (int64_t)0x7FFFFFFF);
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
