// Arrays as spans of memory, for checks on the host that what a call writes lies
// apart from all else.

#ifndef ASYMSPEC_STEP_SPAN_H_
#define ASYMSPEC_STEP_SPAN_H_

#include <cstddef>
#include <cstdint>

namespace asym_step {

// Spans without a byte overlap none.
struct Span {
  uintptr_t from, to;
  Span(const void* p, size_t bytes) : from(bytes != 0 ? (uintptr_t)p : 0), to(from + bytes) {}
};

// Whether one of the first `written` spans shares a byte with any other one.  (No branch
// in the loop: a call that is bound by what the host does compares some 50 pairs.)
inline bool overlap(const Span* s, int written, int n) {
  bool any = false;
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < n; ++j) any |= (s[i].from < s[j].to) & (s[j].from < s[i].to);
  return any;
}

// The same for plan_slots, whose workgroups read all requests while others already
// write.  Arrays that are not given, or not yet, are null.
inline bool slots_overlap(const void* lengths, const void* new_tokens, const void* release, const void* table,
                          int max_blocks, const void* n_blocks, const void* ring, int ring_size, const void* state, int B,
                          int width, int total, const void* slots, const void* starts, const void* short_out,
                          const void* n_blocks_out, const void* state_out) {
  const size_t b = (size_t)B * 4;
  auto of = [](const void* p, size_t bytes) { return Span(p, p != nullptr ? bytes : 0); };
  const Span s[] = {of(table, b * (size_t)max_blocks), of(ring, (size_t)ring_size * 4),
                    of(slots, (width > 0 ? (size_t)B * (size_t)width : (size_t)total) * 8), of(starts, b + 4),
                    of(short_out, b), of(n_blocks_out, b), of(state_out, 8),
                    // what is only read
                    of(lengths, b), of(new_tokens, b), of(release, b), of(n_blocks, b), of(state, 8)};
  return overlap(s, 7, sizeof(s) / sizeof(s[0]));
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_SPAN_H_
