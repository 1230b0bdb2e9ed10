// Argument checks that the C-ABI's entry points share: pointers, alignment, overlap of buffers.  Host code only.
#pragma once
#include <cstddef>
#include <cstdint>

#include "../../include/tvmattn.h"
#include "tvm_common.h"

namespace {

inline bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// A buffer as the overlap check sees it: `dims` levels of (count, byte stride) around an innermost run of
// `inner` bytes.  dims = 0 is a plain range.
struct Buf {
  const void* p;
  int dims;
  long long n[3], s[3];
  long long inner;
  unsigned align = 16;  // what the pointer has to be a multiple of
  long long extent() const {
    long long e = inner;
    for (int i = 0; i < dims; ++i) e += (n[i] - 1) * s[i];
    return e;
  }
  bool same_layout(const Buf& o) const {
    if (dims != o.dims || inner != o.inner) return false;
    for (int i = 0; i < dims; ++i)
      if (n[i] != o.n[i] || s[i] != o.s[i]) return false;
    return true;
  }
};
const void* const skip = reinterpret_cast<const void*>(uintptr_t(1));  // an entry the call's mode does not use
inline Buf plain(const void* p, long long bytes) { return Buf{p, 0, {0, 0, 0}, {0, 0, 0}, bytes}; }
// Do two buffers of ONE layout, `delta` bytes apart, share a byte?  They do iff delta = sum_k d_k s_k + e with
// |d_k| < n_k and |e| < inner.  Where every stride is at least the extent of the levels inside it (any dense or
// sliced tensor), what the inner levels can contribute is smaller than the stride, so only the two multiples of
// s_k around delta can start a solution: a walk of depth `dims` with two branches per level.
inline bool lattice_hit(const Buf& b, int level, long long delta) {
  if (level == b.dims) return delta > -b.inner && delta < b.inner;
  const long long st = b.s[level];
  long long d0 = delta / st;
  if (delta < 0 && d0 * st != delta) --d0;  // floor
  for (long long d = d0; d <= d0 + 1; ++d)
    if (d > -b.n[level] && d < b.n[level] && lattice_hit(b, level + 1, delta - d * st)) return true;
  return false;
}
inline bool nested(const Buf& b) {
  long long inside = b.inner;
  for (int i = b.dims - 1; i >= 0; --i) {
    if (b.s[i] < inside) return false;
    inside = (b.n[i] - 1) * b.s[i] + inside;
  }
  return true;
}
inline bool overlap(const Buf& a, const Buf& b) {
  const long long pa = (long long)reinterpret_cast<uintptr_t>(a.p), pb = (long long)reinterpret_cast<uintptr_t>(b.p);
  if (pa + a.extent() <= pb || pb + b.extent() <= pa) return false;  // disjoint address ranges
  if (a.same_layout(b) && nested(a)) return lattice_hit(a, 0, pb - pa);
  return true;
}
// Every listed pointer must be non-null and aligned, and no output may overlap an input or another
// output.  Entries that the call's mode does not use are passed with p == skip (a null there is fine, and the
// buffer takes no part in the overlap check).  `inout`: pairs (output index, input index) that may be the very
// same buffer (an update in place).
template <size_t NI, size_t NO>
int check_bufs(const Buf (&in)[NI], const Buf (&out)[NO], int same_o = -1, int same_i = -1, int same_o2 = -1,
               int same_i2 = -1) {
  for (size_t i = 0; i < NI; ++i)
    if (in[i].p != skip && (!in[i].p || !aligned(in[i].p, in[i].align))) return TVMATTN_INVALID_ARG;
  for (size_t o = 0; o < NO; ++o) {
    if (out[o].p == skip) continue;
    if (!out[o].p || !aligned(out[o].p, out[o].align)) return TVMATTN_INVALID_ARG;
    for (size_t i = 0; i < NI; ++i) {
      if (in[i].p == skip) continue;
      const bool allowed = ((int)o == same_o && (int)i == same_i) || ((int)o == same_o2 && (int)i == same_i2);
      if (allowed && out[o].p == in[i].p) continue;
      if (overlap(out[o], in[i])) return TVMATTN_INVALID_ARG;
    }
    for (size_t p = 0; p < o; ++p)
      if (out[p].p != skip && overlap(out[o], out[p])) return TVMATTN_INVALID_ARG;
  }
  return TVMATTN_OK;
}
inline Buf unless(bool unused, Buf b) {
  if (unused) b.p = skip;
  return b;
}
inline long long esz_of(int dtype) { return dtype == TVMATTN_F32 ? 4 : 2; }

}  // namespace
