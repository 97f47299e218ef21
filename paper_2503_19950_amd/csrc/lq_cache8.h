// Host-side internals of the 8-bit cache: validated shape bundle, rows of different lengths, launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/logquant.h"

namespace lq {

struct Shape8 {
  int B, Hq, Hkv, d, G, cap;
  int gh;              // query heads of a kv head
  bool bf16;
};
inline int log2_of(int G) { return G == 32 ? 5 : G == 64 ? 6 : 7; }

// What a launch has to know of a batch row.
struct Row8 {
  int n;               // tokens that the row holds (append: before the call; a step: after it)
  int x;               // append: tokens that it takes; attention: its first workgroup
  int parts;           // attention: workgroups that share an item of it (Plan8)
  int b;               // attention: which row
};
// Up to so many rows (2 KB) travel in the launch's own arguments; more are uploaded into the cache's device scratch
// first, on the same stream.  Rows that are all alike travel as one entry.
constexpr int ROWS_IN_ARGS = 128;
typedef const Row8 __attribute__((address_space(4))) * Row8Ptr;
struct RowArg8 {
  const Row8* host;    // B entries, or one
  Row8* dev;
  int n;
  bool same;
};
enum RowMode { ROWS_SAME, ROWS_LISTED };
template <int MODE> struct Rows8 {};                               // a kernel's last argument
template <> struct Rows8<ROWS_LISTED> { Row8 e[ROWS_IN_ARGS]; };

// Fills the last argument, or the device scratch.
hipError_t upload_rows8(Row8* dev, const Row8* host, int n, hipStream_t st);
inline hipError_t hand_over(const RowArg8& a, Rows8<ROWS_LISTED>* in_args, const Row8** dev, hipStream_t st) {
  *dev = nullptr;
  if (a.n <= ROWS_IN_ARGS) {
    for (int i = 0; i < a.n; ++i) in_args->e[i] = a.host[i];
    return hipSuccess;
  }
  *dev = a.dev;
  return upload_rows8(a.dev, a.host, a.n, st);
}

// Kernel side: the rows in device memory, or in the argument block, `offset` bytes from its start.  They are read through
// the segment's address (scalar loads): indexing the by-value parameter would copy all of it into private memory first.
__device__ __forceinline__ Row8Ptr rows_ptr(const Row8* dev, size_t offset) {
  typedef const char __attribute__((address_space(4))) * BytePtr;
  if (dev) return (Row8Ptr)(uintptr_t)dev;
  return (Row8Ptr)((BytePtr)__builtin_amdgcn_kernarg_segment_ptr() + offset);
}

// How attention is dealt to workgroups.  A (row, kv head, head group) is an item; its work is counted in units of 32
// tokens, codes as 1 and rows of the tail, twice as wide, as 2.  A workgroup takes an item, or one of `parts` equal parts
// of it, which the last of them to finish joins.  Rows with the most work come first.
struct Plan8 {
  int groups, hb;      // head groups of a kv head; heads in each (at most 32, two sets of 16; the last has the rest)
  int blocks, waves;
};
// (A fused step counts a block that its token fills up among the rows of the tail, which is what it reads.)
inline int units8(int n, int G, bool step) {
  const int full = (step ? n - 1 : n) / G * G;
  return full / 32 + 2 * ((n - full + 31) / 32);
}

hipError_t launch_append8(const Shape8& s, const lq_cache8& c, const void* k_new, const void* v_new, int n_max, int blocks,
                          const RowArg8& rows, hipStream_t st);
hipError_t launch_read8(const Shape8& s, const lq_cache8& c, int t0, int n, void* k_out, void* v_out, const RowArg8& rows,
                        hipStream_t st);
hipError_t launch_attn8(const Shape8& s, const lq_cache8& c, const void* q, float scale, void* out, void* ws, const Plan8& plan,
                        const void* k_new, const void* v_new, const RowArg8& rows, hipStream_t st);

// A workspace: the counters of the items, each item's (one for all its parts, 16 for sixteen of them each) in a cache line,
// then room for the partial results of the workgroups that share an item (they come first in the grid), and as much again for
// those of sixteen joined.
constexpr int CTR8 = 32;           // ints from one counter to the next
constexpr int MAX_PARTS8 = 1024;
// Head groups of a kv head.  More than 16 heads are two sets in one workgroup, which read the cache once, or two workgroups,
// which share the join's work: the former in launches that read 24 MB or more.
inline int head_groups8(const Shape8& s, bool large) { return (s.gh + (large ? 31 : 15)) / (large ? 32 : 16); }
inline size_t counter_bytes8(const Shape8& s) { return (size_t)s.B * s.Hkv * head_groups8(s, false) * CTR8 * sizeof(int); }
inline int partial_floats8(int hb, int d) { return hb * (d + 4); }   // o, then m and l, padded to 16 bytes
// LDS of a workgroup: each wavefront's results of a set of heads, or a join's (o, m and l of a share for every thread).
inline int lds_bytes8(int waves, int hb, int d) {
  const int merge = waves * partial_floats8(hb < 16 ? hb : 16, d), join = waves * 64 * 6;
  return (merge > join ? merge : join) * (int)sizeof(float);
}

}  // namespace lq
