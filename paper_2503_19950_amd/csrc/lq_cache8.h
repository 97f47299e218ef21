// Host-side internals of the 8-bit cache: validated shape bundle, rows of different lengths, launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>

#include "../../include/logquant.h"
#include "lq_deal8.h"

namespace lq {

// Up to so many rows (2 KB) travel in the launch's own arguments; more are uploaded into the cache's device scratch
// first, on the same stream.  Rows that are all alike travel as one entry.
typedef const Row8 __attribute__((address_space(4))) * Row8Ptr;
struct RowArg8 {
  const Row8* host;    // B entries, or one
  Row8* dev;
  int n;
  bool same;
};
// One entry for each batch row: on the stack for the batches that travel in a launch's arguments, else from the heap.
struct RowList {
  Row8 few[ROWS_IN_ARGS];
  Row8* many = nullptr;
  Row8* e;
  int n;
  explicit RowList(int rows) : e(few), n(rows) {
    if (n > ROWS_IN_ARGS) e = many = static_cast<Row8*>(malloc(n * sizeof(Row8)));
  }
  ~RowList() { free(many); }
  RowList(const RowList&) = delete;
  bool ok() const { return e != nullptr; }
  bool alike() const {
    for (int b = 1; b < n; ++b)
      if (e[b].n != e[0].n || e[b].x != e[0].x) return false;
    return true;
  }
  RowArg8 arg(void* seq_state, bool same) const { return RowArg8{e, (Row8*)seq_state, n, same}; }
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

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

hipError_t launch_append8(const Shape8& s, const lq_cache8& c, const void* k_new, const void* v_new, int n_max, int blocks,
                          const RowArg8& rows, hipStream_t st);
hipError_t launch_read8(const Shape8& s, const lq_cache8& c, int t0, int n, void* k_out, void* v_out, const RowArg8& rows,
                        hipStream_t st);
hipError_t launch_attn8(const Shape8& s, const lq_cache8& c, const void* q, float scale, void* out, void* ws, const Plan8& plan,
                        const void* k_new, const void* v_new, const RowArg8& rows, hipStream_t st);

}  // namespace lq
