// Eviction from a paged cache by accumulated attention weight: which tokens stay, and their way to the new pages.
#include "lq_internal.h"
#include "lq_paged.h"
#include "lq_quant8.h"

namespace lq {

namespace {

struct EvictParams {
  uint16_t *k_pages, *v_pages;
  const int* table;
  float* weights;
  int* slots;                                // [B][Hkv][cap]: slots in the pool of the tokens that stay, -1: without a page
  const Row8* rows;                          // n, x: tokens that stay
  int B, Hkv, log_p, n_pages, max_pages, recent;
};

__device__ __forceinline__ Row8 evicted_row(const EvictParams& P, int i) {
  const Row8Ptr r = rows_ptr(P.rows, sizeof(EvictParams));
  return Row8{r[i].n, r[i].x, 1, r[i].b};
}

// Integers in the order of fp32 numbers; the zeros are equal.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// The tokens that stay, of a (row, kv head): the digits of the smallest of the largest weights are found from the top, 11, 11
// and 10 bits by histograms; then every wavefront counts and places its share of the tokens, in order.
constexpr int SELECT = 1024;                 // threads
__global__ void __launch_bounds__(SELECT) select_kernel(const EvictParams P, const Rows8<ROWS_LISTED> S) {
  (void)S;
  const int item = blockIdx.x, h = item % P.Hkv, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Row8 row = evicted_row(P, item / P.Hkv);
  const int b = row.b < P.B ? row.b : row.b - P.B, other = row.b < P.B ? row.b + P.B : b;
  const int64_t cap = (int64_t)P.max_pages << P.log_p;
  const float* w = P.weights + ((int64_t)row.b * P.Hkv + h) * cap;
  float* w_out = P.weights + ((int64_t)other * P.Hkv + h) * cap;
  int* slots = P.slots + ((int64_t)b * P.Hkv + h) * cap;
  const int* table = P.table + (int64_t)row.b * P.max_pages;
  const int old = row.n - P.recent, need = row.x - P.recent;            // of `old` tokens `need` stay, and all behind them
  auto place = [&](int at, int t) {
    const int id = table[t >> P.log_p];
    slots[at] = is_page(id, P.n_pages) ? (id << P.log_p) + (t & ((1 << P.log_p) - 1)) : -1;
    w_out[at] = w[t];
  };
  for (int i = threadIdx.x; i < P.recent; i += SELECT) place(need + i, old + i);
  if (need == 0) return;

  __shared__ int bins[2048];
  __shared__ int chosen, above;
  uint32_t prefix = 0, mask = 0;
  int left = need;                           // of those that match the prefix, so many stay
  const int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
  for (int d = 0; d < 3; ++d) {
    const int count = 1 << widths[d];
    for (int i = threadIdx.x; i < count; i += SELECT) bins[i] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < old; t += SELECT) {
      const uint32_t u = ordered(w[t]);
      if ((u & mask) == prefix) atomicAdd(&bins[u >> shifts[d] & (count - 1)], 1);
    }
    __syncthreads();
    if (wave == 0) {                         // from the top bin down, count / 64 bins a lane
      const int per = count / 64, top = count - 1 - lane * per;
      int mine = 0;
      for (int i = 0; i < per; ++i) mine += bins[top - i];
      int before = mine;
      for (int x = 1; x < 64; x <<= 1) {
        const int y = __shfl_up(before, x);
        if (lane >= x) before += y;
      }
      before -= mine;
      if (before < left && before + mine >= left) {
        int i = top;
        while (before + bins[i] < left) before += bins[i--];
        chosen = i;
        above = before;
      }
    }
    __syncthreads();
    prefix |= (uint32_t)chosen << shifts[d];
    mask |= (uint32_t)(count - 1) << shifts[d];
    left -= above;
    __syncthreads();
  }
  // tokens over `prefix` stay, and the first `left` of those that are equal to it
  __shared__ int overs[SELECT / 64], equals[SELECT / 64];
  const int share = (old + SELECT - 1) / SELECT * 64, from = wave * share, to = from + share < old ? from + share : old;
  int over = 0, equal = 0;
  for (int t = from + lane; t - lane < to; t += 64) {
    const uint32_t u = t < to ? ordered(w[t]) : 0;
    over += __popcll(__ballot(t < to && u > prefix));
    equal += __popcll(__ballot(t < to && u == prefix));
  }
  if (lane == 0) {
    overs[wave] = over;
    equals[wave] = equal;
  }
  __syncthreads();
  over = equal = 0;
  for (int i = 0; i < wave; ++i) {
    over += overs[i];
    equal += equals[i];
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int t = from + lane; t - lane < to; t += 64) {
    const uint32_t u = t < to ? ordered(w[t]) : 0;
    const uint64_t o = __ballot(t < to && u > prefix), e = __ballot(t < to && u == prefix);
    const int rank = equal + __popcll(e & below);                       // among the equal ones
    const bool stays = (o >> lane & 1) || ((e >> lane & 1) && rank < left);
    if (stays) place(over + __popcll(o & below) + (rank < left ? rank : left), t);
    over += __popcll(o);
    equal += __popcll(e);
  }
}

// Rows to their new places: a wavefront a unit of 32 slots.  grid (units / 4, Hkv, rows)
template <int D>
__global__ void __launch_bounds__(256) move_kernel(const EvictParams P, const Rows8<ROWS_LISTED> S) {
  (void)S;
  constexpr int ND = D / 32, NT = D / 16;
  const int h = blockIdx.y, lane = threadIdx.x & 63, unit = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), a = lane / 16;
  const Row8 row = evicted_row(P, blockIdx.z);
  if (32 * unit >= row.x) return;
  const int b = row.b < P.B ? row.b : row.b - P.B, other = row.b < P.B ? row.b + P.B : b;
  const int id = P.table[(int64_t)other * P.max_pages + (unit >> (P.log_p - 5))];
  if (!is_page(id, P.n_pages)) return;
  const int here = row.x - 32 * unit < 32 ? row.x - 32 * unit : 32;
  const int* slots = P.slots + ((((int64_t)b * P.Hkv + h) * P.max_pages) << P.log_p) + 32 * unit;
  const int64_t off = unit_offset(id, P.Hkv, h, P.log_p, unit, D);
  auto page_of = [&](int slot) { return (((int64_t)(slot >> P.log_p) * P.Hkv + h) << P.log_p) * D; };
  const int in_page = (1 << P.log_p) - 1;
  int ks[2], vs[8];
#pragma unroll
  for (int x = 0; x < 2; ++x) ks[x] = 16 * x + lane % 16 < here ? slots[16 * x + lane % 16] : -1;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int t = 16 * (e >> 2) + 4 * a + (e & 3);
    vs[e] = t < here ? slots[t] : -1;
  }
  u32x4 k[2 * ND];
#pragma unroll
  for (int x = 0; x < 2 * ND; ++x) {
    const int s = ks[x / ND];
    k[x] = u32x4{0, 0, 0, 0};
    if (s >= 0) k[x] = *reinterpret_cast<const u32x4*>(P.k_pages + page_of(s) + k_fp_index(s & in_page, 32 * (x % ND) + 8 * a, ND));
  }
  uint16_t v[NT][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint16_t* from = P.v_pages + (vs[e] >= 0 ? page_of(vs[e]) + v_fp_index(vs[e] & in_page, lane % 16, NT) : 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) v[t][e] = vs[e] >= 0 ? from[t * 512] : 0;
  }
#pragma unroll
  for (int x = 0; x < 2 * ND; ++x)
    if (16 * (x / ND) + lane % 16 < here) *reinterpret_cast<u32x4*>(P.k_pages + off + x * 512 + lane * 8) = k[x];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    uint16_t* to = P.v_pages + off + t * 512 + lane * 8;
    if (here == 32) {
      *reinterpret_cast<u32x4*>(to) = u32x4{v[t][0] | (uint32_t)v[t][1] << 16, v[t][2] | (uint32_t)v[t][3] << 16,
                                            v[t][4] | (uint32_t)v[t][5] << 16, v[t][6] | (uint32_t)v[t][7] << 16};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (16 * (e >> 2) + 4 * a + (e & 3) < here) to[e] = v[t][e];
    }
  }
}

}  // namespace

hipError_t launch_evict_paged(const ShapePaged& s, const lq_cache_paged& c, int recent, int most_kept, void* ws, const RowArg8& rows,
                              int count, hipStream_t st) {
  EvictParams p{(uint16_t*)c.k_pages, (uint16_t*)c.v_pages, c.table, c.weights, split_workspace(s, ws).slots, nullptr, s.B, s.Hkv,
                log2_of(s.P), s.n_pages, s.max_pages, recent};
  Rows8<ROWS_LISTED> listed{};
  hipError_t e = hand_over(rows, &listed, &p.rows, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(select_kernel, dim3(count * s.Hkv), dim3(SELECT), 0, st, p, listed);
  e = launch_status("select");
  if (e != hipSuccess) return e;
  const dim3 grid(((most_kept + 31) / 32 + 3) / 4, s.Hkv, count);
  if (s.d == 64) hipLaunchKernelGGL(move_kernel<64>, grid, dim3(256), 0, st, p, listed);
  else if (s.d == 96) hipLaunchKernelGGL(move_kernel<96>, grid, dim3(256), 0, st, p, listed);
  else hipLaunchKernelGGL(move_kernel<128>, grid, dim3(256), 0, st, p, listed);
  return launch_status("move");
}

}  // namespace lq
