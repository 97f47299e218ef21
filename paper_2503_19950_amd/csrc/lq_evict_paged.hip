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
  int* found;                                // histograms and counts of long rows
  int pieces;                                // of the longest row
  const Row8* rows;                          // n, x: tokens that stay
  int B, Hkv, log_p, n_pages, max_pages, recent;
};

__device__ __forceinline__ Row8 evicted_row(const EvictParams& P, int i) {
  const Row8Ptr r = rows_ptr(P.rows, sizeof(EvictParams));
  return Row8{r[i].n, r[i].x, 1, r[i].b};
}

// Order of LDS accesses within a wavefront (its LDS instructions execute in order: only the compiler has to be told).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Integers in the order of fp32 numbers; the zeros are equal.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// ---- which tokens stay, of a (row, kv head): the smallest weight that stays is found digit by digit, 11, 11 and 10 bits, from
// histograms; what is over it stays, and of what is equal to it the first.  Rows of up to 16384 tokens are a workgroup each, which
// reads the weights once and keeps them in registers; longer ones are cut into pieces of 2048 tokens, whose workgroups add up
// histograms and counts in memory, a launch for each digit, one to count and one to place (131072 tokens x 8 kv heads: as one
// workgroup each, which reads the weights five times, 194 us).
constexpr int THREADS = 1024, WAVES = THREADS / 64, EACH = 16, SHORT = THREADS * EACH, BINS = EVICT_BINS, PIECE = EVICT_PIECE;
static_assert(SHORT == EVICT_SHORT, "what the workspace has room for");
constexpr int SHIFTS[3] = {21, 10, 0}, WIDTHS[3] = {11, 11, 10};

struct Item {
  int b, h, n, keep, old, need;              // of the first `old` tokens `need` stay, and all behind them
  int64_t from, to;                          // row in the weights, before and behind
  const int* table;
};
__device__ __forceinline__ Item item_of(const EvictParams& P, int i) {
  const Row8 row = evicted_row(P, i / P.Hkv);
  Item x;
  x.h = i % P.Hkv;
  x.b = row.b < P.B ? row.b : row.b - P.B;
  x.n = row.n;
  x.keep = row.x;
  x.old = row.n - P.recent;
  x.need = row.x - P.recent;
  const int64_t cap = (int64_t)P.max_pages << P.log_p;
  x.from = ((int64_t)row.b * P.Hkv + x.h) * cap;
  x.to = ((int64_t)(row.b < P.B ? row.b + P.B : x.b) * P.Hkv + x.h) * cap;
  x.table = P.table + (int64_t)row.b * P.max_pages;
  return x;
}
// Token t stays as the at-th.
__device__ __forceinline__ void place(const EvictParams& P, const Item& x, int at, int t, float w) {
  const int id = x.table[t >> P.log_p];
  P.slots[((((int64_t)x.b * P.Hkv + x.h) * P.max_pages) << P.log_p) + at] = is_page(id, P.n_pages) ? (id << P.log_p) + (t & ((1 << P.log_p) - 1)) : -1;
  P.weights[x.to + at] = w;
}

// A histogram in LDS has a word of padding behind every 32 bins: a lane adds up 32.
constexpr int ROOM = BINS + BINS / 32;
__device__ __forceinline__ int bin_at(int i) { return i + i / 32; }
// The bin that the left-th largest falls into, and what is in the bins above it: one wavefront.
__device__ __forceinline__ int2 find_bin(const int* bins, int count, int left) {
  const int lane = threadIdx.x & 63, groups = count / 32, group = groups - 1 - lane;     // the highest first
  int mine = 0;
  if (lane < groups)
#pragma unroll
    for (int i = 0; i < 32; ++i) mine += bins[33 * group + i];
  int upto = mine;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int y = __shfl_up(upto, x);
    if (lane >= x) upto += y;
  }
  const int who = __ffsll(__ballot(upto >= left)) - 1, above = __shfl(upto - mine, who), base = 32 * (groups - 1 - who);
  // its bins, the highest first
  mine = lane < 32 ? bins[bin_at(base + 31 - lane)] : 0;
  upto = mine;
#pragma unroll
  for (int x = 1; x < 32; x <<= 1) {
    const int y = __shfl_up(upto, x);
    if (lane >= x) upto += y;
  }
  const int at = __ffsll(__ballot(above + upto >= left)) - 1;
  return make_int2(base + 31 - at, above + __shfl(upto - mine, at));
}

__global__ void __launch_bounds__(THREADS) select_kernel(const EvictParams P, const Rows8<ROWS_LISTED> S) {
  (void)S;
  const Item x = item_of(P, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float* w = P.weights + x.from;
  for (int i = threadIdx.x; i < P.recent; i += THREADS) place(P, x, x.need + i, x.old + i, w[x.old + i]);
  if (x.need == 0) return;
  if (x.old > SHORT) {                       // (for the launches behind)
    int* memory = P.found + (int64_t)blockIdx.x * (EVICT_MEMORY + 2 * P.pieces);
    for (int i = threadIdx.x; i < 3 * BINS; i += THREADS) memory[i] = 0;
    return;
  }
  // a wavefront's share of the tokens, 64 at a time
  const int rounds = (x.old + THREADS - 1) / THREADS, first = wave * rounds * 64 + lane;
  float mine[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) mine[i] = i < rounds && first + 64 * i < x.old ? w[first + 64 * i] : 0.f;
  __shared__ int bins[ROOM];
  __shared__ int2 found;
  uint32_t prefix = 0, mask = 0;
  int left = x.need;                         // of those that match the prefix, so many stay
#pragma unroll
  for (int d = 0; d < 3; ++d) {
    const int count = 1 << WIDTHS[d];
    for (int i = threadIdx.x; i < bin_at(count); i += THREADS) bins[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint32_t u = ordered(mine[i]);
      if (i < rounds && first + 64 * i < x.old && (u & mask) == prefix) atomicAdd(&bins[bin_at(u >> SHIFTS[d] & (count - 1))], 1);
    }
    __syncthreads();
    if (wave == 0) {
      const int2 f = find_bin(bins, count, left);
      if (lane == 0) found = f;
    }
    __syncthreads();
    prefix |= (uint32_t)found.x << SHIFTS[d];
    mask |= (uint32_t)(count - 1) << SHIFTS[d];
    left -= found.y;
  }
  __shared__ int overs[WAVES], equals[WAVES];
  int over = 0, equal = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const bool in = i < rounds && first + 64 * i < x.old;
    over += __popcll(__ballot(in && ordered(mine[i]) > prefix));
    equal += __popcll(__ballot(in && ordered(mine[i]) == prefix));
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
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const bool in = i < rounds && first + 64 * i < x.old;
    const uint64_t o = __ballot(in && ordered(mine[i]) > prefix), e = __ballot(in && ordered(mine[i]) == prefix);
    const int rank = equal + __popcll(e & below);                       // among the equal ones
    if ((o >> lane & 1) || ((e >> lane & 1) && rank < left)) place(P, x, over + __popcll(o & below) + (rank < left ? rank : left), first + 64 * i, mine[i]);
    over += __popcll(o);
    equal += __popcll(e);
  }
}

// Long rows.  In memory, of an item: three histograms, what each of them says (prefix, and how many of those that match it stay),
// then over and equal of every piece.
constexpr int MEMORY = EVICT_MEMORY;
static_assert(MEMORY == 3 * BINS + 8, "what the workspace has room for");
__device__ __forceinline__ int* memory_of(const EvictParams& P, int i) { return P.found + (int64_t)i * (MEMORY + 2 * P.pieces); }

// After digit D's histogram, all of which is in memory: what it says, from what the one before said.
template <int D>
__device__ __forceinline__ int2 after_digit(int* memory, int need, int* bins, int2* found) {
  const int count = 1 << WIDTHS[D];
  int2* said = reinterpret_cast<int2*>(memory + 3 * BINS);
  for (int i = threadIdx.x; i < count; i += 256) bins[bin_at(i)] = memory[D * BINS + i];
  const int2 before = D ? said[D - 1] : make_int2(0, need);
  __syncthreads();
  if (threadIdx.x < 64) {
    const int2 f = find_bin(bins, count, before.y);
    if (threadIdx.x == 0) {
      *found = make_int2(before.x | f.x << SHIFTS[D], before.y - f.y);
      if (blockIdx.x == 0) said[D] = *found;
    }
  }
  __syncthreads();
  return *found;
}

// grid (pieces, items): digit D's histogram
template <int D>
__global__ void __launch_bounds__(256) histogram_kernel(const EvictParams P, const Rows8<ROWS_LISTED> S) {
  (void)S;
  __shared__ int bins[ROOM];
  __shared__ int2 found;
  const Item x = item_of(P, blockIdx.y);
  const int t0 = blockIdx.x * PIECE + threadIdx.x;
  if (x.need == 0 || x.old <= SHORT || (int)blockIdx.x * PIECE >= x.old) return;
  float w[PIECE / 256];
#pragma unroll
  for (int i = 0; i < PIECE / 256; ++i) w[i] = t0 + 256 * i < x.old ? P.weights[x.from + t0 + 256 * i] : 0.f;
  int* memory = memory_of(P, blockIdx.y);
  uint32_t prefix = 0;
  if constexpr (D > 0) prefix = (uint32_t)after_digit<D - 1>(memory, x.need, bins, &found).x;
  const int count = 1 << WIDTHS[D];
  for (int i = threadIdx.x; i < bin_at(count); i += 256) bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PIECE / 256; ++i) {
    const uint32_t u = ordered(w[i]);
    const bool matches = D == 0 || u >> (D == 1 ? SHIFTS[0] : SHIFTS[1]) == prefix >> (D == 1 ? SHIFTS[0] : SHIFTS[1]);
    if (t0 + 256 * i < x.old && matches) atomicAdd(&bins[bin_at(u >> SHIFTS[D] & (count - 1))], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += 256)
    if (bins[bin_at(i)]) atomicAdd(&memory[D * BINS + i], bins[bin_at(i)]);
}

// grid (pieces, items).  PLACE: with what count_kernel<false> left, else that.
template <bool PLACE>
__global__ void __launch_bounds__(256) count_kernel(const EvictParams P, const Rows8<ROWS_LISTED> S) {
  (void)S;
  constexpr int ROUNDS = PIECE / 256;
  __shared__ int bins[PLACE ? 1 : ROOM];
  __shared__ int2 found;
  __shared__ int overs[4], equals[4], before[2];
  const Item x = item_of(P, blockIdx.y);
  const int piece = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (x.need == 0 || x.old <= SHORT || piece * PIECE >= x.old) return;
  const int first = piece * PIECE + wave * (PIECE / 4) + lane;          // a wavefront's share, 64 at a time
  float w[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) w[i] = first + 64 * i < x.old ? P.weights[x.from + first + 64 * i] : 0.f;
  int* memory = memory_of(P, blockIdx.y);
  int* counts = memory + MEMORY;
  int2 said;
  if constexpr (PLACE) said = reinterpret_cast<const int2*>(memory + 3 * BINS)[2];
  else said = after_digit<2>(memory, x.need, bins, &found);
  const uint32_t prefix = (uint32_t)said.x;
  const int left = said.y;
  int over = 0, equal = 0;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const bool in = first + 64 * i < x.old;
    over += __popcll(__ballot(in && ordered(w[i]) > prefix));
    equal += __popcll(__ballot(in && ordered(w[i]) == prefix));
  }
  if (lane == 0) {
    overs[wave] = over;
    equals[wave] = equal;
  }
  if constexpr (PLACE)
    if (wave == 0) {                         // of the pieces before
      int o = 0, e = 0;
      for (int i = lane; i < piece; i += 64) {
        o += counts[2 * i];
        e += counts[2 * i + 1];
      }
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        o += __shfl_xor(o, m);
        e += __shfl_xor(e, m);
      }
      before[0] = o;
      before[1] = e;
    }
  __syncthreads();
  if constexpr (!PLACE) {
    if (threadIdx.x == 0) {
      counts[2 * piece] = overs[0] + overs[1] + overs[2] + overs[3];
      counts[2 * piece + 1] = equals[0] + equals[1] + equals[2] + equals[3];
    }
    return;
  }
  over = before[0];
  equal = before[1];
  for (int i = 0; i < wave; ++i) {
    over += overs[i];
    equal += equals[i];
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const bool in = first + 64 * i < x.old;
    const uint64_t o = __ballot(in && ordered(w[i]) > prefix), e = __ballot(in && ordered(w[i]) == prefix);
    const int rank = equal + __popcll(e & below);
    if ((o >> lane & 1) || ((e >> lane & 1) && rank < left)) place(P, x, over + __popcll(o & below) + (rank < left ? rank : left), first + 64 * i, w[i]);
    over += __popcll(o);
    equal += __popcll(e);
  }
}

// Rows to their new places: a wavefront a unit of 32 slots.  grid (units / 4, Hkv, rows)
// A token that had no page becomes one of zeros: its new slot lies among others' in a page, and attention knows pages, not slots.
// Keys are pieces of 16 bytes of a token, gathered.  A piece of values holds eight tokens: units that the tokens come from are read
// whole, 16 bytes a lane, and what stays of them is put in its place in LDS, two bytes at a time.  Where the tokens of a unit come
// from more than DENSE others (few stay of many), they are gathered from memory two bytes at a time instead: 8 rows of 16384 tokens x 8
// kv heads, of which a half, a quarter, a sixth and an eighth stay, 229, 165, 145 and 111 us gathered, 182, 148, 136 and 122 read whole,
// 181, 151, 145 and 114 by this rule (149 and 119 of a quarter and an eighth with 8 units, 158 and 112 with 6).
constexpr int DENSE = 7;
template <int D>
__global__ void __launch_bounds__(256) move_kernel(const EvictParams P, const Rows8<ROWS_LISTED> S) {
  (void)S;
  constexpr int ND = D / 32, NT = D / 16;
  __shared__ __align__(16) uint16_t stage[4][32 * D];
  const int h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, unit = (int)blockIdx.x * 4 + wave, a = lane / 16;
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
  const int slot = lane % 32 < here ? slots[lane % 32] : -1;            // lanes 32 .. 63 as 0 .. 31
  u32x4 k[2 * ND];
#pragma unroll
  for (int x = 0; x < 2 * ND; ++x) {
    const int s = __shfl(slot, 16 * (x / ND) + lane % 16);
    k[x] = u32x4{0, 0, 0, 0};
    if (s >= 0) k[x] = *reinterpret_cast<const u32x4*>(P.k_pages + page_of(s) + k_fp_index(s & in_page, 32 * (x % ND) + 8 * a, ND));
  }
  // where a unit of the source begins among the tokens here
  const int from = slot >> 5, last = __shfl_up(slot, 1), before = last >> 5;
  uint32_t starts = (uint32_t)__ballot(slot >= 0 && (lane == 0 || from != before || slot <= last));   // (a page may be named twice)
  auto store_k = [&]() {
#pragma unroll
    for (int x = 0; x < 2 * ND; ++x)
      if (16 * (x / ND) + lane % 16 < here) __builtin_nontemporal_store(k[x], reinterpret_cast<u32x4*>(P.k_pages + off + x * 512 + lane * 8));
  };
  uint16_t* mine = stage[wave];
  if (__popc(starts) <= DENSE) {
    const bool holes = __any(slot < 0);
    if (holes) {
#pragma unroll
      for (int t = 0; t < NT; ++t) *reinterpret_cast<u32x4*>(mine + t * 512 + lane * 8) = u32x4{0, 0, 0, 0};
      wave_lds_order();
    }
    u32x4 v[NT], next[NT];
    auto load = [&](u32x4 (&to)[NT], int at) {                          // the unit of the token at `at`
      const int s = __builtin_amdgcn_readlane(slot, at) & ~31;
      const uint16_t* src = P.v_pages + page_of(s) + (s & in_page) * D;
#pragma unroll
      for (int t = 0; t < NT; ++t) to[t] = *reinterpret_cast<const u32x4*>(src + t * 512 + lane * 8);
    };
    if (starts) load(next, __builtin_ctz(starts));
    store_k();
    while (starts) {
      const int at = __builtin_ctz(starts);
      starts &= starts - 1;
      const int end = starts ? __builtin_ctz(starts) : 32;
#pragma unroll
      for (int t = 0; t < NT; ++t) v[t] = next[t];
      if (starts) load(next, __builtin_ctz(starts));
      // which of the unit's tokens stay; the first of them goes to `at`
      uint32_t stay = lane % 32 >= at && lane % 32 < end && slot >= 0 ? 1u << (slot & 31) : 0;
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) stay |= (uint32_t)__shfl_xor((int)stay, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t0 = 16 * (e >> 2) + 4 * a + (e & 3), to = at + __popc(stay & ((1u << t0) - 1));
        if (!(stay >> t0 & 1)) continue;
        uint16_t* p = mine + ((16 * (to % 16 / 4) + lane % 16) * 8 + 4 * (to / 16) + to % 4);
#pragma unroll
        for (int t = 0; t < NT; ++t) p[t * 512] = (uint16_t)(v[t][e / 2] >> (16 * (e & 1)));
      }
    }
    wave_lds_order();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      uint16_t* to = P.v_pages + off + t * 512 + lane * 8;
      const u32x4 y = *reinterpret_cast<const u32x4*>(mine + t * 512 + lane * 8);
      if (here == 32) {
        __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(to));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (16 * (e >> 2) + 4 * a + (e & 3) < here) to[e] = (uint16_t)(y[e / 2] >> (16 * (e & 1)));
      }
    }
    return;
  }
  uint16_t v[NT][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int s = __shfl(slot, 16 * (e >> 2) + 4 * a + (e & 3));
    const uint16_t* src = P.v_pages + (s >= 0 ? page_of(s) + v_fp_index(s & in_page, lane % 16, NT) : 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) v[t][e] = s >= 0 ? src[t * 512] : 0;
  }
  store_k();
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
  const WorkspacePaged room = split_workspace(s, ws);
  int longest = 0;                                       // tokens of the longest row that may go, among the long rows
  for (int i = 0; i < count; ++i) {
    const int old = rows.host[i].n - recent;
    if (old > longest && old > SHORT && rows.host[i].x > recent) longest = old;
  }
  const int pieces = (longest + PIECE - 1) / PIECE;
  EvictParams p{(uint16_t*)c.k_pages, (uint16_t*)c.v_pages, c.table, c.weights, room.slots, room.found, pieces, nullptr, s.B, s.Hkv,
                log2_of(s.P), s.n_pages, s.max_pages, recent};
  Rows8<ROWS_LISTED> listed{};
  hipError_t e = hand_over(rows, &listed, &p.rows, st);
  if (e != hipSuccess) return e;
  const int items = count * s.Hkv;
  hipLaunchKernelGGL(select_kernel, dim3(items), dim3(THREADS), 0, st, p, listed);
  if (pieces) {
    const dim3 grid(pieces, items), block(256);
    hipLaunchKernelGGL(histogram_kernel<0>, grid, block, 0, st, p, listed);
    hipLaunchKernelGGL(histogram_kernel<1>, grid, block, 0, st, p, listed);
    hipLaunchKernelGGL(histogram_kernel<2>, grid, block, 0, st, p, listed);
    hipLaunchKernelGGL(count_kernel<false>, grid, block, 0, st, p, listed);
    hipLaunchKernelGGL(count_kernel<true>, grid, block, 0, st, p, listed);
  }
  e = launch_status("select");
  if (e != hipSuccess) return e;
  const dim3 grid(((most_kept + 31) / 32 + 3) / 4, s.Hkv, count);
  if (s.d == 64) hipLaunchKernelGGL(move_kernel<64>, grid, dim3(256), 0, st, p, listed);
  else if (s.d == 96) hipLaunchKernelGGL(move_kernel<96>, grid, dim3(256), 0, st, p, listed);
  else hipLaunchKernelGGL(move_kernel<128>, grid, dim3(256), 0, st, p, listed);
  return launch_status("move");
}

}  // namespace lq
