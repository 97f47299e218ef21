// The 8-bit cache: quantizing tokens as they are written, and reading them back.
//
// Both move memory and compute little: per element two conversions and a multiplication against 3 bytes moved.  A wavefront
// works on pieces of 32 tokens x 32 channels, which are 1 KB of codes in one stretch, 16 bytes a lane.  Keys: a lane holds
// eight channels of tokens t and t + 16, as they lie in a row of the prompt.  Values: a lane needs eight tokens of two
// channels c and c + 16; it loads two neighbouring channels of eight tokens (4 bytes each, 64 in a row per 16 lanes) and
// trades half of the packed codes with the lane eight places away.
//
// 131072 tokens x 8 kv heads, bf16 (805 MB): written in 143 us (5.6 TB/s, two thirds of it reads), read back in 150 us (5.4, two
// thirds of it writes); a copy of 1 GB moves 5.05 TB/s.  Eight rows of up to 8191, G = 32 (203 MB): 40.3 us, 5.0 TB/s.  Wavefronts
// with a block of 32 tokens each to themselves, or values staged through LDS, were no faster.
#include "lq_cache8.h"
#include "lq_device.h"
#include "lq_internal.h"
#include "lq_quant8.h"

namespace lq {

namespace {

constexpr int WAVES = 4;

struct Append8Params {
  const uint16_t *k_new, *v_new;
  uint8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
  uint16_t *k_tail, *v_tail;
  const Row8* rows;
  Row8 same;
  int Hkv, cap, n_max;
};

struct Read8Params {
  const uint8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  const uint16_t *k_tail, *v_tail;
  uint16_t *k_out, *v_out;
  const Row8* rows;
  Row8 same;
  int Hkv, cap, log_g, t0, n;         // G = 1 << log_g
};

template <typename P, int MODE>
__device__ __forceinline__ Row8 row_of(const P& p, int b) {
  if constexpr (MODE == ROWS_SAME) return p.same;
  const Row8Ptr r = rows_ptr(p.rows, sizeof(P));
  return Row8{r[b].n, r[b].x, 1, b};
}

// Two values of T from byte pair `hi` of a word of codes, times the scale (exact within T).
template <bool BF16>
__device__ __forceinline__ uint32_t values2(uint32_t w, bool hi, float scale) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 f = hi ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  return (uint32_t)f2t<BF16>(f[0] * scale) | ((uint32_t)f2t<BF16>(f[1] * scale) << 16);
}

__device__ __forceinline__ uint32_t other_half_row(uint32_t v) {   // of the lane eight places away in a row of 16
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false);
}

// Order of LDS accesses within a wavefront (its LDS instructions execute in order: only the compiler has to be told).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ uint32_t load4(__amdgpu_buffer_rsrc_t rs, int off) { return __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0); }

// token within its unit of 32 at position e of the eight that lane row a holds: 16 b + 4 a + e % 4, b = e / 4
__device__ __forceinline__ int value_token(int a, int e) { return 16 * (e >> 2) + 4 * a + (e & 3); }

// grid (most blocks that a row completes, plus one, B * Hkv).  Workgroup i of a slice quantizes the i-th block that becomes
// full; the rows left over go to the tail by workgroup `blocks completed`, or by workgroup 0 where its block takes rows
// from the tail, after it has read them.  These come first in the grid, slice by slice, and the others behind them: in its
// place among a slice's workgroups the last of them, which has up to twice the others' work, was the launch's end (8 rows of
// 8192 tokens x 8 kv heads behind 127 rows of the tail 101 -> 77.5 us, of which 75 without the tail; rows of up to 8191, G = 32,
// 43.9 -> 40.3).
template <bool BF16, int D, int G, int MODE>
__global__ void __launch_bounds__(64 * WAVES) append8_kernel(const Append8Params P, const Rows8<MODE> S) {
  (void)S;
  constexpr int ND = D / 32, PIECES = G / 32 * ND, MINE = (PIECES + WAVES - 1) / WAVES;
  const int slices = gridDim.y, blocks = gridDim.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int at_grid = blockIdx.y * blocks + blockIdx.x, behind = at_grid - slices;
  const int bh = behind < 0 ? at_grid : behind / (blocks - 1);
  const Row8 row = row_of<Append8Params, MODE>(P, bh / P.Hkv);
  const int held = row.n % G, all = held + row.x, full = all / G;   // rows from the first open block on; blocks completed
  const int tail_wg = held && full ? 0 : full;
  const int early = tail_wg < blocks ? tail_wg : blocks - 1, other = behind - bh * (blocks - 1);
  const int i = behind < 0 ? early : other < early ? other : other + 1;
  if (i > full || (i == full && i != tail_wg) || row.x == 0) return;
  const uint16_t* k_new = P.k_new + (int64_t)bh * P.n_max * D;
  const uint16_t* v_new = P.v_new + (int64_t)bh * P.n_max * D;
  uint16_t* k_tail = P.k_tail + (int64_t)bh * G * D;
  uint16_t* v_tail = P.v_tail + (int64_t)bh * G * D;

  if (i < full) {
    const int64_t block = row.n / G + i;
    const bool from_tail = i == 0 && held;
    const int first = i * G - held;                  // of the block's rows among the new ones
    const __amdgpu_buffer_rsrc_t new_v = buffer(v_new, (G - held) * (2 * D));   // those that block 0 takes; elsewhere: zeros, not read
    uint4 k[MINE][2];
    uint32_t v[MINE][8];
    uint32_t top_k = 0, top_v = 0;
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
      const int piece = wave + j * WAVES, unit = piece / ND, nd = piece % ND;
      if (PIECES % WAVES && piece >= PIECES) break;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = 32 * unit + 16 * h + lane % 16, c = 32 * nd + 8 * (lane / 16);
        const uint16_t* src = k_new + (int64_t)(first + t) * D + c;
        if (from_tail && t < held) src = k_tail + k_fp_index(t, c, ND);
        k[j][h] = *reinterpret_cast<const uint4*>(src);
      }
      const int c = 32 * nd + 2 * (lane % 16);
      if (!from_tail) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[j][e] = *reinterpret_cast<const uint32_t*>(v_new + (int64_t)(first + 32 * unit + value_token(lane / 16, e)) * D + c);
      } else {                                       // two pieces of the tail as they lie, eight tokens of c and of c + 1, and the new ones
        const uint4* old = reinterpret_cast<const uint4*>(v_tail + v_fp_index(32 * unit + 4 * (lane / 16), c, 2 * ND));
        const uint4 x = old[0], y = old[1];
        const uint32_t lo[4] = {x.x, x.y, x.z, x.w}, hi[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = 32 * unit + value_token(lane / 16, e);
          const uint32_t was = __builtin_amdgcn_perm(hi[e / 2], lo[e / 2], e & 1 ? 0x07060302 : 0x05040100);
          const uint32_t is = load4(new_v, (t - held) * (2 * D) + 2 * c);
          v[j][e] = t < held ? was : is;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
      if (PIECES % WAVES && wave + j * WAVES >= PIECES) break;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        top_k = max_pair(max_pair(max_pair(max_pair(top_k, k[j][h].x), k[j][h].y), k[j][h].z), k[j][h].w);
#pragma unroll
      for (int e = 0; e < 8; ++e) top_v = max_pair(top_v, v[j][e]);
    }
    // the two tensors' maxima as the halves of one word, then over the wavefront and the workgroup
    uint32_t top = max_pair(top_k & 0xFFFF, top_k >> 16) | (max_pair(top_v & 0xFFFF, top_v >> 16) << 16);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = max_pair(top, (uint32_t)__shfl_xor((int)top, m));
    __shared__ uint32_t tops[WAVES];
    if (lane == 0) tops[wave] = top;
    __syncthreads();                                 // (the tail has been read as well: it may be written below)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = max_pair(top, tops[w]);
    const int ek = scale_exponent<BF16>(top & 0xFFFF), ev = scale_exponent<BF16>(top >> 16);
    const float ik = pow2(-ek), iv = pow2(-ev), cut = t2f<BF16>(cut_bits<BF16>());
    const float mk = fminf(448.f, cut * ik), mv = fminf(448.f, cut * iv);
    const int64_t slice = (int64_t)bh * P.cap * D + block * (G * D);
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
      const int piece = wave + j * WAVES;
      if (PIECES % WAVES && piece >= PIECES) break;
      uint4 w;
      w.x = codes4<BF16>(k[j][0].x, k[j][0].y, ik, mk);
      w.y = codes4<BF16>(k[j][0].z, k[j][0].w, ik, mk);
      w.z = codes4<BF16>(k[j][1].x, k[j][1].y, ik, mk);
      w.w = codes4<BF16>(k[j][1].z, k[j][1].w, ik, mk);
      *reinterpret_cast<uint4*>(P.k_codes + slice + piece * 1024 + lane * 16) = w;
      // channel c (low halves) and c + 1 (high halves) of four tokens each
      auto pick = [&](int e, uint32_t sel) { return __builtin_amdgcn_perm(v[j][e + 1], v[j][e], sel); };
      uint32_t lo[2], hi[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        lo[b] = codes4<BF16>(pick(4 * b, 0x05040100), pick(4 * b + 2, 0x05040100), iv, mv);
        hi[b] = codes4<BF16>(pick(4 * b, 0x07060302), pick(4 * b + 2, 0x07060302), iv, mv);
      }
      // lanes 0..7 of a row hold channels 2c', 2c' + 1 below 16 and take c = 2c' of both halves, lanes 8..15 the odd ones
      const bool upper = lane & 8;
      const uint32_t give0 = upper ? lo[0] : hi[0], give1 = upper ? lo[1] : hi[1];
      const uint32_t got0 = other_half_row(give0), got1 = other_half_row(give1);
      w = upper ? make_uint4(got0, got1, hi[0], hi[1]) : make_uint4(lo[0], lo[1], got0, got1);
      const int cc = 2 * (lane & 7) + (upper ? 1 : 0);
      *reinterpret_cast<uint4*>(P.v_codes + slice + piece * 1024 + (16 * (lane / 16) + cc) * 16) = w;
    }
    if (threadIdx.x == 0) {
      P.k_scale[(int64_t)bh * (P.cap / G) + block] = pow2(ek);
      P.v_scale[(int64_t)bh * (P.cap / G) + block] = pow2(ev);
    }
  }
  if (i != tail_wg) return;
  // slots at .. at + left - 1 get the new rows from `from` on: the rows behind the last full block, or, where a block of the
  // tail has just become full and nothing follows, its new rows, so that the count can be set back into it
  const bool keep = held && all == G;
  const int at = full && !keep ? 0 : held, left = (keep ? G : all - full * G) - at, from = keep ? 0 : full * G + at - held;
  // In pieces of the tail as it lies: 16 rows next to each other for keys; for values two channels of eight rows, of which
  // those that are all new are stored at once, and all loads first (64 slices with 63 rows left over behind 127 blocks: row by
  // row, values 2 bytes at a time, 105 us; so 80).
  const int end = at + left;
  const __amdgpu_buffer_rsrc_t src_k = buffer(k_new + (int64_t)from * D, left * (2 * D)), src_v = buffer(v_new + (int64_t)from * D, left * (2 * D));
  constexpr int T = 64 * WAVES, NK = (G * D / 8 + T - 1) / T, NV = (G * D / 16 + T - 1) / T;
  u32x4 k[NK];
  uint32_t v[NV][8];
#pragma unroll
  for (int j = 0; j < NK; ++j) {
    const int x = threadIdx.x + j * T, t = x / (2 * D) * 16 + x % 16;
    k[j] = load16(src_k, (t - at) * (2 * D) + x / 16 % (D / 8) * 16);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int x = threadIdx.x + j * T, t = x / (2 * D) * 32 + value_token(x / (D / 2) % 4, e);
      v[j][e] = load4(src_v, (t - at) * (2 * D) + x % (D / 2) * 4);
    }
#pragma unroll
  for (int j = 0; j < NK; ++j) {
    const int x = threadIdx.x + j * T, t = x / (2 * D) * 16 + x % 16;
    if (t >= at && t < end) *reinterpret_cast<u32x4*>(k_tail + k_fp_index(t, x / 16 % (D / 8) * 8, ND)) = k[j];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int x = threadIdx.x + j * T, a = x / (D / 2) % 4, t0 = x / (2 * D) * 32 + 4 * a;      // tokens t0 .. t0 + 3, t0 + 16 .. t0 + 19
    if (t0 >= end || t0 + 19 < at) continue;
    uint16_t* to = v_tail + v_fp_index(t0, x % (D / 2) * 2, 2 * ND);     // those of c, and behind them of c + 1
    if (t0 >= at && t0 + 19 < end) {
      auto piece = [&](uint32_t sel) {
        return make_uint4(__builtin_amdgcn_perm(v[j][1], v[j][0], sel), __builtin_amdgcn_perm(v[j][3], v[j][2], sel),
                          __builtin_amdgcn_perm(v[j][5], v[j][4], sel), __builtin_amdgcn_perm(v[j][7], v[j][6], sel));
      };
      reinterpret_cast<uint4*>(to)[0] = piece(0x05040100);
      reinterpret_cast<uint4*>(to)[1] = piece(0x07060302);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = t0 + value_token(0, e);
        if (t < at || t >= end) continue;
        to[e] = (uint16_t)v[j][e];
        to[e + 8] = (uint16_t)(v[j][e] >> 16);
      }
    }
  }
}

// grid (units of 32 tokens that the range touches / WAVES, B * Hkv): a wavefront a unit.
template <bool BF16, int D, int MODE>
__global__ void __launch_bounds__(64 * WAVES) read8_kernel(const Read8Params P, const Rows8<MODE> S) {
  (void)S;
  constexpr int ND = D / 32;
  const int bh = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = P.t0 / 32 + (int)blockIdx.x * WAVES + wave;
  const int held = row_of<Read8Params, MODE>(P, bh / P.Hkv).n;
  const int end = P.t0 + P.n < held ? P.t0 + P.n : held;              // tokens t0 .. end - 1 are wanted and there
  if (32 * unit >= end) return;
  const int full = held >> P.log_g << P.log_g;
  auto wanted = [&](int t) { return t >= P.t0 && t < end; };
  uint16_t* k_out = P.k_out + ((int64_t)bh * P.n - P.t0) * D;
  uint16_t* v_out = P.v_out + ((int64_t)bh * P.n - P.t0) * D;
  // The rows of a unit are put together in LDS, a wavefront for itself, so that a store covers 1 KB of output in one
  // stretch: stored from the lanes that convert them (64 bytes of a row at a time, values 4 bytes a lane) 131072 tokens x
  // 8 heads took 208 us instead of 150, and a tail of 127 rows x 64 slices 11.1 instead of 4.7.
  constexpr int PITCH = 2 * D + 16, CHUNKS = D / 8;          // bytes of a row, 16-byte pieces of it
  __shared__ __align__(16) unsigned char stage[WAVES][32 * PITCH];
  unsigned char* mine = stage[wave];
  auto flush = [&](uint16_t* out) {
    wave_lds_order();
#pragma unroll
    for (int x = 0; x < 32 * CHUNKS / 64; ++x) {
      const int i = lane + 64 * x, t = i / CHUNKS, c = i % CHUNKS;
      const uint4 y = *reinterpret_cast<const uint4*>(mine + t * PITCH + 16 * c);
      if (wanted(32 * unit + t)) *reinterpret_cast<uint4*>(out + (int64_t)(32 * unit + t) * D + 8 * c) = y;
    }
    wave_lds_order();
  };
  if (32 * unit < full) {
    const int64_t slice = ((int64_t)bh * P.cap + 32 * (int64_t)unit) * D;
    const int64_t block = (int64_t)bh * (P.cap >> P.log_g) + (32 * unit >> P.log_g);
    const bool upper = lane & 8;
    const int cc = 2 * (lane & 7) + (upper ? 1 : 0);
    uint4 k[ND], v[ND];
    if (P.k_out)
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) k[nd] = *reinterpret_cast<const uint4*>(P.k_codes + slice + nd * 1024 + lane * 16);
    if (P.v_out)
#pragma unroll
      for (int nd = 0; nd < ND; ++nd)
        v[nd] = *reinterpret_cast<const uint4*>(P.v_codes + slice + nd * 1024 + (16 * (lane / 16) + cc) * 16);
    const float sk = P.k_scale[block], sv = P.v_scale[block];
    if (P.k_out) {
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) {
        const int t = lane % 16, c = 32 * nd + 8 * (lane / 16);
        auto row8 = [&](uint32_t a, uint32_t b) {
          return make_uint4(values2<BF16>(a, false, sk), values2<BF16>(a, true, sk), values2<BF16>(b, false, sk), values2<BF16>(b, true, sk));
        };
        *reinterpret_cast<uint4*>(mine + t * PITCH + 2 * c) = row8(k[nd].x, k[nd].y);
        *reinterpret_cast<uint4*>(mine + (t + 16) * PITCH + 2 * c) = row8(k[nd].z, k[nd].w);
      }
      flush(k_out);
    }
    if (P.v_out) {
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) {
        // the trade of append8_kernel backwards: the lane is left with channels c, c + 1 of eight tokens
        const uint32_t got0 = other_half_row(upper ? v[nd].x : v[nd].z), got1 = other_half_row(upper ? v[nd].y : v[nd].w);
        const uint32_t lo[2] = {upper ? got0 : v[nd].x, upper ? got1 : v[nd].y};
        const uint32_t hi[2] = {upper ? v[nd].z : got0, upper ? v[nd].w : got1};
        const int c = 32 * nd + 2 * (lane % 16);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const uint32_t x = values2<BF16>(lo[b], e != 0, sv), y = values2<BF16>(hi[b], e != 0, sv);
            const int t = value_token(lane / 16, 4 * b + e);
            *reinterpret_cast<uint32_t*>(mine + t * PITCH + 2 * c) = __builtin_amdgcn_perm(y, x, 0x05040100);
            *reinterpret_cast<uint32_t*>(mine + (t + 1) * PITCH + 2 * c) = __builtin_amdgcn_perm(y, x, 0x07060302);
          }
      }
      flush(v_out);
    }
    return;
  }
  // the tail: rows of keys 16 bytes a lane, values as two channels of eight tokens; lanes whose rows are not there read nothing
  const int64_t tail = (((int64_t)bh << P.log_g) + (32 * unit - full)) * D;
  const int live = end - 32 * unit, nothing = 64 * D;
  const __amdgpu_buffer_rsrc_t k_tail = buffer(P.k_tail + tail, 64 * D), v_tail = buffer(P.v_tail + tail, 64 * D);
  u32x4 k[2 * ND], v[2 * ND];
  if (P.k_out)
#pragma unroll
    for (int x = 0; x < 2 * ND; ++x) k[x] = load16(k_tail, 16 * (x / ND) + lane % 16 < live ? x * 1024 + lane * 16 : nothing);
  if (P.v_out)
#pragma unroll
    for (int x = 0; x < 2 * ND; ++x)
      v[x] = load16(v_tail, 4 * (lane / 16) < live ? (int)v_fp_index(4 * (lane / 16), 32 * (x / 2) + 2 * (lane % 16) + x % 2, 2 * ND) * 2 : nothing);
  if (P.k_out) {
#pragma unroll
    for (int x = 0; x < 2 * ND; ++x)
      *reinterpret_cast<u32x4*>(mine + (16 * (x / ND) + lane % 16) * PITCH + 2 * (32 * (x % ND) + 8 * (lane / 16))) = k[x];
    flush(k_out);
  }
  if (P.v_out) {
#pragma unroll
    for (int nd = 0; nd < ND; ++nd) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        *reinterpret_cast<uint32_t*>(mine + value_token(lane / 16, e) * PITCH + 2 * (32 * nd + 2 * (lane % 16))) =
            __builtin_amdgcn_perm(v[2 * nd + 1][e / 2], v[2 * nd][e / 2], e & 1 ? 0x07060302 : 0x05040100);
    }
    flush(v_out);
  }
}

struct Chunk8 { int base, n; Row8 e[ROWS_IN_ARGS]; };
__global__ void upload_rows8_kernel(Row8* dev, const Chunk8 c) {
  const int i = threadIdx.x;
  if (i < c.n) dev[c.base + i] = c.e[i];
}

template <int MODE>
hipError_t append8(const Shape8& s, const Append8Params& p, const Rows8<MODE>& rows, dim3 grid, hipStream_t st) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * WAVES), 0, st, p, rows); };
  auto with_type = [&](auto bf16) {
    constexpr bool T = decltype(bf16)::value;
    switch (s.d * 1000 + s.G) {
      case 64032: return go(append8_kernel<T, 64, 32, MODE>);
      case 64064: return go(append8_kernel<T, 64, 64, MODE>);
      case 64128: return go(append8_kernel<T, 64, 128, MODE>);
      case 96032: return go(append8_kernel<T, 96, 32, MODE>);
      case 96064: return go(append8_kernel<T, 96, 64, MODE>);
      case 96128: return go(append8_kernel<T, 96, 128, MODE>);
      case 128032: return go(append8_kernel<T, 128, 32, MODE>);
      case 128064: return go(append8_kernel<T, 128, 64, MODE>);
      default: return go(append8_kernel<T, 128, 128, MODE>);
    }
  };
  if (s.bf16) with_type(std::true_type{}); else with_type(std::false_type{});
  return launch_status("append8");
}

template <int MODE>
hipError_t read8(const Shape8& s, const Read8Params& p, const Rows8<MODE>& rows, dim3 grid, hipStream_t st) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * WAVES), 0, st, p, rows); };
  auto with_type = [&](auto bf16) {
    constexpr bool T = decltype(bf16)::value;
    if (s.d == 64) return go(read8_kernel<T, 64, MODE>);
    if (s.d == 96) return go(read8_kernel<T, 96, MODE>);
    go(read8_kernel<T, 128, MODE>);
  };
  if (s.bf16) with_type(std::true_type{}); else with_type(std::false_type{});
  return launch_status("read8");
}

}  // namespace

hipError_t upload_rows8(Row8* dev, const Row8* host, int n, hipStream_t st) {
  for (int base = 0; base < n; base += ROWS_IN_ARGS) {
    Chunk8 c{};
    c.base = base;
    c.n = n - base < ROWS_IN_ARGS ? n - base : ROWS_IN_ARGS;
    for (int i = 0; i < c.n; ++i) c.e[i] = host[base + i];
    hipLaunchKernelGGL(upload_rows8_kernel, dim3(1), dim3(ROWS_IN_ARGS), 0, st, dev, c);
  }
  return launch_status("row lengths");
}

hipError_t launch_append8(const Shape8& s, const lq_cache8& c, const void* k_new, const void* v_new, int n_max, int blocks,
                          const RowArg8& rows, hipStream_t st) {
  Append8Params p{(const uint16_t*)k_new, (const uint16_t*)v_new, c.k_codes, c.v_codes, c.k_scale, c.v_scale,
                  (uint16_t*)c.k_tail, (uint16_t*)c.v_tail, nullptr, rows.host[0], s.Hkv, s.cap, n_max};
  const dim3 grid(blocks, s.B * s.Hkv);
  if (rows.same) return append8<ROWS_SAME>(s, p, Rows8<ROWS_SAME>{}, grid, st);
  Rows8<ROWS_LISTED> listed{};
  const hipError_t e = hand_over(rows, &listed, &p.rows, st);
  return e != hipSuccess ? e : append8<ROWS_LISTED>(s, p, listed, grid, st);
}

hipError_t launch_read8(const Shape8& s, const lq_cache8& c, int t0, int n, void* k_out, void* v_out, const RowArg8& rows,
                        hipStream_t st) {
  Read8Params p{c.k_codes, c.v_codes, c.k_scale, c.v_scale, (const uint16_t*)c.k_tail, (const uint16_t*)c.v_tail,
                (uint16_t*)k_out, (uint16_t*)v_out, nullptr, rows.host[0], s.Hkv, s.cap, log2_of(s.G), t0, n};
  const int units = (t0 + n - 1) / 32 - t0 / 32 + 1;
  const dim3 grid((units + WAVES - 1) / WAVES, s.B * s.Hkv);
  if (rows.same) return read8<ROWS_SAME>(s, p, Rows8<ROWS_SAME>{}, grid, st);
  Rows8<ROWS_LISTED> listed{};
  const hipError_t e = hand_over(rows, &listed, &p.rows, st);
  return e != hipSuccess ? e : read8<ROWS_LISTED>(s, p, listed, grid, st);
}

}  // namespace lq
