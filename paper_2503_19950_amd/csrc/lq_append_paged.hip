// The paged cache: writing tokens.
//
// Bound by the bytes.  A workgroup takes a unit of 32 slots of a row and some kv heads, a head a wavefront; with rotary
// positions it computes the unit's cosines and sines once, into LDS.  Keys go over 16 bytes a lane, as they lie in a row of
// the prompt; values as two channels of eight tokens a lane, whose halves are the pieces of the page.
// 8 rows of 8192 tokens x 8 kv heads, d = 128 (537 MB): 104 us, with keys turned on their way 105 (5.1 TB/s, what a copy
// reaches); rows of up to 8191 (270 MB): 60 and 61; one row of 32768 (268 MB) 58, so the workgroups that find their
// row at an end cost some 2 us (a grid without them, whose workgroups look for their row: 1 us less).  Stores past the caches: 121 and 68.
#include "lq_internal.h"
#include "lq_paged.h"
#include "lq_quant8.h"

namespace lq {

namespace {

constexpr int WAVES = 4, PITCH = 66;         // pairs from one token's angles to the next (64 and padding)

struct AppendPagedParams {
  const uint16_t *k_new, *v_new;
  uint16_t *k_pages, *v_pages;
  const int* table;
  float* weights;                            // null unless the cache keeps them
  RopeArg rope;
  const Row8* rows;
  Row8 same;
  int B, Hkv, heads, log_p, n_pages, max_pages, n_max;       // heads: of a workgroup
};

__device__ __forceinline__ uint32_t load4(__amdgpu_buffer_rsrc_t rs, int off) { return __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0); }
__device__ __forceinline__ uint16_t load2(__amdgpu_buffer_rsrc_t rs, int off) { return __builtin_amdgcn_raw_buffer_load_b16(rs, off, 0, 0); }
// token within its unit of 32 at position e of the eight that lane row a holds
__device__ __forceinline__ int value_token(int a, int e) { return 16 * (e >> 2) + 4 * a + (e & 3); }

// How keys are turned: not at all; pairs of neighbours; pairs of halves that are 32 or 64 channels, in the same lane, that are other
// whole pieces of 16 bytes, and that are not.
enum Turn { NONE, NEIGHBOURS, HALVES_32, HALVES_64, HALVES, ODD };

// The other halves of the pairs that channels c0 .. c0+7 of a key (offset `row` of rs) belong to.
template <int TURN>
__device__ __forceinline__ u32x4 other_halves(__amdgpu_buffer_rsrc_t rs, int row, int c0, int dims) {
  const int half = dims / 2, nothing = 0x7FFFF000;
  if constexpr (TURN == HALVES) return load16(rs, c0 < dims ? row + 2 * (c0 < half ? c0 + half : c0 - half) : nothing);
  u32x4 y{0, 0, 0, 0};
  if constexpr (TURN == ODD)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = c0 + e;
      y[e / 2] |= (uint32_t)load2(rs, c < dims ? row + 2 * (c < half ? c + half : c - half) : nothing) << (16 * (e & 1));
    }
  return y;
}
// Channels c0 .. c0+7 turned; y: other_halves; angle: that token's, PITCH of them, of which dims / 2 have been computed and others are
// read for channels that stay alone.  (The results of turn_pair, bit for bit.)
template <bool BF16, int TURN>
__device__ __forceinline__ u32x4 turned(int c0, u32x4 x, u32x4 y, int dims, const float2* angle) {
  if constexpr (TURN == NEIGHBOURS) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint16_t p = (uint16_t)x[w], o = (uint16_t)(x[w] >> 16);
      turn_pair<BF16>(p, o, angle[c0 / 2 + w]);
      if (c0 + 2 * w < dims) x[w] = p | (uint32_t)o << 16;
    }
    return x;
  }
  const int half = dims / 2;
  const float2* of_piece = angle + (TURN == HALVES ? angle_of(c0, dims, 8) : c0 < half ? c0 : c0 - half);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = c0 + e, sh = 16 * (e & 1);
    const bool first = TURN == ODD ? c < half : c0 < half;
    const float2 cs = TURN == ODD ? angle[angle_of(c, dims, 1)] : of_piece[e];
    const float own = t2f<BF16>((uint16_t)(x[e / 2] >> sh)), other = t2f<BF16>((uint16_t)(y[e / 2] >> sh));
    const uint32_t z = f2t<BF16>(fmaf(own, cs.x, other * (first ? -cs.y : cs.y)));
    if (c < dims) x[e / 2] = (x[e / 2] & ~(0xFFFFu << sh)) | z << sh;
  }
  return x;
}

// grid (units that a row's new tokens touch, shares of the kv heads, B).  HALVES_64 has registers for three wavefronts on a SIMD and
// four of them spilled (one kv head, 65536 tokens: 15.8 us, with two wavefronts and none spilled 19.7; 8 kv heads 61.0 and 62.0).
template <bool BF16, int D, int MODE, int TURN>
__global__ void __launch_bounds__(64 * WAVES, TURN == HALVES_64 ? 3 : 1) append_paged_kernel(const AppendPagedParams P, const Rows8<MODE> S) {
  (void)S;
  constexpr int ND = D / 32;
  const int b = blockIdx.z, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), a = lane / 16;
  Row8 row = P.same;
  if constexpr (MODE == ROWS_LISTED) {
    const Row8Ptr r = rows_ptr(P.rows, sizeof(AppendPagedParams));
    row = Row8{r[b].n, r[b].x, 1, r[b].b};
  } else {
    row.b += b;
  }
  const int unit = row.n / 32 + (int)blockIdx.x, end = row.n + row.x;
  if (32 * unit >= end || row.x == 0) return;
  const int low = row.n > 32 * unit ? row.n - 32 * unit : 0, high = end - 32 * unit < 32 ? end - 32 * unit : 32;
  const int head0 = blockIdx.y * P.heads, head1 = head0 + P.heads < P.Hkv ? head0 + P.heads : P.Hkv;
  const int64_t new0 = 32 * (int64_t)unit + low - row.n;                // token `low` of the unit among the new ones
  if (P.weights)
    for (int x = threadIdx.x; x < 32 * (head1 - head0); x += 64 * WAVES)
      if (x % 32 >= low && x % 32 < high)
        P.weights[((((int64_t)row.b * P.Hkv + head0 + x / 32) * P.max_pages) << P.log_p) + 32 * unit + x % 32] = 0.f;
  const int id = P.table[(int64_t)row.b * P.max_pages + (unit >> (P.log_p - 5))];
  // A lane computes the angles of one pair for every fourth token.  What it takes to compute them is loaded first (loads arrive in
  // order), then the first head's rows, which are under way meanwhile.
  const int pairs = P.rope.dims / 2;
  constexpr int TOKENS = 32 / WAVES;
  double freq = 0.0;
  int position[TOKENS];
  if constexpr (TURN) {
    if (lane < pairs) freq = P.rope.freq[lane];
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
      const int t = wave + j * WAVES;
      position[j] = 32 * unit + t;
      if (P.rope.positions && t >= low && t < high) position[j] = P.rope.positions[(int64_t)b * P.n_max + new0 + t - low];
    }
  }
  __amdgpu_buffer_rsrc_t rk;
  constexpr bool APART = TURN == HALVES || TURN == ODD;                 // the other halves are loaded
  constexpr int OTHER = TURN == HALVES_32 ? 1 : TURN == HALVES_64 ? 2 : 0;
  u32x4 k[2 * ND], y[ND];
  uint32_t v[ND][8];
  auto load_y = [&](int tile) {
    if constexpr (APART)
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) y[nd] = other_halves<TURN>(rk, (16 * tile + lane % 16 - low) * (2 * D), 32 * nd + 8 * a, P.rope.dims);
  };
  auto load = [&](int h) {                                              // tokens outside low .. high - 1: zeros, not read
    const int64_t from = (((int64_t)b * P.Hkv + h) * P.n_max + new0) * D;
    rk = buffer(P.k_new + from, (high - low) * D * 2);
    const __amdgpu_buffer_rsrc_t rv = buffer(P.v_new + from, (high - low) * D * 2);
#pragma unroll
    for (int x = 0; x < 2 * ND; ++x) k[x] = load16(rk, (16 * (x / ND) + lane % 16 - low) * (2 * D) + 2 * (32 * (x % ND) + 8 * a));
    load_y(0);
#pragma unroll
    for (int nd = 0; nd < ND; ++nd)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[nd][e] = load4(rv, (value_token(a, e) - low) * (2 * D) + 2 * (32 * nd + 2 * (lane % 16)));
  };
  int h = head0 + wave;
  if (h < head1) load(h);
  __shared__ __align__(16) float2 cs[TURN ? 32 * PITCH : 1];
  if constexpr (TURN) {
#pragma unroll
    for (int j = 0; j < TOKENS; ++j)
      if (lane < pairs) cs[(wave + j * WAVES) * PITCH + lane] = turn_of(freq, position[j], P.rope.factor);
    __syncthreads();
  }
  if (!is_page(id, P.n_pages)) return;                                  // (loads do not wait for the table: 0 to 2 % by size)
  for (; h < head1; h += WAVES) {
    const int64_t off = unit_offset(id, P.Hkv, h, P.log_p, unit, D);
#pragma unroll
    for (int x = 0; x < 2 * ND; ++x) {
      const int t = 16 * (x / ND) + lane % 16, c = 32 * (x % ND) + 8 * a;
      if (x == ND) load_y(1);
      if (t < low || t >= high) continue;
      u32x4 z = k[x];
      if constexpr (OTHER > 0) {
        if (x % ND < 2 * OTHER) z = turned<BF16, TURN>(c, z, k[x % ND < OTHER ? x + OTHER : x - OTHER], 64 * OTHER, cs + t * PITCH);
      } else if constexpr (TURN) {
        z = turned<BF16, TURN>(c, z, y[x % ND], P.rope.dims, cs + t * PITCH);
      }
      *reinterpret_cast<u32x4*>(P.k_pages + off + x * 512 + lane * 8) = z;
    }
#pragma unroll
    for (int nd = 0; nd < ND; ++nd) {
      const int t0 = 4 * a, c = 32 * nd + 2 * (lane % 16);              // tokens t0 .. t0 + 3, t0 + 16 .. t0 + 19
      if (t0 >= high || t0 + 19 < low) continue;
      uint16_t* to = P.v_pages + off + v_fp_index(t0, c, 2 * ND);      // those of c, and behind them of c + 1
      if (t0 >= low && t0 + 19 < high) {
        auto piece = [&](uint32_t sel) {
          return u32x4{__builtin_amdgcn_perm(v[nd][1], v[nd][0], sel), __builtin_amdgcn_perm(v[nd][3], v[nd][2], sel),
                       __builtin_amdgcn_perm(v[nd][5], v[nd][4], sel), __builtin_amdgcn_perm(v[nd][7], v[nd][6], sel)};
        };
        reinterpret_cast<u32x4*>(to)[0] = piece(0x05040100);
        reinterpret_cast<u32x4*>(to)[1] = piece(0x07060302);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = t0 + value_token(0, e);
          if (t < low || t >= high) continue;
          to[e] = (uint16_t)v[nd][e];
          to[e + 8] = (uint16_t)(v[nd][e] >> 16);
        }
      }
    }
    if (h + WAVES < head1) load(h + WAVES);
  }
}

template <int MODE>
hipError_t append_paged(const ShapePaged& s, const AppendPagedParams& p, const Rows8<MODE>& rows, dim3 grid, hipStream_t st) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * WAVES), 0, st, p, rows); };
  auto with = [&](auto t, auto turn) {
    constexpr bool T = decltype(t)::value;
    constexpr int TURN = decltype(turn)::value;
    if constexpr (TURN != HALVES_64) {                                  // (of 128 channels)
      if (s.d == 64) return go(append_paged_kernel<T, 64, MODE, TURN>);
      if (s.d == 96) return go(append_paged_kernel<T, 96, MODE, TURN>);
    }
    go(append_paged_kernel<T, 128, MODE, TURN>);
  };
  auto with_type = [&](auto t) {
    if (p.rope.interleaved) return with(t, std::integral_constant<int, NEIGHBOURS>{});
    if (p.rope.dims % 16) return with(t, std::integral_constant<int, ODD>{});
    if (p.rope.dims == 64) return with(t, std::integral_constant<int, HALVES_32>{});
    if (p.rope.dims == 128) return with(t, std::integral_constant<int, HALVES_64>{});
    with(t, std::integral_constant<int, HALVES>{});
  };
  if (!p.rope.freq) with(std::false_type{}, std::integral_constant<int, NONE>{});      // (the type does not matter)
  else if (s.bf16) with_type(std::true_type{});
  else with_type(std::false_type{});
  return launch_status("append_paged");
}

}  // namespace

hipError_t launch_append_paged(const ShapePaged& s, const lq_cache_paged& c, const RopeArg& rope, const void* k_new, const void* v_new,
                               int n_max, int units, const RowArg8& rows, hipStream_t st) {
  // A head a wavefront: two share the angles, but there are fewer workgroups to fill the GPU (8 rows of up to 8191 tokens x 8 kv heads
  // 64.8 and 67.0 us; 8 rows of 8192 109.8 and 111.3), which only pays where turning takes longest, halves that are no whole pieces
  // (136.4 and 125.7).
  const bool odd = rope.freq && !rope.interleaved && rope.dims % 16;
  const int heads = odd && s.Hkv > WAVES ? 2 * WAVES : WAVES;
  AppendPagedParams p{(const uint16_t*)k_new, (const uint16_t*)v_new, (uint16_t*)c.k_pages, (uint16_t*)c.v_pages, c.table,
                      s.weighted ? c.weights : nullptr, rope, nullptr, rows.host[0], s.B, s.Hkv, heads, log2_of(s.P), s.n_pages, s.max_pages,
                      n_max};
  const dim3 grid(units, (s.Hkv + heads - 1) / heads, s.B);
  if (rows.same) return append_paged<ROWS_SAME>(s, p, Rows8<ROWS_SAME>{}, grid, st);
  Rows8<ROWS_LISTED> listed{};
  const hipError_t e = hand_over(rows, &listed, &p.rows, st);
  return e != hipSuccess ? e : append_paged<ROWS_LISTED>(s, p, listed, grid, st);
}

}  // namespace lq
