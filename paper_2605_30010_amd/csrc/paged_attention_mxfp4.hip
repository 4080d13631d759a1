// Attention of one new token per sequence over a paged key-value cache in 4 bits.
#include <algorithm>
#include <type_traits>

#include "paged_attention.h"

namespace et {

// Keys in 4 bits.  A lane's load serves several steps of 32 dimensions, and so does its exponent: where a row is a multiple of 128,
// 32 dimensions (a block) for four steps, elsewhere 16 (half a block) for two, and the third step has the dimensions from 64 on.
template <int HD>
struct MxKeys {
  using Lay = KvLayout<HD, ET_KV_MXFP4>;
  static constexpr int STEPS = (HD + 31) / 32, NREG = STEPS;
  static constexpr bool WIDE = HD % 128 == 0;
  static constexpr int UNITS = WIDE ? STEPS / 4 : STEPS - 1;             // exponents of a lane
  static __device__ __forceinline__ int dim(int s, int g) {
    return WIDE ? s / 4 * 128 + g * 32 + s % 4 * 8 : s < 2 ? g * 16 + s * 8 : 64 + g * 8;
  }
  // Past the row's end the last dimensions are read again (and not used).
  static __device__ __forceinline__ void load(const char *base, int r, int g, uint32_t (&w)[NREG]) {
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < STEPS / 4; ++i) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(base + (uint32_t)(r * Lay::kRow + i * 64 + g * 16));
        w[4 * i] = v[0], w[4 * i + 1] = v[1], w[4 * i + 2] = v[2], w[4 * i + 3] = v[3];
      }
    } else {
      const uint2 v = *reinterpret_cast<const uint2 *>(base + (uint32_t)(r * Lay::kRow + g * 8));
      w[0] = v.x, w[1] = v.y;
      if constexpr (STEPS > 2) w[2] = *reinterpret_cast<const uint32_t *>(base + (uint32_t)(r * Lay::kRow + min(32 + g * 4, Lay::kRow - 4)));
    }
  }
  static __device__ __forceinline__ void load_units(const char *exponents, int r, int g, uint32_t (&u)[UNITS]) {
    const uint8_t *e = reinterpret_cast<const uint8_t *>(exponents) + (uint32_t)(r * Lay::kBlocks);
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < UNITS; ++i) u[i] = (uint32_t)e[4 * i + g];
    } else {
      u[0] = (uint32_t)e[g / 2];
      if constexpr (STEPS > 2) u[1] = (uint32_t)e[2];
    }
  }
  static __device__ __forceinline__ u32x4 operand(const uint32_t (&w)[NREG], const uint32_t (&u)[UNITS], int s, int g) {
    const u32x4 v = mx_decode8(w[s], u[WIDE ? s / 4 : s / 2]);
    return HD % 32 && s == STEPS - 1 && 64 + g * 8 >= HD ? u32x4{0, 0, 0, 0} : v;
  }
};
// Values in 4 bits: a lane's dimensions of a token are one load of 2 or 4 bytes, become bfloat16 pairs with the exponent of their block,
// and go on as bfloat16 values do.
template <int HD>
struct MxValues {
  using Lay = KvLayout<HD, ET_KV_MXFP4>;
  using Wide = Values<HD, ET_KV_BF16>;
  static constexpr int DPL = Wide::DPL, BLOCKS = Wide::BLOCKS, NREG = Wide::NREG;
  // the codes of the lane's dimensions
  static __device__ __forceinline__ uint32_t load(const char *base, int token, int r, int blk) {
    const char *at = base + (uint32_t)(token * Lay::kRow + (blk * 128 + min(r, HD / DPL - 1) * DPL) / 2);
    if constexpr (DPL == 8) return *reinterpret_cast<const uint32_t *>(at);
    else return *reinterpret_cast<const uint16_t *>(at);
  }
  // the exponents of four tokens from `token` on, a byte each
  static __device__ __forceinline__ uint32_t load_units(const char *exponents, int page_size, int token, int r, int blk) {
    const int block = blk * 4 + min(r, HD / DPL - 1) * DPL / kMxBlock;
    return *reinterpret_cast<const uint32_t *>(exponents + (uint32_t)(block * page_size + token));
  }
  // token e of those four (its exponent moves to where float32 has it; what comes along does not count)
  static __device__ __forceinline__ void widen(uint32_t code, uint32_t units, int e, uint32_t (&w)[NREG]) {
    const uint32_t unit = e == 0 ? units << 23 : e == 1 ? units << 15 : e == 2 ? units << 7 : units >> 1;
    w[0] = mx_pair<0>(code, unit), w[1] = mx_pair<1>(code, unit);
    if constexpr (DPL == 8) w[2] = mx_pair<2>(code, unit), w[3] = mx_pair<3>(code, unit);
  }
  static __device__ __forceinline__ u32x4 operand(const uint32_t (&w)[8][NREG], int j) { return Wide::operand(w, j); }
};

// Largest of three (without the canonicalisation that fmaxf asks for: these are results of arithmetic).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// What lane r's column of the products is: COLS columns are one query head's, r / COLS.  One: column h is head h, and an accumulator's rows
// are the j-th of DPL dimensions each.  Two: the even and the odd dimensions; a row of the values' operand is then a pair of dimensions as
// codes become them, (token, even), (token, odd) in turn along the summed axis, and a weight stands in the place of its column's parity, 0 in
// the other.  Four: both, with a weight's two halves apart.  A head's columns have the same logits; each takes a share of their softmax.
template <int COLS>
struct Cols {
  static constexpr int WIDTH = COLS == 1 ? 1 : 2;         // dimensions of an operand's row
  int head, index, odd, low;
  bool first, writes;                                     // of the head's columns; of those that are added up
  __device__ __forceinline__ Cols(int r)
      : head(r / COLS), index(r % COLS), odd(COLS == 1 ? 0 : r & 1), low(COLS == 4 ? r >> 1 & 1 : 0), first(index == 0), writes(!low) {}
  __device__ __forceinline__ int dim(int j) const { return j * WIDTH + odd; }
  // of four logits that all columns of a head have: the i-th of the column's own
  __device__ __forceinline__ float pick(f32x4 d, int i) const {
    if constexpr (COLS == 1) return d[i];
    else if constexpr (COLS == 2) return odd ? d[2 * i + 1] : d[2 * i];
    else return low ? (odd ? d[3] : d[2]) : (odd ? d[1] : d[0]);
  }
  // what the head's column I has
  template <int I>
  __device__ __forceinline__ uint32_t from(uint32_t x) const {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, COLS == 4 ? I * 0x55 : I * 0x55 + 0xA0, 0xf, 0xf, true);
  }
};

// The end of a workgroup's part: its wavefronts' results (accumulators, reference m and this lane's sum of query head r) together, and out,
// or to where the parts are joined.  `factor`: what the values are multiplied with.  WAVES: wavefronts of the workgroup, of which the first kWaves
// have results.
template <int HD, int DPL, int BLOCKS, int WAVES, int COLS>
__device__ __forceinline__ void finish_part(const PagedMore &o, const Part &part, const f32x4 (&acc)[BLOCKS * DPL / Cols<COLS>::WIDTH], float m, float sum, float factor,
                                            int wave, int live, int64_t head, int64_t slot, float (&lds_o)[kWaves][HD / BLOCKS][16],
                                            float2 (&lds_ml)[kWaves][16]) {
  constexpr int BD = HD / BLOCKS;                         // dimensions that the wavefronts add up at a time
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, h = threadIdx.x & 15;
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  const Cols<COLS> col(r);
  if (g == 0 && col.first && (WAVES == kWaves || wave < kWaves)) lds_ml[wave][col.head] = make_float2(m, sum);
  float top = -INFINITY, total = 0.f, f[kWaves];
#pragma unroll
  for (int blk = 0; blk < BLOCKS; ++blk) {
    if (blk) __syncthreads();
    if (col.writes && col.head < live && (WAVES == kWaves || wave < kWaves)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = (4 * g + e) * DPL;
        if (d < BD)
#pragma unroll
          for (int j = 0; j < DPL / col.WIDTH; ++j) lds_o[wave][d + col.dim(j)][col.head] = acc[blk * DPL / col.WIDTH + j][e];
      }
    }
    __syncthreads();
    if (blk == 0) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds_ml[w][h].x);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 ml = lds_ml[w][h];
        f[w] = part_factor(ml, top);
        total += f[w] * ml.y;
      }
    }
    for (int d = (threadIdx.x >> 4) * 8; h < live && d < BD; d += 4 * kWaves * 8) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x[e] = fmaf(f[w], lds_o[w][d + e][h], x[e]);
      }
      if (part.count == 1) {
        const float inv = factor / total;
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = total == 0.f ? 0 : cvt_pk_bf16(x[2 * e] * inv, x[2 * e + 1] * inv);  // (0 times x could be NaN)
        *reinterpret_cast<u32x4 *>(o.out + head * HD + blk * BD + d) = v;
      } else {
        float *to = o.part_o + slot * HD + blk * BD + d;
        *reinterpret_cast<f32x4 *>(to) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4 *>(to + 4) = f32x4{x[4], x[5], x[6], x[7]};
      }
    }
  }
  if (part.count > 1 && threadIdx.x < live) o.part_ml[slot] = make_float2(top, total);
}

// As paged_attention_kernel: a workgroup takes one part of a sequence's tokens for up to 16 query heads of one key-value head, its
// wavefronts tiles of 32 tokens in turn, S^T = K Q^T and O^T += V^T P^T by matrix instructions on bfloat16 numbers, which codes and their power of two
// are exactly; a weight is the sum of two of them, within 2^-15.  A tile's registers are loaded again as soon as they have become operands, so the next
// tile's keys come in during the softmax and the second product, its values during that and the next logits.  Bound by memory where there is much
// to read: 64 x 1000 to 16384 tokens of 8 heads of 128, 606 MB in 110 us, 5.5 TB/s, with vector instructions issued 40 % of the time (160 for 32 tokens);
// 9 x 1 to 2047 of 24 heads of 80, 32 MB in 13.1 us: a start of 4.5 us, then the longest part's eight turns, a chain of 0.9 us each (12.4 us where the
// other eight sequences have one token).  A
// tile more in flight: 120 -> 118 us there, 13.3 -> 14.0 here, 32 x 0 to 5309 of 4 heads 15.6 -> 16.7; sixteen wavefronts 13.3 -> 14.4.
template <int HD, bool ONE, int WAVES, int COLS>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_mxfp4_kernel(const int32_t *len, const int32_t *table, int n_seqs, int share, int bound,
                                                                 int window, int units, int row_tiles, int page_shift, int table_stride,
                                                                 int group, PagedMore o) {
  using Lay = KvLayout<HD, ET_KV_MXFP4>;
  using K = MxKeys<HD>;
  using V = MxValues<HD>;
  constexpr int ACCS = V::DPL / Cols<COLS>::WIDTH, ACC = V::BLOCKS * ACCS, OWN = 8 / COLS;
  __shared__ float lds_o[kWaves][HD / V::BLOCKS][16];
  __shared__ float2 lds_ml[kWaves][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const Cols<COLS> col(r);
  const PagedArgs a{len, n_seqs, bound, window, share};
  // (row tiles of one part and key-value head eight workgroups apart, as there)
  const int kv_heads = units / row_tiles;
  int place = blockIdx.x, rt = 0;
  if (row_tiles > 1) {
    const int turn = 8 * row_tiles, first = place / turn * 8, width = min(8, (int)gridDim.x / row_tiles - first);
    rt = place % turn / width;
    place = first + place % turn % width;
  }
  const int item = place / kv_heads, kv = place % kv_heads;
  const int n_heads = group * kv_heads, ps = 1 << page_shift;
  const int live = min(16, group - rt * 16);              // query heads of this workgroup
  Part part{item, 0, 1, 0, 0, 0};
  if (a.share) {
    part = find_part<ONE>(a, item, -1);
    if (part.seq < 0) return;
  } else {
    part.len = a.len[item];
  }
  const int b = __builtin_amdgcn_readfirstlane(part.seq);
  const SeqRange sr(__builtin_amdgcn_readfirstlane(part.len), a.bound, a.window);
  const int start = sr.lo + part.index * (int)part.per * kBlock;
  const int end = a.share ? (int)min((int64_t)sr.hi, (int64_t)start + (int64_t)part.per * kBlock) : sr.hi;
  const int tiles = end > start ? (end - start + kTile - 1) / kTile : 0;

  f32x4 acc[ACC];
#pragma unroll
  for (int j = 0; j < ACC; ++j) acc[j] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, sum = 0.f;                         // of query head r; sum: this lane's tokens only

  const int32_t *row = table + (int64_t)b * table_stride;
  const int mine = (tiles - wave + WAVES - 1) / WAVES;  // tiles of this wavefront
  int page_of = -1;                                       // lane i: page of the i-th group of 16 tokens of 32 tiles of the wavefront
  // (A group of 16 tokens without a page reads the first page's bytes, and its tokens do not count.)
  auto head_of = [&](int page) { return o.data + max(page, 0) * o.page_bytes + (int64_t)kv * Lay::head_bytes(ps); };
  struct Tile {
    uint32_t kw[2][K::NREG], ku[2][K::UNITS], code[V::BLOCKS][8], vu[V::BLOCKS][2];
    int page[2];
  };
  Tile x;
  auto load_keys = [&](int n) {                         // of the wavefront's n-th tile
    const int t = wave + n * WAVES;
    if ((n & 31) == 0) {
      const int pos = start + (t + (lane >> 1) * WAVES) * kTile + (lane & 1) * 16;
      page_of = pos < end ? row[pos >> page_shift] : -1;
      if (page_of >= o.n_pages) page_of = -1;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x.page[u] = __builtin_amdgcn_readlane(page_of, 2 * (n & 31) + u);
      const int at = (start + t * kTile + 16 * u) & (ps - 1);
      const char *head = head_of(x.page[u]);
      K::load(head + at * Lay::kRow, r, g, x.kw[u]);
      K::load_units(head + Lay::key_scale(ps) + at * Lay::kBlocks, r, g, x.ku[u]);
    }
  };
  auto load_values = [&](int n, int blk) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int at = (start + (wave + n * WAVES) * kTile + 16 * u) & (ps - 1);
      const char *head = head_of(x.page[u]);
#pragma unroll
      for (int i = 0; i < 4; ++i) x.code[blk][4 * u + i] = V::load(head + Lay::values(ps) + at * Lay::kRow, 4 * g + i, r, blk);
      x.vu[blk][u] = V::load_units(head + Lay::value_scale(ps), ps, at + 4 * g, r, blk);
    }
  };
  // (no branches around these loads, and the queries' awaited here: a turn then waits for its own operands alone)
  u32x4 qf[K::STEPS];
#pragma unroll
  for (int st = 0; st < K::STEPS; ++st)
    qf[st] = *reinterpret_cast<const u32x4 *>(o.q + b * o.q_stride + ((int64_t)kv * group + rt * 16 + min(col.head, live - 1)) * HD +
                                              min(K::dim(st, g), HD - 8));
  if (mine > 0) {
    load_keys(0);
#pragma unroll
    for (int blk = 0; blk < V::BLOCKS; ++blk) load_values(0, blk);
  }
#pragma unroll
  for (int st = 0; st < K::STEPS; ++st) {
    asm volatile("" : "+v"(qf[st]));
    if (col.head >= live || K::dim(st, g) >= HD) qf[st] = u32x4{0, 0, 0, 0};
  }
  // selectors of a weight's half in the place of the column's parity, 0 in the other: the upper one's (four columns: the column's own), the lower one's
  const uint32_t half = col.low ? (col.odd ? 0x03020C0Cu : 0x0C0C0302u) : (col.odd ? 0x01000C0Cu : 0x0C0C0100u);
  const uint32_t half2 = col.odd ? 0x03020C0Cu : 0x0C0C0302u;
  for (int n = 0; n < mine; ++n) {
    const int pos0 = start + (wave + n * WAVES) * kTile;
    // tokens that do not count: no page, past the end, before the window
    const bool paged[2] = {x.page[0] >= 0, x.page[1] >= 0};
    const bool whole = paged[0] && paged[1] && pos0 >= sr.first && pos0 + kTile <= end;
    const int next = min(n + 1, mine - 1);              // (the last tile again, from the caches, so that every turn has the same loads)
    float z[OWN];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 d{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < K::STEPS; ++st) d = mfma16(K::operand(x.kw[u], x.ku[u], st, g), qf[st], d);
#pragma unroll
      for (int i = 0; i < 4 / COLS; ++i) z[4 / COLS * u + i] = whole_product(col.pick(d, i), o.scale_log2);
    }
    load_keys(next);
    uint32_t dead = 0;
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int pos = pos0 + 16 * (i / 4) + 4 * g + (i & 3);
        if (!paged[i / 4] || pos < sr.first || pos >= end) {
          dead |= 1u << i;
        }
      }
#pragma unroll
      for (int i = 0; i < OWN; ++i)
        if (dead >> (COLS * i + col.index) & 1) z[i] = -INFINITY;
    }
    // The reference of the exponentials moves when a logit exceeds it by 2^8: below that nothing overflows.
    float top = max3(z[0], z[1], z[OWN > 2 ? 2 : 1]);
#pragma unroll
    for (int i = 3; i < OWN; i += 2) top = max3(top, z[i], z[min(i + 1, OWN - 1)]);
    if (__ballot(top > m + 8.f)) {
#pragma unroll
      for (int i = 1; i < COLS; i *= 2) top = fmaxf(top, __shfl_xor(top, i, 64));
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float m2 = fmaxf(m, top), f = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      sum *= f;
#pragma unroll
      for (int j = 0; j < ACC; ++j) acc[j] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float p[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      p[i] = __builtin_amdgcn_exp2f(z[i] - ref);
      sum += p[i];
    }
    // the weights' halves: what bfloat16 cuts off goes into the second
    u32x4 pf[2], pl[2];
    if constexpr (COLS == 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pf[0][i] = __builtin_amdgcn_perm(__float_as_uint(p[2 * i + 1]), __float_as_uint(p[2 * i]), 0x07060302u);
        pl[0][i] = cvt_pk_bf16(p[2 * i] - bf16lo_to_f32(pf[0][i]), p[2 * i + 1] - bf16hi_to_f32(pf[0][i]));
      }
    } else {
      // both halves of a lane's weights in one register, which the head's other columns read from there
      uint32_t both[OWN];
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        const float high = __uint_as_float(__float_as_uint(p[i]) & 0xFFFF0000u);
        both[i] = cvt_pk_bf16(high, p[i] - high);
      }
      const auto place = [&](auto token) {
        constexpr int i = decltype(token)::value;
        const uint32_t w = col.template from<i % COLS>(both[i / COLS]);
        pf[i / 4][i & 3] = __builtin_amdgcn_perm(w, w, half);
        if constexpr (COLS == 2) pl[i / 4][i & 3] = __builtin_amdgcn_perm(w, w, half2);
      };
      place(std::integral_constant<int, 0>()), place(std::integral_constant<int, 1>()), place(std::integral_constant<int, 2>());
      place(std::integral_constant<int, 3>()), place(std::integral_constant<int, 4>()), place(std::integral_constant<int, 5>());
      place(std::integral_constant<int, 6>()), place(std::integral_constant<int, 7>());
    }
#pragma unroll
    for (int blk = 0; blk < V::BLOCKS; ++blk) {
      uint32_t vw[8][V::NREG];
#pragma unroll
      for (int i = 0; i < 8; ++i) V::widen(x.code[blk][i], x.vu[blk][i / 4], i & 3, vw[i]);
      load_values(next, blk);
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int j = 0; j < V::NREG; ++j) vw[i][j] = dead >> i & 1 ? 0 : vw[i][j];   // (0 times what lies there could be NaN)
      }
#pragma unroll
      for (int j = 0; j < ACCS; ++j) {
        f32x4 &to = acc[blk * ACCS + j];
        if constexpr (COLS == 1) {
          const u32x4 values = V::operand(vw, j);
          to = mfma16(values, pf[0], mfma16(values, pl[0], to));
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const u32x4 values{vw[4 * u][j], vw[4 * u + 1][j], vw[4 * u + 2][j], vw[4 * u + 3][j]};
            if constexpr (COLS == 2) to = mfma16(values, pl[u], to);
            to = mfma16(values, pf[u], to);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 1; i < COLS; i *= 2) sum += __shfl_xor(sum, i, 64);
  if constexpr (COLS == 4) {
#pragma unroll
    for (int j = 0; j < ACC; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] += __shfl_xor(acc[j][i], 2, 64);
  }
  if constexpr (WAVES > kWaves) {
    // the upper half's results go to the lower half, block by block of dimensions
    float all = sum;
    all += __shfl_xor(all, 16, 64);
    all += __shfl_xor(all, 32, 64);
    const int to = wave & (kWaves - 1);
    const bool upper = wave >= kWaves;
    if (upper && g == 0) lds_ml[to][r] = make_float2(m, all);
    float f = 0.f, f2 = 0.f;
#pragma unroll
    for (int blk = 0; blk < V::BLOCKS; ++blk) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = (4 * g + i) * V::DPL;
        if (upper && col.writes && d < HD / V::BLOCKS)
#pragma unroll
          for (int j = 0; j < ACCS; ++j) lds_o[to][d + col.dim(j)][col.head] = acc[blk * ACCS + j][i];
      }
      __syncthreads();
      if (!upper) {
        if (blk == 0) {
          const float2 other = lds_ml[to][r];
          const float top = fmaxf(m, other.x);
          f = part_factor(make_float2(m, all), top), f2 = part_factor(other, top);
          sum = sum * f + (g == 0 ? other.y * f2 : 0.f);
          m = top;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = (4 * g + i) * V::DPL;
          if (d < HD / V::BLOCKS)
#pragma unroll
            for (int j = 0; j < ACCS; ++j) {
              f32x4 &x = acc[blk * ACCS + j];
              x[i] = fmaf(f2, lds_o[to][d + col.dim(j)][col.head], f * x[i]);
            }
        }
      }
      __syncthreads();
    }
  }
  const int h = threadIdx.x & 15;
  const int64_t head = (int64_t)b * n_heads + (int64_t)kv * group + rt * 16 + h;
  const int64_t slot = (int64_t)item * n_heads + kv * group + rt * 16 + h;       // of a part that is one of several
  finish_part<HD, V::DPL, V::BLOCKS, WAVES, COLS>(o, part, acc, m, sum, 1.f, wave, live, head, slot, lds_o, lds_ml);
}

int launch_paged_mxfp4(int head_dim, const PagedLaunch &l) {
  const int span = l.window > 0 ? (int)std::min<int64_t>(l.bound, (int64_t)l.window + 15) : l.bound;
  // Eight wavefronts where a part is long and a compute unit has one at most, us with eight / four: 9 x 2048 of 24 heads of 128 13.9 / 16.7, of 64
  // 11.3 / 14.2, 32 x 800 of 8 heads of 128 7.8 / 8.9; but 32 x 200 of 4 5.6 / 5.2, 64 x 1500 of 8 20.6 / 19.4.
  const bool wide = l.share == 0 && span > 512 && l.blocks <= 256;
  return kv_dispatch_mxfp4(head_dim, [&](auto hd) {
    auto launch = [&](auto kernel, int waves) {
      kernel<<<l.blocks, 64 * waves, 0, l.stream>>>(l.len, l.table, l.n_seqs, l.share, l.bound, l.window, l.units, l.row_tiles, l.page_shift,
                                                    l.table_stride, l.group, l.more);
      ET_LAUNCH_CHECK();
      return ET_OK;
    };
    // As many columns of a head as there is room for.  us with 1 / 2 / 4: 9 x 1 to 2047 tokens of 24 heads of 80 15.5 / 14.6 / 14.0, 32 x 800 of
    // 8 of 128 with four query heads each 9.0 / 8.3 / 8.2, 32 x 1000 of 4 with seven 9.6 / 8.9; where memory is the bound they are level, 64 x
    // 1000 to 16384 tokens of 8 122.
    auto pick = [&](auto cols) {
      if (wide) return launch(paged_mxfp4_kernel<hd.value, false, 2 * kWaves, cols.value>, 2 * kWaves);
      return l.n_seqs == 1 ? launch(paged_mxfp4_kernel<hd.value, true, kWaves, cols.value>, kWaves)
                           : launch(paged_mxfp4_kernel<hd.value, false, kWaves, cols.value>, kWaves);
    };
    if (l.group <= 4) return pick(std::integral_constant<int, 4>());
    if (l.group <= 8) return pick(std::integral_constant<int, 2>());
    return pick(std::integral_constant<int, 1>());
  });
}

}  // namespace et
