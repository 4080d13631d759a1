// Attention of one new token per sequence over a paged key-value cache.
#include <type_traits>

#include "kv_cache.h"
#include "mfma_common.h"
#include "select_common.h"

namespace et {

constexpr int kTile = 32;                                // tokens that a wavefront takes at a time
constexpr int kWaves = 4;                                // wavefronts of a workgroup
constexpr int kBlock = kWaves * kTile;
// Workgroups that a call is shared out over: two per compute unit (us at 512 / 768 / 1024: 32 x 0 to 5309 int8 tokens 21.9 / 23.2 / 25.0,
// 131072 bfloat16 tokens 96 / 98 / 97); and how many times as many at most (see part_blocks).
constexpr int kShare = 512, kFiner = 4;

// a * b rounded, never part of a fused multiply-add: a logit less the maximum has to be 0 for the maximum itself, however large.
__device__ __forceinline__ float whole_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// How a call's work is shared out.  The tokens of all sequences, in blocks of kBlock, are dealt out evenly over about `share`
// workgroups per query-head tile; a workgroup gets up to `per` consecutive blocks of one sequence (a part of it), so that lengths
// that differ leave no workgroup with more than another.  Only the device knows the lengths: each workgroup finds its part by a
// scan over them, 64 at a time.  There are at most kFiner share + n_seqs parts, whatever the lengths are.
struct PagedArgs {
  const int32_t *len;
  int n_seqs, bound, window;                             // bound: no position from here on counts
  int share;                                             // 0: every sequence is one part
};
// Tokens [first, hi) of a sequence count; lo = first rounded down to 16.
struct SeqRange {
  int lo, hi, first;
  __device__ __forceinline__ SeqRange(int len, int bound, int window) {
    hi = min(len, bound);
    first = window > 0 && len > window ? len - window : 0;
    lo = first & ~15;
  }
  __device__ __forceinline__ uint32_t blocks() const { return hi > lo ? (uint32_t)(hi - lo + kBlock - 1) / kBlock : 0; }
};
// Blocks of a part.  Sequences seldom end with a whole part, so where there are several and the parts are long, shorter ones even
// out what the last parts leave over: 64 x 1000 to 16384 e4m3 tokens 247 -> 215 us, 12 x 2000 to 8000 with heads of 256 116 -> 101.
__device__ __forceinline__ uint32_t part_blocks(const PagedArgs &a, uint32_t total) {
  const uint32_t per = max((total + a.share - 1) / a.share, 1u);
  return a.n_seqs > 1 && per > 8 ? max((per + kFiner - 1) / kFiner, 8u) : per;
}
struct Part {
  int seq, index, count;                                 // the index-th of sequence seq's `count`; seq < 0: none
  int len;                                               // of the sequence
  uint32_t per, before;                                  // blocks of a part; parts of the sequences before this one
};
// Part number `item`, or (of_seq >= 0) what belongs to that sequence.  The same in all lanes.  ONE: there is one sequence; without the
// scans' code beside it each kernel of such a call is 0.2 us shorter.
template <bool ONE>
__device__ __forceinline__ Part find_part(const PagedArgs &a, int item, int of_seq) {
  const int lane = threadIdx.x & 63;
  Part p{-1, 0, 0, 0, 1, 0};
  if constexpr (ONE) {
    p.len = a.len[0];
    const uint32_t blocks = SeqRange(p.len, a.bound, a.window).blocks();
    p.per = part_blocks(a, blocks);
    p.count = (blocks + p.per - 1) / p.per;
    p.index = item;
    if (of_seq >= 0 || item < p.count) p.seq = 0;
    return p;
  }
  auto len_of = [&](int i) { return i < a.n_seqs ? a.len[i] : 0; };
  int len = len_of(lane), ahead = 0, total = (int)SeqRange(len, a.bound, a.window).blocks();
  if (a.n_seqs > 64) ahead = len_of(lane + 64);
  for (int i = lane + 64; i - lane < a.n_seqs; i += 256) {  // (four loads in flight)
    int l[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) l[u] = len_of(i + 64 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u) total += (int)SeqRange(l[u], a.bound, a.window).blocks();
  }
  total = __builtin_amdgcn_readlane(wave_inclusive_scan(total), 63);
  p.per = part_blocks(a, total);
  for (int i0 = 0; i0 < a.n_seqs; i0 += 64) {
    int after = 0;
    if (i0 + 128 < a.n_seqs) after = len_of(i0 + 128 + lane);
    const int parts = (SeqRange(len, a.bound, a.window).blocks() + p.per - 1) / p.per, upto = wave_inclusive_scan(parts);
    const uint64_t found = of_seq < 0 ? __ballot((uint32_t)item < p.before + upto) : of_seq < i0 + 64 ? 1ull << (of_seq & 63) : 0;
    if (found) {
      const int at = __builtin_ctzll(found);
      p.seq = i0 + at;
      p.len = __builtin_amdgcn_readlane(len, at);
      p.count = __builtin_amdgcn_readlane(parts, at);
      p.before += __builtin_amdgcn_readlane(upto, at) - p.count;
      p.index = item - (int)p.before;
      return p;
    }
    p.before += __builtin_amdgcn_readlane(upto, 63);
    len = ahead;
    ahead = after;
  }
  return p;
}

// Weight of a part (or a wavefront's share) whose largest logit and sum are ml, against the largest of all.  One without tokens has
// none; a NaN in its sum stays.
__device__ __forceinline__ float part_factor(float2 ml, float top) {
  return ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(ml.x - top);
}
// What the values' codes are multiplied with at the end (their rows' maxima went into the weights, times 2^-9).
template <int FMT>
__device__ __forceinline__ float value_factor() { return FMT == ET_KV_BF16 ? 1.f : 1.f / (kv_qmax<FMT>() * 0x1p-9f); }

// bf16 pair of two 8-bit codes, bytes 2 SEL and 2 SEL + 1 of w; exact in both formats.
template <int FMT, int SEL>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
  if constexpr (FMT == ET_KV_E4M3) {
    const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, SEL != 0);
    return __builtin_bit_cast(uint32_t, v);
  } else {
    const float a = (float)(int8_t)(w >> (16 * SEL)), b = (float)(int8_t)(w >> (16 * SEL + 8));
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  }
}

// Keys.  S^T = K Q^T by 16x16x32 MFMAs: a token is a row of operand A, a query head a column of operand B, and lane (r, g) holds
// of token r (head r) eight of a step's 32 dimensions.  Which ones is free, as long as both sides agree: g's eighths in turn for
// bfloat16; in 8 bits a lane's 16-byte load serves two steps.
template <int HD, int FMT>
struct Keys {
  static constexpr int STEPS = (HD + 31) / 32, kRow = KvLayout<HD, FMT>::kRow;
  static constexpr bool WIDE = FMT == ET_KV_BF16;
  static constexpr int PAIRS = WIDE ? 0 : STEPS / 2, NREG = WIDE ? STEPS * 4 : PAIRS * 4 + (STEPS % 2) * 2;
  static __device__ __forceinline__ int dim(int s, int g) {
    return WIDE || s >= 2 * PAIRS ? s * 32 + g * 8 : (s / 2) * 64 + g * 16 + (s % 2) * 8;
  }
  // Past the row's end the last dimensions are read again (and not used).
  static __device__ __forceinline__ void load(const char *base, int r, int g, uint32_t (&w)[NREG]) {
    if constexpr (WIDE) {
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const int d = s * 32 + g * 8;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(base + (uint32_t)(r * kRow + 2 * (HD % 32 && d >= HD ? HD - 8 : d)));
        w[4 * s] = v[0], w[4 * s + 1] = v[1], w[4 * s + 2] = v[2], w[4 * s + 3] = v[3];
      }
    } else {
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(base + (uint32_t)(r * kRow + p * 64 + g * 16));
        w[4 * p] = v[0], w[4 * p + 1] = v[1], w[4 * p + 2] = v[2], w[4 * p + 3] = v[3];
      }
      if constexpr (STEPS % 2) {
        const int d = (STEPS - 1) * 32 + g * 8;
        const uint2 v = *reinterpret_cast<const uint2 *>(base + (uint32_t)(r * kRow + (d >= HD ? HD - 8 : d)));
        w[4 * PAIRS] = v.x, w[4 * PAIRS + 1] = v.y;
      }
    }
  }
  static __device__ __forceinline__ u32x4 operand(const uint32_t (&w)[NREG], int s, int g) {
    u32x4 v;
    if constexpr (WIDE) v = u32x4{w[4 * s], w[4 * s + 1], w[4 * s + 2], w[4 * s + 3]};
    else {
      const int at = s < 2 * PAIRS ? 4 * (s / 2) + 2 * (s % 2) : 4 * PAIRS;
      v = u32x4{code_pair<FMT, 0>(w[at]), code_pair<FMT, 1>(w[at]), code_pair<FMT, 0>(w[at + 1]), code_pair<FMT, 1>(w[at + 1])};
    }
    if (HD % 32 && s == STEPS - 1 && s * 32 + g * 8 >= HD) v = u32x4{0, 0, 0, 0};
    return v;
  }
};

// Values.  O^T = V^T P^T: a lane loads DPL neighbouring dimensions of each of its eight tokens, so that 16 lanes read whole
// rows; operand A number j is the j-th dimension of every lane's eight tokens, put together by byte permutes in the lane.
template <int HD, int FMT>
struct Values {
  static constexpr int DPL = HD <= 64 ? 4 : 8, BLOCKS = HD > 128 ? 2 : 1, kRow = KvLayout<HD, FMT>::kRow, B = KvLayout<HD, FMT>::kBytes;
  static constexpr int NREG = DPL * B / 4;                               // per token and block
  static __device__ __forceinline__ void load(const char *base, int token, int r, int blk, uint32_t (&w)[NREG]) {
    const uint32_t off = token * kRow + (blk * 128 + min(r, HD / DPL - 1) * DPL) * B;
    if constexpr (NREG == 4) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(base + off);
      w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
    } else if constexpr (NREG == 2) {
      const uint2 v = *reinterpret_cast<const uint2 *>(base + off);
      w[0] = v.x, w[1] = v.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t *>(base + off);
    }
  }
  // operand A of dimension j from the eight tokens' registers
  static __device__ __forceinline__ u32x4 operand(const uint32_t (&w)[8][NREG], int j) {
    u32x4 v;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
      if constexpr (FMT == ET_KV_BF16) v[p] = __builtin_amdgcn_perm(w[2 * p + 1][j / 2], w[2 * p][j / 2], sel);
      else if constexpr (FMT == ET_KV_INT8) {
        const float a = (float)(int8_t)(w[2 * p][j / 4] >> (8 * (j & 3))), b = (float)(int8_t)(w[2 * p + 1][j / 4] >> (8 * (j & 3)));
        v[p] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
      } else {
        const uint32_t a = w[2 * p][j / 4], b = w[2 * p + 1][j / 4];
        v[p] = j & 2 ? __builtin_amdgcn_perm(code_pair<FMT, 1>(b), code_pair<FMT, 1>(a), sel)
                     : __builtin_amdgcn_perm(code_pair<FMT, 0>(b), code_pair<FMT, 0>(a), sel);
      }
    }
    return v;
  }
};

struct PagedMore {                                       // the kernel's arguments that its first loads do not need
  const uint16_t *q;
  int64_t q_stride;
  char *data;
  int64_t page_bytes;
  float *part_o;
  float2 *part_ml;
  uint16_t *out;
  int n_pages;
  float scale_log2;
};
// A workgroup takes one part of a sequence's tokens for up to 16 query heads of one key-value head; its wavefronts take tiles of
// 32 tokens in turn: logits S^T = K Q^T, weights against a running reference, O^T += V^T P^T, where the accumulators that hold S^T are,
// exponentiated and rounded, operand B of the second product (which tokens a lane's eight places of the contraction stand for is free, and the
// values are loaded to match).  The cache's bytes go to registers in operand order, with no LDS on the way, the next tile's keys while a
// tile is worked on; up to 16 query heads per key-value head read everything once, more of them once for each 16.  A weight is taken as
// the sum of two bfloat16 numbers (within 2^-15 of it) by two matrix instructions on the same values, so that what is left of its
// rounding is far below the result's own, 2^-8; logits, reference, sums and accumulators are float32.
// Bound by the memory side from some 10 MB on: 537 MB of bfloat16 (one sequence of 131072 tokens, 8 key-value heads of 128) in 91 us,
// 5.9 TB/s, 1.16 GB of e4m3 (64 sequences) in 209, 5.6 TB/s, by the counters 1.00 of these bytes; below that by the chain launch -
// length - page - keys - products - joined wavefronts, 4.1 us at the least.  Two workgroups per compute unit are asked for: without that the compiler
// moves the accumulators to and fro between the two halves of the registers, and 32 int8 sequences of up to 5309 tokens take 24.0
// instead of 21.9 us, 12 of 2000 to 8000 with 16 heads of 256 134 instead of 101.
template <int HD, int FMT, bool ONE>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_kernel(const int32_t *len, const int32_t *table, int n_seqs,
                                                                      int share, int bound, int window, int units, int row_tiles,
                                                                      int page_shift, int table_stride, int group, PagedMore o) {
  using Lay = KvLayout<HD, FMT>;
  using K = Keys<HD, FMT>;
  using V = Values<HD, FMT>;
  constexpr int ACC = V::BLOCKS * V::DPL;
  constexpr bool kAhead = HD <= 128;                      // a tile's keys are fetched during the one before: heads of 256 have no registers for it
  constexpr int BD = HD / V::BLOCKS;                      // dimensions that the wavefronts add up at a time
  __shared__ float lds_o[kWaves][BD][16];
  __shared__ float2 lds_ml[kWaves][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const PagedArgs a{len, n_seqs, bound, window, share};
  // The row tiles of one part and key-value head are eight workgroups apart: on the same XCD, whose L2 gives them the bytes twice.
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
  const SeqRange sr(part.len, a.bound, a.window);
  const int start = sr.lo + part.index * (int)part.per * kBlock;
  const int end = a.share ? (int)min((int64_t)sr.hi, (int64_t)start + (int64_t)part.per * kBlock) : sr.hi;
  const int tiles = end > start ? (end - start + kTile - 1) / kTile : 0;

  f32x4 acc[ACC];
#pragma unroll
  for (int j = 0; j < ACC; ++j) acc[j] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, sum = 0.f;                         // of query head r; sum: this lane's tokens only

  const int32_t *row = table + (int64_t)b * table_stride;
  int page_of = -1;                                       // lane i: page of the wavefront's i-th group of 16 tokens, of 64
  auto fetch_pages = [&](int t) {
    const int pos = start + (t + (lane >> 1) * kWaves) * kTile + (lane & 1) * 16;
    page_of = pos < end ? row[pos >> page_shift] : -1;
    if (page_of >= o.n_pages) page_of = -1;
  };
  // (A group without a page reads the first page's bytes, and its tokens do not count.)
  auto head_of = [&](int page) { return o.data + max(page, 0) * o.page_bytes + (int64_t)kv * Lay::head_bytes(ps); };
  struct Tile {
    uint32_t kw[2][K::NREG];
    uint2 km[2], vm[2];
    int page[2];
  };
  auto load_keys = [&](Tile &x, int t, int i) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x.page[u] = __builtin_amdgcn_readlane(page_of, i + u);
      const int at = (start + t * kTile + 16 * u) & (ps - 1);
      const char *head = head_of(x.page[u]);
      K::load(head + at * Lay::kRow, r, g, x.kw[u]);
      if constexpr (FMT != ET_KV_BF16) {
        x.km[u] = *reinterpret_cast<const uint2 *>(head + Lay::key_max(ps) + (at + 4 * g) * 2);
        x.vm[u] = *reinterpret_cast<const uint2 *>(head + Lay::value_max(ps) + (at + 4 * g) * 2);
      }
    }
  };
  Tile next;
  fetch_pages(wave);                                      // (in front of the queries' loads: the keys' wait for it)
  u32x4 qf[K::STEPS];
#pragma unroll
  for (int st = 0; st < K::STEPS; ++st) {
    const int d = K::dim(st, g);
    qf[st] = u32x4{0, 0, 0, 0};
    if (r < live && d < HD)
      qf[st] = *reinterpret_cast<const u32x4 *>(o.q + b * o.q_stride + ((int64_t)kv * group + rt * 16 + r) * HD + d);
  }
  if (wave < tiles) load_keys(next, wave, 0);
  for (int t = wave, i = 0; t < tiles; t += kWaves) {
    if (!kAhead && t != wave) load_keys(next, t, i);
    const Tile cur = next;
    const int pos0 = start + t * kTile;
    const uint2 *km = cur.km, *vm = cur.vm;
    const int *page = cur.page;
    const auto &kw = cur.kw;
    uint32_t vw[8][V::NREG];
    auto load_values = [&](int blk) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const char *values = head_of(page[u]) + Lay::values(ps) + ((pos0 + 16 * u) & (ps - 1)) * Lay::kRow;
#pragma unroll
        for (int e = 0; e < 4; ++e) V::load(values, 4 * g + e, r, blk, vw[4 * u + e]);
      }
    };
    load_values(0);
    i = (i + 2) & 63;
    if (i == 0) fetch_pages(t + kWaves);
    float z[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 d{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < K::STEPS; ++st) d = mfma16(K::operand(kw[u], st, g), qf[st], d);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float f = o.scale_log2;
        if constexpr (FMT != ET_KV_BF16) f *= e & 1 ? bf16hi_to_f32(e & 2 ? km[u].y : km[u].x) : bf16lo_to_f32(e & 2 ? km[u].y : km[u].x);
        z[4 * u + e] = whole_product(d[e], f);
      }
    }
    if (kAhead && t + kWaves < tiles) load_keys(next, t + kWaves, i);
    // tokens that do not count: no page, past the end, before the window
    const bool whole = page[0] >= 0 && page[1] >= 0 && pos0 >= sr.first && pos0 + kTile <= end;
    uint32_t dead = 0;
    if (!whole) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int pos = pos0 + 16 * (e / 4) + 4 * g + (e & 3);
        if (page[e / 4] < 0 || pos < sr.first || pos >= end) {
          dead |= 1u << e;
          z[e] = -INFINITY;
        }
      }
    }
    // The reference of the exponentials moves when a logit exceeds it by 2^8: below that nothing overflows.
    float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
    if (__ballot(top > m + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float m2 = fmaxf(m, top), f = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      sum *= f;
#pragma unroll
      for (int j = 0; j < ACC; ++j) acc[j] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(z[e] - ref);
      sum += p[e];
      if constexpr (FMT != ET_KV_BF16) {
        const uint32_t w = e & 2 ? vm[e / 4].y : vm[e / 4].x;
        p[e] *= (e & 1 ? bf16hi_to_f32(w) : bf16lo_to_f32(w)) * 0x1p-9f;
        if (!whole && (dead >> e & 1)) p[e] = 0.f;
      }
    }
    // The weights' halves: what bfloat16 cuts off goes into the second.  Neither is 0 or negative where the weight is not (2^-20 of it is
    // added), so that an infinite value stays one.
    u32x4 pf, pl;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      pf[e] = __builtin_amdgcn_perm(__float_as_uint(p[2 * e + 1]), __float_as_uint(p[2 * e]), 0x07060302u);
      pl[e] = cvt_pk_bf16(fmaf(p[2 * e], 0x1p-20f, p[2 * e] - bf16lo_to_f32(pf[e])),
                          fmaf(p[2 * e + 1], 0x1p-20f, p[2 * e + 1] - bf16hi_to_f32(pf[e])));
    }
#pragma unroll
    for (int blk = 0; blk < V::BLOCKS; ++blk) {
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int x = 0; x < V::NREG; ++x) vw[e][x] = dead >> e & 1 ? 0 : vw[e][x];     // (0 times what lies there could be NaN)
      }
#pragma unroll
      for (int j = 0; j < V::DPL; ++j) {
        const u32x4 values = V::operand(vw, j);
        f32x4 &to = acc[blk * V::DPL + j];
        to = mfma16(values, pf, mfma16(values, pl, to));
      }
      if (blk + 1 < V::BLOCKS) load_values(blk + 1);
    }
  }

  // the wavefronts' results together
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (g == 0) lds_ml[wave][r] = make_float2(m, sum);
  const int h = threadIdx.x & 15;
  const int64_t head = (int64_t)b * n_heads + (int64_t)kv * group + rt * 16 + h;
  const int64_t slot = (int64_t)item * n_heads + kv * group + rt * 16 + h;       // of a part that is one of several
  float top = -INFINITY, total = 0.f, f[kWaves];
#pragma unroll
  for (int blk = 0; blk < V::BLOCKS; ++blk) {
    if (blk) __syncthreads();
    if (r < live) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = (4 * g + e) * V::DPL;
        if (d < BD)
#pragma unroll
          for (int j = 0; j < V::DPL; ++j) lds_o[wave][d + j][r] = acc[blk * V::DPL + j][e];
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
        const float inv = value_factor<FMT>() / total;
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

// Joins the parts of one query head, always in the same order: groups of lanes, four dimensions a lane, take every GROUPS-th part
// with a running maximum and sum, eight parts' loads in flight, and the groups' results are added up in the groups' order.
// A head whose sequence is one part has its result already.  THREADS: 64 where a sequence has few parts.  Bound by latency: 28 heads of
// 40 parts take 3.1 us, 32 of 64 5.0, 2048 of four 5.1.
template <int HD, int FMT, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void paged_join_kernel(const int32_t *len, const float *part_o, const float2 *part_ml, int n_seqs,
                                                             int share, int bound, int window, int n_heads, uint16_t *out) {
  constexpr int LANES = HD / 4, GROUPS = THREADS / LANES, BATCH = 8;
  __shared__ float lds_o[GROUPS][HD];
  __shared__ float2 lds_ml[GROUPS];
  const PagedArgs a{len, n_seqs, bound, window, share};
  const int b = blockIdx.x / n_heads, h = blockIdx.x % n_heads;
  const int tid = threadIdx.x, lane = tid % LANES, grp = tid / LANES;
  f32x4 v[BATCH];
  float2 s[BATCH];
  auto load = [&](int before, int first, int last) {
    const int64_t base = (int64_t)before * n_heads + h;
    const float2 *my_ml = part_ml + base;
    const float *my_o = part_o + base * HD;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const uint32_t at = (uint32_t)min(first + i * GROUPS, last) * n_heads;
      s[i] = my_ml[at];
      v[i] = *reinterpret_cast<const f32x4 *>(my_o + (at * HD + lane * 4));
    }
  };
  // a single sequence's parts come first, however many there are: their loads need not wait for its length
  if (ONE && grp < GROUPS) load(0, grp, share - 1);
  const Part p = find_part<ONE>(a, 0, b);
  if (p.count == 1) return;
  if (!ONE && grp < GROUPS && p.count) load(p.before, grp, p.count - 1);
  if (grp < GROUPS) {
    f32x4 x{0, 0, 0, 0};
    float top = -INFINITY, total = 0.f;
    for (int first = grp; first < p.count; first += BATCH * GROUPS) {
      if (first != grp) load(p.before, first, p.count - 1);
      float most = top;
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
        if (first + i * GROUPS < p.count) most = fmaxf(most, s[i].x);
      const float old = part_factor(make_float2(top, total), most);
      total *= old;
      top = most;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= old;
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
        if (first + i * GROUPS < p.count) {
          const float f = part_factor(s[i], top);
          total = fmaf(f, s[i].y, total);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = fmaf(f, v[i][e], x[e]);
        }
    }
    *reinterpret_cast<f32x4 *>(&lds_o[grp][lane * 4]) = x;
    if (lane == 0) lds_ml[grp] = make_float2(top, total);
  }
  __syncthreads();
  float top = -INFINITY, total = 0.f, f[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) top = fmaxf(top, lds_ml[i].x);
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    f[i] = part_factor(lds_ml[i], top);
    total = fmaf(f[i], lds_ml[i].y, total);
  }
  for (int d = tid; d < HD; d += THREADS) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) x = fmaf(f[i], lds_o[i][d], x);
    out[(int64_t)blockIdx.x * HD + d] = f32_to_bf16_bits(total == 0.f ? 0.f : x * (value_factor<FMT>() / total));
  }
}

struct PagedPlan {
  int group, row_tiles, units, bound, share;
  int64_t items;                                         // workgroups per unit
  size_t slots, bytes;                                   // of the workspace
};
static PagedPlan paged_plan(const et_kv_cache &c, const et_kv_seqs &s, int n_heads, int max_len, int window) {
  PagedPlan p;
  p.group = n_heads / c.n_kv_heads;
  p.row_tiles = (p.group + 15) / 16;
  p.units = p.row_tiles * c.n_kv_heads;
  p.bound = std::min(max_len, s.pages_per_seq * c.page_size);
  const int span = window > 0 ? (int)std::min<int64_t>(p.bound, (int64_t)window + 15) : p.bound;
  const int64_t blocks = (int64_t)s.n_seqs * ((span + kBlock - 1) / kBlock);
  // One part each where that is as fast: short sequences, and longer ones that fill the chip by themselves.  us as one part / shared out:
  // 1 x 197 tokens 4.8 / 7.7, 256 x 500 of 4 key-value heads 50 / 58, 4 x 1000 of 32 13.7 / 16.7, 1024 x 100 to 2048 of 4 223 / 261;
  // but 1 x 700 of 8 10.0 / 7.8, 4 x 1500 of 4 16.8 / 8.6, 64 x 1000 to 16384 of 8 255 / 215.  The host knows the bound only, so a
  // generous one takes the second figure; and the rule counts tokens, not their bytes (64 x 1024 of one bfloat16 head of 256, one part
  // each: 24.0 / 20.3).
  // Beyond 4096 sequences too: every workgroup of a call that is shared out looks at all lengths, which would come to a minute for
  // a million sequences.  Bound 131072: 4097 x 60 tokens of 8 195 / 1200, 0 to 8000 8768 / 9167, 60 with one of 131072 among them
  // 1419 / 1261 (of one key-value head 1113 / 277).
  const int64_t all = (int64_t)s.n_seqs * p.units;
  const bool whole = span <= 512 || (span <= 1024 && all >= 64) || (span <= 2048 && all >= 1024) || s.n_seqs > 4096;
  p.share = whole ? 0 : (int)std::min<int64_t>(blocks, (kShare + p.units - 1) / p.units);
  p.items = p.share * (s.n_seqs > 1 ? kFiner : 1) + (int64_t)s.n_seqs;
  p.slots = p.share ? (size_t)p.items * n_heads : 0;
  p.bytes = p.slots * (c.head_dim * sizeof(float) + sizeof(float2));
  return p;
}

static int check_paged(const et_kv_cache *cache, const et_kv_seqs *seqs, int n_heads, int max_len, int window) {
  int rc;
  if ((rc = check_kv(cache, seqs))) return rc;
  ET_REQUIRE(n_heads >= 1 && n_heads % cache->n_kv_heads == 0 && n_heads <= 65536,
             "n_heads = %d must be a multiple of n_kv_heads = %d, at most 65536", n_heads, cache->n_kv_heads);
  ET_REQUIRE(max_len >= 1, "max_len = %d must be at least 1", max_len);
  ET_REQUIRE(window >= 0, "window = %d is negative", window);
  ET_REQUIRE((int64_t)seqs->n_seqs * n_heads <= 1 << 24, "n_seqs * n_heads = %lld is above 2^24", (long long)seqs->n_seqs * n_heads);
  ET_REQUIRE((int64_t)seqs->n_seqs * std::min(max_len, seqs->pages_per_seq * cache->page_size) <= 1ll << 36,
             "n_seqs * max_len is above 2^36");
  // (a launch takes fewer than 2^32 lanes)
  const PagedPlan p = paged_plan(*cache, *seqs, n_heads, max_len, window);
  ET_REQUIRE(p.items * p.units < (1ll << 32) / (64 * kWaves), "n_seqs * n_kv_heads = %lld is too much for one launch",
             (long long)seqs->n_seqs * cache->n_kv_heads);
  return ET_OK;
}

}  // namespace et

using namespace et;

extern "C" {

size_t et_attention_paged_workspace_bytes(const et_kv_cache *cache, const et_kv_seqs *seqs, int32_t n_heads, int32_t max_len,
                                          int32_t window) {
  if (check_paged(cache, seqs, n_heads, max_len, window) || seqs->n_seqs == 0) return 0;
  return paged_plan(*cache, *seqs, n_heads, max_len, window).bytes;
}

int et_attention_paged(const et_kv_cache *cache, const et_kv_seqs *seqs, const uint16_t *q_dev, int64_t q_stride, int32_t n_heads,
                       int32_t max_len, int32_t window, float scale, void *workspace_dev, size_t workspace_bytes, uint16_t *out_dev,
                       void *hip_stream) {
  int rc;
  if ((rc = check_paged(cache, seqs, n_heads, max_len, window))) return rc;
  ET_REQUIRE(scale - scale == 0.f, "scale must be finite");
  if (seqs->n_seqs == 0) return ET_OK;
  ET_REQUIRE(q_dev && out_dev && (uintptr_t)q_dev % 16 == 0 && (uintptr_t)out_dev % 16 == 0,
             "q_dev or out_dev is NULL or not aligned to 16 bytes");
  ET_REQUIRE(q_stride % 8 == 0 && q_stride >= (int64_t)n_heads * cache->head_dim, "q_stride = %lld must be a multiple of 8 and at least %lld",
             (long long)q_stride, (long long)n_heads * cache->head_dim);
  const PagedPlan p = paged_plan(*cache, *seqs, n_heads, max_len, window);
  if (p.bytes) {
    ET_REQUIRE(workspace_dev != nullptr && (uintptr_t)workspace_dev % 16 == 0, "workspace_dev is NULL or not aligned to 16 bytes");
    if (workspace_bytes < p.bytes) {
      set_error("workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, p.bytes);
      return ET_ERR_WORKSPACE;
    }
  }
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  float *part_o = static_cast<float *>(workspace_dev);
  float2 *part_ml = reinterpret_cast<float2 *>(part_o + p.slots * cache->head_dim);
  const float scale_log2 = scale * 1.4426950408889634f * (cache->format == ET_KV_BF16 ? 1.f : cache->format == ET_KV_INT8 ? 1.f / 127.f : 1.f / 448.f);
  const KvPages c = kv_pages(*cache);
  return kv_dispatch(cache->head_dim, cache->format, [&](auto hd, auto fmt) {
    const bool one = seqs->n_seqs == 1;
    (one ? paged_attention_kernel<hd.value, fmt.value, true> : paged_attention_kernel<hd.value, fmt.value, false>)<<<
        (unsigned)(p.items * p.units), 64 * kWaves, 0, stream>>>(
        seqs->kv_len_dev, seqs->page_table_dev, seqs->n_seqs, p.share, p.bound, window, p.units, p.row_tiles, c.page_shift, seqs->table_stride,
        p.group, PagedMore{q_dev, q_stride, c.data, c.page_bytes, part_o, part_ml, out_dev, c.n_pages, scale_log2});
    ET_LAUNCH_CHECK();
    if (p.share) {
      // (64 / 256 lanes a head, us: 64 x 100 to 2048 tokens, 32 heads 61.6 / 64.9; 2 x 60000, 16 heads, 196 parts each 30.1 / 20.2)
      const bool few = !one && p.share <= 16 * (int64_t)seqs->n_seqs;
      const unsigned heads = (unsigned)(seqs->n_seqs * n_heads);
      (one ? paged_join_kernel<hd.value, fmt.value, 256, true> : few ? paged_join_kernel<hd.value, fmt.value, 64, false>
                                                                     : paged_join_kernel<hd.value, fmt.value, 256, false>)<<<
          heads, few ? 64 : 256, 0, stream>>>(seqs->kv_len_dev, part_o, part_ml, seqs->n_seqs, p.share, p.bound, window, n_heads, out_dev);
      ET_LAUNCH_CHECK();
    }
    return ET_OK;
  });
}

}  // extern "C"
