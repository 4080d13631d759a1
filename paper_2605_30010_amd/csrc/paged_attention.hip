// Attention of one new token per sequence over a paged key-value cache.
#include <type_traits>

#include "kv_cache.h"
#include "mfma_common.h"

namespace et {

constexpr int kTile = 32;                                // tokens that a wavefront takes at a time
constexpr int kMostSplits = 1024;                        // parts of a sequence

// a * b rounded, never part of a fused multiply-add: a logit less the maximum has to be 0 for the maximum itself, however large.
__device__ __forceinline__ float whole_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// How a call is split.  Each sequence's tokens are shared out over up to `splits` workgroups, at least a tile per wavefront each.
struct PagedSplit {
  int splits, row_tiles;                                 // row_tiles: groups of 16 query heads of one key-value head
};
struct SeqRange {
  int lo, hi, first;                                     // tokens [first, hi) count; lo = first rounded down to 16
  int chunk, parts;
};
__device__ __forceinline__ SeqRange seq_range(int len, int bound, int window, int splits) {
  constexpr int kStep = 4 * kTile;
  SeqRange r;
  r.hi = min(len, bound);
  r.first = window > 0 && len > window ? len - window : 0;
  r.lo = r.first & ~15;
  const int span = max(r.hi - r.lo, 0);
  r.chunk = max((span + splits - 1) / splits, 1);
  r.chunk = (r.chunk + kStep - 1) / kStep * kStep;
  r.parts = (span + r.chunk - 1) / r.chunk;
  return r;
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
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const bf16x2_t v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, SEL != 0);
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
  static __device__ __forceinline__ uint32_t lane_off(int r, int g) { return r * kRow + g * 16; }
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

// A workgroup takes one part of a sequence's tokens for up to 16 query heads of one key-value head; its wavefronts take tiles of
// 32 tokens in turn.  The cache's bytes go to registers in MFMA operand order, no LDS on the way.
// The kernel is bound by reading the cache, once.
template <int HD, int FMT, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void paged_attention_kernel(KvPages c, KvSeqs s, const uint16_t *q, int64_t q_stride,
                                                                      int group, int bound, int window, float scale_log2,
                                                                      PagedSplit split, float *part_o, float2 *part_ml,
                                                                      uint16_t *out) {
  using Lay = KvLayout<HD, FMT>;
  using K = Keys<HD, FMT>;
  using V = Values<HD, FMT>;
  constexpr int ACC = V::BLOCKS * V::DPL;
  constexpr int BD = HD / V::BLOCKS;                      // dimensions that the wavefronts add up at a time
  __shared__ float lds_o[kWaves][BD][16];
  __shared__ float2 lds_ml[kWaves][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int part = blockIdx.x % split.splits, unit = blockIdx.x / split.splits;
  const int rt = unit % split.row_tiles, kv = unit / split.row_tiles % c.kv_heads, b = unit / (split.row_tiles * c.kv_heads);
  const int n_heads = group * c.kv_heads, ps = 1 << c.page_shift;
  const int live = min(16, group - rt * 16);              // query heads of this workgroup
  const SeqRange sr = seq_range(s.len[b], bound, window, split.splits);
  if (part >= max(sr.parts, 1)) return;
  const int start = sr.lo + part * sr.chunk, end = min(sr.hi, start + sr.chunk);
  const int tiles = end > start ? (end - start + kTile - 1) / kTile : 0;

  u32x4 qf[K::STEPS];
#pragma unroll
  for (int st = 0; st < K::STEPS; ++st) {
    const int d = K::dim(st, g);
    qf[st] = u32x4{0, 0, 0, 0};
    if (r < live && d < HD)
      qf[st] = *reinterpret_cast<const u32x4 *>(q + b * q_stride + ((int64_t)kv * group + rt * 16 + r) * HD + d);
  }
  f32x4 acc[ACC];
#pragma unroll
  for (int j = 0; j < ACC; ++j) acc[j] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, sum = 0.f;                         // of query head r; sum: this lane's tokens only

  const int32_t *row = s.table + (int64_t)b * s.table_stride;
  int page_of = -1;                                       // lane i: page of the wavefront's i-th group of 16 tokens, of 64
  for (int t = wave, i = 0; t < tiles; t += kWaves, i = (i + 2) & 63) {
    if (i == 0) {
      const int pos = start + (t + (lane >> 1) * kWaves) * kTile + (lane & 1) * 16;
      page_of = pos < end ? row[pos >> c.page_shift] : -1;
      if (page_of >= c.n_pages) page_of = -1;
    }
    const int pos0 = start + t * kTile;
    uint32_t kw[2][K::NREG], vw[V::BLOCKS][8][V::NREG];
    uint2 km[2], vm[2];
    int page[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      page[u] = __builtin_amdgcn_readlane(page_of, i + u);
      const int at = (pos0 + 16 * u) & (ps - 1);
      const char *head = c.data + max(page[u], 0) * c.page_bytes + (int64_t)kv * Lay::head_bytes(ps);
      K::load(head + at * Lay::kRow, r, g, kw[u]);
      const char *values = head + Lay::values(ps) + at * Lay::kRow;
#pragma unroll
      for (int blk = 0; blk < V::BLOCKS; ++blk)
#pragma unroll
        for (int e = 0; e < 4; ++e) V::load(values, 4 * g + e, r, blk, vw[blk][4 * u + e]);
      if constexpr (FMT != ET_KV_BF16) {
        km[u] = *reinterpret_cast<const uint2 *>(head + Lay::key_max(ps) + (at + 4 * g) * 2);
        vm[u] = *reinterpret_cast<const uint2 *>(head + Lay::value_max(ps) + (at + 4 * g) * 2);
      }
    }
    float z[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 d{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < K::STEPS; ++st) d = mfma16(K::operand(kw[u], st, g), qf[st], d);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float f = scale_log2;
        if constexpr (FMT != ET_KV_BF16) f *= e & 1 ? bf16hi_to_f32(e & 2 ? km[u].y : km[u].x) : bf16lo_to_f32(e & 2 ? km[u].y : km[u].x);
        z[4 * u + e] = whole_product(d[e], f);
      }
    }
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
#pragma unroll
          for (int blk = 0; blk < V::BLOCKS; ++blk)
#pragma unroll
            for (int x = 0; x < V::NREG; ++x) vw[blk][e][x] = 0;           // (0 times what lies there could be NaN)
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
    const u32x4 pf{cvt_pk_bf16(p[0], p[1]), cvt_pk_bf16(p[2], p[3]), cvt_pk_bf16(p[4], p[5]), cvt_pk_bf16(p[6], p[7])};
#pragma unroll
    for (int blk = 0; blk < V::BLOCKS; ++blk)
#pragma unroll
      for (int j = 0; j < V::DPL; ++j) acc[blk * V::DPL + j] = mfma16(V::operand(vw[blk], j), pf, acc[blk * V::DPL + j]);
  }

  // the wavefronts' results together
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (g == 0) lds_ml[wave][r] = make_float2(m, sum);
  const int h = threadIdx.x & 15;
  const int64_t head = (int64_t)b * n_heads + (int64_t)kv * group + rt * 16 + h;
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
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) o[e] = fmaf(f[w], lds_o[w][d + e][h], o[e]);
      }
      if (split.splits == 1) {
        const float inv = total == 0.f ? 0.f : value_factor<FMT>() / total;
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = cvt_pk_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
        *reinterpret_cast<u32x4 *>(out + head * HD + blk * BD + d) = v;
      } else {
        float *to = part_o + (head * split.splits + part) * HD + blk * BD + d;
        *reinterpret_cast<f32x4 *>(to) = f32x4{o[0], o[1], o[2], o[3]};
        *reinterpret_cast<f32x4 *>(to + 4) = f32x4{o[4], o[5], o[6], o[7]};
      }
    }
  }
  if (split.splits > 1 && threadIdx.x < live) part_ml[head * split.splits + part] = make_float2(top, total);
}

// Joins the parts of one query head, always in the same order: groups of lanes, four dimensions a lane, take every GROUPS-th part,
// and their sums are added up in the groups' order.  Every load is issued before the first is needed: parts that the
// sequence does not have are read (they lie in the workspace) and left out.
template <int HD, int FMT>
__global__ __launch_bounds__(256) void paged_join_kernel(const float *part_o, const float2 *part_ml, const int32_t *len, int n_heads,
                                                         int splits, int bound, int window, uint16_t *out) {
  constexpr int LANES = HD / 4, GROUPS = 256 / LANES, BATCH = 8;
  __shared__ float lds_f[kMostSplits], lds_o[GROUPS][HD], lds_top[4], lds_sum[4];
  const int64_t head = blockIdx.x;
  const int tid = threadIdx.x, lane = tid % LANES, grp = tid / LANES;
  const f32x4 *o = reinterpret_cast<const f32x4 *>(part_o + head * splits * HD) + lane;
  f32x4 v[BATCH];
  if (grp < GROUPS)
#pragma unroll
    for (int i = 0; i < BATCH; ++i) v[i] = o[(int64_t)min(grp + i * GROUPS, splits - 1) * (HD / 4)];
  float2 ml[kMostSplits / 256];
#pragma unroll
  for (int i = 0; i < kMostSplits / 256; ++i) ml[i] = part_ml[head * splits + min(tid + 256 * i, splits - 1)];
  const int parts = max(seq_range(len[head / n_heads], bound, window, splits).parts, 1);
  float top = -INFINITY, total = 0.f;
#pragma unroll
  for (int i = 0; i < kMostSplits / 256; ++i)
    if (tid + 256 * i < parts) top = fmaxf(top, ml[i].x);
  top = wave_max(top);
  if (tid % 64 == 0) lds_top[tid / 64] = top;
  __syncthreads();
  top = fmaxf(fmaxf(lds_top[0], lds_top[1]), fmaxf(lds_top[2], lds_top[3]));
#pragma unroll
  for (int i = 0; i < kMostSplits / 256; ++i)
    if (tid + 256 * i < parts) {
      const float f = part_factor(ml[i], top);
      lds_f[tid + 256 * i] = f;
      total += f * ml[i].y;
    }
  total = wave_sum(total);
  if (tid % 64 == 0) lds_sum[tid / 64] = total;
  __syncthreads();
  total = (lds_sum[0] + lds_sum[1]) + (lds_sum[2] + lds_sum[3]);
  if (grp < GROUPS) {
    f32x4 x{0, 0, 0, 0};
    for (int first = grp;;) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int at = first + i * GROUPS;
        if (at < parts) {
          const float f = lds_f[at];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = fmaf(f, v[i][e], x[e]);
        }
      }
      first += BATCH * GROUPS;
      if (first >= parts) break;
#pragma unroll
      for (int i = 0; i < BATCH; ++i) v[i] = o[(int64_t)min(first + i * GROUPS, splits - 1) * (HD / 4)];
    }
    *reinterpret_cast<f32x4 *>(&lds_o[grp][lane * 4]) = x;
  }
  __syncthreads();
  const float inv = total == 0.f ? 0.f : value_factor<FMT>() / total;
  if (tid < HD) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) x += lds_o[i][tid];
    out[head * HD + tid] = f32_to_bf16_bits(x * inv);
  }
}

// Splits so that about 1024 workgroups share the work, if each gets a tile per wavefront.
static PagedSplit paged_split(int n_seqs, int kv_heads, int group, int64_t span) {
  PagedSplit p;
  p.row_tiles = (group + 15) / 16;
  const int64_t units = (int64_t)n_seqs * kv_heads * p.row_tiles;
  #ifndef TARGET
#define TARGET 1024
#endif
#ifndef WV
#define WV 4
#endif
  const int64_t most = (span + 4 * kTile - 1) / (4 * kTile), want = (TARGET + units - 1) / units;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kMostSplits, std::min(most, want)));
  return p;
}

static int64_t paged_span(const et_kv_cache &c, const et_kv_seqs &s, int max_len, int window) {
  const int64_t bound = std::min<int64_t>(max_len, (int64_t)s.pages_per_seq * c.page_size);
  return window > 0 ? std::min<int64_t>(bound, (int64_t)window + 15) : bound;
}

static size_t paged_workspace(int64_t rows, int head_dim, int splits) {
  return splits == 1 ? 0 : (size_t)rows * splits * (head_dim * sizeof(float) + sizeof(float2));
}

static int check_paged(const et_kv_cache *cache, const et_kv_seqs *seqs, int n_heads, int max_len, int window) {
  int rc;
  if ((rc = check_kv(cache, seqs))) return rc;
  ET_REQUIRE(n_heads >= 1 && n_heads % cache->n_kv_heads == 0 && n_heads <= 65536,
             "n_heads = %d must be a multiple of n_kv_heads = %d, at most 65536", n_heads, cache->n_kv_heads);
  ET_REQUIRE(max_len >= 1, "max_len = %d must be at least 1", max_len);
  ET_REQUIRE(window >= 0, "window = %d is negative", window);
  ET_REQUIRE((int64_t)seqs->n_seqs * n_heads <= INT32_MAX / 1024, "n_seqs * n_heads = %lld is above %d", (long long)seqs->n_seqs * n_heads,
             INT32_MAX / 1024);
  return ET_OK;
}

}  // namespace et

using namespace et;

extern "C" {

size_t et_attention_paged_workspace_bytes(const et_kv_cache *cache, const et_kv_seqs *seqs, int32_t n_heads, int32_t max_len,
                                          int32_t window) {
  if (check_paged(cache, seqs, n_heads, max_len, window) || seqs->n_seqs == 0) return 0;
  const PagedSplit p = paged_split(seqs->n_seqs, cache->n_kv_heads, n_heads / cache->n_kv_heads, paged_span(*cache, *seqs, max_len, window));
  return paged_workspace((int64_t)seqs->n_seqs * n_heads, cache->head_dim, p.splits);
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
  const int group = n_heads / cache->n_kv_heads, bound = (int)std::min<int64_t>(max_len, (int64_t)seqs->pages_per_seq * cache->page_size);
  const PagedSplit p = paged_split(seqs->n_seqs, cache->n_kv_heads, group, paged_span(*cache, *seqs, max_len, window));
  const int64_t rows = (int64_t)seqs->n_seqs * n_heads;
  const size_t need = paged_workspace(rows, cache->head_dim, p.splits);
  if (need) {
    ET_REQUIRE(workspace_dev != nullptr && (uintptr_t)workspace_dev % 16 == 0, "workspace_dev is NULL or not aligned to 16 bytes");
    if (workspace_bytes < need) {
      set_error("workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
      return ET_ERR_WORKSPACE;
    }
  }
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  float *part_o = static_cast<float *>(workspace_dev);
  float2 *part_ml = reinterpret_cast<float2 *>(part_o + (need ? rows * p.splits * cache->head_dim : 0));
  const float scale_log2 = scale * 1.4426950408889634f * (cache->format == ET_KV_BF16 ? 1.f : cache->format == ET_KV_INT8 ? 1.f / 127.f : 1.f / 448.f);
  const int64_t grid = (int64_t)seqs->n_seqs * cache->n_kv_heads * p.row_tiles * p.splits;
  return kv_dispatch(cache->head_dim, cache->format, [&](auto hd, auto fmt) {
    paged_attention_kernel<hd.value, fmt.value, WV><<<(unsigned)grid, 64 * WV, 0, stream>>>(
        kv_pages(*cache), kv_seqs(*seqs), q_dev, q_stride, group, bound, window, scale_log2, p, part_o, part_ml, out_dev);
    ET_LAUNCH_CHECK();
    if (p.splits > 1) {
      paged_join_kernel<hd.value, fmt.value><<<(unsigned)rows, 256, 0, stream>>>(part_o, part_ml, seqs->kv_len_dev, n_heads, p.splits, bound,
                                                                                 window, out_dev);
      ET_LAUNCH_CHECK();
    }
    return ET_OK;
  });
}

}  // extern "C"
