// Rotary positions: queries and keys turned by angles that grow with their position.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>

#include "mfma_common.h"

namespace et {

struct RotaryRows {
  const uint16_t *in;
  int64_t in_stride;
  uint16_t *out;
  int64_t out_stride;
};
struct RotaryArgs {
  RotaryRows q, k;
  const uint64_t *steps;
  int n_heads, heads;                                     // of q, of both
  int head_dim, pairs, units;                             // units: of 2 VEC values, of a head
  float amplitude, sign;
};

// Cosine and sine of 2 pi t / 2^32.  t's nearest quarter turn is taken off, which leaves at most an eighth, x in [-pi/4, pi/4], for the
// power series: what they leave out is below x^11 / 11! and x^10 / 10!, 2^-29 and 2^-25.
__device__ __forceinline__ void turn(uint32_t t, float &c, float &s) {
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(t - (quarter << 30)) * (float)(6.283185307179586 / 4294967296.0), y = x * x;
  const float sx = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float cx = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = quarter & 1 ? sx : cx, b = quarter & 1 ? cx : sx;
  c = (quarter + 1) & 2 ? -a : a;
  s = quarter & 2 ? -b : b;
}

// N bfloat16 values as they lie, L of them a load.  PAST: past the caches.
template <int L>
struct Bits;
template <> struct Bits<1> { using type = uint16_t; };
template <> struct Bits<2> { using type = uint32_t; };
template <> struct Bits<4> { using type = uint2; };
template <> struct Bits<8> { using type = u32x4; };
template <int L, bool PAST, int N>
__device__ __forceinline__ void load_bits(const uint16_t *p, uint16_t (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += L) {
    const auto *from = reinterpret_cast<const typename Bits<L>::type *>(p + i);
    typename Bits<L>::type b;
    if constexpr (PAST) b = __builtin_nontemporal_load(from);
    else b = *from;
    __builtin_memcpy(&v[i], &b, 2 * L);
  }
}
template <int L, bool PAST, int N>
__device__ __forceinline__ void store_bits(uint16_t *p, const uint16_t (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += L) {
    typename Bits<L>::type b;
    __builtin_memcpy(&b, &v[i], 2 * L);
    auto *to = reinterpret_cast<typename Bits<L>::type *>(p + i);
    if constexpr (PAST) __builtin_nontemporal_store(b, to);
    else *to = b;
  }
}

// (a, b) -> A (a cos - b sin, b cos + a sin) for every pair of a head's first 2 * pairs dimensions; the rest is copied where it goes to another
// place.  The angle of pair i at position p is kept as a fraction of a turn in 64 bits, p * steps[i] mod 2^64, so that a far
// position loses nothing; its upper half goes on.  A workgroup puts the cosines and sines of its rows into LDS, once for all heads; then its lanes
// take units of VEC pairs (half: two loads of VEC values, interleaved: one of twice as many), all heads of all its rows in turn.  Bound by
// memory: 64 987 rows of 32 heads of 128, 533 MB read and as many written in 168 us, 6.3 TB/s; few rows are one chain of position, angle, cosine
// and load, 3 us.  PAST: past the caches.
template <int VEC, int L, bool HALF, bool PAST>
__global__ __launch_bounds__(256) void rotary_kernel(const int32_t *positions, int rows, int per_block, RotaryArgs a) {
  extern __shared__ float lds_turn[];                     // cosines [per_block, pairs], sines
  const int first = blockIdx.x * per_block, count = min(per_block, rows - first), pairs = a.pairs;
  float *lds_cos = lds_turn, *lds_sin = lds_turn + per_block * pairs;
  for (int i = threadIdx.x; i < count * pairs; i += 256) {
    const int row = i / pairs;
    const uint64_t phase = (uint64_t)(int64_t)positions[first + row] * a.steps[i - row * pairs];
    float c, s;
    turn((uint32_t)(phase >> 32), c, s);
    lds_cos[i] = c * a.amplitude;
    lds_sin[i] = s * a.amplitude * a.sign;
  }
  __syncthreads();
  const int slots = 256 / a.units, u = threadIdx.x % a.units, slot = threadIdx.x / a.units;
  if (slot >= slots) return;
  const int turning = pairs / VEC;                        // units that are turned
  for (int i = slot; i < count * a.heads; i += slots) {
    const int row = i / a.heads, h = i - row * a.heads;
    const bool key = h >= a.n_heads;
    const int64_t at = first + (int64_t)row;
    const int from = (key ? h - a.n_heads : h) * a.head_dim;
    const uint16_t *in = (key ? a.k.in + at * a.k.in_stride : a.q.in + at * a.q.in_stride) + from;
    uint16_t *out = (key ? a.k.out + at * a.k.out_stride : a.q.out + at * a.q.out_stride) + from;
    // (units that are copied take the same loads and stores as those that are turned)
    const bool turns = u < turning;
    const float *c = lds_cos + row * pairs + VEC * (turns ? u : 0), *s = lds_sin + row * pairs + VEC * (turns ? u : 0);
    const auto pair = [&](uint16_t &x, uint16_t &y, int e) {
      const float fx = bf16_to_f32(x), fy = bf16_to_f32(y);
      const uint32_t two = cvt_pk_bf16(fmaf(fx, c[e], -(fy * s[e])), fmaf(fy, c[e], fx * s[e]));
      x = (uint16_t)two;
      y = (uint16_t)(two >> 16);
    };
    if constexpr (HALF) {
      const int at0 = turns ? VEC * u : pairs + VEC * u, at1 = turns ? pairs + VEC * u : a.head_dim / 2 + VEC * u;
      uint16_t x[VEC], y[VEC];
      load_bits<L, PAST>(in + at0, x);
      load_bits<L, PAST>(in + at1, y);
      if (turns) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) pair(x[e], y[e], e);
      }
      store_bits<L, PAST>(out + at0, x);
      store_bits<L, PAST>(out + at1, y);
    } else {
      uint16_t v[2 * VEC];
      load_bits<L, PAST>(in + 2 * VEC * u, v);
      if (turns) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) pair(v[2 * e], v[2 * e + 1], e);
      }
      store_bits<L, PAST>(out + 2 * VEC * u, v);
    }
  }
}

// Values that can be moved at a time: a power of two up to 8 that divides all of what is given (in values of two bytes).
static int widest(std::initializer_list<int64_t> all) {
  int w = 8;
  for (const int64_t x : all)
    while (x % w) w /= 2;
  return w;
}

static int check_rows(const et_rotary_rows *r, const char *name, int head_dim, int rows) {
  ET_REQUIRE(r->n_heads >= 0 && r->n_heads <= 65536, "%s has %d heads: 0 to 65536 are possible", name, r->n_heads);
  if (r->n_heads == 0 || rows == 0) return ET_OK;
  const int64_t width = (int64_t)r->n_heads * head_dim;
  ET_REQUIRE(r->in_dev && r->out_dev && (uintptr_t)r->in_dev % 2 == 0 && (uintptr_t)r->out_dev % 2 == 0, "a pointer of %s is NULL or not aligned",
             name);
  ET_REQUIRE(r->in_stride >= width && r->out_stride >= width, "row strides %lld and %lld of %s must be at least %lld", (long long)r->in_stride,
             (long long)r->out_stride, name, (long long)width);
  ET_REQUIRE(r->in_dev != r->out_dev || r->in_stride == r->out_stride || rows == 1, "%s in place has strides %lld and %lld", name,
             (long long)r->in_stride, (long long)r->out_stride);
  return ET_OK;
}

// Whether rows of `width` values at p (stride between rows) and at q have values in common.  Columns of one wider matrix have the same stride and
// keep apart within it; rows of different strides have to be apart as a whole.
struct Span {
  const uint16_t *p;
  int64_t stride, width;
};
static bool overlap(Span x, Span y, int rows) {
  if (x.p > y.p) std::swap(x, y);
  const int64_t off = ((uintptr_t)y.p - (uintptr_t)x.p + 1) / 2;
  if (off >= (__int128)(rows - 1) * x.stride + x.width) return false;
  if (rows == 1 || x.stride != y.stride) return true;
  const int64_t at = off % x.stride;
  return at < x.width || at + y.width > x.stride;
}

static constexpr int kMaxHead = 512;                      // (a unit of two values a lane: a head is at most one workgroup)
// A launch takes fewer than 2^32 lanes, 256 a workgroup of up to 8 rows.
static constexpr int kMaxBlocks = (1 << 24) - 1, kMaxRows = 8 * kMaxBlocks;

}  // namespace et

using namespace et;

extern "C" {

int et_rotary_steps(const et_rotary_scaling *sc, int32_t rot_dim, double base, uint64_t *steps, float *amplitude) {
  ET_REQUIRE(steps != nullptr && amplitude != nullptr, "steps or amplitude is NULL");
  ET_REQUIRE(rot_dim >= 2 && rot_dim <= kMaxHead && rot_dim % 2 == 0, "rot_dim = %d must be even and in [2, %d]", rot_dim, kMaxHead);
  ET_REQUIRE(base >= 1.0 && base <= 1e30, "base = %g must be in [1, 1e30]", base);
  const int kind = sc ? sc->kind : ET_ROTARY_PLAIN;
  ET_REQUIRE(kind >= ET_ROTARY_PLAIN && kind <= ET_ROTARY_TURNS, "unknown scaling %d", kind);
  const double factor = kind == ET_ROTARY_PLAIN ? 1.0 : sc->factor;
  ET_REQUIRE(factor >= 1.0 && factor <= 1e9, "factor = %g must be in [1, 1e9]", factor);
  // (A step counts 2^-64 of a turn, and a far position multiplies its error by 2^31: with the host's 64-bit significands it is within two units, with
  // double's 53 up to some hundreds.)
  const long double two_pi = 6.283185307179586476925286766559L;
  const int n = rot_dim;
  if (kind == ET_ROTARY_YARN || kind == ET_ROTARY_TURNS) {
    ET_REQUIRE(sc->original_len >= 1 && sc->original_len <= 1e15, "original_len = %g must be in [1, 1e15]", sc->original_len);
    ET_REQUIRE(sc->slow > 0 && sc->fast > sc->slow && sc->fast <= 1e9, "slow = %g and fast = %g must be 0 < slow < fast <= 1e9", sc->slow, sc->fast);
    ET_REQUIRE(kind != ET_ROTARY_YARN || base > 1.0, "base = %g must be above 1 here", base);
  }
  double first = 0, last = 0;
  long double stretched = base;
  if (kind == ET_ROTARY_NTK && n > 2) stretched *= std::pow((long double)factor, n / (n - 2.0L));
  if (kind == ET_ROTARY_YARN) {
    const auto index = [&](double turns) { return n * std::log(sc->original_len / ((double)two_pi * turns)) / (2.0 * std::log(base)); };
    first = std::max(std::floor(index(sc->fast)), 0.0);
    last = std::min(std::ceil(index(sc->slow)), n - 1.0);
  }
  for (int i = 0; i < n / 2; ++i) {
    long double f = std::pow(stretched, -2.0L * i / n);
    long double share = kind == ET_ROTARY_LINEAR || (kind == ET_ROTARY_NTK && n == 2) ? 1.0L : 0.0L;    // of the frequency that is stretched
    if (kind == ET_ROTARY_YARN) share = std::min(std::max((i - first) / std::max((long double)last - first, 0.001L), 0.0L), 1.0L);
    if (kind == ET_ROTARY_TURNS)
      share = 1.0L - std::min(std::max((sc->original_len * f / two_pi - sc->slow) / ((long double)sc->fast - sc->slow), 0.0L), 1.0L);
    f = f / factor * share + f * (1.0L - share);
    steps[i] = (uint64_t)std::nearbyint(f / two_pi * 18446744073709551616.0L);         // (f is at most 1: a sixth of a turn)
  }
  *amplitude = kind == ET_ROTARY_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return ET_OK;
}

int et_rotary_apply(const et_rotary *rotary, const int32_t *positions_dev, int32_t rows, const et_rotary_rows *q, const et_rotary_rows *k,
                    int32_t transpose, void *hip_stream) {
  ET_REQUIRE(rotary != nullptr && q != nullptr, "rotary or q is NULL");
  const et_rotary &r = *rotary;
  ET_REQUIRE(r.head_dim >= 2 && r.head_dim <= kMaxHead && r.head_dim % 2 == 0, "head_dim = %d must be even and in [2, %d]", r.head_dim, kMaxHead);
  ET_REQUIRE(r.rot_dim >= 2 && r.rot_dim <= r.head_dim && r.rot_dim % 2 == 0, "rot_dim = %d must be even and in [2, head_dim = %d]", r.rot_dim,
             r.head_dim);
  ET_REQUIRE(r.layout == ET_ROTARY_HALF || r.layout == ET_ROTARY_INTERLEAVED, "unknown layout %d", r.layout);
  ET_REQUIRE(r.amplitude - r.amplitude == 0.f, "amplitude must be finite");
  ET_REQUIRE(transpose == 0 || transpose == 1, "transpose = %d must be 0 or 1", transpose);
  ET_REQUIRE(rows >= 0 && rows <= kMaxRows, "rows = %d must be in [0, 2^27 - 8]", rows);
  int rc;
  et_rotary_rows none{};
  const et_rotary_rows &kr = k ? *k : none;
  if ((rc = check_rows(q, "q", r.head_dim, rows)) || (rc = check_rows(&kr, "k", r.head_dim, rows))) return rc;
  const int heads = q->n_heads + kr.n_heads;
  if (rows == 0 || heads == 0) return ET_OK;
  // What is written may be read as the same tensor's values only, and is written once.
  const Span spans[2][2] = {{{q->in_dev, q->in_stride, (int64_t)q->n_heads * r.head_dim}, {q->out_dev, q->out_stride, (int64_t)q->n_heads * r.head_dim}},
                            {{kr.in_dev, kr.in_stride, (int64_t)kr.n_heads * r.head_dim}, {kr.out_dev, kr.out_stride, (int64_t)kr.n_heads * r.head_dim}}};
  for (int i = 0; i < 2; ++i) {
    const Span &in = spans[i][0], &out = spans[i][1], &other = spans[1 - i][1];
    if (in.width == 0) continue;
    ET_REQUIRE(in.p == out.p || !overlap(in, out, rows), "%s has its result in part where it lies itself", i ? "k" : "q");
    ET_REQUIRE(other.width == 0 || (!overlap(in, other, rows) && !overlap(out, other, rows)), "the result of %s lies on %s", i ? "q" : "k", i ? "k" : "q");
  }
  ET_REQUIRE(positions_dev != nullptr && r.steps_dev != nullptr && (uintptr_t)r.steps_dev % 8 == 0,
             "positions_dev or steps_dev is NULL or steps_dev is not aligned to 8 bytes");
  const int pairs = r.rot_dim / 2;
  const bool half = r.layout == ET_ROTARY_HALF;
  // values a load: whole units of pairs (half: of either side), whole heads, and everything aligned to it
  int load = half ? widest({pairs, (r.head_dim - r.rot_dim) / 2, r.head_dim}) : widest({r.rot_dim, r.head_dim});
  for (const et_rotary_rows *x : {q, &kr})
    if (x->n_heads)
      load = std::min(load, widest({rows > 1 ? x->in_stride : 0, rows > 1 ? x->out_stride : 0, (int64_t)((uintptr_t)x->in_dev / 2),
                                    (int64_t)((uintptr_t)x->out_dev / 2)}));
  const int vec = half ? load : std::max(1, load / 2);
  const bool in_place = (q->n_heads == 0 || q->in_dev == q->out_dev) && (kr.n_heads == 0 || kr.in_dev == kr.out_dev);
  RotaryArgs a{{q->in_dev, q->in_stride, q->out_dev, q->out_stride}, {kr.in_dev, kr.in_stride, kr.out_dev, kr.out_stride}, r.steps_dev, q->n_heads,
               heads, r.head_dim, pairs, (in_place ? r.rot_dim : r.head_dim) / (2 * vec), r.amplitude, transpose ? -1.f : 1.f};
  // Rows of a workgroup: as many as give its lanes fewer than two units each, at most 8, and 512 workgroups at least.  Wide rows gain nothing by
  // sharing one: us at one / 2 / 4 / 8 rows of 32 heads of 128 (256 units), 65 536 rows 191 / 193 / 197 / 205, 300 rows 3.1 / 3.3 / 4.0 / 5.8; of 40
  // interleaved heads of 80 (400 units) 168 / 174 / 194 / 218; but of 5 heads of 64 (20 units) 46.8 / 26.0 / 19.4 / 14.9.  With fewer than
  // one unit a lane instead: 65 536 rows of 4 heads of 80 in units of 4 (80 units) 21.3 -> 27.1, of 16 heads of 64 39.4 -> 41.0.
  const int least = (rows + kMaxBlocks - 1) / kMaxBlocks;
  const int per_block = std::max({1, least, std::min({8, rows / 512, 511 / (heads * a.units)})});
  const unsigned blocks = (unsigned)((rows + per_block - 1) / per_block);
  const size_t lds = (size_t)per_block * pairs * 2 * sizeof(float);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  auto launch = [&](auto kernel) {
    kernel<<<blocks, 256, lds, stream>>>(positions_dev, rows, per_block, a);
    ET_LAUNCH_CHECK();
    return ET_OK;
  };
  // Past the caches where what is read and written exceeds the memory side's (256 MB) anyway, and every store writes whole lines of 128 bytes: runs of
  // dimensions that lie together are half of rot_dim and of a head's rest (half), the whole row, or, in place, rot_dim (interleaved).  us cached / past:
  // 64 987 rows of 32 heads of 128 191 / 168, 40 interleaved ones of 80, 32 dimensions turned, 147 / 139; 16 000 rows of 32 (131 MB each way)
  // 46.4 / 43.2, again and again on the same rows 41.2 / 42.6; 4000 rows 12.1 / 13.3; 64 987 of 10 of 128, 64 turned (runs of 64 bytes), 64.6 / 69.8.
  const int run = half ? pairs | r.head_dim | (in_place ? 0 : (r.head_dim - r.rot_dim) / 2) : in_place && r.rot_dim < r.head_dim ? r.rot_dim | r.head_dim : 0;
  bool past = run % 64 == 0 && (int64_t)rows * heads * a.units * vec * 4 >= 128 << 20;
  for (const et_rotary_rows *x : {q, &kr})
    past = past && (x->n_heads == 0 || ((uintptr_t)x->out_dev % 128 == 0 && x->out_stride % 64 == 0 && (int64_t)x->n_heads * r.head_dim % 64 == 0));
  switch (load) {
    case 8:
      if (past) return launch(half ? rotary_kernel<8, 8, true, true> : rotary_kernel<4, 8, false, true>);
      return launch(half ? rotary_kernel<8, 8, true, false> : rotary_kernel<4, 8, false, false>);
    case 4: return launch(half ? rotary_kernel<4, 4, true, false> : rotary_kernel<2, 4, false, false>);
    case 2: return launch(half ? rotary_kernel<2, 2, true, false> : rotary_kernel<1, 2, false, false>);
    default: return launch(half ? rotary_kernel<1, 1, true, false> : rotary_kernel<1, 1, false, false>);
  }
}

}  // extern "C"
