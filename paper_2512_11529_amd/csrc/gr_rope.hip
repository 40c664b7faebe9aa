// gr_qk_norm_rope, gr_page_append: what stands between a projection and attention.
//
// A head x of d elements is normed, y = x w / sqrt(mean(x^2) + eps), and its first `rot` elements are turned in pairs by the angles of the row's position,
//     y_a' = y_a cos - y_b sin,   y_b' = y_b cos + y_a sin,
// with (a, b) = (i, i + rot / 2) or (2 i, 2 i + 1) for i < rot / 2.  All of it is in fp32; the only rounding to fewer bits is the store's.
// A code of FP4 is a whole step away from its neighbours, so that next to a border the last bit of an fp32 value decides between values that are far apart.  So every operation is rounded by
// itself (this file is compiled without contraction), in the order in which the formulas read: the squares' sum by neighbours (fours in a chain, of heads up to 64 in pairs, then pairs of
// sums: any order will do, and this is how a mean over the last axis in plain torch operations adds heads of 64 and 128), times 1 / d, plus eps, its reciprocal root rounded to nearest, x times
// that, times w; two products, then their difference or sum.  A plain evaluation in fp32, operation by operation, has the same bits.  (With r w first, another order of sums and fused
// rotations 14 to 22 of the 134 million codes of 32 x 4096 keys of 8 x 128 were others than that evaluation's.)
//
// Bound: memory, 4 bytes an element in and out (bf16).  A lane holds 16 elements of a head in two runs of eight, so that both of every pair are its own: elements 8 j .. and
// rot / 2 + 8 j .., or 16 j .. .  4, 8 or 16 lanes hold the head, and a wavefront the same head of 16, 8 or 4 consecutive rows: what it writes into an FP4 page is then one
// run of codes and one of scales, and a lane's cosines and sines serve all of its heads.  The wavefronts of a workgroup take different heads of the same rows.
// With 16 consecutive elements a lane and the other halves of its pairs loaded a second time, 32 x 256 rows of 32 + 8 + 8 heads of 128, normed, took 69.6 us, now 41.4 (4.9 TB/s; a copy of
// 1 GiB reaches 5.15), 32 x 4096 tokens of 8 heads into FP4 361 us, now 147 (4.7; bf16 216, 5.0, FP8 163, 5.0; heads of 64 4.4-4.8).  The launch is all there is of 16 rows of 8 + 8 + 8
// heads of 64: 2.8 us.  16 prompts of 60-700 tokens of 8 heads into FP8 take 10.1 us, 7.5 without norm and rotation: all wavefronts are resident at once, and each waits for one chain of loads,
// position, angles, and the rows and weights behind them, those that hold only heads of V too, which need no angles.
#include <initializer_list>
#include <type_traits>
#include "gr_pages.hpp"

namespace {

__device__ __forceinline__ unsigned div_by(unsigned n, unsigned d, uint32_t inv) {      // inv = (2^32 - 1) / d, rounded down: the product's high word is n / d or one less
  const unsigned q = __umulhi(n, inv);
  return q + (n - q * d >= d ? 1u : 0u);
}

// Of a neighbouring lane
template <int CTRL>
__device__ __forceinline__ float lanes_of(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}
// Sum of a head's squares; a and b: those of a lane's two runs of eight.  Whatever the lane layout, neighbouring eights meet first, then neighbouring pairs of them, and so on: where the first
// `split` lanes hold runs that lie apart, the sums of the two are kept apart until one run of all of them is whole (rot / 16 a power of two; for other numbers of lanes the order is another).
template <int LG, bool PAIRS>
__device__ __forceinline__ float head_sum(float a, float b, int split, bool apart) {
  a += PAIRS || !apart ? b : 0.f;
  b = PAIRS || !apart ? 0.f : b;
  auto meet = [&](int lanes, auto of) __attribute__((always_inline)) {
    if (!PAIRS && split == lanes) { a += b; b = 0.f; }
    a += of(a);
    if (!PAIRS) b += of(b);
  };
  meet(1, [](float v) { return lanes_of<0xb1>(v); });                   // lane ^ 1
  meet(2, [](float v) { return lanes_of<0x4e>(v); });                   // lane ^ 2
  if (LG >= 8) meet(4, [](float v) { return lanes_of<0x141>(v); });     // the other four of eight (in reverse, but they are alike)
  if (LG >= 16) meet(8, [](float v) { return lanes_of<0x140>(v); });
  return PAIRS ? a : a + b;
}

// 1 / sqrt(x) rounded to nearest (for all 2^25 significands and parities of the exponent): the instruction's, a unit of fp32 off at most, and two terms of the root's series around it in
// 64 bits.  Of 0, infinities and NaN the instruction's.
__device__ __forceinline__ float reciprocal_root(float x) {
  const float r = __builtin_amdgcn_rsqf(x);
  const double e = __builtin_fma(-((double)x * (double)r), (double)r, 1.0);          // (the first product is exact)
  const float y = (float)__builtin_fma((double)r * e, __builtin_fma(0.375, e, 0.5), (double)r);
  return __builtin_fabs(e) < 1.0 ? y : r;
}

struct TurnCtx {
  uint32_t T, chunks, inv_chunks;      // rows; workgroups of a row's heads
  int d, rot, n_pos;
  float inv_d, eps;
  const float* table;                  // [n_pos, rot]
  const int32_t* pos;
};

// A wavefront's rows and a lane's part of them.
template <int LG, bool PAIRS>
struct Place {
  uint32_t row, chunk;                 // (rows past the last one as that one)
  int at, e[2];                        // position; first of the lane's elements, of each eight
  bool live, holds, turns;             // the row is written; the head has these elements; they are rotated
  __device__ __forceinline__ Place(const TurnCtx& c) {
    const uint32_t group = div_by(blockIdx.x, c.chunks, c.inv_chunks);
    const int lane = (int)threadIdx.x & 63, j = lane % LG;
    chunk = blockIdx.x - group * c.chunks;
    row = group * (64 / LG) + (uint32_t)(lane / LG);
    live = row < c.T;
    row = min(row, c.T - 1);
    holds = 16 * j < c.d;
    turns = 16 * j < c.rot;
    const bool split = !PAIRS && turns;
    e[0] = holds ? (split ? 8 : 16) * j : 0;                                    // (lanes past the head load what the first does)
    e[1] = split ? (c.rot >> 1) + e[0] : e[0] + 8;
    at = 0;
    if (c.rot > 0) {
      at = c.pos[row];
      if ((unsigned)at >= (unsigned)c.n_pos) { live = false; at = 0; }
    }
  }
};

__device__ __forceinline__ void load8(const float* p, float* to) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  to[0] = a.x; to[1] = a.y; to[2] = a.z; to[3] = a.w; to[4] = b.x; to[5] = b.y; to[6] = b.z; to[7] = b.w;
}

// Cosines and sines of a lane's eight pairs.
struct Angles {
  float cs[8], sn[8];
  template <class P>
  __device__ __forceinline__ Angles(const TurnCtx& c, const P& p, bool pairs) {
    if (!p.turns) return;
    const float* t = c.table + (size_t)(unsigned)p.at * (unsigned)c.rot + (pairs ? p.e[0] >> 1 : p.e[0]);
    load8(t, cs);
    load8(t + (c.rot >> 1), sn);
  }
};

struct Head {
  kv_u32x4 x[2];
  template <class P>
  __device__ __forceinline__ void load(const uint16_t* head, const P& p) {
    x[0] = *(const kv_u32x4*)(head + p.e[0]);
    x[1] = *(const kv_u32x4*)(head + p.e[1]);
  }
  __device__ __forceinline__ void numbers(float (&y)[16]) const {
#pragma unroll
    for (int e = 0; e < 16; e++) y[e] = bf16_at(x[e / 8][e % 8 / 2], e & 1);
  }
};

// A norm's weights for the lane's elements; a wavefront's next head mostly has the same.
struct Weights {
  const float* from = nullptr;
  float w[16];
  template <class P>
  __device__ __forceinline__ void of(const float* weight, const P& p) {
    if (weight == from || !weight) return;
    from = weight;
    load8(weight + p.e[0], w);
    load8(weight + p.e[1], w + 8);
  }
};

// The lane's 16 elements, normed where there is a weight (of the head's elements) and turned.
template <int LG, bool PAIRS>
__device__ __forceinline__ void turned(float (&y)[16], const Head& h, const Angles& a, const float* weight, Weights& ws, const TurnCtx& c, const Place<LG, PAIRS>& p) {
  h.numbers(y);
  ws.of(weight, p);
  if (weight) {
    auto eight = [&](const float* v) __attribute__((always_inline)) {        // (squares of bf16 values are exact in fp32: nothing is lost or won by adding them in one instruction)
      auto four = [](const float* v) __attribute__((always_inline)) {
        return LG == 4 ? fmaf(v[1], v[1], v[0] * v[0]) + fmaf(v[3], v[3], v[2] * v[2]) : fmaf(v[3], v[3], fmaf(v[2], v[2], fmaf(v[1], v[1], v[0] * v[0])));
      };
      return four(v) + four(v + 4);
    };
    const float sum = head_sum<LG, PAIRS>(p.holds ? eight(y) : 0.f, p.holds ? eight(y + 8) : 0.f, c.rot >> 4, p.turns && c.rot > 16);
    const float r = reciprocal_root(sum * c.inv_d + c.eps);
#pragma unroll
    for (int e = 0; e < 16; e++) y[e] = y[e] * r * ws.w[e];
  }
  if (p.turns) {
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const int i = PAIRS ? 2 * k : k, j = PAIRS ? 2 * k + 1 : k + 8;
      const float u = y[i], v = y[j];
      y[i] = u * a.cs[k] - v * a.sn[k];
      y[j] = v * a.cs[k] + u * a.sn[k];
    }
  }
}

template <class P>
__device__ __forceinline__ void store16(uint16_t* head, const P& p, const float (&y)[16]) {
#pragma unroll
  for (int r = 0; r < 2; r++) {
    const kv_u32x4 w = {bf16_pair(y[8 * r], y[8 * r + 1]), bf16_pair(y[8 * r + 2], y[8 * r + 3]), bf16_pair(y[8 * r + 4], y[8 * r + 5]), bf16_pair(y[8 * r + 6], y[8 * r + 7])};
    *(kv_u32x4*)(head + p.e[r]) = w;
  }
}

// ------------------------------------------------------------------------------------------------ queries and keys
struct NormRopeCtx {
  TurnCtx t;
  int Hq, Hkv, heads;                  // heads: of q, k and v together
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride, v_out_stride;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const float* q_weight;
  const float* k_weight;
  uint16_t* q_out;
  uint16_t* k_out;
  uint16_t* v_out;
};

// U: heads of a wavefront.  In place: a lane reads and writes the same elements.
template <int LG, bool PAIRS, int U>
__global__ void __launch_bounds__(256) k_qk_norm_rope(NormRopeCtx c) {
  const Place<LG, PAIRS> at(c.t);
  const int h0 = ((int)at.chunk * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)) * U;
  Head x[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int h = min(h0 + u, c.heads - 1);
    x[u].load(h < c.Hq              ? c.q + (int64_t)at.row * c.q_stride + h * c.t.d
              : h < c.Hq + c.Hkv    ? c.k + (int64_t)at.row * c.k_stride + (h - c.Hq) * c.t.d
                                    : c.v + (int64_t)at.row * c.v_stride + (h - c.Hq - c.Hkv) * c.t.d, at);
  }
  const Angles a(c.t, at, PAIRS);
  Weights ws;
  const bool stores = at.live && at.holds;
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int h = h0 + u;
    if (h >= c.heads) return;
    if (h >= c.Hq + c.Hkv) {
      uint16_t* to = c.v_out + (int64_t)at.row * c.v_out_stride + (h - c.Hq - c.Hkv) * c.t.d;
      if (stores) {
        *(kv_u32x4*)(to + at.e[0]) = x[u].x[0];
        *(kv_u32x4*)(to + at.e[1]) = x[u].x[1];
      }
      continue;
    }
    const bool is_q = h < c.Hq;
    float y[16];
    turned<LG, PAIRS>(y, x[u], a, is_q ? c.q_weight : c.k_weight, ws, c.t, at);
    uint16_t* to = is_q ? c.q_out + (int64_t)at.row * c.q_out_stride + h * c.t.d : c.k_out + (int64_t)at.row * c.k_out_stride + (h - c.Hq) * c.t.d;
    if (stores) store16(to, at, y);
  }
}

// ------------------------------------------------------------------------------------------------ into pages
struct AppendCtx {
  TurnCtx t;
  int Hkv, shift;
  uint32_t n_slots;
  int64_t k_stride, v_stride;
  float k_scale, v_scale, k_rcp, v_rcp;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* slot;
  const float* k_weight;
  uint8_t* k_pages;
  uint8_t* v_pages;
};

// FP4: the scale of 32 values is the smallest power of two 2^e, -120 <= e <= 125, with |y| <= 7 * 2^e, so that no value is further from its code's than half the distance of the two
// codes around it (the largest is 6, 7 half a step above it; with 2^(floor(log2 max) - 2), the usual choice, values between 7 and 8 are up to a whole step off).  Finite values above 7 * 2^125 have no such power: they are cut to 6 * 2^125.  `most`: the bits of the
// largest, of which 1.75 * 2^k + 0x1fffff are the last that keep their exponent.
__device__ __forceinline__ uint32_t fp4_power(uint32_t most) { return min(max((most + 0x1fffffu) >> 23, 9u) - 2u, 252u); }
// Eight values as codes under the scale 2^(power - 127), to nearest, ties to even
__device__ __forceinline__ uint32_t fp4_codes8(const float* y, uint32_t power) {
  const float step = __uint_as_float(power << 23);
  uint32_t v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], step, 0);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[2], y[3], step, 1);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[4], y[5], step, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[6], y[7], step, 3);
}

// KV: GR_KV_BF16, GR_KV_FP8, GR_KV_FP4, or 3: FP8 under scales that are divided by (see fp8_quotient).
template <int LG, bool PAIRS, int KV, int U>
__global__ void __launch_bounds__(256) k_page_append(AppendCtx c) {
  const Place<LG, PAIRS> at(c.t);
  const uint32_t slot = (uint32_t)c.slot[at.row];
  const bool stores = at.live && at.holds && slot < c.n_slots;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h0 = ((int)at.chunk * 4 + wave) * U, heads = 2 * c.Hkv;
  const int64_t k_row = (int64_t)at.row * c.k_stride, v_row = (int64_t)at.row * c.v_stride;
  Head x[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int h = min(h0 + u, heads - 1);
    x[u].load(h < c.Hkv ? c.k + h * c.t.d + k_row : c.v + (h - c.Hkv) * c.t.d + v_row, at);
  }
  const Angles a(c.t, at, PAIRS);
  Weights ws;
  // FP4: bytes from a pool's first record of a head to the row's codes, and from these to its powers
  const uint32_t ps = 1u << c.shift, d = (uint32_t)c.t.d, tok = slot & (ps - 1), record = gr_fp4_record(ps, d), powers_at = gr_fp4_codes(ps, d) + tok * (d / 32) - tok * (d / 2);
  const size_t codes_at = (size_t)(slot >> c.shift) * ((unsigned)c.Hkv * record) + tok * (d / 2);
  // largest of each eight of the wavefront's heads: a block's are four neighbours there, wherever its lanes are
  __shared__ __attribute__((aligned(16))) uint32_t s_most[KV == GR_KV_FP4 ? 4 * 128 : 4];
#pragma unroll
  for (int u = 0; u < U; u++) {
    int h = h0 + u;
    if (h >= heads) return;
    const bool is_k = h < c.Hkv;
    h -= is_k ? 0 : c.Hkv;
    float y[16];
    if (is_k) turned<LG, PAIRS>(y, x[u], a, c.k_weight, ws, c.t, at);
    else x[u].numbers(y);
    uint8_t* pages = is_k ? c.k_pages : c.v_pages;
    if (KV == GR_KV_FP4) {
      uint32_t* most = s_most + wave * 128 + ((int)threadIdx.x & 63) / LG * (2 * LG);
      if (at.holds) {
#pragma unroll
        for (int r = 0; r < 2; r++) {
          float m = 0.f;
#pragma unroll
          for (int e = 0; e < 8; e++) m = __builtin_elementwise_maximum(m, __builtin_fabsf(y[8 * r + e]));        // (NaN stays)
          most[at.e[r] >> 3] = __float_as_uint(m) & 0x7fffffffu;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");             // (the wavefront's own places, and LDS serves it in order)
      uint8_t* codes = pages + (unsigned)h * record + codes_at;
#pragma unroll
      for (int r = 0; r < 2; r++) {
        const uint32_t e = (uint32_t)at.e[r];
        const uint4 m4 = *(const uint4*)(most + (e >> 5) * 4);
        const uint32_t m = max(max(m4.x, m4.y), max(m4.z, m4.w)), power = fp4_power(m);                 // (as whole numbers: NaN is above the infinite)
        if (stores) {
          *(uint32_t*)(codes + e / 2) = fp4_codes8(y + 8 * r, power);
          // (an infinite value or NaN makes the scale one that says NaN for all 32)
          if ((e & 31) == 0) codes[powers_at + e / 32] = (uint8_t)(m >= 0x7f800000u ? 255u : power);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else {
      const size_t i = (size_t)slot * ((unsigned)c.Hkv * d) + (unsigned)h * d;
      if (KV == GR_KV_BF16) {
        if (stores) store16((uint16_t*)pages + i, at, y);
      } else {
        const float scale = is_k ? c.k_scale : c.v_scale, rcp = is_k ? c.k_rcp : c.v_rcp;
#pragma unroll
        for (int r = 0; r < 2; r++) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; e++) f[e] = fp8_quotient<KV == GR_KV_FP8>(y[8 * r + e], scale, rcp);
          const kv_u32x2 w = {fp8_codes4(f[0], f[1], f[2], f[3]), fp8_codes4(f[4], f[5], f[6], f[7])};
          if (stores) *(kv_u32x2*)(pages + i + at.e[r]) = w;
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ host
bool any_misaligned(std::initializer_list<const void*> of, uintptr_t mask) {
  for (const void* p : of)
    if ((uintptr_t)p & mask) return true;
  return false;
}

bool is_one_of(const void* out, std::initializer_list<const void*> of) {
  for (const void* p : of)
    if (out && out == p) return true;
  return false;
}

// What both calls ask of a rotation and of a head's size
gr_status turn_ok(int32_t d, int32_t rot, int32_t pairs, int32_t n_pos, float eps, bool norms, const float* table, const int32_t* pos, int64_t T) {
  if (d <= 0 || rot < 0 || rot > d || (pairs != 0 && pairs != 1)) return GR_ERR_INVALID_ARG;
  if (rot > 0 && (n_pos <= 0 || (T > 0 && (!table || !pos)))) return GR_ERR_INVALID_ARG;
  if (norms && !(eps >= 0.f && eps < INFINITY)) return GR_ERR_INVALID_ARG;
  if (d % 16 || d > 256 || rot % 16) return GR_ERR_UNSUPPORTED;
  return GR_OK;
}
void fill_turn(TurnCtx* t, int64_t T, int32_t d, int32_t rot, int32_t n_pos, float eps, const float* table, const int32_t* pos) {
  t->T = (uint32_t)T; t->d = d; t->rot = rot; t->n_pos = n_pos; t->inv_d = 1.0f / (float)d; t->eps = eps; t->table = table; t->pos = pos;
}
// The launch: 0 where it has too many threads
unsigned grid_of(TurnCtx* t, int lg, int heads, int per_wave) {
  t->chunks = (uint32_t)((heads + 4 * per_wave - 1) / (4 * per_wave));
  t->inv_chunks = 0xffffffffu / t->chunks;
  const int64_t rows = 64 / lg, grid = ((int64_t)t->T + rows - 1) / rows * t->chunks;
  return gr_grid_fits(grid, 256) ? (unsigned)grid : 0;
}
// (Head sizes between powers of two leave lanes without work: 67000 rows of 8 heads into bf16 pages, d = 80 85 us, 96 91, 160 139, 208 183, 4.0 to 4.9 TB/s; gr_page_write, which has no heads,
// 71, 82, 135, 174.  Of 64, 128, 192 and 256 both take the same.)
int lanes_of_head(int d) { return d <= 64 ? 4 : d <= 128 ? 8 : 16; }

template <class F>
gr_status with_lanes(int lg, F&& f) {
  return lg == 4 ? f(std::integral_constant<int, 4>()) : lg == 8 ? f(std::integral_constant<int, 8>()) : f(std::integral_constant<int, 16>());
}
// Heads of a wavefront: four, which share their angles and the norm's weights, once the launch fills the chip so (4096 wavefronts, four to a SIMD).  us with one and with four: prompts
// of 36 thousand tokens, 32 and 8 heads of 128, 154.9, 143.9; 32 x 4096 tokens of 8 heads into FP4 (and back) 298.7, 282.3; 32 x 256 rows of 32 + 8 + 8 heads 42.0, 41.7; 16 prompts of
// 60-700 tokens into FP8 10.8, 11.0.
template <class F>
gr_status with_heads(int64_t T, int lg, int heads, F&& f) {
  const int64_t waves = (T + 64 / lg - 1) / (64 / lg) * heads;
  return waves >= 4 * 4096 ? f(std::integral_constant<int, 4>()) : f(std::integral_constant<int, 1>());
}
template <class F>
gr_status with_bool(bool b, F&& f) { return b ? f(std::true_type()) : f(std::false_type()); }

}  // namespace

extern "C" gr_status gr_qk_norm_rope(const gr_qk_norm_rope_params* p, void* stream_) {
  if (!p) return GR_ERR_INVALID_ARG;
  const bool has_q = p->q != nullptr, has_k = p->k != nullptr, has_v = p->v != nullptr;
  if (p->T < 0 || p->Hq < 0 || p->Hkv < 0 || (has_q && p->Hq == 0) || ((has_k || has_v) && p->Hkv == 0)) return GR_ERR_INVALID_ARG;
  if (!has_q && !has_k && p->T > 0) return GR_ERR_INVALID_ARG;
  if (has_q != (p->q_out != nullptr) || has_k != (p->k_out != nullptr) || has_v != (p->v_out != nullptr)) return GR_ERR_INVALID_ARG;
  if (p->T > 0 && ((p->q_weight && !has_q) || (p->k_weight && !has_k))) return GR_ERR_INVALID_ARG;         // (tensors of no rows may have no address)
  if (const gr_status st = turn_ok(p->d, p->rot, p->pairs, p->n_pos, p->eps, p->q_weight || p->k_weight, p->table, p->pos, p->T)) return st;
  const int64_t nq = (int64_t)p->Hq * p->d, nk = (int64_t)p->Hkv * p->d;
  if ((has_q && (p->q_stride < nq || p->q_out_stride < nq)) || (has_k && (p->k_stride < nk || p->k_out_stride < nk)) || (has_v && (p->v_stride < nk || p->v_out_stride < nk)))
    return GR_ERR_INVALID_ARG;
  if ((p->q_out == p->q && has_q && p->q_out_stride != p->q_stride) || (p->k_out == p->k && has_k && p->k_out_stride != p->k_stride)) return GR_ERR_INVALID_ARG;
  if (is_one_of(p->q_out, {p->k, p->v, p->q_weight, p->k_weight, p->table, p->pos, p->k_out, p->v_out}) || is_one_of(p->k_out, {p->q, p->v, p->q_weight, p->k_weight, p->table, p->pos, p->v_out}) ||
      is_one_of(p->v_out, {p->q, p->k, p->v, p->q_weight, p->k_weight, p->table, p->pos}))
    return GR_ERR_INVALID_ARG;                               // (other wavefronts would read rows that are written over already)
  if (any_misaligned({p->q, p->k, p->v, p->q_weight, p->k_weight, p->table, p->q_out, p->k_out, p->v_out}, 15) || any_misaligned({p->pos}, 3)) return GR_ERR_INVALID_ARG;
  auto odd = [](bool has, int64_t a, int64_t b) { return has && (a % 8 || b % 8); };
  if (odd(has_q, p->q_stride, p->q_out_stride) || odd(has_k, p->k_stride, p->k_out_stride) || odd(has_v, p->v_stride, p->v_out_stride)) return GR_ERR_UNSUPPORTED;
  if (p->T >= (int64_t)1 << 31 || nq > 1 << 20 || nk > 1 << 20) return GR_ERR_UNSUPPORTED;
  if (p->T == 0) return GR_OK;
  NormRopeCtx c;
  fill_turn(&c.t, p->T, p->d, p->rot, p->n_pos, p->eps, p->table, p->pos);
  c.Hq = has_q ? p->Hq : 0; c.Hkv = has_k ? p->Hkv : 0; c.heads = c.Hq + c.Hkv + (has_v ? p->Hkv : 0);
  c.q_stride = p->q_stride; c.k_stride = p->k_stride; c.v_stride = p->v_stride;
  c.q_out_stride = p->q_out_stride; c.k_out_stride = p->k_out_stride; c.v_out_stride = p->v_out_stride;
  c.q = (const uint16_t*)p->q; c.k = (const uint16_t*)p->k; c.v = (const uint16_t*)p->v; c.q_weight = p->q_weight; c.k_weight = p->k_weight;
  c.q_out = (uint16_t*)p->q_out; c.k_out = (uint16_t*)p->k_out; c.v_out = (uint16_t*)p->v_out;
  const int lg = lanes_of_head(p->d);
  const gr_status st = with_lanes(lg, [&](auto lanes) {
    return with_bool(p->pairs != 0, [&](auto pairs) {
      return with_heads(p->T, lg, c.heads, [&](auto per_wave) {
        constexpr int U = decltype(per_wave)::value;
        const unsigned grid = grid_of(&c.t, lg, c.heads, U);
        if (!grid) return (gr_status)GR_ERR_UNSUPPORTED;
        hipLaunchKernelGGL((k_qk_norm_rope<decltype(lanes)::value, decltype(pairs)::value, U>), dim3(grid), dim3(256), 0, (hipStream_t)stream_, c);
        return (gr_status)GR_OK;
      });
    });
  });
  if (st) return st;
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}

extern "C" gr_status gr_page_append(const gr_page_append_params* p, void* stream_) {
  if (!p) return GR_ERR_INVALID_ARG;
  if (p->T < 0 || p->Hkv <= 0 || p->n_pages <= 0) return GR_ERR_INVALID_ARG;
  if (p->kv_type != GR_KV_BF16 && p->kv_type != GR_KV_FP8 && p->kv_type != GR_KV_FP4) return GR_ERR_INVALID_ARG;
  if (p->kv_type == GR_KV_FP8 && (!gr_scale_ok(p->k_scale) || !gr_scale_ok(p->v_scale))) return GR_ERR_INVALID_ARG;
  if (!p->k_pages || !p->v_pages || p->k_pages == p->v_pages) return GR_ERR_INVALID_ARG;
  for (const void* pool : {p->k_pages, p->v_pages})
    if (is_one_of(pool, {p->k, p->v, p->slot, p->pos, p->table, p->k_weight})) return GR_ERR_INVALID_ARG;
  if (p->T > 0 && (!p->k || !p->v || !p->slot)) return GR_ERR_INVALID_ARG;
  if (const gr_status st = turn_ok(p->d, p->rot, p->pairs, p->n_pos, p->eps, p->k_weight != nullptr, p->table, p->pos, p->T)) return st;
  const int64_t n = (int64_t)p->Hkv * p->d;
  if (p->k_stride < n || p->v_stride < n) return GR_ERR_INVALID_ARG;
  if (any_misaligned({p->k, p->v, p->k_pages, p->v_pages, p->k_weight, p->table}, 15) || any_misaligned({p->slot, p->pos}, 3)) return GR_ERR_INVALID_ARG;
  if (!gr_page_size_ok(p->page_size) || p->k_stride % 8 || p->v_stride % 8 || n > 1 << 20) return GR_ERR_UNSUPPORTED;
  if (p->kv_type == GR_KV_FP4 && p->d % 32) return GR_ERR_UNSUPPORTED;
  if ((int64_t)p->n_pages * p->page_size >= ((int64_t)1 << 31) || p->T >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  if (p->T == 0) return GR_OK;
  AppendCtx c;
  fill_turn(&c.t, p->T, p->d, p->rot, p->n_pos, p->eps, p->table, p->pos);
  c.Hkv = p->Hkv; c.shift = __builtin_ctz((unsigned)p->page_size); c.n_slots = (uint32_t)(p->n_pages * p->page_size);
  c.k_stride = p->k_stride; c.v_stride = p->v_stride; c.k_scale = p->k_scale; c.v_scale = p->v_scale; c.k_rcp = 1.0f / p->k_scale; c.v_rcp = 1.0f / p->v_scale;
  c.k = (const uint16_t*)p->k; c.v = (const uint16_t*)p->v; c.slot = p->slot; c.k_weight = p->k_weight; c.k_pages = (uint8_t*)p->k_pages; c.v_pages = (uint8_t*)p->v_pages;
  auto ordinary = [](float s) { return s >= 0x1p-60f && s <= 0x1p60f; };
  const int lg = lanes_of_head(p->d);
  const gr_status st = with_lanes(lg, [&](auto lanes) {
    return with_bool(p->pairs != 0, [&](auto pairs) {
      auto go = [&](auto type) {
        return with_heads(p->T, lg, 2 * p->Hkv, [&](auto per_wave) {
          constexpr int U = decltype(per_wave)::value;
          const unsigned grid = grid_of(&c.t, lg, 2 * p->Hkv, U);
          if (!grid) return (gr_status)GR_ERR_UNSUPPORTED;
          hipLaunchKernelGGL((k_page_append<decltype(lanes)::value, decltype(pairs)::value, decltype(type)::value, U>), dim3(grid), dim3(256), 0, (hipStream_t)stream_, c);
          return (gr_status)GR_OK;
        });
      };
      if (p->kv_type == GR_KV_BF16) return go(std::integral_constant<int, GR_KV_BF16>());
      if (p->kv_type == GR_KV_FP4) return go(std::integral_constant<int, GR_KV_FP4>());
      if (ordinary(p->k_scale) && ordinary(p->v_scale)) return go(std::integral_constant<int, GR_KV_FP8>());
      return go(std::integral_constant<int, 3>());
    });
  });
  if (st) return st;
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
