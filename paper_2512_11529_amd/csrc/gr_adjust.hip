// gr_logits_adjust: what a serving program does to the logits before the item step.  For a live beam w of request b with logits x:
//     c(v) = rows h of the request's history with h[0..step) = the beam's tokens and h[step] = v
//     y = x(v) > 0 ? x(v) / r_b : x(v) r_b,  y -= f_b c(v) + p_b     where c(v) > 0, else y = x(v)
//     y += bias(v);   y = -inf where the beam's mask forbids v
//
// c is zero nearly everywhere, so it never meets the stream of logits: a workgroup finds its row's counts in LDS (only the counters that the history
// touches are cleared and read) and one thread per counted token changes that token alone, before the row is streamed where it is changed in place, behind it
// where it is copied.  A row that is changed in place without a bias is not streamed at all: forbidden tokens are overwritten without being read.
// Bound: memory, 8 bytes a logit for rows that are copied.
#include "gr_internal.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kStreamTile = 8192;        // tokens of a workgroup, at most: of streamed rows (32 KB of counters, five workgroups to a CU),
constexpr int kSparseTile = 16384;       // of rows whose counted tokens alone are touched
constexpr int kMaxV = 32768;
constexpr int kMaxDepth = 8;
constexpr int kKept = 32;                // history rows per thread whose match is kept in a bit

struct AdjustCtx {
  int B, W, V, depth, step, words, n_history, n_allowed, tiles, tile;
  int64_t bias_stride;                   // 0: one bias for all requests
  const float* logits;
  float* out;
  const float* scores;
  const int32_t* prefix;
  const int32_t* history;
  const int32_t* cu_history;
  const float* repetition;
  const float* frequency;
  const float* presence;
  const float* bias;
  const uint32_t* allowed;
  const int32_t* allowed_row;
};

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));       // a row begins at any multiple of 4 bytes

template <bool COUNT, bool INPLACE>
__global__ void __launch_bounds__(kThreads) k_logits_adjust(AdjustCtx c) {
  extern __shared__ uint32_t s_count[];
  const int tid = (int)threadIdx.x;
  const unsigned row = blockIdx.x / (unsigned)c.tiles;
  const int v0 = (int)(blockIdx.x - row * (unsigned)c.tiles) * c.tile, v1 = min(v0 + c.tile, c.V);
  if (c.scores && !(c.scores[row] > -INFINITY)) return;            // a dead beam's row is left as it is
  const unsigned b = row / (unsigned)c.W;
  const float* x = c.logits + (size_t)row * (unsigned)c.V;
  float* y = c.out + (size_t)row * (unsigned)c.V;
  const float* bias = c.bias ? c.bias + (int64_t)b * c.bias_stride : nullptr;
  const uint32_t* allowed = nullptr;
  if (c.allowed) {
    const int at = c.allowed_row ? c.allowed_row[row] : 0;
    if ((unsigned)at < (unsigned)c.n_allowed) allowed = c.allowed + (size_t)(unsigned)at * (unsigned)c.words;
  }

  // the tokens that the history counts, each by one thread
  auto counted = [&]() {
    const int h0 = min(max(c.cu_history[b], 0), c.n_history), h1 = min(max(c.cu_history[b + 1], h0), c.n_history);
    if (h0 == h1) return;
    int mine[kMaxDepth];
    const int32_t* prefix = c.step > 0 ? c.prefix + (size_t)row * (unsigned)c.depth : nullptr;
#pragma unroll
    for (int t = 0; t < kMaxDepth - 1; t++) mine[t] = t < c.step ? prefix[t] : 0;
    auto token = [&](int h) { return c.history[(size_t)(unsigned)h * (unsigned)c.depth + (unsigned)c.step]; };
    auto match = [&](int h) {
      const int32_t* item = c.history + (size_t)(unsigned)h * (unsigned)c.depth;
      bool same = true;
#pragma unroll
      for (int t = 0; t < kMaxDepth - 1; t++)
        if (t < c.step) same &= item[t] == mine[t];
      const int v = item[c.step];
      return same && v >= v0 && v < v1;
    };
    uint32_t hit = 0;
    for (int i = 0, h = h0 + tid; h < h1; i++, h += kThreads)
      if (match(h)) { hit |= i < kKept ? 1u << i : 0; s_count[token(h) - v0] = 0; }
    // f(token) of this thread's matches
    auto each = [&](auto&& f) {
      for (uint32_t m = hit; m; m &= m - 1) f(token(h0 + tid + (__ffs((int)m) - 1) * kThreads));
      for (int h = h0 + tid + kKept * kThreads; h < h1; h += kThreads)
        if (match(h)) f(token(h));
    };
    __syncthreads();
    each([&](int v) { atomicAdd(&s_count[v - v0], 1u); });
    __syncthreads();
    const float r = c.repetition ? c.repetition[b] : 1.f, f = c.frequency ? c.frequency[b] : 0.f, p = c.presence ? c.presence[b] : 0.f;
    each([&](int v) {
      const uint32_t n = atomicExch(&s_count[v - v0], 0u);         // (of equal tokens one thread gets the count)
      if (n == 0) return;
      const bool forbidden = allowed && !((allowed[v >> 5] >> (v & 31)) & 1);
      if (forbidden && (!INPLACE || !bias)) return;                // (the row's stream has it as -inf, or will)
      float z = x[v];
      z = z > 0.f ? z / r : z * r;
      z -= fmaf(f, (float)n, p);
      if (!INPLACE && bias) z += bias[v];
      y[v] = z;
    });
  };

  if (INPLACE && COUNT) {
    counted();
    if (!bias && !allowed) return;
    __syncthreads();
  }
  if (INPLACE && !bias && !allowed) return;
  constexpr int U = 4;
  for (int base = v0; base < v1; base += kThreads * 4 * U) {
    f32x4u z[U], more[U];
    uint32_t ok[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int v = base + 4 * (tid + kThreads * u);
      ok[u] = 15;
      if (v + 4 <= v1) {
        if (!INPLACE || bias) z[u] = *(const f32x4u*)(x + v);
        if (bias) more[u] = *(const f32x4u*)(bias + v);
        if (allowed) ok[u] = allowed[v >> 5] >> (v & 31);
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int v = base + 4 * (tid + kThreads * u);
      if (v + 4 <= v1) {
        if (!INPLACE || bias) {
          if (bias) z[u] += more[u];
#pragma unroll
          for (int k = 0; k < 4; k++) z[u][k] = (ok[u] >> k) & 1 ? z[u][k] : -INFINITY;
          *(f32x4u*)(y + v) = z[u];
        } else if ((ok[u] & 15) == 0) {
          *(f32x4u*)(y + v) = f32x4u{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        } else {
#pragma unroll
          for (int k = 0; k < 4; k++)
            if (!((ok[u] >> k) & 1)) y[v + k] = -INFINITY;
        }
      } else {
        for (int k = v; k < v1; k++) {                             // the row's last one to three tokens
          const bool good = !allowed || ((allowed[k >> 5] >> (k & 31)) & 1);
          if (!good) y[k] = -INFINITY;
          else if (!INPLACE || bias) y[k] = x[k] + (bias ? bias[k] : 0.f);
        }
      }
    }
  }
  if (!INPLACE && COUNT) {
    __syncthreads();
    counted();
  }
}

}  // namespace

extern "C" gr_status gr_logits_adjust(const gr_logits_adjust_params* p, void* stream_) {
  if (!p) return GR_ERR_INVALID_ARG;
  if (p->B <= 0 || p->W <= 0 || p->V <= 0 || p->depth <= 0 || p->step < 0 || p->step >= p->depth || p->n_history < 0 || p->n_allowed < 0)
    return GR_ERR_INVALID_ARG;
  if (!p->logits || !p->out) return GR_ERR_INVALID_ARG;
  const bool penalties = p->repetition || p->frequency || p->presence;
  if (penalties && (!p->cu_history || (p->n_history > 0 && !p->history) || (p->step > 0 && !p->prefix))) return GR_ERR_INVALID_ARG;
  if (p->bias && p->bias_rows != 1 && p->bias_rows != p->B) return GR_ERR_INVALID_ARG;
  if ((p->allowed_row && !p->allowed) || (p->allowed && p->n_allowed == 0)) return GR_ERR_INVALID_ARG;
  if (((uintptr_t)p->logits | (uintptr_t)p->out | (uintptr_t)p->scores | (uintptr_t)p->prefix | (uintptr_t)p->history | (uintptr_t)p->cu_history |
       (uintptr_t)p->repetition | (uintptr_t)p->frequency | (uintptr_t)p->presence | (uintptr_t)p->bias | (uintptr_t)p->allowed |
       (uintptr_t)p->allowed_row) & 3)
    return GR_ERR_INVALID_ARG;
  if (p->V > kMaxV || p->depth > kMaxDepth) return GR_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)p->B * p->W;
  const uint64_t bytes = (uint64_t)rows * p->V * 4, from = (uint64_t)(uintptr_t)p->logits, to = (uint64_t)(uintptr_t)p->out;
  const bool inplace = from == to;
  if (!inplace && from < to + bytes && to < from + bytes) return GR_ERR_INVALID_ARG;       // out lies across the logits
  const bool count = penalties && p->n_history > 0;
  if (inplace && !count && !p->bias && !p->allowed) return GR_OK;                          // nothing to change
  AdjustCtx c;
  c.B = p->B; c.W = p->W; c.V = p->V; c.depth = p->depth; c.step = p->step; c.words = (p->V + 31) / 32; c.n_history = p->n_history; c.n_allowed = p->n_allowed;
  c.bias_stride = p->bias_rows == 1 ? 0 : p->V;
  c.logits = p->logits; c.out = p->out; c.scores = p->scores; c.prefix = p->prefix; c.history = p->history; c.cu_history = p->cu_history;
  c.repetition = p->repetition; c.frequency = p->frequency; c.presence = p->presence; c.bias = p->bias; c.allowed = p->allowed; c.allowed_row = p->allowed_row;
  const int most = inplace && !p->bias && !p->allowed ? kSparseTile : kStreamTile;
  c.tiles = (p->V + most - 1) / most;
  c.tile = ((p->V + c.tiles - 1) / c.tiles + 31) / 32 * 32;
  const int64_t grid = rows * c.tiles;
  if (grid >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  const size_t lds = count ? (size_t)c.tile * 4 : 0;
  const hipStream_t stream = (hipStream_t)stream_;
#define GR_LAUNCH(C_, I_) hipLaunchKernelGGL((k_logits_adjust<C_, I_>), dim3((unsigned)grid), dim3(kThreads), lds, stream, c)
  if (count) { if (inplace) GR_LAUNCH(true, true); else GR_LAUNCH(true, false); }
  else { if (inplace) GR_LAUNCH(false, true); else GR_LAUNCH(false, false); }
#undef GR_LAUNCH
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
