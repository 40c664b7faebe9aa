// gr_logits_adjust: what a serving program does to the logits before the item step.  For a live beam w of request b with logits x:
//     c(v) = rows h of the request's history with h[0..step) = the beam's tokens and h[step] = v
//     y = x(v) > 0 ? x(v) / r_b : x(v) r_b,  y -= f_b c(v) + p_b     where c(v) > 0, else y = x(v)
//     y += bias(v);   y = -inf where the beam's mask forbids v
//
// c is zero nearly everywhere, so it never meets the stream of logits: the tokens that the history continues a row with go to a list in LDS, equal ones are
// counted (few against each other, more in bins, 4096 at a time, from the history once more where the list is too short for them), and one thread per counted
// token changes that token alone, before the row is streamed where it is changed in place, behind it where it is copied.  A row that
// is changed in place without a bias or a mask is not streamed at all, and a workgroup looks through the history for eight such rows at once.
// Bound: memory, 8 bytes a logit of streamed rows.  8192 rows x 8192 logits copied with a bias and a mask take 103 us (5.2 TB/s); with counters for all
// tokens in LDS, looked for behind the stream, the history of 200-600 rows cost another 36.
#include <type_traits>
#include "gr_internal.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 8192;              // tokens of a workgroup, at most, of a streamed row
constexpr int kSparseRows = 8;           // rows of a workgroup that streams none
constexpr int kMaxV = 32768;
constexpr int kMaxDepth = 8;
constexpr int kMaxHistory = 1 << 28;     // (kSparseRows rows that all of them continue: the list's length is an int)
constexpr int kFew = 256;                 // counted against each other
constexpr int kList = 1024;
constexpr int kBins = 4096;
// History rows of a thread on their way at once.  us at the first step (one live row a request) with one and with four: 32 requests of 1000-3000 history rows, 4096 tokens in place,
// 16.5, 11.4; 35 of 364-1091, 928 tokens copied, 7.3, 5.6.
constexpr int kAhead = 4;

struct AdjustCtx {
  int W, V, depth, step, words, n_history, n_allowed, tiles, tile;
  unsigned row_blocks;                   // SPARSE: blocks of kSparseRows rows per request
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

// The mask row of a beam, nullptr: nothing is forbidden.
__device__ __forceinline__ const uint32_t* mask_of(const AdjustCtx& c, size_t row) {
  if (!c.allowed) return nullptr;
  const int at = c.allowed_row ? c.allowed_row[row] : 0;
  return (unsigned)at < (unsigned)c.n_allowed ? c.allowed + (size_t)(unsigned)at * (unsigned)c.words : nullptr;
}

__device__ __forceinline__ bool dead(const AdjustCtx& c, size_t row) { return c.scores && !(c.scores[row] > -INFINITY); }

// A workgroup's counted tokens: those v0 <= v < v1 of the live ones of rows row0 .. row0 + rows - 1 of request b.
// find() looks through the history; apply(f) then calls f(row, token, count) once for each counted token, by some thread.
template <int R>
struct Counted {
  struct Lds { int n, h0, h1; unsigned live; alignas(16) int list[kList]; uint32_t bins[kBins]; int prefix[R][kMaxDepth]; };
  const AdjustCtx& c;
  Lds& s;
  const unsigned b;
  const size_t row0;
  const int rows, v0, v1;

  // History rows h, h + kThreads, ... (U of them, on their way together): bit r: it counts for row0 + r; and the tokens
  template <int U>
  __device__ __forceinline__ void match(int h, unsigned (&hit)[U], int (&token)[U]) const {
    const int32_t* item[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      hit[u] = h + u * kThreads < s.h1 ? s.live : 0;
      item[u] = c.history + (size_t)(unsigned)min(h + u * kThreads, s.h1 - 1) * (unsigned)c.depth;
    }
    for (int t = 0; t < c.step; t++) {
      int x[U];
#pragma unroll
      for (int u = 0; u < U; u++) x[u] = item[u][t];
#pragma unroll
      for (int r = 0; r < R; r++)
#pragma unroll
        for (int u = 0; u < U; u++) hit[u] &= x[u] == s.prefix[r][t] ? ~0u : ~(1u << r);
    }
#pragma unroll
    for (int u = 0; u < U; u++) token[u] = item[u][c.step];
#pragma unroll
    for (int u = 0; u < U; u++) hit[u] = token[u] >= v0 && token[u] < v1 ? hit[u] : 0;
  }
  __device__ __forceinline__ void find() {
    const int tid = (int)threadIdx.x;
    if (tid == 0) {
      s.n = 0;
      s.h0 = min(max(c.cu_history[b], 0), c.n_history);
      s.h1 = min(max(c.cu_history[b + 1], s.h0), c.n_history);
    }
    if (tid < 64) {
      const bool is_live = tid < rows && !dead(c, row0 + tid);
      const unsigned live = (unsigned)__ballot(is_live);
      if (tid == 0) s.live = live;
    }
    if (c.step > 0 && tid < R * kMaxDepth) {
      const int r = tid / kMaxDepth, t = tid % kMaxDepth;
      if (r < rows && t < c.step) s.prefix[r][t] = c.prefix[(row0 + r) * (size_t)(unsigned)c.depth + t];
    }
    __syncthreads();
    const int h1 = s.h1;
    // (wavefront by wavefront: one lane asks for the places of all)
    auto look = [&](int h0, auto ahead) {
      constexpr int U = decltype(ahead)::value;
      unsigned hit[U];
      int v[U];
      match<U>(h0 + tid, hit, v);
#pragma unroll
      for (int u = 0; u < U; u++) {
        if (!__any(hit[u])) continue;
#pragma unroll
        for (int r = 0; r < R; r++) {
          const uint64_t all = __ballot((hit[u] >> r) & 1);
          if (all == 0) continue;
          int at = 0;
          if ((tid & 63) == 0) at = atomicAdd(&s.n, __popcll(all));
          at = __builtin_amdgcn_readfirstlane(at) + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
          if (((hit[u] >> r) & 1) && at < kList) s.list[at] = r * kMaxV + v[u];
        }
      }
    };
    int h0 = s.h0;
    for (; h1 - h0 > kThreads; h0 += kThreads * kAhead) look(h0, std::integral_constant<int, kAhead>());
    if (h0 < h1) look(h0, std::integral_constant<int, 1>());
    __syncthreads();
  }
  template <class F>
  __device__ __forceinline__ void apply(F&& f) {
    const int n = s.n, tid = (int)threadIdx.x;
    if (n <= kFew) {
      for (int i = tid; i < n; i += kThreads) {
        const int mine = s.list[i];
        int count = 0, before = 0;
#pragma unroll 4
        for (int j = 0; j < n; j += 4) {
          const int4 four = *(const int4*)&s.list[j];              // (what is behind the list's end counts nothing)
          const int same[4] = {four.x == mine, four.y == mine, four.z == mine, four.w == mine};
#pragma unroll
          for (int k = 0; k < 4; k++) {
            count += j + k < n ? same[k] : 0;
            before += j + k < i ? same[k] : 0;
          }
        }
        if (before == 0) f(mine / kMaxV, mine % kMaxV, count);     // (of equal tokens the first one's thread)
      }
      return;
    }
    if (n <= kList) {                            // only the bins that the list touches are cleared and read
      for (int r = 0; r < rows; r++) {
        if (!((s.live >> r) & 1)) continue;
        for (int base = v0; base < v1; base += kBins) {
          auto each = [&](auto&& g) {
            for (int i = tid; i < n; i += kThreads) {
              const int v = s.list[i] - r * kMaxV;
              if (v >= base && v < min(base + kBins, v1)) g(v);
            }
            __syncthreads();
          };
          each([&](int v) { s.bins[v - base] = 0; });
          each([&](int v) { atomicAdd(&s.bins[v - base], 1u); });
          each([&](int v) {
            const uint32_t count = atomicExch(&s.bins[v - base], 0u);
            if (count) f(r, v, (int)count);
          });
        }
      }
      return;
    }
    // the history once more for as many rows as have room in the bins together, or for each part of one row (4 requests of 6667-20000 history rows that all continue their one live
    // row of 32768 tokens: 73 us, 131 with two live rows each; through it three times for each part, to clear, count and read only what it touches, 241)
    const int width = min(v1 - v0, kBins), together = min(kBins / width, R);
    for (int r0 = 0; r0 < rows; r0 += together) {
      if (!((s.live >> r0) & ((1u << together) - 1u))) continue;
      for (int base = v0; base < v1; base += width) {
        for (int i = tid; i < together * width; i += kThreads) s.bins[i] = 0;
        __syncthreads();
        for (int h0 = s.h0; h0 < s.h1; h0 += kThreads * kAhead) {
          unsigned hit[kAhead];
          int v[kAhead];
          match<kAhead>(h0 + tid, hit, v);
#pragma unroll
          for (int u = 0; u < kAhead; u++) {
            if (v[u] < base || v[u] >= base + width) continue;
            for (int k = 0; k < together; k++)
              if ((hit[u] >> (r0 + k)) & 1) atomicAdd(&s.bins[k * width + v[u] - base], 1u);
          }
        }
        __syncthreads();
        for (int k = 0; k < together; k++)
          for (int i = (s.live >> (r0 + k)) & 1 ? tid : width; i < width; i += kThreads) {
            const uint32_t count = s.bins[k * width + i];
            if (count) f(r0 + k, base + i, (int)count);
          }
        __syncthreads();
      }
    }
  }
};

struct Penalties { float r, f, p; };
__device__ __forceinline__ Penalties penalties_of(const AdjustCtx& c, unsigned b) {
  return {c.repetition ? c.repetition[b] : 1.f, c.frequency ? c.frequency[b] : 0.f, c.presence ? c.presence[b] : 0.f};
}
__device__ __forceinline__ float penalised(float x, const Penalties& p, int n) {
  const float y = x > 0.f ? x / p.r : x * p.r;
  return y - fmaf(p.f, (float)n, p.p);
}

// COPY: out is another tensor; BIAS: in place, with a bias (and masks); MASK: in place, masks alone.
enum { COPY = 0, BIAS = 1, MASK = 2 };
template <bool COUNT, int MODE>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(6))) k_logits_adjust(AdjustCtx c) {
  __shared__ typename Counted<1>::Lds s_counted;
  constexpr bool INPLACE = MODE != COPY;
  const int tid = (int)threadIdx.x;
  const unsigned row = blockIdx.x / (unsigned)c.tiles;
  const int v0 = (int)(blockIdx.x - row * (unsigned)c.tiles) * c.tile, v1 = min(v0 + c.tile, c.V);
  if (dead(c, row)) return;                                        // a dead beam's row is left as it is
  const unsigned b = row / (unsigned)c.W;
  const float* x = c.logits + (size_t)row * (unsigned)c.V;
  float* y = c.out + (size_t)row * (unsigned)c.V;
  const float* bias = MODE != MASK && c.bias ? c.bias + (int64_t)b * c.bias_stride : nullptr;
  const uint32_t* allowed = mask_of(c, row);
  Counted<1> counted{c, s_counted, b, row, 1, v0, v1};
  if (COUNT) counted.find();
  auto change = [&](int, int v, int n) {
    const bool forbidden = allowed && !((allowed[v >> 5] >> (v & 31)) & 1);
    if (forbidden) return;                                         // (the row's stream has it as -inf, or will)
    const float z = penalised(x[v], penalties_of(c, b), n);
    y[v] = MODE == COPY && bias ? z + bias[v] : z;
  };
  if (INPLACE && COUNT) {
    counted.apply(change);
    __syncthreads();
  }
  if (MODE == MASK && !allowed) return;
  // (one base and 32-bit offsets: 64-bit addresses of twelve loads were a third of the registers)
  auto at = [](const float* base, int v) { return (const f32x4u*)((const char*)base + (uint32_t)v * 4u); };
  constexpr int U = 4;
#pragma unroll 1
  for (int base = v0; base < v1; base += kThreads * 4 * U) {
    f32x4u z[U], more[U];
    uint32_t ok[U];
    bool partly = MODE != MASK;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int v = base + 4 * (tid + kThreads * u);
      ok[u] = 15;
      if (allowed && v + 4 <= v1) ok[u] = (allowed[v >> 5] >> (v & 31)) & 15;
      partly = partly || (ok[u] != 15 && ok[u] != 0);
    }
    // (masks alone: four that are forbidden are written unread, four that are not left alone.  Where a wavefront has some of which part is forbidden, it reads and
    // writes them whole; 8192 rows of 8192 under random masks, with penalties, take 116 us so, 2 more where single logits are written; the call that copies, adds a bias and masks 107)
    partly = MODE != MASK || __any(partly);
    if (partly) {
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int v = base + 4 * (tid + kThreads * u);
        if (v + 4 <= v1) z[u] = *at(x, v);
      }
    }
    if (bias) {
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int v = base + 4 * (tid + kThreads * u);
        if (v + 4 <= v1) more[u] = *at(bias, v);
      }
#pragma unroll
      for (int u = 0; u < U; u++) z[u] += more[u];
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int v = base + 4 * (tid + kThreads * u);
      if (v + 4 <= v1) {
        if (MODE == MASK && ok[u] == 15) continue;
#pragma unroll
        for (int k = 0; k < 4; k++) z[u][k] = (ok[u] >> k) & 1 ? z[u][k] : -INFINITY;
        *const_cast<f32x4u*>(at(y, v)) = z[u];
      } else {
        for (int k = v; k < v1; k++) {                             // the row's last one to three tokens
          const bool good = !allowed || ((allowed[k >> 5] >> (k & 31)) & 1);
          if (!good) y[k] = -INFINITY;
          else if (MODE != MASK) y[k] = x[k] + (bias ? bias[k] : 0.f);
        }
      }
    }
  }
  if (!INPLACE && COUNT) {
    __syncthreads();
    counted.apply(change);
  }
}

// In place, penalties alone: nothing but the counted tokens is touched.
__global__ void __launch_bounds__(kThreads) k_logits_penalise(AdjustCtx c) {
  __shared__ typename Counted<kSparseRows>::Lds s_counted;
  const unsigned b = blockIdx.x / c.row_blocks, w0 = (blockIdx.x - b * c.row_blocks) * kSparseRows;
  const size_t row0 = (size_t)b * (unsigned)c.W + w0;
  Counted<kSparseRows> counted{c, s_counted, b, row0, min(kSparseRows, c.W - (int)w0), 0, c.V};
  counted.find();
  const Penalties p = penalties_of(c, b);
  counted.apply([&](int r, int v, int n) {
    float* y = c.out + (row0 + r) * (size_t)(unsigned)c.V + v;
    *y = penalised(*y, p, n);
  });
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
  if (p->V > kMaxV || p->depth > kMaxDepth || p->n_history >= kMaxHistory) return GR_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)p->B * p->W;
  if (rows >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  const uint64_t bytes = (uint64_t)rows * p->V * 4, from = (uint64_t)(uintptr_t)p->logits, to = (uint64_t)(uintptr_t)p->out;
  const bool inplace = from == to;
  if (!inplace && from < to + bytes && to < from + bytes) return GR_ERR_INVALID_ARG;       // out lies across the logits
  const bool count = penalties && p->n_history > 0;
  if (inplace && !count && !p->bias && !p->allowed) return GR_OK;                          // nothing to change
  AdjustCtx c;
  c.W = p->W; c.V = p->V; c.depth = p->depth; c.step = p->step; c.words = (p->V + 31) / 32; c.n_history = p->n_history; c.n_allowed = p->n_allowed;
  c.bias_stride = p->bias_rows == 1 ? 0 : p->V;
  c.logits = p->logits; c.out = p->out; c.scores = p->scores; c.prefix = p->prefix; c.history = p->history; c.cu_history = p->cu_history;
  c.repetition = p->repetition; c.frequency = p->frequency; c.presence = p->presence; c.bias = p->bias; c.allowed = p->allowed; c.allowed_row = p->allowed_row;
  // a workgroup looks through its request's history, so a long row is one workgroup's where there are rows enough (8 x 128 rows of 20000 tokens, 1333-4000 history rows a request,
  // bias and masks: 48.1 us; 8 x 127 with three workgroups to a row 50.9); not at the first step, where most rows are dead
  c.tiles = count && p->step > 0 && rows >= 1024 ? 1 : (p->V + kTile - 1) / kTile;
  c.tile = ((p->V + c.tiles - 1) / c.tiles + 31) / 32 * 32;
  c.row_blocks = (unsigned)((p->W + kSparseRows - 1) / kSparseRows);
  const bool sparse = inplace && !p->bias && !p->allowed;
  const int64_t grid = sparse ? (int64_t)p->B * c.row_blocks : rows * c.tiles;
  if (!gr_grid_fits(grid, kThreads)) return GR_ERR_UNSUPPORTED;
  const hipStream_t stream = (hipStream_t)stream_;
#define GR_LAUNCH(...) hipLaunchKernelGGL((__VA_ARGS__), dim3((unsigned)grid), dim3(kThreads), 0, stream, c)
  if (sparse) GR_LAUNCH(k_logits_penalise);
  else if (!inplace) { if (count) GR_LAUNCH(k_logits_adjust<true, COPY>); else GR_LAUNCH(k_logits_adjust<false, COPY>); }
  else if (p->bias) { if (count) GR_LAUNCH(k_logits_adjust<true, BIAS>); else GR_LAUNCH(k_logits_adjust<false, BIAS>); }
  else { if (count) GR_LAUNCH(k_logits_adjust<true, MASK>); else GR_LAUNCH(k_logits_adjust<false, MASK>); }
#undef GR_LAUNCH
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
