// gr_page_map, gr_page_write: a prompt cache kept in pages of a pool.
//
// Request b has s_b tokens in its pages and gets n_b more.  With ps tokens to a page it needs
//     need_b = ceil((s_b + n_b) / ps) - ceil(s_b / ps)
// fresh pages; off_b, the sum of need over the requests before it, is where they begin in the list of free pages, and cu_b, the sum of n,
// where its tokens begin among the new ones.  Both sums are of whole numbers in a fixed order, so the same lengths and the same free list
// always give the same tables.
#include "gr_internal.hpp"

namespace {

constexpr int kMapThreads = 256;
constexpr int kMapTokens = 4;         // consecutive tokens of a thread: one search for their request, one 16-byte store
constexpr int kMapMaxB = 4096;        // requests whose sums fit in LDS

struct MapCtx {
  int B, shift, max_pages, n_free, n_pages, total;
  const int32_t* seq;
  const int32_t* fresh;        // new tokens of a request
  const int32_t* free_pages;
  int32_t* table;
  int32_t* lens;
  int32_t* cu;
  int32_t* slot;
  int32_t* taken;
};

// Sums stop at 2^31 - 1: adding so is associative, and a request behind such a sum cannot be served anyway.
__device__ __forceinline__ uint32_t add_capped(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }

// Every workgroup adds up all requests for itself (a second launch would cost more than the sums of 128 requests, and takes
// nothing from the tokens' part, which is a store) and then writes the slots of its 1024 tokens.  The token that opens a fresh page writes the page's table entry:
// entries in front are only read and entries from there on only written, so no workgroup waits for another.
__global__ void __launch_bounds__(kMapThreads) k_page_map(MapCtx c) {
  extern __shared__ int32_t s_map[];
  int32_t* s_cu = s_map;                     // [B + 1]
  int32_t* s_off = s_cu + c.B + 1;           // [B] first fresh page in the free list, -1: not served
  int32_t* s_seq = s_off + c.B;              // [B]
  __shared__ uint2 s_wave[kMapThreads / 64];
  __shared__ int s_last[2];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ps1 = (1 << c.shift) - 1;
  const uint32_t most = (uint32_t)c.max_pages << c.shift;
  const int per = (c.B + kMapThreads - 1) / kMapThreads, b0 = min(tid * per, c.B), b1 = min(b0 + per, c.B);
  if (tid < 2) s_last[tid] = 0;
  auto lengths = [&](int b, uint32_t* s, uint32_t* n, uint32_t* need) {
    *s = (uint32_t)max(c.seq[b], 0);
    *n = (uint32_t)max(c.fresh[b], 0);
    // (a request too long for its row of the table gets nothing, and takes no pages from those behind it)
    *need = *s + *n <= most ? ((*s + *n + ps1) >> c.shift) - ((*s + ps1) >> c.shift) : 0;
  };
  uint2 sum = make_uint2(0, 0);
  for (int b = b0; b < b1; b++) {
    uint32_t s, n, need;
    lengths(b, &s, &n, &need);
    sum.x = add_capped(sum.x, n);
    sum.y = add_capped(sum.y, need);
  }
  uint2 upto = sum;                          // of this thread and those before it in the wavefront
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = (uint32_t)__shfl_up((int)upto.x, d, 64), y = (uint32_t)__shfl_up((int)upto.y, d, 64);
    if (lane >= d) { upto.x = add_capped(upto.x, x); upto.y = add_capped(upto.y, y); }
  }
  if (lane == 63) s_wave[wave] = upto;
  uint2 at;                                  // of all threads before this one
  at.x = (uint32_t)__shfl_up((int)upto.x, 1, 64);
  at.y = (uint32_t)__shfl_up((int)upto.y, 1, 64);
  if (lane == 0) at = make_uint2(0, 0);
  __syncthreads();
  for (int w = 0; w < wave; w++) { at.x = add_capped(at.x, s_wave[w].x); at.y = add_capped(at.y, s_wave[w].y); }
  const bool writes = blockIdx.x == 0;
  int refused = 0, last = 0;
  for (int b = b0; b < b1; b++) {
    uint32_t s, n, need;
    lengths(b, &s, &n, &need);
    const uint32_t cu1 = add_capped(at.x, n), off1 = add_capped(at.y, need);
    const bool served = s + n <= most && cu1 <= (uint32_t)c.total && (need == 0 || off1 <= (uint32_t)c.n_free);
    s_cu[b] = (int)at.x;
    s_off[b] = served ? (int)at.y : -1;
    s_seq[b] = (int)s;
    if (b == c.B - 1) s_cu[c.B] = (int)cu1;
    if (writes) {
      c.lens[b] = (int)(served ? s + n : s);
      c.cu[b] = (int)at.x;
      if (b == c.B - 1) c.cu[c.B] = (int)cu1;
    }
    // (pages go out from the first on, and where one request finds too few, so do all behind it that need any: the last one served says how many)
    if (served && need > 0) last = (int)off1;
    refused += !served && n > 0;
    at = make_uint2(cu1, off1);
  }
  if (writes) {                              // (one lane for all: atomics of 64 lanes are made one after the other; 575 requests of two tokens 10.9 us with them)
    const uint64_t some = __ballot(last > 0);
    if (some) last = __builtin_amdgcn_readlane(last, 63 - __clzll((long long)some));
    if (__any(refused)) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) refused += __shfl_xor(refused, d, 64);
    }
    if (lane == 0) {
      if (some) atomicMax(&s_last[0], last);
      if (refused) atomicAdd(&s_last[1], refused);
    }
  }
  __syncthreads();
  if (writes && tid < 2) c.taken[tid] = s_last[tid];

  const int64_t j0 = ((int64_t)blockIdx.x * kMapThreads + tid) * kMapTokens;
  if (j0 >= c.total) return;
  int lo = 0, hi = c.B;                      // s_cu[lo] <= j0, s_cu[hi] > j0 or hi = B
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s_cu[mid] <= (int)j0) lo = mid; else hi = mid;
  }
  int out[kMapTokens], b = lo;
#pragma unroll
  for (int k = 0; k < kMapTokens; k++) {
    const int j = (int)j0 + k;
    while (b < c.B && j >= s_cu[b + 1]) b++;
    out[k] = -1;
    if (b < c.B && s_off[b] >= 0) {
      const int s = s_seq[b], pos = s + (j - s_cu[b]), first = (s + ps1) >> c.shift, p = pos >> c.shift;
      int32_t* entry = c.table + (size_t)b * (unsigned)c.max_pages + (unsigned)p;
      int page;
      if (p >= first) {
        page = c.free_pages[s_off[b] + p - first];
        if ((pos & ps1) == 0) *entry = page;
      } else {
        page = *entry;
      }
      if ((unsigned)page < (unsigned)c.n_pages) out[k] = (page << c.shift) + (pos & ps1);
    }
  }
  if (j0 + kMapTokens <= c.total && ((uintptr_t)c.slot & 15) == 0) {
    *(int4*)(c.slot + j0) = make_int4(out[0], out[1], out[2], out[3]);
  } else {
#pragma unroll
    for (int k = 0; k < kMapTokens; k++)
      if (j0 + k < c.total) c.slot[j0 + k] = out[k];
  }
}

// ------------------------------------------------------------------------------------------------ write
struct WriteCtx {
  uint32_t T, pieces, inv_pieces;      // rows; 8-element pieces of a row
  uint32_t rows_wg;                    // rows of a workgroup
  uint32_t n_slots;
  int64_t k_stride, v_stride;          // elements between rows of the inputs
  float k_scale, v_scale, k_rcp, v_rcp;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* slot;
  void* k_pages;
  void* v_pages;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Eight bf16 values as E4M3 codes of x / scale: the division in fp32 as IEEE has it, saturated, rounded to nearest even; NaN stays NaN.
// FAST: the quotient from the scale's reciprocal r (rounded to nearest) and one correction by the exact remainder, q = q0 + (x - q0 scale) r with q0 = x r, which rounds as the
// division does (Markstein's theorem; of the 2^30 pairs of a scale's significand and a bf16 value's none differs from the division.  Powers of two beside them change nothing
// for scales from 2^-60 to 2^60, where the remainder of a value whose code is not 0 is far from underflow).
// q0 is held within +-512, so that an infinite one does not make the remainder NaN: the result saturates all the same.  16 x 60-700 rows of 8 x 128 from a fused projection
// 10.0 us with the division.
template <bool FAST>
__device__ __forceinline__ u32x2 codes8(u32x4 w, float scale, float r) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const float x = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    float y;
    if (FAST) {
      const float q0 = fminf(fmaxf(x * r, -512.f), 512.f);
      y = copysignf(fmaf(fmaf(-q0, scale, x), r, q0), x);        // (-0 lost its sign)
    } else {
      y = x / scale;
    }
    f[i] = x != x ? x : fminf(fmaxf(y, -448.f), 448.f);
  }
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], a, true);
  int b = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], 0, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], b, true);
  return u32x2{(uint32_t)a, (uint32_t)b};
}

// Bound: memory, 4 bytes an element in and out (FP8: 3).  A thread moves U pieces of 16 bytes of K and of V; all its rows are on their way before the
// slots are needed.
template <int FP8, int U>      // FP8: 0 bf16, 1 codes by the corrected reciprocal, 2 by the division
__global__ void __launch_bounds__(256) k_page_write(WriteCtx c) {
  const uint32_t row0 = blockIdx.x * c.rows_wg, n = min(c.rows_wg, c.T - row0) * c.pieces;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += 256 * U) {
    u32x4 kx[U], vx[U];
    int to[U];
    uint32_t piece[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const uint32_t i = min(i0 + 256 * u, n - 1), q = __umulhi(i, c.inv_pieces), r = q + (i - q * c.pieces >= c.pieces ? 1u : 0u);
      const size_t row = row0 + r;
      piece[u] = i - r * c.pieces;
      to[u] = i0 + 256 * u < n ? c.slot[row] : -1;
      kx[u] = *(const u32x4*)(c.k + (int64_t)row * c.k_stride + piece[u] * 8);
      vx[u] = *(const u32x4*)(c.v + (int64_t)row * c.v_stride + piece[u] * 8);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      if ((uint32_t)to[u] >= c.n_slots) continue;
      const size_t at = (size_t)(uint32_t)to[u] * c.pieces + piece[u];
      if (FP8) {
        ((u32x2*)c.k_pages)[at] = codes8<FP8 == 1>(kx[u], c.k_scale, c.k_rcp);
        ((u32x2*)c.v_pages)[at] = codes8<FP8 == 1>(vx[u], c.v_scale, c.v_rcp);
      } else {
        ((u32x4*)c.k_pages)[at] = kx[u];
        ((u32x4*)c.v_pages)[at] = vx[u];
      }
    }
  }
}

bool page_size_ok(int32_t ps) { return ps >= 16 && ps <= 1024 && (ps & (ps - 1)) == 0; }
bool scale_ok(float s) { return s > 0.f && s < INFINITY; }

}  // namespace

extern "C" gr_status gr_page_map(const gr_page_map_params* p, void* stream_) {
  if (!p) return GR_ERR_INVALID_ARG;
  if (p->B <= 0 || p->max_pages <= 0 || p->n_free < 0 || p->n_pages <= 0 || p->total_new < 0) return GR_ERR_INVALID_ARG;
  if (!p->seq_lens || !p->new_lens || !p->block_table || !p->lens_out || !p->cu_new || !p->taken) return GR_ERR_INVALID_ARG;
  if ((p->n_free > 0 && !p->free_pages) || (p->total_new > 0 && !p->slot)) return GR_ERR_INVALID_ARG;
  if (p->lens_out == p->seq_lens || p->lens_out == p->new_lens || p->cu_new == p->seq_lens || p->cu_new == p->new_lens) return GR_ERR_INVALID_ARG;
  if (((uintptr_t)p->seq_lens | (uintptr_t)p->new_lens | (uintptr_t)p->free_pages | (uintptr_t)p->block_table | (uintptr_t)p->lens_out |
       (uintptr_t)p->cu_new | (uintptr_t)p->slot | (uintptr_t)p->taken) & 3)
    return GR_ERR_INVALID_ARG;
  if (!page_size_ok(p->page_size) || p->B > kMapMaxB) return GR_ERR_UNSUPPORTED;
  if (p->total_new >= ((int64_t)1 << 31) - 1024 || (int64_t)p->max_pages * p->page_size >= ((int64_t)1 << 31) ||
      (int64_t)p->n_pages * p->page_size >= ((int64_t)1 << 31))
    return GR_ERR_UNSUPPORTED;                                 // positions and slots are 32-bit numbers
  MapCtx c;
  c.B = p->B; c.shift = __builtin_ctz((unsigned)p->page_size); c.max_pages = p->max_pages; c.n_free = p->n_free; c.n_pages = p->n_pages;
  c.total = (int)p->total_new;
  c.seq = p->seq_lens; c.fresh = p->new_lens; c.free_pages = p->free_pages; c.table = p->block_table; c.lens = p->lens_out; c.cu = p->cu_new;
  c.slot = p->slot; c.taken = p->taken;
  const int64_t per_wg = kMapThreads * kMapTokens, grid = p->total_new > 0 ? (p->total_new + per_wg - 1) / per_wg : 1;
  hipLaunchKernelGGL(k_page_map, dim3((unsigned)grid), dim3(kMapThreads), (size_t)(3 * p->B + 1) * 4, (hipStream_t)stream_, c);
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}

extern "C" gr_status gr_page_write(const gr_page_write_params* p, void* stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  if (!p) return GR_ERR_INVALID_ARG;
  if (p->T < 0 || p->Hkv <= 0 || p->d <= 0 || p->n_pages <= 0) return GR_ERR_INVALID_ARG;
  if (p->kv_type != GR_KV_BF16 && p->kv_type != GR_KV_FP8) return GR_ERR_INVALID_ARG;
  const bool fp8 = p->kv_type == GR_KV_FP8;
  if (fp8 && (!scale_ok(p->k_scale) || !scale_ok(p->v_scale))) return GR_ERR_INVALID_ARG;
  const int64_t n = (int64_t)p->Hkv * p->d;
  if (!p->k_pages || !p->v_pages || p->k_pages == p->v_pages) return GR_ERR_INVALID_ARG;
  if (p->T > 0 && (!p->k || !p->v || !p->slot)) return GR_ERR_INVALID_ARG;
  if (p->k_stride < n || p->v_stride < n) return GR_ERR_INVALID_ARG;
  if (((uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->k_pages | (uintptr_t)p->v_pages) & 15 || ((uintptr_t)p->slot & 3)) return GR_ERR_INVALID_ARG;
  if (!page_size_ok(p->page_size) || n % 8 || p->k_stride % 8 || p->v_stride % 8 || n > 1 << 20) return GR_ERR_UNSUPPORTED;
  if ((int64_t)p->n_pages * p->page_size >= ((int64_t)1 << 31) || p->T >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  if (p->T == 0) return GR_OK;
  WriteCtx c;
  c.T = (uint32_t)p->T; c.pieces = (uint32_t)(n / 8); c.inv_pieces = 0xffffffffu / c.pieces;
  c.n_slots = (uint32_t)(p->n_pages * p->page_size);
  c.k_stride = p->k_stride; c.v_stride = p->v_stride; c.k_scale = p->k_scale; c.v_scale = p->v_scale; c.k_rcp = 1.0f / p->k_scale; c.v_rcp = 1.0f / p->v_scale;
  c.k = (const uint16_t*)p->k; c.v = (const uint16_t*)p->v; c.slot = p->slot; c.k_pages = p->k_pages; c.v_pages = p->v_pages;
  const int64_t all = (int64_t)c.T * c.pieces;
  const int u = all >= (int64_t)256 * 4 * 512 ? 4 : 1;
  c.rows_wg = (uint32_t)((256 * u + c.pieces - 1) / c.pieces);
  const unsigned grid = (c.T + c.rows_wg - 1) / c.rows_wg;
  if (!gr_grid_fits(grid, 256)) return GR_ERR_UNSUPPORTED;
#define GR_LAUNCH(F, U_) hipLaunchKernelGGL((k_page_write<F, U_>), dim3(grid), dim3(256), 0, stream, c)
  auto ordinary = [](float s) { return s >= 0x1p-60f && s <= 0x1p60f; };
  const int type = !fp8 ? 0 : ordinary(p->k_scale) && ordinary(p->v_scale) ? 1 : 2;
  if (u == 4) { if (type == 0) GR_LAUNCH(0, 4); else if (type == 1) GR_LAUNCH(1, 4); else GR_LAUNCH(2, 4); }
  else { if (type == 0) GR_LAUNCH(0, 1); else if (type == 1) GR_LAUNCH(1, 1); else GR_LAUNCH(2, 1); }
#undef GR_LAUNCH
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
