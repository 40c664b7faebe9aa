// gr_page_map, gr_page_write, gr_page_read: a prompt cache kept in pages of a pool.
//
// Request b has s_b tokens in its pages and gets n_b more.  With ps tokens to a page it needs
//     need_b = ceil((s_b + n_b) / ps) - ceil(s_b / ps)
// fresh pages; off_b, the sum of need over the requests before it, is where they begin in the list of free pages, and cu_b, the sum of n,
// where its tokens begin among the new ones.  Both sums are of whole numbers in a fixed order, so the same lengths and the same free list
// always give the same tables.
#include <type_traits>
#include "gr_pages.hpp"

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

// Eight bf16 values as E4M3 codes of x / scale: the division in fp32 as IEEE has it, saturated, rounded to nearest even; NaN stays NaN.
template <bool FAST>
__device__ __forceinline__ kv_u32x2 codes8(kv_u32x4 w, float scale, float r) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; i++) f[i] = fp8_quotient<FAST>(bf16_at(w[i / 2], i & 1), scale, r);
  return kv_u32x2{fp8_codes4(f[0], f[1], f[2], f[3]), fp8_codes4(f[4], f[5], f[6], f[7])};
}

// Bound: memory, 4 bytes an element in and out (FP8: 3).  A thread moves U pieces of 16 bytes of K and of V; all its rows are on their way before the
// slots are needed.
template <int FP8, int U>      // FP8: 0 bf16, 1 codes by the corrected reciprocal, 2 by the division
__global__ void __launch_bounds__(256) k_page_write(WriteCtx c) {
  const uint32_t row0 = blockIdx.x * c.rows_wg, n = min(c.rows_wg, c.T - row0) * c.pieces;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += 256 * U) {
    kv_u32x4 kx[U], vx[U];
    int to[U];
    uint32_t piece[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const uint32_t i = min(i0 + 256 * u, n - 1), q = __umulhi(i, c.inv_pieces), r = q + (i - q * c.pieces >= c.pieces ? 1u : 0u);
      const size_t row = row0 + r;
      piece[u] = i - r * c.pieces;
      to[u] = i0 + 256 * u < n ? c.slot[row] : -1;
      kx[u] = *(const kv_u32x4*)(c.k + (int64_t)row * c.k_stride + piece[u] * 8);
      vx[u] = *(const kv_u32x4*)(c.v + (int64_t)row * c.v_stride + piece[u] * 8);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      if ((uint32_t)to[u] >= c.n_slots) continue;
      const size_t at = (size_t)(uint32_t)to[u] * c.pieces + piece[u];
      if (FP8) {
        ((kv_u32x2*)c.k_pages)[at] = codes8<FP8 == 1>(kx[u], c.k_scale, c.k_rcp);
        ((kv_u32x2*)c.v_pages)[at] = codes8<FP8 == 1>(vx[u], c.v_scale, c.v_rcp);
      } else {
        ((kv_u32x4*)c.k_pages)[at] = kx[u];
        ((kv_u32x4*)c.v_pages)[at] = vx[u];
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ read
struct ReadCtx {
  uint32_t T, chunks, inv_chunks;      // rows; workgroups of a row's heads
  int Hkv, d, shift;
  uint32_t n_slots;
  int64_t k_stride, v_stride;
  float k_scale, v_scale;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const int32_t* slot;
  uint16_t* k;
  uint16_t* v;
};

// Bound: memory, 4 bytes an element in and out (FP8 3, FP4 2.5).  A lane takes 16 consecutive elements of a head, a wavefront the same head of 64 / LG consecutive rows: of
// FP4 pages, whose tokens of a head lie together, it reads runs of codes and of scales.  Two heads a wavefront: 32 x 4096 tokens of 8 heads of 128 out of FP4 124 us (5.5 TB/s; a copy
// of 1 GiB reaches 5.15), 32 prompts of 512-3700 tokens 78 us (4.7); one 130 and 79, four 159 and 95.
constexpr int kReadHeads = 2;
template <int LG, int KV>
__global__ void __launch_bounds__(256) k_page_read(ReadCtx c) {
  uint32_t group = __umulhi(blockIdx.x, c.inv_chunks);
  group += blockIdx.x - group * c.chunks >= c.chunks ? 1u : 0u;
  const uint32_t chunk = blockIdx.x - group * c.chunks;
  const int lane = (int)threadIdx.x & 63, heads = 2 * c.Hkv;
  const uint32_t row = group * (64 / LG) + (uint32_t)(lane / LG), e0 = (uint32_t)(lane % LG) * 16, d = (uint32_t)c.d;
  if (row >= c.T || e0 >= d) return;
  const uint32_t slot = (uint32_t)c.slot[row];
  if (slot >= c.n_slots) return;
  const int h0 = ((int)chunk * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)) * kReadHeads;
  kv_u32x4 y[kReadHeads][2];
  uint32_t power[kReadHeads];
#pragma unroll
  for (int u = 0; u < kReadHeads; u++) {
    const int h = min(h0 + u, heads - 1);
    const bool is_k = h < c.Hkv;
    const unsigned hk = (unsigned)(is_k ? h : h - c.Hkv);
    const uint8_t* pages = is_k ? c.k_pages : c.v_pages;
    if (KV == GR_KV_FP4) {
      const uint32_t ps = 1u << c.shift, tok = slot & (ps - 1);
      const uint8_t* record = pages + ((size_t)(slot >> c.shift) * (unsigned)c.Hkv + hk) * gr_fp4_record(ps, d);
      const kv_u32x2 w = *(const kv_u32x2*)(record + tok * (d / 2) + e0 / 2);
      y[u][0] = kv_u32x4{w[0], w[1], 0, 0};
      power[u] = record[gr_fp4_codes(ps, d) + tok * (d / 32) + e0 / 32];
    } else {
      const uint8_t* from = pages + (((size_t)slot * (unsigned)c.Hkv + hk) * d + e0) * (KV == GR_KV_FP8 ? 1 : 2);
      y[u][0] = *(const kv_u32x4*)from;
      if (KV == GR_KV_BF16) y[u][1] = *(const kv_u32x4*)(from + 16);
    }
  }
#pragma unroll
  for (int u = 0; u < kReadHeads; u++) {
    const int h = h0 + u;
    if (h >= heads) return;
    const bool is_k = h < c.Hkv;
    if (KV == GR_KV_FP4) {
      const uint32_t w[2] = {y[u][0][0], y[u][0][1]};
#pragma unroll
      for (int p = 0; p < 2; p++) y[u][p] = power[u] == 255u ? kv_u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u} : fp4_values8(w[p], power[u]);      // (255: no numbers)
    } else if (KV == GR_KV_FP8) {
      const kv_u32x4 w = y[u][0];
      const float scale = is_k ? c.k_scale : c.v_scale;
#pragma unroll
      for (int k = 0; k < 4; k++) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
        y[u][k / 2][2 * (k % 2)] = bf16_pair(lo[0] * scale, lo[1] * scale);
        y[u][k / 2][2 * (k % 2) + 1] = bf16_pair(hi[0] * scale, hi[1] * scale);
      }
    }
    kv_u32x4* to = (kv_u32x4*)(is_k ? c.k + (int64_t)row * c.k_stride + h * c.d + e0 : c.v + (int64_t)row * c.v_stride + (h - c.Hkv) * c.d + e0);
    to[0] = y[u][0];
    to[1] = y[u][1];
  }
}

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
  if (!gr_page_size_ok(p->page_size) || p->B > kMapMaxB) return GR_ERR_UNSUPPORTED;
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
  if (fp8 && (!gr_scale_ok(p->k_scale) || !gr_scale_ok(p->v_scale))) return GR_ERR_INVALID_ARG;
  const int64_t n = (int64_t)p->Hkv * p->d;
  if (!p->k_pages || !p->v_pages || p->k_pages == p->v_pages) return GR_ERR_INVALID_ARG;
  if (p->T > 0 && (!p->k || !p->v || !p->slot)) return GR_ERR_INVALID_ARG;
  if (p->k_stride < n || p->v_stride < n) return GR_ERR_INVALID_ARG;
  if (((uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->k_pages | (uintptr_t)p->v_pages) & 15 || ((uintptr_t)p->slot & 3)) return GR_ERR_INVALID_ARG;
  if (!gr_page_size_ok(p->page_size) || n % 8 || p->k_stride % 8 || p->v_stride % 8 || n > 1 << 20) return GR_ERR_UNSUPPORTED;
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

extern "C" size_t gr_kv_fp4_page_bytes(int32_t page_size, int32_t d) {
  return gr_page_size_ok(page_size) && d > 0 && d % 32 == 0 && d <= 256 ? gr_fp4_record((uint32_t)page_size, (uint32_t)d) : 0;
}

extern "C" gr_status gr_page_read(const gr_page_read_params* p, void* stream_) {
  if (!p) return GR_ERR_INVALID_ARG;
  if (p->T < 0 || p->Hkv <= 0 || p->d <= 0 || p->n_pages <= 0) return GR_ERR_INVALID_ARG;
  if (p->kv_type != GR_KV_BF16 && p->kv_type != GR_KV_FP8 && p->kv_type != GR_KV_FP4) return GR_ERR_INVALID_ARG;
  if (p->kv_type == GR_KV_FP8 && (!gr_scale_ok(p->k_scale) || !gr_scale_ok(p->v_scale))) return GR_ERR_INVALID_ARG;
  const int64_t n = (int64_t)p->Hkv * p->d;
  if (!p->k_pages || !p->v_pages) return GR_ERR_INVALID_ARG;
  if (p->T > 0 && (!p->k || !p->v || !p->slot || p->k == p->v)) return GR_ERR_INVALID_ARG;
  for (const void* out : {p->k, p->v})
    if (out && (out == p->k_pages || out == p->v_pages || out == p->slot)) return GR_ERR_INVALID_ARG;
  if (p->k_stride < n || p->v_stride < n) return GR_ERR_INVALID_ARG;
  if (((uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->k_pages | (uintptr_t)p->v_pages) & 15 || ((uintptr_t)p->slot & 3)) return GR_ERR_INVALID_ARG;
  if (!gr_page_size_ok(p->page_size) || p->d % 16 || p->d > 256 || p->k_stride % 8 || p->v_stride % 8 || n > 1 << 20) return GR_ERR_UNSUPPORTED;
  if (p->kv_type == GR_KV_FP4 && p->d % 32) return GR_ERR_UNSUPPORTED;
  if ((int64_t)p->n_pages * p->page_size >= ((int64_t)1 << 31) || p->T >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  if (p->T == 0) return GR_OK;
  ReadCtx c;
  c.T = (uint32_t)p->T; c.Hkv = p->Hkv; c.d = p->d; c.shift = __builtin_ctz((unsigned)p->page_size); c.n_slots = (uint32_t)(p->n_pages * p->page_size);
  c.k_stride = p->k_stride; c.v_stride = p->v_stride; c.k_scale = p->k_scale; c.v_scale = p->v_scale;
  c.k_pages = (const uint8_t*)p->k_pages; c.v_pages = (const uint8_t*)p->v_pages; c.slot = p->slot; c.k = (uint16_t*)p->k; c.v = (uint16_t*)p->v;
  auto go = [&](auto lanes, auto type) {
    constexpr int LG = decltype(lanes)::value, KV = decltype(type)::value;
    c.chunks = (uint32_t)((2 * p->Hkv + 4 * kReadHeads - 1) / (4 * kReadHeads));
    c.inv_chunks = 0xffffffffu / c.chunks;
    const int64_t grid = (p->T + 64 / LG - 1) / (64 / LG) * c.chunks;
    if (!gr_grid_fits(grid, 256)) return (gr_status)GR_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((k_page_read<LG, KV>), dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream_, c);
    return (gr_status)GR_OK;
  };
  auto of_type = [&](auto lanes) {
    return p->kv_type == GR_KV_BF16  ? go(lanes, std::integral_constant<int, GR_KV_BF16>())
           : p->kv_type == GR_KV_FP8 ? go(lanes, std::integral_constant<int, GR_KV_FP8>())
                                     : go(lanes, std::integral_constant<int, GR_KV_FP4>());
  };
  const gr_status st = p->d <= 64    ? of_type(std::integral_constant<int, 4>())
                       : p->d <= 128 ? of_type(std::integral_constant<int, 8>())
                                     : of_type(std::integral_constant<int, 16>());
  if (st) return st;
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
