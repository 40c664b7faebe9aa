// What the kernels over pages in bf16 and FP8 (gr_paged.hip) and in FP4 (gr_paged4.hip) have in common: the launch and its rule, and the kernel that joins partials.  Not part of the ABI.
#pragma once
#include <math.h>
#include "gr_attn_rows.hpp"
#include "gr_pages.hpp"

namespace {

// Joins a row's partials: those of part 0, whose rows are all requests' in one, then those of part 1.  A lane takes four columns of a row; eight rows of eight
// neighbouring lanes are a line.  Four segments are requested together.
struct JoinCtx {
  int B, W, Hq, Hkv, g, ns0, ns1;     // segments of part 0 and of part 1
  const float* part_o;
  const float* part_ml;
  uint16_t* out;
  float* lse;
};
template <int D>
__global__ void __launch_bounds__(256) k_paged_join(JoinCtx c) {
  constexpr int RPW = 1024 / D;
  static_assert(RPW % 8 == 0 && 32 % RPW == 0, "whole lines of one block");
  const unsigned M = (unsigned)(c.W * c.g), per_pair = (M + RPW - 1) / RPW, pair = blockIdx.x / per_pair;
  const unsigned b = pair / (unsigned)c.Hkv, kvh = pair - b * (unsigned)c.Hkv;
  const int t = (int)threadIdx.x, piece = (t >> 3) % (D / 4);
  const unsigned r = (blockIdx.x - pair * per_pair) * RPW + (unsigned)((t & 7) + 8 * (t / (2 * D)));
  if (r >= M) return;
  const int ns0 = c.ns0, ns = ns0 + c.ns1;
  const unsigned M0 = (unsigned)c.B * M, r0 = b * M + r;
  auto row_of = [&](int s) {
    return s < ns0 ? ((size_t)(unsigned)s * (unsigned)c.Hkv + kvh) * M0 + r0
                   : (size_t)(unsigned)ns0 * (unsigned)c.Hkv * M0 + (((size_t)b * (unsigned)c.ns1 + (unsigned)(s - ns0)) * (unsigned)c.Hkv + kvh) * M + r;
  };
  float M2 = -INFINITY, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
#pragma unroll 1
  for (int s0 = 0; s0 < ns; s0 += U) {
    f32x2 ml[U];
    f32x4 o[U];
#pragma unroll
    for (int k = 0; k < U; k++) {
      const int s = min(s0 + k, ns - 1);
      const unsigned rr = s < ns0 ? r0 : r, all = s < ns0 ? M0 : M, left = min(32u, all - (rr & ~31u));
      const size_t row = row_of(s);
      ml[k] = *(const f32x2*)(c.part_ml + row * 2);
      o[k] = *(const f32x4*)(c.part_o + (row - (rr & 31)) * D + 4 * (piece * left + (rr & 31)));
    }
    float mx = M2;
#pragma unroll
    for (int k = 0; k < U; k++) {
      if (s0 + k >= ns) ml[k].y = 0.f;           // (a repeated segment counts nothing)
      if (ml[k].y > 0.f) mx = fmaxf(mx, ml[k].x);
    }
    if (!(mx > -INFINITY)) continue;
    const float alpha = __builtin_amdgcn_exp2f(M2 - mx);
    L *= alpha;
#pragma unroll
    for (int e = 0; e < 4; e++) acc[e] *= alpha;
#pragma unroll
    for (int k = 0; k < U; k++) {
      if (!(ml[k].y > 0.f)) continue;
      const float sc = __builtin_amdgcn_exp2f(ml[k].x - mx);
      L += ml[k].y * sc;
#pragma unroll
      for (int e = 0; e < 4; e++) acc[e] += o[k][e] * sc;
    }
    M2 = mx;
  }
  const float inv = L > 0.f ? 1.0f / L : 0.f;
  bf16x4 h;
#pragma unroll
  for (int e = 0; e < 4; e++) h[e] = (__bf16)(acc[e] * inv);
  const unsigned w = r / (unsigned)c.g;
  const size_t row = ((size_t)b * (unsigned)c.W + w) * (unsigned)c.Hq + kvh * (unsigned)c.g + (r - w * (unsigned)c.g);
  *(bf16x4*)(c.out + row * D + 4 * piece) = h;
  if (c.lse && piece == 0) c.lse[row] = L > 0.f ? (M2 + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

// The launch.  rows: of a workgroup of part 1 (32, 128, 256); ns: segments of the prefix in part 0 (0: there is none) and of the list in part 1; ks and find as in gr_beam_attn.
struct PagedPlan { int rows, ns[2], ks; bool find; };

// More than 80 rows of a (request, KV head) pair are launched as gr_beam_attn launches them, and never share a prefix: part 1 exists in blocks of 32 rows alone.  For fewer, the cheapest of these is taken, by their estimated time in us: blocks of 32 rows or of 128
// over the whole list, or the prefix packed, each with 1 to 16 segments.  The estimate of a launch is `start`, and (the fourth root of the sum of the fourth powers: a little more than the longer) of
//   - what its keys take at `rate`;
//   - its workgroups' time: `few` + `few_step` for every 128 tokens (blocks of 32), `unit` + `tile1` for every 64 (128; two sets of wavefronts where there is at most one workgroup per CU:
//     `tile2` for every 128), `shared` + `shared_tile` for every 64 (part 0), times the rounds that an XCD's 32 CUs take them in (`few_per_cu` workgroups to a CU, two of part 0 and 1);
// and, where there are several segments, `join` and the partials written and read at 2.7 TB/s.  Fitted to 870 random calls of 1 to 128 requests of 10 to 16384 tokens with 1 to 80 rows,
// 430 of them behind a prefix of 64 to 8192 tokens, each timed in up to 40 ways: the mean call takes 1.03 times the best of them, the worst 1.63, and 120 others 1.047 and 1.35 (packed wherever that saves half of the
// blocks, with segments for about one or two workgroups per CU, 1.07 without a prefix and 1.14 with one; with the longer of the two times alone 16 requests of 1500-3000 tokens x 8 beams
// took 49.0 us in one segment each, now 39.7 in two, 64 x 8 of 2 KV heads 46.6, 40.7).  One call in twenty takes more than 1.15 times its best: mostly lists of thousands of tokens and
// ragged lengths of head size 64, left in one segment (53 requests of 972-4736 x 1 beam of 8 heads in FP8 79 us, 57 in eight; 28 of 642-7763 x 54 in bf16 92, 66 in three), a few long lists in
// sixteen (6 of 2342 x 2, 16 and 4 heads of 128, 17.9, 13.8 in eight), and prefixes of 64-800 tokens packed, or not, the wrong way (58 requests of 604 x 24 behind 512, 8 heads of 64, 27.5,
// 21.3 not packed).
struct PagedCost { double start, few, few_step, few_per_cu, unit, tile1, tile2, shared, shared_tile, join, rate; };
constexpr PagedCost kPagedCost[2][2] = {      // [head size 128][FP8]; rate in bytes a us
    {{3.3, 1.5, 1.2, 2.0, 2.0, 1.05, 0.95, 1.5, 0.7, 3.1, 8.0e6}, {3.3, 1.5, 1.4, 2.0, 2.0, 1.05, 0.95, 1.5, 0.8, 3.1, 4.0e6}},
    {{0.7, 0.15, 1.9, 1.95, 2.1, 0.9, 1.25, 0.4, 0.9, 1.95, 7.9e6}, {1.5, 2.35, 2.05, 1.6, 4.0, 1.45, 1.35, 1.25, 0.9, 2.2, 5.4e6}}};

// FP4: the same choice by estimated time, for any number of rows: blocks of 16 rows (32 for more than 16) with four or, ks = 2, eight wavefronts for up to 160 rows of a pair, of 128 (ks = 2 with
// two sets of wavefronts where there is at most one to a CU) for more than 24, of 256 for more than 128, each with 1 to 16 (32) segments, and up to 80 rows the prefix packed.  A block's time is a
// fixed part and a step for its tokens, 128 of them (few16, few32; `eight` more, and half the steps, with eight wavefronts) or 64 (rows128, two sets, rows256), times the rounds that an XCD's 32 CUs
// take the blocks in, between their number (weight 1 - ceil) and the whole one above (weight ceil), with per_cu16, per_cu32, 2, 1 and 1 blocks to a CU; the fourth root of the sum of its fourth power and
// that of the keys' time at `rate`; and for several segments `join`, `join_one` for each, and partials at `partials` bytes a us.
// Fitted to half of 13450 random calls of 1 to 128 requests of 10 to 16384 tokens with 1 to 2048 rows, half of them behind a prefix of 64 to 8192 tokens, each timed in up to 50 ways: of the other half
// the mean call takes 1.019 times the best of its ways, one in twenty more than 1.11, the worst 1.6 (a few ragged or very long lists left in one segment).  With gr_beam_attn's rule for FP8 the calls
// of more than 80 rows took 1.043 times their best (16 x 4000 tokens x 200 beams 240 us in blocks of 128 rows, which widen every key more often, 229 in blocks of 256).
struct Fp4Cost {
  double start, few16, step16, per_cu16, few32, step32, per_cu32, eight, ceil_few, rows128, tile128, sets, tile_sets, rows256, tile256, ceil_rows, shared, shared_tile, join, join_one, partials, rate;
};
constexpr Fp4Cost kFp4Cost[2] = {{4.23, 1.70, 0.562, 3.67, 2.36, 0.725, 1.88, 0.38, 0.30, 2.96, 1.05, 1.97, 1.12, 3.08, 1.05, 0.45, 1.09, 0.66, 1.44, 0.26, 4.0e6, 4.8e6},
                                 {6.02, 1.42, 0.763, 1.88, 2.36, 1.115, 1.76, 0.56, 0.18, 1.82, 1.49, 2.38, 1.58, 4.10, 1.25, 0.67, 0.76, 1.27, 1.20, 0.21, 3.8e6, 6.75e6}};
PagedPlan plan_fp4(const gr_attn_paged_params* p) {
  PagedPlan plan{};
  const int64_t M = (int64_t)p->W * (p->Hq / p->Hkv), all = p->B * M, pairs = (int64_t)p->B * p->Hkv, list = (int64_t)p->prefix_L + p->max_L;
  const Fp4Cost& c = kFp4Cost[p->d == 128];
  const int rows = M <= 16 ? 16 : 32;
  const double few0 = rows == 16 ? c.few16 : c.few32, step = rows == 16 ? c.step16 : c.step32, per_cu = rows == 16 ? c.per_cu16 : c.per_cu32;
  const double partial_us = 2.0 * p->B * p->W * p->Hq * p->d * 4 / c.partials, token_bytes = 17.0 / 16 * p->Hkv * p->d;
  auto parts = [](int64_t n, int64_t of) { return (n + of - 1) / of; };
  auto larger = [](double a, double b) { return a > b ? a : b; };
  auto both = [](double a, double b) { return sqrt(sqrt(a * a * a * a + b * b * b * b)); };
  auto rounds = [&](double blocks, double places, double weight) { return larger(1.0, weight * ceil(blocks / places) + (1.0 - weight) * (blocks / places)); };
  double least = 0;
  auto look_at = [&](int r, int n0, int n1, int ks, double us) {
    const int n = n0 + n1;
    us += n > 1 ? c.join + (c.join_one + partial_us) * n : 0.0;
    if (plan.rows && !(us < least)) return;
    least = us;
    plan.rows = r; plan.ns[0] = n0; plan.ns[1] = n1; plan.ks = ks;
  };
  const double list_us = list * p->B * token_bytes / c.rate;
  for (const int n : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
    if (n > 1 && n * 64 > list) break;
    const double tiles = (double)parts(parts(list, n), KT);
    const int64_t on_xcd = parts(pairs * n, 8);
    if (M <= 160) {
      for (const int ks : {1, 2}) {
        const double few = few0 + step * tiles / (2 * ks) + (ks == 2 ? c.eight : 0.0);
        look_at(rows, 0, n, ks, both(few * rounds((double)(on_xcd * parts(M, rows) * ks), 32 * per_cu, c.ceil_few), list_us));
      }
    }
    if (M <= 24 || n > 16 || (n > 1 && n * 96 > list)) continue;
    for (const int r : {128, 256}) {
      const int64_t units = pairs * parts(M, r) * n, of_xcd = on_xcd * parts(M, r);
      if ((r == 256 && M <= 128) || (n > 1 && units > 1100)) continue;
      const bool sets = r == 128 && units <= 256 && list > KT;
      const double unit = r == 256 ? c.rows256 + c.tile256 * tiles : sets ? c.sets + c.tile_sets * (double)(((int64_t)tiles + 1) >> 1) : c.rows128 + c.tile128 * tiles;
      look_at(r, 0, n, sets ? 2 : 1, both(unit * rounds((double)of_xcd, r == 256 || sets ? 32 : 64, c.ceil_rows), list_us));
    }
  }
  // packed, as the beams of one request (offsets inside its rows fit 32 bits)
  if (M <= 80 && p->prefix_L > 0 && p->B > 1 && all < ((int64_t)1 << 22) && all * p->Hkv * p->d < ((int64_t)1 << 31)) {
    const double packed_us = (p->prefix_L + (double)p->max_L * p->B) * token_bytes / c.rate;
    for (const int n0 : {1, 2, 3, 4, 6, 8, 12, 16}) {
      if (n0 > 1 && n0 * 96 > p->prefix_L) break;
      const double shared = c.shared + c.shared_tile * (double)parts(parts(p->prefix_L, n0), KT), shared_blocks = (double)(parts((int64_t)p->Hkv * n0, 8) * parts(all, 128));
      for (const int n1 : {1, 2, 4}) {
        if (n1 > 1 && n1 * 128 > p->max_L) break;
        const double few = few0 + step * (double)parts(parts(p->max_L, n1), KT) / 2, few_blocks = (double)(parts(pairs * n1, 8) * parts(M, rows));
        look_at(rows, n0, n1, 1, both(larger(larger(few, shared), (shared * shared_blocks + few * few_blocks * 2 / per_cu) / 64), packed_us));
      }
    }
  }
  plan.find = plan.rows >= 128 && plan.ks == 1 && pairs * parts(M, plan.rows) * plan.ns[1] > 256 && p->B >= 2 && p->B <= kRankB;
  return plan;
}

PagedPlan plan_paged(const gr_attn_paged_params* p) {
  if (p->kv_type == GR_KV_FP4) return plan_fp4(p);
  PagedPlan plan{};
  const int64_t g = p->Hq / p->Hkv, M = p->W * g, all = p->B * M, pairs = (int64_t)p->B * p->Hkv;
  const bool kv8 = p->kv_type == GR_KV_FP8;
  auto parts = [](int64_t n, int64_t of) { return (n + of - 1) / of; };
  if (M > 80) {
    gr_attn_params q{};
    q.B = p->B; q.W = p->W; q.Hq = p->Hq; q.Hkv = p->Hkv; q.d = p->d; q.max_L = p->prefix_L + p->max_L;
    q.total_L = (int64_t)q.B * q.max_L;                      // (the lengths are on the GPU)
    const AttnPlan a = plan_attn(&q, kv8);
    plan.rows = a.mwg; plan.ns[1] = a.nsplit; plan.ks = a.ks;
    plan.find = a.many && a.ks == 1 && p->B >= 2 && p->B <= kRankB;
    return plan;
  }
  const PagedCost& c = kPagedCost[p->d == 128][kv8];
  const double partial_us = 2.0 * p->B * p->W * p->Hq * p->d * 4 / 2.7e6, token_bytes = 2.0 * p->Hkv * p->d * (kv8 ? 1 : 2);
  constexpr int kCounts[] = {1, 2, 3, 4, 6, 8, 12, 16};
  double least = 0;
  auto look_at = [&](int rows, int n0, int n1, int ks, double us) {
    const int n = n0 + n1;
    us += n > 1 ? c.join + partial_us * n : 0.0;
    if (plan.rows && !(us < least)) return;
    least = us;
    plan.rows = rows; plan.ns[0] = n0; plan.ns[1] = n1; plan.ks = ks;
  };
  auto larger = [](double a, double b) { return a > b ? a : b; };
  auto both = [](double a, double b) { return sqrt(sqrt(a * a * a * a + b * b * b * b)); };
  const int64_t list = (int64_t)p->prefix_L + p->max_L;
  const double list_us = list * p->B * token_bytes / c.rate;
  for (const int n : kCounts) {
    if (n > 1 && n * 96 > list) break;
    const double tiles = (double)parts(parts(list, n), KT);
    const double few = (c.few + c.few_step * tiles / 2) * larger(1.0, parts(pairs * n, 8) * parts(M, 32) / (32 * c.few_per_cu));
    look_at(32, 0, n, 1, both(few, list_us));
    const bool sets = list > KT && pairs * parts(M, 128) * n <= 256;
    const int64_t on_xcd = parts(pairs * n, 8) * parts(M, 128);
    const double unit = sets ? (c.unit + c.tile2 * (double)(((int64_t)tiles + 1) >> 1)) * (double)parts(on_xcd, 32) : (c.unit + c.tile1 * tiles) * larger(1.0, on_xcd / 64.0);
    look_at(128, 0, n, sets ? 2 : 1, both(unit, list_us));
  }
  // packed, as the beams of one request (offsets inside its rows fit 32 bits)
  if (p->prefix_L > 0 && p->B > 1 && all < ((int64_t)1 << 22) && (int64_t)p->B * p->W * p->Hq * p->d < ((int64_t)1 << 31)) {
    for (const int n0 : kCounts) {
      if (n0 > 1 && n0 * 96 > p->prefix_L) break;
      const double shared = c.shared + c.shared_tile * (double)parts(parts(p->prefix_L, n0), KT), shared_all = shared * (double)(parts((int64_t)p->Hkv * n0, 8) * parts(all, 128));
      for (const int n1 : {1, 2, 4}) {
        if (n1 > 1 && n1 * 128 > p->max_L) break;
        const double few = c.few + c.few_step * (double)parts(parts(p->max_L, n1), KT) / 2;
        look_at(32, n0, n1, 1, larger(larger(few, shared), (shared_all + few * (double)(parts(pairs * n1, 8) * parts(M, 32))) / 64));
      }
    }
  }
  plan.find = plan.rows == 128 && plan.ks == 1 && pairs * parts(M, 128) * plan.ns[1] > 256 && p->B >= 2 && p->B <= kRankB;
  return plan;
}

size_t paged_workspace(const gr_attn_paged_params* p, const PagedPlan& plan) {
  const int n = plan.ns[0] + plan.ns[1];                     // (a packed prefix always joins: part 1 has the lists and the own tokens)
  if (n == 1) return 0;
  const size_t rows = (size_t)p->B * p->W * p->Hq * n;
  return gr_align256(rows * p->d * 4) + gr_align256(rows * 8);
}

constexpr int64_t kMaxKeys = (int64_t)1 << 30;               // request_of_rank looks no further (a table may name the same page again and again)
bool shapes_ok(const gr_attn_paged_params* p) {
  return p->B > 0 && p->W > 0 && p->Hq > 0 && p->Hkv > 0 && p->d > 0 && p->Hq % p->Hkv == 0 && p->page_size > 0 && p->prefix_L >= 0 && p->max_L >= 0 &&
         (int64_t)p->prefix_L + p->max_L < kMaxKeys;
}

template <auto KERNEL, class... Args>
gr_status launch(size_t lds, unsigned threads, unsigned grid, hipStream_t stream, const Args&... args) {
  if (const gr_status st = gr_allow_lds<KERNEL>(lds)) return st;
  hipLaunchKernelGGL(KERNEL, dim3(grid), dim3(threads), lds, stream, args...);
  return GR_OK;
}

// One call, whose arguments have been looked at.  kernels(plan, c0, c, grid, blocks0): launches the kernel of the plan: c0, c: the arguments of part 0 and part 1.
template <class Kernels>
gr_status run_paged(const gr_attn_paged_params* p, void* workspace, size_t workspace_bytes, hipStream_t stream, Kernels&& kernels) {
  const bool kv8 = p->kv_type == GR_KV_FP8;
  const int64_t g = p->Hq / p->Hkv;
  const PagedPlan plan = plan_paged(p);
  const bool pack = plan.ns[0] > 0;
  const int64_t M1 = p->W * g, M0 = p->B * M1;
  AttnCtx c;                                                  // part 1
  c.B = p->B; c.W = p->W; c.Hq = p->Hq; c.Hkv = p->Hkv; c.g = (int)g; c.ND = p->ND; c.u = p->u;
  c.M = (int)M1; c.MB = (int)((M1 + plan.rows - 1) / plan.rows); c.nsplit = plan.ns[1];
  c.rcp_hkv = 0.f; c.rcp_g = 1.0f / (float)g; c.rcp_u = 1.0f / (float)(p->u > 1 ? p->u : 1);
  c.inv_hkv = div_inv((uint32_t)p->Hkv);
  c.c = p->sm_scale * kLog2e; c.k_scale = kv8 ? p->k_scale : 1.f; c.v_scale = kv8 ? p->v_scale : 1.f;
  c.q = (const uint16_t*)p->q; c.ks = (const uint16_t*)p->k_pages; c.vs = (const uint16_t*)p->v_pages; c.cu = nullptr;
  c.ku = (const uint16_t*)p->k_unshared; c.vu = (const uint16_t*)p->v_unshared;
  c.out = (uint16_t*)p->out; c.lse = p->lse_out; c.part_o = nullptr; c.part_ml = nullptr; c.order = nullptr; c.slot = p->slot;
  c.front = pack ? 0 : p->prefix_L; c.max_L = p->max_L; c.max_pages = p->max_pages; c.n_pages = p->n_pages; c.shift = __builtin_ctz((unsigned)p->page_size);
  c.prefix_pages = p->prefix_pages; c.table = p->block_table; c.lens = p->seq_lens;
  AttnCtx c0 = c;                                             // part 0: all requests' beams as one request's, whose list is the prefix
  c0.B = 1; c0.W = p->B * p->W; c0.ND = 0; c0.u = 0; c0.M = (int)M0; c0.MB = (int)((M0 + 127) / 128); c0.nsplit = plan.ns[0];
  c0.front = p->prefix_L; c0.max_L = 0; c0.slot = nullptr;
  int64_t blocks[2] = {0, 0};
  for (int k = pack ? 0 : 1; k < 2; k++) {
    AttnCtx& x = k == 0 ? c0 : c;
    const int64_t groups = (int64_t)x.B * x.Hkv * x.nsplit;
    blocks[k] = (groups + 7) / 8 * 8 * x.MB;
    if (groups >= ((int64_t)1 << 31) || !gr_grid_fits(blocks[0] + blocks[1], plan.rows == 256 || plan.ks == 2 ? 512 : 256)) return GR_ERR_UNSUPPORTED;
    x.n_groups = (int)groups; x.inv_mb = div_inv((uint32_t)x.MB); x.inv_split = div_inv((uint32_t)x.nsplit);
  }
  const unsigned grid = (unsigned)(blocks[0] + blocks[1]), blocks0 = (unsigned)blocks[0];
  JoinCtx j{p->B, p->W, p->Hq, p->Hkv, (int)g, plan.ns[0], plan.ns[1], nullptr, nullptr, c.out, c.lse};
  const int64_t join = (int64_t)p->B * p->Hkv * ((M1 + 1024 / p->d - 1) / (1024 / p->d));
  if (const size_t need = paged_workspace(p, plan)) {
    if (!workspace || ((uintptr_t)workspace & 255)) return GR_ERR_INVALID_ARG;
    if (workspace_bytes < need) return GR_ERR_WORKSPACE_TOO_SMALL;
    if (!gr_grid_fits(join, 256)) return GR_ERR_UNSUPPORTED;
    const size_t rows = (size_t)p->B * p->W * p->Hq, first = rows * plan.ns[0];          // part 1's partials lie behind part 0's
    c0.part_o = (float*)workspace;
    c0.part_ml = (float*)((char*)workspace + gr_align256(rows * (plan.ns[0] + plan.ns[1]) * p->d * 4));
    c.part_o = c0.part_o + first * p->d;
    c.part_ml = c0.part_ml + first * 2;
    j.part_o = c0.part_o; j.part_ml = c0.part_ml;
  }
  if (const gr_status st = kernels(plan, c0, c, grid, blocks0)) return st;
  if (j.part_o) {
    if (p->d == 128) hipLaunchKernelGGL((k_paged_join<128>), dim3((unsigned)join), dim3(256), 0, stream, j);
    else hipLaunchKernelGGL((k_paged_join<64>), dim3((unsigned)join), dim3(256), 0, stream, j);
  }
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}

}  // namespace
