// gr_beam_attn: shared-prefix beam attention on gfx950 (paper Sections 5.1, 5.2).
//
// Work unit = (request b, KV head h, block of query rows, L segment).  The W*g query rows that share
// KV head h of request b (g = Hq/Hkv) form the N side of a transposed score matrix
//     S^T[kv, q] = K[kv, :] . Q[q, :]          (v_mfma_f32_32x32x16_bf16, A = K tile from LDS, B = Q in registers)
// so that every lane owns ONE query column: the online-softmax max / sum / rescale are per-lane
// scalars and the exponentiated scores leave the accumulators already in the B-operand layout of
//     O^T[d, q] += V^T[d, kv] . P^T[kv, q]     (A = V tile read from LDS with the transposing ds_read_b64_tr_b16).
// Each prompt K/V tile is brought in once per workgroup (direct global -> LDS loads into unpadded, XOR-swizzled
// tiles) and used by all query rows of the block.  The unshared stage (each beam's own u decode tokens) and the merge
// run in the epilogue of one segment on the same per-lane state; when the prompt is split into
// segments, partial (max, sum, O) go to the workspace and k_attn_merge combines them.
#include "gr_attn_rows.hpp"

namespace {

template <int D, int NCB, int NWAVES, bool CAUSAL, bool KV8, int KS, bool FIND>
__global__ void __launch_bounds__(NWAVES * 64 * KS) __attribute__((amdgpu_waves_per_eu(NCB == 1 ? 2 : 1, NCB == 1 ? 2 : 1)))
k_beam_attn(AttnCtx c) {
  constexpr bool PAGED = false, WHOLE = false;
#include "gr_attn_rows.inc"
}

// Merge of the per-segment partials (Section 5.2 merge stage).  They lie as k_beam_attn's lanes hold them: per (request, segment, KV head) its M rows
// in blocks of up to 32, of a block first columns 0..3 of all its rows, then columns 4..7, and so on.  A lane takes four columns of a row; the
// eight rows of eight neighbouring lanes are a line, and the eight lanes of a row write 64 bytes of it.  The (max, sum) pairs
// and the partials of four segments are requested together, so a row waits for memory once per four segments.  Bound: the
// partials' bytes; 4096 rows x 5 segments of 128 (10.5 MB) take 4.3 us (6.7 us with 4-byte loads, one segment at a time).
template <int D>
__global__ void __launch_bounds__(256) k_attn_merge(AttnCtx c) {
  constexpr int RPW = 1024 / D;                            // rows per workgroup, of one (request, KV head) pair
  static_assert(RPW % 8 == 0 && 32 % RPW == 0, "whole lines of one block");
  const unsigned per_pair = ((unsigned)c.M + RPW - 1) / RPW, pair = blockIdx.x / per_pair;
  const int b = (int)(pair / (unsigned)c.Hkv), kvh = (int)(pair - (unsigned)b * (unsigned)c.Hkv);
  const int t = (int)threadIdx.x, piece = (t >> 3) % (D / 4), r = (int)(blockIdx.x - pair * per_pair) * RPW + (t & 7) + 8 * (t / (2 * D));
  if (r >= c.M) return;
  const int left = min(32, c.M - (r & ~31));               // rows of this row's block
  const size_t per_seg = (size_t)c.Hkv * c.M;              // rows of a segment of the request
  const size_t row0 = ((size_t)b * c.nsplit * c.Hkv + kvh) * c.M + r;
  const float* part = c.part_o + (row0 - (r & 31)) * D + 4 * (piece * left + (r & 31));
  float M2 = -INFINITY, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
#pragma unroll 1
  for (int s0 = 0; s0 < c.nsplit; s0 += U) {
    f32x2 ml[U];
    f32x4 o[U];
#pragma unroll
    for (int k = 0; k < U; k++) {
      const size_t skip = (size_t)min(s0 + k, c.nsplit - 1) * per_seg;
      ml[k] = *(const f32x2*)(c.part_ml + (row0 + skip) * 2);
      o[k] = *(const f32x4*)(part + skip * D);
    }
    float mx = M2;
#pragma unroll
    for (int k = 0; k < U; k++) {
      if (s0 + k >= c.nsplit) ml[k].y = 0.f;               // (a repeated segment counts nothing)
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
  const float inv = (L > 0.f) ? 1.0f / L : 0.f;
  bf16x4 h;
#pragma unroll
  for (int e = 0; e < 4; e++) h[e] = (__bf16)(acc[e] * inv);
  const int w = (int)((unsigned)r / (unsigned)c.g);
  const size_t row = ((size_t)b * c.W + w) * c.Hq + kvh * c.g + (r - w * c.g);
  *(bf16x4*)(c.out + row * D + 4 * piece) = h;
  if (c.lse && piece == 0) c.lse[row] = (L > 0.f) ? (M2 + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

// Requests by decreasing prompt length (ties by index), so that the longest units are dispatched first
// and the tail of a ragged batch is made of short ones.  Rank by counting; B is at most kMaxOrderB.
constexpr int kMaxOrderB = 4096;
__global__ void __launch_bounds__(256) k_attn_order(const int32_t* cu, int B, int32_t* order) {
  __shared__ int s_len[kMaxOrderB];
  for (int i = threadIdx.x; i < B; i += 256) s_len[i] = cu[i + 1] - cu[i];
  __syncthreads();
  for (int i = threadIdx.x; i < B; i += 256) {
    const int li = s_len[i];
    int rank = 0;
    for (int j = 0; j < B; j++) rank += (s_len[j] > li) || (s_len[j] == li && j < i);
    order[rank] = i;
  }
}

// Ragged batches with more units than CUs are worth ordering by length (measured: 4 % on 128 requests of
// 512..8192 tokens); a uniform batch (total_L == B * max_L) is not touched.  Up to kRankB requests every workgroup finds its own by
// rank (FIND), beyond that a kernel of one workgroup writes the order first: 128 of 40-120 tokens x 30 beams, 32 query and 8 KV
// heads of 128, 36.9 us with that kernel, 33.2 without; 100 of 50-500 x 40, 8 and 2 heads of 64, 16.0, 12.6.
bool attn_wants_order(const gr_attn_params* p, const AttnPlan& plan) {
  return p->B >= 2 && p->B <= kMaxOrderB && p->total_L != (int64_t)p->B * p->max_L && plan.many;
}

int g_plan_rows = 0, g_plan_segments = 0;                  // gr_diag_attn_plan: 0 = use the rule
AttnPlan plan_of(const gr_attn_params* p, bool kv8) {
  if (!g_plan_rows) return plan_attn(p, kv8);
  const int64_t cap = p->max_L / KT, M = (int64_t)p->W * (p->Hq / p->Hkv);       // a sweep asked for this tiling; keep at least one tile per segment
  AttnPlan plan;
  plan.mwg = g_plan_rows;
  plan.nsplit = (int)(g_plan_segments < cap ? g_plan_segments : (cap < 1 ? 1 : cap));
  plan.ks = sets_of(p, plan);
  plan.many = (int64_t)p->B * p->Hkv * ((M + plan.mwg - 1) / plan.mwg) * plan.nsplit > 256;
  return plan;
}

}  // namespace

extern "C" gr_status gr_diag_attn_plan(int32_t rows_per_workgroup, int32_t l_segments) {
  if (rows_per_workgroup == 0 && l_segments == 0) { g_plan_rows = g_plan_segments = 0; return GR_OK; }
  if ((rows_per_workgroup != 128 && rows_per_workgroup != 256) || l_segments < 1 || l_segments > 16) return GR_ERR_INVALID_ARG;
  g_plan_rows = rows_per_workgroup; g_plan_segments = l_segments;
  return GR_OK;
}

extern "C" size_t gr_beam_attn_workspace_bytes(const gr_attn_params* p) {
  if (!p || p->B <= 0 || p->W <= 0 || p->Hq <= 0 || p->Hkv <= 0 || p->Hq % p->Hkv) return 0;
  const AttnPlan plan = plan_of(p, false);               // (what it says about the workspace is the same for FP8 codes)
  size_t need = attn_wants_order(p, plan) ? gr_align256((size_t)p->B * 4) : 0;      // (up to kRankB requests: asked for as ever, and not used)
  if (plan.nsplit > 1) {
    const size_t rows = (size_t)p->B * plan.nsplit * p->W * p->Hq;
    need += gr_align256(rows * p->d * 4) + gr_align256(rows * 8);
  }
  return need;
}

namespace {
gr_status attn_run(const gr_attn_params* p, const int32_t* slot, bool kv8, float k_scale, float v_scale, void* workspace, size_t workspace_bytes,
                   void* stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  if (!p) return GR_ERR_INVALID_ARG;
  if (kv8 && (!(k_scale > 0.f) || !(k_scale < INFINITY) || !(v_scale > 0.f) || !(v_scale < INFINITY))) return GR_ERR_INVALID_ARG;
  if (p->B <= 0 || p->W <= 0 || p->Hq <= 0 || p->Hkv <= 0 || p->d <= 0 || p->ND < 0 || p->u < 0 || p->u > p->ND)
    return GR_ERR_INVALID_ARG;
  if (p->max_L < 0 || p->total_L < 0 || p->total_L > (int64_t)p->max_L * p->B) return GR_ERR_INVALID_ARG;
  if (!p->q || !p->cu_seqlens || !p->out) return GR_ERR_INVALID_ARG;
  if (p->total_L > 0 && (!p->k_shared || !p->v_shared)) return GR_ERR_INVALID_ARG;
  if (p->u > 0 && (!p->k_unshared || !p->v_unshared)) return GR_ERR_INVALID_ARG;
  if (p->Hq % p->Hkv) return GR_ERR_INVALID_ARG;
  if ((((uintptr_t)p->q | (uintptr_t)p->k_shared | (uintptr_t)p->v_shared | (uintptr_t)p->k_unshared | (uintptr_t)p->v_unshared |
        (uintptr_t)p->out) & 15) || ((uintptr_t)p->cu_seqlens & 3) || ((uintptr_t)p->lse_out & 3) || ((uintptr_t)slot & 3))
    return GR_ERR_INVALID_ARG;                                                          // every tensor is moved in 16-byte pieces
  if (!(p->sm_scale > 0.f) || !(p->sm_scale < INFINITY)) return GR_ERR_INVALID_ARG;   // (also rejects NaN: the largest score is taken before it is scaled)
  if (p->d != 64 && p->d != 128) return GR_ERR_UNSUPPORTED;
  if (p->total_L >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  if ((int64_t)p->max_L * p->Hkv * p->d * 2 >= ((int64_t)1 << 32)) return GR_ERR_UNSUPPORTED;   // one request's K (or V) must fit a buffer descriptor
  const int g = p->Hq / p->Hkv;
  if ((int64_t)p->W * g >= ((int64_t)1 << 22)) return GR_ERR_UNSUPPORTED;      // row indices go through small_div, whose bound is 2^22
  if ((int64_t)p->W * p->Hq * p->d >= ((int64_t)1 << 31) || (int64_t)p->W * p->ND * p->Hkv * p->d >= ((int64_t)1 << 31))
    return GR_ERR_UNSUPPORTED;                                                   // offsets inside one request fit 32 bits

  AttnCtx c;
  c.B = p->B; c.W = p->W; c.Hq = p->Hq; c.Hkv = p->Hkv; c.g = g; c.ND = p->ND; c.u = p->u;
  c.M = p->W * g;
  const AttnPlan plan = plan_of(p, kv8);
  c.MB = (c.M + plan.mwg - 1) / plan.mwg;
  c.nsplit = plan.nsplit;
  c.n_groups = p->B * p->Hkv * c.nsplit;
  c.rcp_g = 1.0f / (float)g; c.rcp_u = 1.0f / (float)(p->u > 1 ? p->u : 1);
  c.inv_mb = div_inv((uint32_t)c.MB); c.inv_split = div_inv((uint32_t)c.nsplit); c.inv_hkv = div_inv((uint32_t)c.Hkv);
  c.c = p->sm_scale * kLog2e;
  c.k_scale = kv8 ? k_scale : 1.f; c.v_scale = kv8 ? v_scale : 1.f;
  c.q = (const uint16_t*)p->q; c.ks = (const uint16_t*)p->k_shared; c.vs = (const uint16_t*)p->v_shared;
  c.cu = p->cu_seqlens; c.ku = (const uint16_t*)p->k_unshared; c.vu = (const uint16_t*)p->v_unshared;
  c.out = (uint16_t*)p->out; c.lse = p->lse_out;
  c.part_o = nullptr; c.part_ml = nullptr; c.order = nullptr; c.slot = slot; c.rcp_hkv = 0.f;
  const size_t need = gr_beam_attn_workspace_bytes(p);
  const bool ordered = attn_wants_order(p, plan), find = ordered && p->B <= kRankB;       // (these have one set of wavefronts: two are for at most 256 workgroups)
  if (need > 0) {
    if (!workspace || ((uintptr_t)workspace & 255)) return GR_ERR_INVALID_ARG;
    if (workspace_bytes < need) return GR_ERR_WORKSPACE_TOO_SMALL;
    char* ws = (char*)workspace;
    if (ordered && !find) {
      hipLaunchKernelGGL(k_attn_order, dim3(1), dim3(256), 0, stream, p->cu_seqlens, p->B, (int32_t*)ws);
      c.order = (const int32_t*)ws;
    }
    if (ordered) ws += gr_align256((size_t)p->B * 4);
    if (c.nsplit > 1) {
      const size_t rows = (size_t)p->B * c.nsplit * p->W * p->Hq;
      c.part_o = (float*)ws;
      c.part_ml = (float*)(ws + gr_align256(rows * p->d * 4));
    }
  }
  const int64_t groups_padded = ((int64_t)c.n_groups + 7) / 8 * 8;
  const int64_t grid = groups_padded * c.MB;
  if (grid >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  const size_t lds = attn_lds_bytes(p->d, plan.mwg, plan.ks);
#define GR_LAUNCH(...)                                                                                       \
  do {                                                                                                       \
    if (const gr_status st = gr_allow_lds<k_beam_attn<__VA_ARGS__>>(lds)) return st;                         \
    hipLaunchKernelGGL((k_beam_attn<__VA_ARGS__>), dim3((unsigned)grid), dim3(threads), lds, stream, c);     \
  } while (0)
#define GR_LAUNCH_ATTN(DD, NW_)                                                                              \
  do {                                                                                                       \
    if (find) { if (kv8) GR_LAUNCH(DD, 1, NW_, false, true, 1, true); else GR_LAUNCH(DD, 1, NW_, false, false, 1, true); }      \
    else { if (kv8) GR_LAUNCH(DD, 1, NW_, false, true, 1, false); else GR_LAUNCH(DD, 1, NW_, false, false, 1, false); }         \
  } while (0)
#define GR_LAUNCH_SETS(DD)                                                                                   \
  do { if (kv8) GR_LAUNCH(DD, 1, 4, false, true, 2, false); else GR_LAUNCH(DD, 1, 4, false, false, 2, false); } while (0)
  const unsigned threads = plan.mwg == 256 || plan.ks == 2 ? 512 : 256;
  if (p->d == 128) {
    if (plan.mwg == 256) GR_LAUNCH_ATTN(128, 8); else if (plan.ks == 2) GR_LAUNCH_SETS(128); else GR_LAUNCH_ATTN(128, 4);
  } else {
    if (plan.mwg == 256) GR_LAUNCH_ATTN(64, 8); else if (plan.ks == 2) GR_LAUNCH_SETS(64); else GR_LAUNCH_ATTN(64, 4);
  }
#undef GR_LAUNCH_SETS
#undef GR_LAUNCH_ATTN
  if (c.nsplit > 1) {
    const int rpw = 1024 / p->d;                           // rows per workgroup
    const unsigned mgrid = (unsigned)((int64_t)p->B * p->Hkv * ((c.M + rpw - 1) / rpw));
    if (p->d == 128) hipLaunchKernelGGL((k_attn_merge<128>), dim3(mgrid), dim3(256), 0, stream, c);
    else hipLaunchKernelGGL((k_attn_merge<64>), dim3(mgrid), dim3(256), 0, stream, c);
  }
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
}  // namespace

extern "C" gr_status gr_beam_attn(const gr_attn_params* p, void* workspace, size_t workspace_bytes, void* stream) {
  return attn_run(p, nullptr, false, 1.f, 1.f, workspace, workspace_bytes, stream);
}

// The same attention with the own-token caches read through a slot table: nothing is moved between decode steps, the
// table (gr_beam_slot_update) says which row of the request's block holds token t of beam w.
extern "C" gr_status gr_beam_attn_slots(const gr_attn_params* p, const int32_t* slot, void* workspace, size_t workspace_bytes, void* stream) {
  if (!slot) return GR_ERR_INVALID_ARG;
  return attn_run(p, slot, false, 1.f, 1.f, workspace, workspace_bytes, stream);
}

// The same attention over a prompt cache stored as FP8 E4M3 codes with one scale per tensor.
extern "C" gr_status gr_beam_attn_fp8kv(const gr_attn_fp8kv_params* p, void* workspace, size_t workspace_bytes, void* stream) {
  if (!p) return GR_ERR_INVALID_ARG;
  return attn_run(&p->attn, nullptr, true, p->k_scale, p->v_scale, workspace, workspace_bytes, stream);
}

// Causal prompt attention through the same kernel (CAUSAL = true).
extern "C" gr_status gr_prefill_attn(const gr_prefill_params* p, void* stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  if (!p) return GR_ERR_INVALID_ARG;
  if (p->B <= 0 || p->Hq <= 0 || p->Hkv <= 0 || p->d <= 0 || p->Hq % p->Hkv) return GR_ERR_INVALID_ARG;
  if (p->max_L < 0 || p->total_L < 0 || p->total_L > (int64_t)p->max_L * p->B) return GR_ERR_INVALID_ARG;
  if (!p->cu_seqlens) return GR_ERR_INVALID_ARG;
  if (p->total_L > 0 && (!p->q || !p->k || !p->v || !p->out)) return GR_ERR_INVALID_ARG;
  if ((((uintptr_t)p->q | (uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->out) & 15) || ((uintptr_t)p->cu_seqlens & 3) ||
      ((uintptr_t)p->lse_out & 3))
    return GR_ERR_INVALID_ARG;
  if (!(p->sm_scale > 0.f) || !(p->sm_scale < INFINITY)) return GR_ERR_INVALID_ARG;
  if (p->d != 64 && p->d != 128) return GR_ERR_UNSUPPORTED;
  if (p->total_L >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  if ((int64_t)p->max_L * p->Hkv * p->d * 2 >= ((int64_t)1 << 32)) return GR_ERR_UNSUPPORTED;   // one request's K (or V) must fit a buffer descriptor
  const int g = p->Hq / p->Hkv;
  if ((int64_t)p->max_L * g >= ((int64_t)1 << 22)) return GR_ERR_UNSUPPORTED;                   // row indices go through small_div, whose bound is 2^22
  if ((int64_t)p->max_L * p->Hq * p->d >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;        // offsets inside one request fit 32 bits
  if (p->total_L == 0 || p->max_L == 0) return GR_OK;

  AttnCtx c;
  c.B = p->B; c.W = 0; c.Hq = p->Hq; c.Hkv = p->Hkv; c.g = g; c.ND = 0; c.u = 0;
  c.M = p->max_L * g;                                        // the longest request's rows size the grid
  // 128 rows, two workgroups to a CU: one computes while the other waits for its queries or stores its output, which is most of
  // the life of a block of a short prompt.  256 rows stage every K/V tile half as often, which counts for long prompts of head size
  // 128, and for shorter ones where an XCD has one or two (prompt, KV head) pairs and 1.25 to 2 such blocks per CU (counted by
  // the tokens there are), so that the few heaviest blocks are what the call waits for.  us with 256 and 128 rows (32 query and 8 KV heads of 128 unless noted):
  // 1 x 1024 tokens 29.7, 22.3; 16 prompts of 62-512 38.2, 33.9; 4 x 1024 56, 49; 1 x 2048 55.1, 47.6; 16 x 2048 596, 579; 4 of
  // 190-1500 with 16 query and 4 KV heads 43.6, 36.7; but 1 x 4096 128, 138 and 8 of 1024-8192 1674, 1700; 2 x 2048 74.5, 77.9 and 1 to 4 x 2048 of 16 query and 2 KV heads 69-75, 75-79.  8 heads of 64:
  // 1 x 4096 71, 50; 16 x 4096 383, 344.
  const int64_t pairs = (int64_t)p->B * p->Hkv, rows_per_xcd = p->total_L * p->Hq / (pairs < 8 ? pairs : 8);
  const bool heavy = p->max_L > 2048 || (pairs <= 16 && rows_per_xcd > 40 * 256 && rows_per_xcd <= 64 * 256);
  const int mwg = p->d == 64 || !heavy || c.M <= 128 ? 128 : 256;
  c.MB = (c.M + mwg - 1) / mwg;
  c.nsplit = 1;
  c.n_groups = p->B * p->Hkv;
  c.rcp_g = 1.0f / (float)g; c.rcp_u = 1.f;
  c.inv_mb = div_inv((uint32_t)c.MB); c.inv_split = div_inv(1); c.inv_hkv = div_inv((uint32_t)c.Hkv);
  c.c = p->sm_scale * kLog2e;
  c.k_scale = 1.f; c.v_scale = 1.f;
  c.q = (const uint16_t*)p->q; c.ks = (const uint16_t*)p->k; c.vs = (const uint16_t*)p->v;
  c.cu = p->cu_seqlens; c.ku = nullptr; c.vu = nullptr;
  c.out = (uint16_t*)p->out; c.lse = p->lse_out;
  c.part_o = nullptr; c.part_ml = nullptr; c.order = nullptr; c.slot = nullptr;
  const int64_t groups_padded = ((int64_t)c.n_groups + 7) / 8 * 8;
  const int64_t grid = groups_padded * c.MB;
  // Row blocks dealt heaviest first over all pairs of an XCD: the blocks that prompts shorter than the longest do not have come last
  // (pair by pair they come first, and hold a place while they find that out), and the call ends with light blocks.  Against that stand
  // 0.4 us at the start of every block and K/V that is read again when it has left the L2.  So: where not all blocks have a place at once,
  //   an XCD's pairs times the rows of a token in each are at most 48 (head size 128) or 128 (64), or more, up to 64 with head size 128,
  //     where the prompts are on average shorter than two thirds of the longest, and
  //   the K/V of an XCD's pairs times the rows of a token take at most 24 MiB: 64 x 4500 tokens of 8 heads of 64 1647 us pair by pair, 2266 by
  //     weight, 32 x 3000 with 32 and 8 heads 1397, 1532, 48 of 960-1200 with 8 heads of 128 162, 188; but 32 x 3000 with 8 heads 405, 387.
  // 2400 shapes of 250 to 11000 tokens: where the rule deals by weight that takes 0.94 of pair by pair in the mean (head size 64 0.91, 128
  // 0.95), and in one of 90 more than 1.06.  us pair by pair, by weight: 16 prompts of 60-700 tokens, 32 query and 8 KV heads of 128, 44.7, 41.6; 8 of
  // 200-2000 136.7, 133; 10 of 300-1000 57.5, 55.8; 40 of 100-900, 8 and 2 heads, 47.2, 44.1; 8 heads of 64: 12 of 100-1000 18.9, 15.1, 16 of
  // 1000-4000 153, 140.  But 32 of 100-600, 32 and 8 heads of 128, 69, 78; 16 x 600 70, 74; 64 of 100-600, 16 and 2 heads, 68, 71.
  const int64_t rows_of_token = groups_padded / 8 * g;
  const bool uneven = p->total_L * 3 < (int64_t)p->B * p->max_L * 2;
  const bool by_weight = groups_padded <= 512 && grid > 512 && mwg == 128 && p->total_L * p->Hq * p->d <= (int64_t)48 << 20 &&
                         (rows_of_token <= (p->d == 64 ? 128 : 48) || (uneven && (p->d == 64 || rows_of_token <= 64)));
  c.rcp_hkv = 1.0f / (float)p->Hkv * 1.00001f;
  if (grid >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  const size_t lds = attn_lds_bytes(p->d, mwg, 1);
  const unsigned threads = 2 * mwg;
  if (p->d == 128) {
    if (mwg == 256) GR_LAUNCH(128, 1, 8, true, false, 1, false);
    else if (by_weight) GR_LAUNCH(128, 1, 4, true, false, 1, true);
    else GR_LAUNCH(128, 1, 4, true, false, 1, false);
  } else {
    if (by_weight) GR_LAUNCH(64, 1, 4, true, false, 1, true); else GR_LAUNCH(64, 1, 4, true, false, 1, false);
  }
#undef GR_LAUNCH
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
