// What the attention kernels of gr_attn.hip (keys packed by request) and of gr_paged.hip (keys in pages of a pool) have in common beside their body
// (gr_attn_rows.inc): arguments, LDS, index helpers and the launch rule.  Not part of the ABI.
#pragma once
#include <type_traits>
#include "gr_attn_tile.hpp"
#include "gr_pages.hpp"

namespace {

// Dynamic LDS of k_beam_attn: K and V tiles, double-buffered; the Q hand-over, behind the tiles for workgroups of 8 wavefronts and in the V
// tiles' place for those of 4.  After the prompt loop a wavefront's 32 own-token rows take the K tiles' place (of K; Q's where 8 wavefronts hold
// 256 rows) and the V tiles' (of V; all tiles' there), and its 32 rows of output K's again.  All of it in unpadded, swizzled rows.  Behind it 256
// bytes per wave that loads issued only to bring lines into L2 write to.
// Workgroups whose two halves share the prompt (ks = 2): each half's tiles and a place for one more (a third V tile where the head size is 128), which
// takes half of Q at first and, after the loop, the second half's (maximum, sum).
constexpr int attn_tiles_bytes(int d) { return 4 * KT * d * 2; }
constexpr int attn_lds_used(int d, int mwg) { return attn_tiles_bytes(d) + (mwg == 256 ? mwg * d * 2 : 0); }
constexpr int attn_lds_bytes(int d, int mwg, int ks) {
  return ks == 2 ? 2 * 5 * KT * d * 2 : attn_lds_used(d, mwg) + mwg / 32 * 256;
}

struct AttnCtx {
  int B, W, Hq, Hkv, g, ND, u;
  int M;            // W * g query rows per (b, kv head)
  int MB;           // row blocks per (b, kv head)
  int nsplit;       // L segments per request
  int n_groups;     // B * Hkv * nsplit
  float rcp_hkv;    // 1 / Hkv, a little high: n * rcp_hkv is n / Hkv rounded down for 0 <= n < 512
  float rcp_g, rcp_u;       // 1 / g, 1 / max(u, 1)
  uint32_t inv_mb, inv_split, inv_hkv;       // for div_by
  float c;          // sm_scale * log2(e)
  float k_scale, v_scale;   // FP8 prompt cache: value = code * scale (1 for the bf16 cache)
  const uint16_t* q;
  const uint16_t* ks;
  const uint16_t* vs;
  const int32_t* cu;
  const uint16_t* ku;
  const uint16_t* vu;
  uint16_t* out;
  float* lse;
  float* part_o;    // [B, nsplit, Hkv, M rows in blocks of 32: D / 4, row, 4] fp32, unnormalised
  float* part_ml;   // [B, nsplit, Hkv, M, 2] (max in log2 domain, sum)
  const int32_t* order;   // [B] requests by decreasing prompt length, or nullptr (requests taken in index order)
  const int32_t* slot;    // [B, W, ND] row of the request's own-token block that holds (beam, token), or nullptr (= w * ND + t)
  // keys in pages (PAGED; cu and order are not used): the first `front` tokens of every request's list are in the pages of prefix_pages, the others in those of its
  // row of the table
  int front, max_L, max_pages, n_pages, shift;      // shift: log2 of a page's tokens
  const int32_t* prefix_pages;
  const int32_t* table;   // [B, max_pages]
  const int32_t* lens;    // [B] tokens behind the front
};

// The kernel's arguments, read where this stands and not before: what only rare or late code needs takes no scalar registers through the prompt loop.
typedef const __attribute__((address_space(4))) AttnCtx* LateArgs;
__device__ __forceinline__ LateArgs late_args() {
  LateArgs a = (LateArgs)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return a;
}

__device__ __forceinline__ int wave_total(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);      // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);      // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);      // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // lane 15 of rows 0, 2 to rows 1, 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // lane 31 to rows 2, 3
  return __builtin_amdgcn_readlane(v, 63);
}

__device__ __forceinline__ int rank_in(uint64_t mask) {     // lanes of the mask in front of this one
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
// The request of rank `rank` by decreasing prompt length (ties by index), its first row and its length; every wavefront by itself, lane i
// with requests i and i + 64.  About 0.2 us, which the two dependent loads that it takes the place of (the order, then the
// request's rows) cost as well; a kernel for the order is 5.6 us in front of the call.
constexpr int kRankB = 128;
__device__ __forceinline__ int request_of_rank(const int (&first)[2], const int (&l)[2], int rank, int lane, int* row0, int* len) {
  auto reach = [&](int n) { return __popcll(__ballot(l[0] >= n)) + __popcll(__ballot(l[1] >= n)); };
  int lo = 0, hi = 64;                                       // more than `rank` requests reach lo, not so many hi
  while (hi < 1 << 30 && reach(hi) > rank) { lo = hi; hi <<= 1; }
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (reach(mid) > rank) lo = mid; else hi = mid;
  }
  rank -= reach(hi);                                         // among those of length lo
  const uint64_t same0 = __ballot(l[0] == lo), same1 = __ballot(l[1] == lo);
  const bool upper = rank >= __popcll(same0);
  const uint64_t same = upper ? same1 : same0;
  rank -= upper ? __popcll(same0) : 0;
  const uint64_t it = __ballot(((same >> lane) & 1) && rank_in(same) == rank);
  const int at = __ffsll((unsigned long long)it) - 1;
  *row0 = __builtin_amdgcn_readlane(upper ? first[1] : first[0], at);
  *len = lo;
  return at + (upper ? 64 : 0);
}
__device__ __forceinline__ int request_by_length(const int32_t* cu, int B, int rank, int lane, int* row0, int* len) {
  int first[2], l[2];
#pragma unroll
  for (int k = 0; k < 2; k++) {
    first[k] = 0; l[k] = -1;
    if (lane + 64 * k < B) { first[k] = cu[lane + 64 * k]; l[k] = cu[lane + 64 * k + 1] - first[k]; }
  }
  return request_of_rank(first, l, rank, lane, row0, len);
}

// ---- keys in pages
// Tokens of request b behind the front; a length outside [0, max_L] counts as the nearer end.
__device__ __forceinline__ int paged_length(const AttnCtx& c, int b) { return c.max_L == 0 ? 0 : min(max(c.lens[b], 0), c.max_L); }
__device__ __forceinline__ int request_by_own_length(const AttnCtx& c, int rank, int lane, int* len) {
  int first[2] = {0, 0}, l[2], none;
#pragma unroll
  for (int k = 0; k < 2; k++) l[k] = lane + 64 * k < c.B ? paged_length(c, lane + 64 * k) : -1;
  return request_of_rank(first, l, rank, lane, &none, len);
}
// Number of page p of a request's list (behind the last one: that one's), as its table has it; one outside the pool counts as 0.
template <class C>
__device__ __forceinline__ int page_entry(const C& c, unsigned b, int p, int last) {
  p = min(p, last);
  const int q = p - (c.front >> c.shift);
  return q < 0 ? c.prefix_pages[p] : c.table[(size_t)b * (unsigned)c.max_pages + (unsigned)q];
}
template <class C>
__device__ __forceinline__ int page_number(const C& c, unsigned b, int p, int last) {
  const int number = page_entry(c, b, p, last);
  return (unsigned)number < (unsigned)c.n_pages ? number : 0;
}
// Slot of token t of the list in the pools.
template <class C>
__device__ __forceinline__ size_t slot_of(const C& c, unsigned b, int t, int last_page) {
  return ((size_t)(unsigned)page_number(c, b, t >> c.shift, last_page) << c.shift) + (unsigned)(t & ((1 << c.shift) - 1));
}

// Host-side launch plan, fitted to measured sweeps over (B, L, W) on the MI355X.  8-wave workgroups of 256 query rows stage each
// K/V tile once per 256 rows and win for long prompts once there are at least 256 of them (one per CU); else, workgroups of 128 rows: two of
// 4 waves to a CU, or, where there is at most one per CU, one of 8 waves in two sets that share the prompt (ks = 2: 8 requests of
// 2048 tokens x 128 beams, 256 workgroups, 46.3 -> 41.8 us; 2 x 256 x 16 of head size 64 8.4 -> 7.7).
// Splitting the prompt into L segments costs fp32 partials through memory and the merge kernel.  With fewer workgroups than
// CUs, the number of segments is the one for which this sum is least, in us: for every round of workgroups of an XCD (32 CUs, one or two
// to a CU; a segment of a (request, KV head) pair stays on one XCD) 6 and 1.6 (head size 128) or 1.07 (64) for a tile of each
// set that a segment holds, 3.5 for the merge, and the partials written and read at 3 TB/s (64: 3.5).  Over 48 shapes of 400 to 12000 tokens it is 2 %
// above the best number on average (3.4 % without the rounds and with 4 TB/s): 2 requests of 8000 tokens x 200
// beams, 8 query and 2 KV heads of 64: 29.2 us with 9 segments, whose 36 pairs put 35 workgroups on some XCDs, 20.5 with 8; 4 x 2048 x 128 of 8
// heads of 64 20.9 with 8, 15.9 with 4; one of 800 x 128 of these 13.9, 13.7, 12.5, 11.5, 12.8 with 1 to 5.
// Up to two workgroups per CU are looked at: with one at most, long prompts whose pairs and row blocks are somewhat more than half of 256, or a third, left
// places empty: 9 of 2860-4376 x 195 beams of 16 query and 4 KV heads 97.4 us, now 74.4; 7 x 12959 x 66 178.7, 145.6; 12 of 1504-2443 x 39, 8 heads
// of 64, 23.2, 21.0; of 180 shapes none is more than 2 % slower.
//
// With 256 workgroups of 256 rows or more, 128 rows win nevertheless, us with 128 and 256 rows:
//   where they waste fewer rows of the last block (more than 5 %; 8 % for FP8 codes, which every workgroup widens for itself): 128 requests of
//     100-900 tokens x 200 beams, 32 query and 8 KV heads of 128: 319, 350 (FP8 329, 350); 48 of 512-8192 x 300, 8 heads of 64: 210, 271;
//   for prompts of up to 1024 tokens on average in more than one round: two workgroups to a CU cover each other's queries, own tokens and
//     output, which are 40 % of the life of a unit of 8 tiles: 64 x 512 x 128 96.8, 101.6; 32 x 1024 x 256 149.6, 153.9; 128 x 128 x 256 of
//     16 query and 2 KV heads 93, 103, of 8 and 2 heads of 64 28.3, 32.0.  But 64 x 1500 x 256 425, 421, 32 x 4096 x 256 504, 498, with FP8 codes
//     128 x 512 x 256 385, 373, and where queries and outputs are twice what the Infinity Cache holds 128 x 128 x 256 of 32 heads 223, 216.
struct AttnPlan { int mwg, nsplit, ks; bool many; };       // many: more workgroups than CUs before the choice of 128 rows for their own sake
int sets_of(const gr_attn_params* p, const AttnPlan& plan) {
  const int64_t M = (int64_t)p->W * (p->Hq / p->Hkv);
  return plan.mwg == 128 && p->max_L > KT && (int64_t)p->B * p->Hkv * ((M + 127) / 128) * plan.nsplit <= 256 ? 2 : 1;
}
AttnPlan plan_attn(const gr_attn_params* p, bool kv8) {
  const int g = p->Hq / p->Hkv;
  const int64_t M = (int64_t)p->W * g;
  AttnPlan plan;
  const int64_t units256 = (int64_t)p->B * p->Hkv * ((M + 255) / 256);
  plan.mwg = (M <= 128 || units256 < 256) ? 128 : 256;     // 256-row workgroups only when they fill the chip by themselves
  const int64_t units = (int64_t)p->B * p->Hkv * ((M + plan.mwg - 1) / plan.mwg);
  plan.nsplit = 1;
  if (units < 256 && p->max_L > 4 * KT) {
    const int64_t want = (512 + units / 2) / units, cap = p->max_L / ((p->d == 64 ? 3 : 4) * KT);      // about two workgroups per CU; at least so many tiles per segment
    const int most = (int)(want < cap ? (want < 16 ? want : 16) : (cap < 16 ? cap : 16));
    const int tiles = (p->max_L + KT - 1) / KT;
    const double partial_us = 2.0 * p->B * p->W * p->Hq * p->d * 4 / (p->d == 64 ? 3.5e6 : 3e6);             // of one segment
    double least = 0;
    for (int n = 1; n <= most; n++) {
      const int ks = units * n <= 256 ? 2 : 1, per_set = ((tiles + n - 1) / n + ks - 1) / ks;
      const int64_t on_xcd = ((int64_t)p->B * p->Hkv * n + 7) / 8 * ((M + 127) / 128), rounds = (on_xcd + 64 / ks - 1) / (64 / ks);
      const double us = (double)rounds * (6.0 + (p->d == 64 ? 1.07 : 1.6) * per_set) + (n > 1 ? 3.5 + partial_us * n : 0.0);
      if (n == 1 || us < least) { least = us; plan.nsplit = n; }
    }
  }
  plan.many = units * plan.nsplit > 256;
  if (plan.mwg == 256) {
    const int64_t rows128 = (M + 127) / 128 * 128, rows256 = (M + 255) / 256 * 256;
    const bool fewer_rows = rows256 * 100 > rows128 * (kv8 ? 108 : 105);
    const bool short_prompts = !kv8 && p->total_L <= (int64_t)p->B * 1024 && units256 > 256 && (int64_t)p->B * p->W * p->Hq * p->d * 4 <= ((int64_t)400 << 20);
    if (fewer_rows || short_prompts) plan.mwg = 128;
  }
  plan.ks = sets_of(p, plan);
  return plan;
}

}  // namespace
