// gr_beam_attn_paged: the decode step's attention over a prompt cache in pages of a pool, behind a prefix that all requests share.
//
// The kernel is gr_beam_attn's (gr_attn_rows.inc).  What differs is where the tokens lie and which rows meet which tokens:
//   - Token t of a row's keys is in page t / page_size of its list of pages: the prefix's pages, then the request's.  A prefix is whole
//     pages, so both are one list.  A wavefront brings 1 KiB of a tile at a time, 4 or 8 consecutive tokens, which lie in one page
//     (pages hold 16 tokens at least): its address is scalar work beside the MFMAs, from page numbers that a lane each holds.
//   - Softmax partials (maximum, sum, O) of disjoint sets of keys join exactly, so the prefix may be met by other workgroups than the rest.  A workgroup's
//     128 or 256 rows share their keys: the rows of one (request, KV head) pair share all of them (W * g rows), the rows of ALL requests
//     share the prefix.  Where a request's rows leave most of a workgroup empty, part 0 of the launch packs all requests' rows against the prefix, as if they were
//     the beams of one request, and part 1 takes each request's own pages; a second kernel joins the partials.  Else, and with more than 80 rows of a pair
//     always, a row walks the whole list by itself.
//   - Where a request's rows of a KV head are few, 32 of them meet the keys in a workgroup whose wavefronts share out the keys and not the rows.
#include "gr_paged.hpp"

namespace {

// A pointer that is the same in all lanes, in scalar registers (where a load's address has to be, and the compiler has it in vector ones).
template <class P>
__device__ __forceinline__ P* scalar(P* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p;
  uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
  // (a vector instruction's scalar result may be a load's address five wait states later, which the compiler keeps to only for loads that it sees)
  asm volatile("s_nop 4" : "+s"(lo), "+s"(hi));
  return (P*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

// Up to 32 rows of a (request, KV head) pair: 32 rows of a workgroup of 128 would be all there is, and what counts is how soon the keys arrive.  Every wavefront
// holds the rows and takes every fourth 32 tokens of the segment through places of its own in LDS: K's next 32 are asked for as soon as the scores
// are made, V's as soon as its products are, and nobody waits for anybody until the four (maximum, sum, O) are joined in LDS.  The beams' own tokens are the
// list's last tiles.  Bound: memory; two workgroups of four wavefronts to a CU have up to 128 KB of loads on their way.
constexpr int paged_few_lds_bytes(int d) { return (4 * 2 * 32 + 32) * d * 2; }      // a K and a V place per wavefront, and Q

// ARG: which of the kernel's arguments c is.
template <int D, bool KV8, int ARG>
__device__ __forceinline__ void few_rows(const AttnCtx& c, const unsigned id) {
  using T = AttnTile<D, 1>;
  constexpr int PPR = D / 8, RPC = 1024 / (D * 2), FT = 32, PLACE = FT * D, NLD = FT / RPC;      // NLD: loads of a place
  constexpr int EB = KV8 ? 1 : 2;
  extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];
  const int tid = (int)threadIdx.x, wave = tid >> 6, lane = tid & 63, G = lane >> 5, n32 = lane & 31;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const unsigned place = id >> 3, nth = div_by(place, (unsigned)c.MB, c.inv_mb);
  const int group = (int)(nth * 8 + (id & 7u)), mbi = (int)(place - nth * (unsigned)c.MB), ns = c.nsplit, M = c.M;
  if (group >= c.n_groups) return;
  const unsigned gq = div_by((unsigned)group, (unsigned)ns, c.inv_split);
  const int sp = group - (int)gq * ns;
  const unsigned bu = div_by(gq, (unsigned)c.Hkv, c.inv_hkv), kvh = gq - bu * (unsigned)c.Hkv;
  auto dma = [&](uint32_t lds_addr, const char* gbase, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(off), "s"(gbase) : "memory", "m0");
  };
  const uint32_t lds_0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)smem;

  // ---- Q, in one place for all
  const int row_w = mbi * 32, beam0 = __builtin_amdgcn_readfirstlane(small_div(row_w, c.rcp_g));
  const char* q_b = (const char*)scalar(c.q + (((size_t)bu * (unsigned)c.W + (unsigned)beam0) * (unsigned)c.Hq + kvh * (unsigned)c.g) * D);
  constexpr int q_place = 8 * PLACE;
  const int k_place = wave_u * 2 * PLACE, v_place = k_place + PLACE;
#pragma unroll
  for (int i = 0; i < NLD / 4; i++) {
    const int ch = i * 4 + wave_u, rl = ch * RPC + lane / PPR, r = min(row_w + rl, M - 1), beam = small_div(r, c.rcp_g);
    dma(lds_0 + (uint32_t)(q_place + ch * RPC * D) * 2, q_b,
        (uint32_t)((beam - beam0) * c.Hq + (r - beam * c.g)) * (D * 2) + (uint32_t)(((lane % PPR) ^ T::swz_k(rl)) * 16));
  }

  // ---- page numbers: lane i has that of page window + i of the list.  The first segment's are asked for beside the length, whatever it will be (what a table holds
  // behind a request's pages is of no use to anybody): the first loads of K wait for one of the two after the other less
  const int most_pages = (c.front + c.max_L + (1 << c.shift) - 1) >> c.shift;
  auto numbers_from = [&](int first) { return most_pages > 0 ? page_number(c, bu, first + lane, most_pages - 1) : 0; };
  int window = 0, numbers = sp == 0 ? numbers_from(0) : 0;
  const int keys = c.front + __builtin_amdgcn_readfirstlane(paged_length(c, (int)bu));
  int chunk = (int)div_by((unsigned)keys + (unsigned)ns - 1u, (unsigned)ns, c.inv_split);
  chunk = (chunk + KT - 1) / KT * KT;
  const int seg0 = min(keys, sp * chunk), seg1 = min(keys, seg0 + chunk);
  const int nt = (seg1 - seg0 + FT - 1) / FT;
  const bool own_stage = c.u > 0 && sp == (max(0, keys - (ns - 1) * chunk) < chunk ? ns - 1 : 0);
  const int qrow = row_w + n32 < M ? row_w + n32 : -1;
  const int beam_q = small_div(max(qrow, 0), c.rcp_g);
  const int Ru = own_stage ? (__builtin_amdgcn_readfirstlane(small_div(min(row_w + 31, M - 1), c.rcp_g)) - beam0 + 1) * c.u : 0;
  const int my_lo = (beam_q - beam0) * c.u;
  const int total = nt + (Ru + FT - 1) / FT;

  const int mask = (1 << c.shift) - 1, last_tok = seg1 - 1, last_chunk = last_tok & ~(RPC - 1);
  if (sp > 0) { window = seg0 >> c.shift; numbers = numbers_from(window); }
  const uint32_t tok_bytes = (uint32_t)c.Hkv * D * EB, own_bytes = (uint32_t)c.Hkv * D * 2;
  const char* k_base = (const char*)c.ks + (size_t)kvh * D * EB;
  const char* v_base = (const char*)c.vs + (size_t)kvh * D * EB;
  const char* ku_b = (const char*)(c.ku + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  const char* vu_b = (const char*)(c.vu + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  // byte offset of a chunk of tile j in its pool, and of this lane's row in the chunk (rows behind the segment: its last token)
  auto chunk_at = [&](int j, int i, uint32_t* lane_row) {
    const int tok = seg0 + j * FT + i * RPC, t = min(tok, last_chunk), p = t >> c.shift;
    if (p - window >= 64) { window = (seg0 + j * FT) >> c.shift; numbers = numbers_from(window); }      // (wave-uniform; a tile lies in four pages at most)
    const int number = __builtin_amdgcn_readlane(numbers, p - window);
    *lane_row = (uint32_t)(min(tok + lane / PPR, last_tok) - t) * tok_bytes;
    return (size_t)((unsigned)(number << c.shift) + (unsigned)(t & mask)) * tok_bytes;
  };
  uint32_t own_off = 0;                          // byte offset in the request's own-token block of row lane % 32 of a tile of own tokens
  auto own_rows = [&](int j) {
    const int rho = (j - nt) * FT + n32;
    int bl, tok;
    divmod_small(rho < Ru ? rho : 0, c.u, c.rcp_u, &bl, &tok);
    int prow = (beam0 + bl) * c.ND + tok;
    if (c.slot) {                                // (an entry outside the block falls back to the beam's own row)
      const int sl = c.slot[(size_t)bu * (unsigned)(c.W * c.ND) + (unsigned)prow];
      prow = (unsigned)sl < (unsigned)(c.W * c.ND) ? sl : prow;
    }
    own_off = (uint32_t)prow * own_bytes;
  };
  struct Stage8 { uint2 r[KV8 ? NLD : 1]; };
  Stage8 k8, v8;
  auto ask = [&](bool is_k, int j) __attribute__((always_inline)) {
    if (j < nt) {
#pragma unroll
      for (int i = 0; i < NLD; i++) {
        uint32_t row;
        const size_t at = chunk_at(j, i, &row);
        const int r = i * RPC + lane / PPR;
        if (KV8) (is_k ? k8 : v8).r[i] = *(const uint2*)((is_k ? k_base : v_base) + at + row + (uint32_t)(lane % PPR) * 8);
        else dma(lds_0 + (uint32_t)((is_k ? k_place : v_place) * 2 + i * 1024), (is_k ? k_base : v_base) + at, row + (uint32_t)(((lane % PPR) ^ (is_k ? T::swz_k(r) : T::swz_v(r))) * 16));
      }
    } else {
#pragma unroll
      for (int i = 0; i < NLD; i++) {
        const int r = i * RPC + lane / PPR, piece = (lane % PPR) ^ (is_k ? T::swz_k(r) : T::swz_v(r));
        dma(lds_0 + (uint32_t)((is_k ? k_place : v_place) * 2 + i * 1024), is_k ? ku_b : vu_b, (uint32_t)__shfl((int)own_off, r, 64) + (uint32_t)piece * 16);
      }
    }
  };
  // the tile is in its place: `later`: a tile's loads of the other kind came behind it
  auto there = [&](bool is_k, int j, bool later) __attribute__((always_inline)) {
    if (KV8 && j < nt) {
#pragma unroll
      for (int i = 0; i < NLD; i++) {
        const uint2 w = (is_k ? k8 : v8).r[i];
        const int r = i * RPC + lane / PPR;
        const bf16x2 e01 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.x, 1.0f, false), e23 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.x, 1.0f, true);
        const bf16x2 e45 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.y, 1.0f, false), e67 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.y, 1.0f, true);
        uint4 x;
        x.x = __builtin_bit_cast(uint32_t, e01); x.y = __builtin_bit_cast(uint32_t, e23);
        x.z = __builtin_bit_cast(uint32_t, e45); x.w = __builtin_bit_cast(uint32_t, e67);
        *(uint4*)(smem + (is_k ? k_place : v_place) + r * D + ((lane % PPR) ^ (is_k ? T::swz_k(r) : T::swz_v(r))) * 8) = x;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else if (!KV8 && later) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"i"(NLD) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
  };

  f32x16 o_acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; db++)
#pragma unroll
    for (int i = 0; i < 16; i++) o_acc[db][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float cp = KV8 ? c.c * c.k_scale : c.c;
  const typename T::Rd rdo = T::make_rd(lane, (int)lds_0);
  int j = wave_u;
  if (j < total) {
    if (j >= nt) own_rows(j);
    ask(true, j);
    ask(false, j);
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(2 * NLD) : "memory");           // (Q came before them)
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __syncthreads();
  bf16x8 qop[D / 16];
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) qop[ks] = T::read_k(q_place, rdo, 0, ks);
  bool own_units = !KV8;                         // O is in true units, not in those of the FP8 codes
  for (; j < total; j += 4) {
    const bool own = j >= nt, more = j + 4 < total;
    there(true, j, true);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; i++) s[i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(T::read_k(k_place, rdo, 0, ks), qop[ks], s, 0, 0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                       // (K has been read)
    if (more) {
      if (j + 4 >= nt) own_rows(j + 4);
      ask(true, j + 4);
    }
    // what the column may see of the tile: rows [lo, lo + n)
    const int lo = own ? my_lo - (j - nt) * FT : 0;
    const unsigned n = own ? (qrow >= 0 ? (unsigned)c.u : 0u) : (unsigned)(seg1 - (seg0 + j * FT));
    const float cs = own ? c.c : cp;
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; i++) {
      s[i] = (unsigned)(8 * (i / 4) + 4 * G + (i % 4) - lo) < n ? s[i] : -INFINITY;
      mx = fmaxf(mx, s[i]);
    }
    mx = halves_max(mx) * cs;
    if (KV8 && own && !own_units) {
      own_units = true;
#pragma unroll
      for (int db = 0; db < D / 32; db++)
#pragma unroll
        for (int i = 0; i < 16; i++) o_acc[db][i] *= c.v_scale;
    }
    if (__any(mx > m_run)) {
      const float m_new = fmaxf(m_run, mx), scale = mx > m_run ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
      l_run *= scale;
      m_run = m_new;
#pragma unroll
      for (int db = 0; db < D / 32; db++)
#pragma unroll
        for (int i = 0; i < 16; i++) o_acc[db][i] *= scale;
    }
    const float ref = m_run > -INFINITY ? m_run : 0.f;
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], cs, -ref));
      l_run += p[i];
    }
    bf16x8 pop[2];
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int e = 0; e < 8; e++) pop[t][e] = (__bf16)p[8 * t + e];
    there(false, j, more);
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int db = 0; db < D / 32; db++) o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(T::read_v(v_place, rdo, t, db), pop[t], o_acc[db], 0, 0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                       // (V has been read)
    if (more) ask(false, j + 4);
  }
  if (!own_units) {
#pragma unroll
    for (int db = 0; db < D / 32; db++)
#pragma unroll
      for (int i = 0; i < 16; i++) o_acc[db][i] *= c.v_scale;
  }

  // ---- the four wavefronts' parts join in LDS, each in its own places; then every one has columns of its own to write
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  f32x2* s_ml = (f32x2*)(smem + q_place);        // (everybody had read Q when it first asked for K again; with one tile or none: at the barrier above)
  f32x4* mine = (f32x4*)(smem + k_place) + lane;
#pragma unroll
  for (int e = 0; e < D / 8; e++) mine[64 * e] = f32x4{o_acc[e / 4][4 * (e % 4)], o_acc[e / 4][4 * (e % 4) + 1], o_acc[e / 4][4 * (e % 4) + 2], o_acc[e / 4][4 * (e % 4) + 3]};
  __syncthreads();
  if (G == 0) s_ml[wave * 32 + n32] = f32x2{l_tot > 0.f ? m_run : -INFINITY, l_tot};
  __syncthreads();
  if (qrow < 0) return;
  float top = -INFINITY, l = 0.f, a[4];
#pragma unroll
  for (int w = 0; w < 4; w++) top = fmaxf(top, s_ml[w * 32 + n32].x);
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const f32x2 ml = s_ml[w * 32 + n32];
    a[w] = ml.x > -INFINITY ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
    l += ml.y * a[w];
  }
  const LateArgs late = late_args() + ARG;
  const float inv = late->part_o ? 1.f : l > 0.f ? 1.0f / l : 0.f;
  const size_t row = ((size_t)bu * (unsigned)late->W + (unsigned)beam_q) * (unsigned)late->Hq + kvh * (unsigned)late->g + (unsigned)(qrow - beam_q * late->g);
  const int left = min(32, M - row_w);
  const size_t row_p = (((size_t)bu * (unsigned)ns + (unsigned)sp) * (unsigned)late->Hkv + kvh) * (unsigned)M + (unsigned)row_w;
  f32x4* part = (f32x4*)(late->part_o + row_p * D) + G * left + n32;
  constexpr int EW = D / 32;                     // pieces of four columns (8 e + 4 G ..) of a row that a wavefront has
#pragma unroll
  for (int k = 0; k < EW; k++) {
    const int e = wave_u * EW + k;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const f32x4 x = *((const f32x4*)(smem + w * 2 * PLACE) + 64 * e + lane);
#pragma unroll
      for (int i = 0; i < 4; i++) o[i] += x[i] * a[w];
    }
    if (late->part_o) {
      part[2 * e * left] = o;
    } else {
      bf16x4 h;
#pragma unroll
      for (int i = 0; i < 4; i++) h[i] = (__bf16)(o[i] * inv);
      *(bf16x4*)(late->out + row * D + 8 * e + 4 * G) = h;
    }
  }
  if (wave == 0 && G == 0) {
    if (late->part_o) *(f32x2*)(late->part_ml + (row_p + n32) * 2) = f32x2{top, l};
    else if (late->lse) late->lse[row] = l > 0.f ? (top + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
}

constexpr int paged_mix_lds_bytes(int d) { return attn_lds_bytes(d, 128, 1) > paged_few_lds_bytes(d) ? attn_lds_bytes(d, 128, 1) : paged_few_lds_bytes(d); }

// All rows by blocks of 128 or 256; all by blocks of 32; the prefix by blocks of 128 of all requests' rows, which are dealt first (arguments c), and each request's
// list by blocks of 32 (arguments few).  WHOLE: pages of 64 tokens and more.
template <int D, int NWAVES, bool KV8, int KS, bool FIND, bool WHOLE>
__global__ void __launch_bounds__(NWAVES * 64 * KS) __attribute__((amdgpu_waves_per_eu(2, 2))) k_paged_attn(AttnCtx c) {
  constexpr int NCB = 1;
  constexpr bool CAUSAL = false, PAGED = true;
#include "gr_attn_rows.inc"
}
template <int D, bool KV8>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, D == 64 ? 4 : 2))) k_paged_few(AttnCtx c) {
  few_rows<D, KV8, 0>(c, blockIdx.x);
}
template <int D, bool KV8, bool WHOLE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) k_paged_mix(AttnCtx c, AttnCtx few, unsigned blocks0) {
  if (blockIdx.x >= blocks0) {
    few_rows<D, KV8, 1>(few, blockIdx.x - blocks0);
    return;
  }
  constexpr int NCB = 1, NWAVES = 4, KS = 1;
  constexpr bool CAUSAL = false, FIND = false, PAGED = true;
#include "gr_attn_rows.inc"
}

}  // namespace

extern "C" size_t gr_beam_attn_paged_workspace_bytes(const gr_attn_paged_params* p) {
  if (!p || !shapes_ok(p)) return 0;
  return paged_workspace(p, plan_paged(p));
}

extern "C" gr_status gr_diag_attn_paged_plan(const gr_attn_paged_params* p, int32_t* plan) {
  if (!p || !plan || !shapes_ok(p)) return GR_ERR_INVALID_ARG;
  const PagedPlan a = plan_paged(p);
  plan[0] = a.rows; plan[1] = a.ns[0]; plan[2] = a.ns[1]; plan[3] = a.ks; plan[4] = a.find;
  return GR_OK;
}

extern "C" gr_status gr_beam_attn_paged(const gr_attn_paged_params* p, void* workspace, size_t workspace_bytes, void* stream_) {
  const hipStream_t stream = (hipStream_t)stream_;
  if (!p || p->prefix_L < 0 || p->max_L < 0) return GR_ERR_INVALID_ARG;
  if ((int64_t)p->prefix_L + p->max_L >= kMaxKeys) return GR_ERR_UNSUPPORTED;
  if (!shapes_ok(p)) return GR_ERR_INVALID_ARG;
  if (p->ND < 0 || p->u < 0 || p->u > p->ND || p->max_pages < 0 || p->n_pages < 0) return GR_ERR_INVALID_ARG;
  if (p->kv_type != GR_KV_BF16 && p->kv_type != GR_KV_FP8 && p->kv_type != GR_KV_FP4) return GR_ERR_INVALID_ARG;
  const bool kv8 = p->kv_type == GR_KV_FP8;
  auto positive = [](float s) { return s > 0.f && s < INFINITY; };
  if (!positive(p->sm_scale) || (kv8 && (!positive(p->k_scale) || !positive(p->v_scale)))) return GR_ERR_INVALID_ARG;
  if (!p->q || !p->out) return GR_ERR_INVALID_ARG;
  if (p->prefix_L + (int64_t)p->max_L > 0 && (!p->k_pages || !p->v_pages || p->n_pages == 0)) return GR_ERR_INVALID_ARG;
  if (p->prefix_L > 0 && !p->prefix_pages) return GR_ERR_INVALID_ARG;
  if (p->max_L > 0 && (!p->block_table || !p->seq_lens || p->max_L > (int64_t)p->max_pages * p->page_size)) return GR_ERR_INVALID_ARG;
  if (p->u > 0 && (!p->k_unshared || !p->v_unshared)) return GR_ERR_INVALID_ARG;
  if ((((uintptr_t)p->q | (uintptr_t)p->k_pages | (uintptr_t)p->v_pages | (uintptr_t)p->k_unshared | (uintptr_t)p->v_unshared | (uintptr_t)p->out) & 15) ||
      (((uintptr_t)p->prefix_pages | (uintptr_t)p->block_table | (uintptr_t)p->seq_lens | (uintptr_t)p->slot | (uintptr_t)p->lse_out) & 3))
    return GR_ERR_INVALID_ARG;
  if (p->d != 64 && p->d != 128) return GR_ERR_UNSUPPORTED;
  if (p->page_size < 16 || p->page_size > 1024 || (p->page_size & (p->page_size - 1)) || p->prefix_L % p->page_size) return GR_ERR_UNSUPPORTED;
  const int64_t g = p->Hq / p->Hkv;
  if ((int64_t)p->n_pages * p->page_size >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
  if ((int64_t)p->n_pages * p->page_size * p->Hkv * p->d >= ((int64_t)1 << 41)) return GR_ERR_UNSUPPORTED;      // (a page's address in 32 bits of 1 KiB)
  if ((int64_t)p->Hkv * p->d > 65536 || p->W * g >= ((int64_t)1 << 22)) return GR_ERR_UNSUPPORTED;          // row numbers go through small_div, whose bound is 2^22
  if ((int64_t)p->W * p->Hq * p->d >= ((int64_t)1 << 31) || (int64_t)p->W * p->ND * p->Hkv * p->d >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;

  if (p->kv_type == GR_KV_FP4) return gr_paged_fp4(p, workspace, workspace_bytes, stream);
  return run_paged(p, workspace, workspace_bytes, stream, [&](const PagedPlan& plan, const AttnCtx& c0, const AttnCtx& c, unsigned grid, unsigned blocks0) {
    const bool pack = plan.ns[0] > 0;
    auto rows = [&](auto dim, auto fp8, auto whole) -> gr_status {
      constexpr int D = decltype(dim)::value;
      constexpr bool K8 = decltype(fp8)::value, WH = decltype(whole)::value;
      if (pack) return launch<k_paged_mix<D, K8, WH>>(paged_mix_lds_bytes(D), 256, grid, stream, c0, c, blocks0);
      if (plan.rows == 32) return launch<k_paged_few<D, K8>>(paged_few_lds_bytes(D), 256, grid, stream, c);
      if (plan.ks == 2) return launch<k_paged_attn<D, 4, K8, 2, false, WH>>(attn_lds_bytes(D, 128, 2), 512, grid, stream, c);
      if (plan.rows == 128) {
        if (plan.find) return launch<k_paged_attn<D, 4, K8, 1, true, WH>>(attn_lds_bytes(D, 128, 1), 256, grid, stream, c);
        return launch<k_paged_attn<D, 4, K8, 1, false, WH>>(attn_lds_bytes(D, 128, 1), 256, grid, stream, c);
      }
      if (plan.find) return launch<k_paged_attn<D, 8, K8, 1, true, WH>>(attn_lds_bytes(D, 256, 1), 512, grid, stream, c);
      return launch<k_paged_attn<D, 8, K8, 1, false, WH>>(attn_lds_bytes(D, 256, 1), 512, grid, stream, c);
    };
    auto of_page = [&](auto dim, auto fp8) { return p->page_size >= KT ? rows(dim, fp8, std::true_type()) : rows(dim, fp8, std::false_type()); };
    auto of_type = [&](auto dim) { return kv8 ? of_page(dim, std::true_type()) : of_page(dim, std::false_type()); };
    return p->d == 128 ? of_type(std::integral_constant<int, 128>()) : of_type(std::integral_constant<int, 64>());
  });
}
