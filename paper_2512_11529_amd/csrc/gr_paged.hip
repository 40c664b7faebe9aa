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
#include "gr_attn_rows.hpp"

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

PagedPlan plan_paged(const gr_attn_paged_params* p) {
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
  if (p->kv_type != GR_KV_BF16 && p->kv_type != GR_KV_FP8) return GR_ERR_INVALID_ARG;
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
  if (const gr_status st = p->d == 128 ? of_type(std::integral_constant<int, 128>()) : of_type(std::integral_constant<int, 64>())) return st;
  if (j.part_o) {
    if (p->d == 128) hipLaunchKernelGGL((k_paged_join<128>), dim3((unsigned)join), dim3(256), 0, stream, j);
    else hipLaunchKernelGGL((k_paged_join<64>), dim3((unsigned)join), dim3(256), 0, stream, j);
  }
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
