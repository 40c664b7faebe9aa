// gr_beam_attn_paged: the decode step's attention over a prompt cache in pages of a pool, behind a prefix that all requests share.
//
// The tiles, their layout in LDS and the loop that keeps matrix and vector pipes busy together are gr_beam_attn's (gr_attn_tile.hpp).  What differs is where the
// tokens lie and which rows meet which tokens:
//   - Token t of a row's keys is in page t / page_size of its list of pages: the prefix's pages, then the request's.  A prefix is whole
//     pages, so both are one list.  A wavefront brings 1 KiB of a tile at a time, 4 or 8 consecutive tokens, which lie in one page
//     (pages hold 16 tokens at least): its address is scalar work beside the MFMAs, from page numbers that a lane each holds.
//   - Softmax partials (maximum, sum, O) of disjoint sets of keys join exactly, so the prefix may be met by other workgroups than the rest.  A workgroup's
//     128 or 256 rows share their keys: the rows of one (request, KV head) pair share all of them (W * g rows), the rows of ALL requests
//     share the prefix.  Where a request's rows leave most of a workgroup empty, part 0 of the launch packs all requests' rows against the prefix and
//     part 1 takes each request's own pages; a second kernel joins the partials.  Else a row walks the whole list by itself.
//   - Where a request's rows of a KV head are few, 32 of them meet the keys in a workgroup whose wavefronts share out the keys and not the rows.
#include <type_traits>
#include "gr_attn_tile.hpp"

namespace {

constexpr int kSegPages = 2048;       // pages of a segment, at most: their numbers wait in LDS

struct PagedPart {
  int M, MB, ns, groups;              // rows that share their keys, blocks of them, segments of the keys, workgroups / MB
  uint32_t inv_mb, inv_ns;            // for div_by
};
struct PagedCtx {
  int B, W, Hq, Hkv, g, ND, u;
  int prefix, own_prefix;             // tokens of the prefix, and those of it that part 1 meets (all or none)
  int max_L, max_pages, n_pages, shift;
  unsigned grid0;                     // workgroups of part 0
  PagedPart part0, part1;
  uint32_t inv_hkv;
  float rcp_g, rcp_u;
  float c;                            // sm_scale * log2(e)
  float k_scale, v_scale;             // FP8 pools: value = code * scale (1 for bf16)
  const uint16_t* q;
  const char* kp;
  const char* vp;
  const int32_t* prefix_pages;
  const int32_t* table;
  const int32_t* lens;
  const uint16_t* ku;
  const uint16_t* vu;
  const int32_t* slot;
  uint16_t* out;
  float* lse;
  float* part_o;                      // rows of D fp32 in blocks of 32 (D / 4, row, 4), unnormalised; nullptr: rows are not split
  float* part_ml;                     // (maximum in log2 units, sum) of each
};

// A pointer that is the same in all lanes, in scalar registers (where a load's address has to be, and the compiler has it in vector ones).
template <class P>
__device__ __forceinline__ P* scalar(P* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p;
  uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
  // (a vector instruction's scalar result may be a load's address five wait states later, which the compiler keeps to only for loads that it sees)
  asm volatile("s_nop 4" : "+s"(lo), "+s"(hi));
  return (P*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

// The kernel's arguments, read where this stands and not before: what only late code needs takes no scalar registers through the loop.
typedef const __attribute__((address_space(4))) PagedCtx* LateArgs;
__device__ __forceinline__ LateArgs late_args() {
  LateArgs a = (LateArgs)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return a;
}

constexpr int paged_lds_bytes(int d, int mwg) { return 4 * KT * d * 2 + (mwg == 256 ? mwg * d * 2 : 0) + kSegPages * 4; }

// One workgroup of NWAVES wavefronts and as many blocks of 32 rows.  SHARED: rows of all requests against the prefix (part 0), without own tokens; else rows of one
// request against its whole list (part 1).
template <int D, int NWAVES, bool KV8, bool SHARED>
__device__ __forceinline__ void tile_rows(const PagedCtx& c, const unsigned id) {
  using T = AttnTile<D, 1>;
  constexpr int NT = NWAVES * 64, MWG = NWAVES * 32;
  constexpr int PPR = D / 8;                     // 16-byte pieces of a bf16 row
  constexpr int TILE = KT * D;                   // elements of a K or V tile in LDS
  constexpr int CPW = TILE * 2 / 1024 / NWAVES;  // chunks of 1 KiB (FP8: of 512 bytes of codes) per wave and tile
  constexpr int RPC = 1024 / (D * 2);            // tokens of a chunk
  constexpr int EB = KV8 ? 1 : 2;                // bytes of a stored element
  constexpr int UR = 32;                         // rows of a mini-tile of own tokens
  // LDS: K and V tiles, two of each, K(j) and V(j) in slot (j + flip) % 2; then, for 8 waves, the Q hand-over, which 4 waves have in the V tiles' place; then
  // the page numbers.  After the loop a wave's own-token rows and its output take the tiles' place (8 waves: K rows and output Q's).
  extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];
  constexpr bool kQSeparate = NWAVES == 8;
  constexpr int HEAD = NWAVES == 4 ? 0 : D == 128 ? 3 : 2;
  uint16_t* s_k = smem;
  uint16_t* s_v = smem + 2 * TILE;
  int* s_pages = (int*)(smem + 4 * TILE + (kQSeparate ? MWG * D : 0));
  constexpr int q_place = (kQSeparate ? 4 : 2) * TILE;
  const int tid = (int)threadIdx.x, wave = tid >> 6, lane = tid & 63, G = lane >> 5, n32 = lane & 31;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);

  // ---- the unit: a block of rows and a segment of their keys.  Workgroups are dealt round-robin to the 8 XCDs: ids congruent mod 8 share an L2, and the
  // row blocks that read the same keys get consecutive slots of one XCD.
  const PagedPart pt = SHARED ? c.part0 : c.part1;
  const int M = pt.M, ns = pt.ns;
  const unsigned place = id >> 3, nth = div_by(place, (unsigned)pt.MB, pt.inv_mb);
  const int group = (int)(nth * 8 + (id & 7u)), mbi = (int)(place - nth * (unsigned)pt.MB);
  if (group >= pt.groups) return;
  const unsigned gq = div_by((unsigned)group, (unsigned)ns, pt.inv_ns);
  const int sp = group - (int)gq * ns;
  const unsigned bu = SHARED ? 0u : div_by(gq, (unsigned)c.Hkv, c.inv_hkv);
  const unsigned kvh = SHARED ? gq : gq - bu * (unsigned)c.Hkv;
  const int L = __builtin_amdgcn_readfirstlane(SHARED || c.max_L == 0 ? 0 : min(max(c.lens[bu], 0), c.max_L));

  // ---- Q: the workgroup's rows come into LDS like K tiles, rows past the last one as that one (their columns are dropped)
  auto dma = [&](uint32_t lds_addr, const char* gbase, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(off), "s"(gbase) : "memory", "m0");
  };
  const uint32_t lds_0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)smem;
  const int beam_wg = __builtin_amdgcn_readfirstlane(small_div(mbi * MWG, c.rcp_g));
  const uint16_t* q_b = scalar(c.q + (((size_t)bu * (unsigned)c.W + (unsigned)beam_wg) * (unsigned)c.Hq + kvh * (unsigned)c.g) * D);
#pragma unroll
  for (int i = 0; i < MWG / RPC / NWAVES; i++) {
    const int ch = i * NWAVES + wave_u, rl = ch * RPC + lane / PPR, r = min(mbi * MWG + rl, M - 1), beam = small_div(r, c.rcp_g);
    dma(lds_0 + (uint32_t)(q_place + ch * RPC * D) * 2, (const char*)q_b,
        (uint32_t)((beam - beam_wg) * c.Hq + (r - beam * c.g)) * (D * 2) + (uint32_t)(((lane % PPR) ^ T::swz_k(rl)) * 16));
  }

  const int front = SHARED ? c.prefix : c.own_prefix, keys = front + L;        // tokens of the list
  int chunk = (int)div_by((unsigned)keys + (unsigned)ns - 1u, (unsigned)ns, pt.inv_ns);
  chunk = (chunk + KT - 1) / KT * KT;
  const int seg0 = min(keys, sp * chunk), seg1 = min(keys, seg0 + chunk);
  const int ntiles = (seg1 - seg0 + KT - 1) / KT, tl = ntiles - 1;
  const int flip = tl & 1;
  // the segment that takes the beams' own tokens: the first, or the last where it has fewer tiles
  const int own_sp = max(0, keys - (ns - 1) * chunk + KT - 1) / KT < chunk / KT ? ns - 1 : 0;
  const bool own_stage = !SHARED && c.u > 0 && sp == own_sp;

  // ---- page numbers of the segment; one outside the pool is read as page 0
  const int mask = (1 << c.shift) - 1, page0 = seg0 >> c.shift, n_seg = ntiles > 0 ? ((seg1 - 1) >> c.shift) - page0 + 1 : 0;
  for (int i = tid; i < n_seg; i += NT) {
    const int p = page0 + i - (front >> c.shift);
    const int number = p < 0 ? c.prefix_pages[page0 + i] : c.table[(size_t)bu * (unsigned)c.max_pages + (unsigned)p];
    s_pages[i] = (unsigned)number < (unsigned)c.n_pages ? number : 0;
  }
  __syncthreads();
  int window = 0, numbers = n_seg > 0 ? s_pages[min(lane, n_seg - 1)] : 0;      // lane i: number of page window + i of the segment

  const int row_w = mbi * MWG + wave_u * 32;     // the wave's first row
  const int qrow = row_w + n32 < M ? row_w + n32 : -1;
  const int beam_q = small_div(max(qrow, 0), c.rcp_g);
  const float cp = KV8 ? c.c * c.k_scale : c.c;  // exponent scale of the prompt loop
  const typename T::Rd rdo = T::make_rd(lane, (int)lds_0);

  // ---- tiles.  Wave w brings chunks w, w + NWAVES, ... of a tile: lane l fills slot l % PPR of row chunk * RPC + l / PPR with the piece that belongs
  // there.  Rows behind the segment's end (last tile only) re-read its last token: what their slots hold may be no number at all, which
  // a score of -inf and a probability of 0 would not cancel.  V's tile is the K tile before, at the same place of its own pool.
  const uint32_t tok_bytes = (uint32_t)c.Hkv * D * EB;
  const char* k_base = c.kp + (size_t)kvh * D * EB;
  const char* v_base = c.vp + (size_t)kvh * D * EB;
  const int last_tok = seg1 - 1, last_chunk = last_tok & ~(RPC - 1);
  const uint32_t k_piece = KV8 ? (uint32_t)(lane % PPR) * 8 : (uint32_t)((lane % PPR) ^ T::swz_k(wave * RPC + lane / PPR)) * 16;      // (swizzles repeat every 16 rows)
  const uint32_t v_piece = KV8 ? k_piece : (uint32_t)((lane % PPR) ^ T::swz_v(wave * RPC + lane / PPR)) * 16;
  static_assert(NWAVES * RPC % 16 == 0, "a lane's chunks are alike");
  uint32_t koff[CPW], voff[CPW];
  uint32_t k_row[CPW], v_row[CPW];               // chunks' first slots in the pools
  int kt = 0;                                    // the tile that k_row is of
  auto locate = [&]() __attribute__((always_inline)) {
    const int tok = seg0 + kt * KT;
    if (__builtin_expect((min(tok + KT - 1, last_tok) >> c.shift) - page0 - window >= 64, 0)) {
      window = (tok >> c.shift) - page0;
      numbers = s_pages[min(window + lane, n_seg - 1)];
    }
#pragma unroll
    for (int i = 0; i < CPW; i++) {
      const int t = min(tok + (i * NWAVES + wave_u) * RPC, last_chunk);
      const int number = __builtin_amdgcn_readlane(numbers, (t >> c.shift) - page0 - window);
      k_row[i] = (unsigned)(number << c.shift) + (unsigned)(t & mask);
    }
  };
  auto offsets_of_last = [&](uint32_t (&off)[CPW], uint32_t piece) {
#pragma unroll
    for (int i = 0; i < CPW; i++) {
      const int t = seg0 + tl * KT + (i * NWAVES + wave_u) * RPC;
      off[i] = (uint32_t)(min(t + lane / PPR, last_tok) - min(t, last_chunk)) * tok_bytes + piece;
    }
  };
  auto next_tile = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < CPW; i++) v_row[i] = k_row[i];
    if (__builtin_expect(kt >= tl, 0)) offsets_of_last(voff, v_piece);
    // (a value that the compiler knows nothing of between the two: it joins their stores through a pointer, and both arrays go to memory)
    asm volatile("" : "+s"(kt));
    if (__builtin_expect(kt < tl, 1)) {
      kt++;
      locate();
      if (kt == tl) offsets_of_last(koff, k_piece);
    }
  };
  auto tload_chunk = [&](bool is_k, int slot, int i) {
    dma(lds_0 + (uint32_t)((is_k ? 0 : 2 * TILE) + slot * TILE) * 2 + (uint32_t)(i * NWAVES + wave_u) * 1024, is_k ? k_base + (size_t)k_row[i] * tok_bytes : v_base + (size_t)v_row[i] * tok_bytes,
        is_k ? koff[i] : voff[i]);
  };
  auto tload = [&](bool is_k, int slot) {
#pragma unroll
    for (int i = 0; i < CPW; i++) tload_chunk(is_k, slot, i);
  };
  auto all_landed = [&]() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
  // FP8: eight codes a lane and chunk, in registers for a tile, then widened (exactly) into the same places
  struct Stage8 { uint2 r[CPW]; };
  auto gload8_piece = [&](bool is_k, int i) { return *(const uint2*)((is_k ? k_base + (size_t)k_row[i] * tok_bytes : v_base + (size_t)v_row[i] * tok_bytes) + (is_k ? koff[i] : voff[i])); };
  auto gload8 = [&](bool is_k) {
    Stage8 st;
#pragma unroll
    for (int i = 0; i < CPW; i++) st.r[i] = gload8_piece(is_k, i);
    return st;
  };
  auto widen8 = [](uint2 r) {
    const bf16x2 e01 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r.x, 1.0f, false);
    const bf16x2 e23 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r.x, 1.0f, true);
    const bf16x2 e45 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r.y, 1.0f, false);
    const bf16x2 e67 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r.y, 1.0f, true);
    uint4 v;
    v.x = __builtin_bit_cast(uint32_t, e01); v.y = __builtin_bit_cast(uint32_t, e23);
    v.z = __builtin_bit_cast(uint32_t, e45); v.w = __builtin_bit_cast(uint32_t, e67);
    return v;
  };
  const int row8 = tid / PPR, k8_to = row8 * D + ((tid % PPR) ^ T::swz_k(row8)) * 8, v8_to = row8 * D + ((tid % PPR) ^ T::swz_v(row8)) * 8;
  auto lstore8_piece = [&](uint16_t* dst, bool is_k, uint2 codes, int i) { *(uint4*)(dst + (is_k ? k8_to : v8_to) + i * (NT / PPR) * D) = widen8(codes); };
  auto lstore8 = [&](uint16_t* dst, bool is_k, const Stage8& st) {
#pragma unroll
    for (int i = 0; i < CPW; i++) lstore8_piece(dst, is_k, st.r[i], i);
  };

  // ---- geometry of the own tokens: a wave's 32 rows belong to a few beams, whose rows (beam_local * u + token) form mini-tiles of 32
  int beam0 = 0, Ru = 0;
  if (own_stage && row_w < M) {
    beam0 = __builtin_amdgcn_readfirstlane(small_div(row_w, c.rcp_g));
    Ru = (__builtin_amdgcn_readfirstlane(small_div(min(row_w + 31, M - 1), c.rcp_g)) - beam0 + 1) * c.u;
  }
  const int my_lo = qrow >= 0 ? (beam_q - beam0) * c.u : -1;
  const uint32_t own_bytes = (uint32_t)c.Hkv * D * 2;
  auto own_row = [&](int pass) {                 // byte offset in the request's own-token block of row pass * 32 + lane % 32 (past the last: of the first)
    const int rho = pass * UR + n32;
    int bl, tok;
    divmod_small(rho < Ru ? rho : 0, c.u, c.rcp_u, &bl, &tok);
    int prow = (beam0 + bl) * c.ND + tok;
    if (c.slot && Ru > 0) {                      // (an entry outside the block falls back to the beam's own row)
      const int sl = c.slot[(size_t)bu * (unsigned)(c.W * c.ND) + (unsigned)prow];
      prow = (unsigned)sl < (unsigned)(c.W * c.ND) ? sl : prow;
    }
    return (uint32_t)prow * own_bytes;
  };
  const char* ku_b = (const char*)(c.ku + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  const char* vu_b = (const char*)(c.vu + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  const int own_k = (NWAVES == 8 ? 4 * TILE : 0) + wave_u * UR * D, own_v = (NWAVES == 8 ? 0 : 2 * TILE) + wave_u * UR * D;
  auto uload = [&](bool is_k, uint32_t row_off, int rows) {
#pragma unroll
    for (int i = 0; i < UR / RPC; i++) {
      if (i * RPC >= rows) break;                // (wave-uniform)
      const int row = i * RPC + lane / PPR, piece = (lane % PPR) ^ (is_k ? T::swz_k(row) : T::swz_v(row));
      dma(lds_0 + (uint32_t)((is_k ? own_k : own_v) * 2 + i * 1024), is_k ? ku_b : vu_b, (uint32_t)__shfl((int)row_off, row, 64) + (uint32_t)piece * 16);
    }
  };

  f32x16 o_acc[D / 32][1];
#pragma unroll
  for (int db = 0; db < D / 32; db++)
#pragma unroll
    for (int i = 0; i < 16; i++) o_acc[db][0][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;          // reference of the exponentials in log2 units, and sum

  // ---- the first tiles
#pragma unroll
  for (int i = 0; i < CPW; i++) {
    koff[i] = (uint32_t)(lane / PPR) * tok_bytes + k_piece;
    voff[i] = (uint32_t)(lane / PPR) * tok_bytes + v_piece;
    k_row[i] = v_row[i] = 0;
  }
  Stage8 k8, v8, k8b;
  if (ntiles > 0) {
    locate();
    if (tl == 0) offsets_of_last(koff, k_piece);
    if (KV8) {
      k8 = gload8(true);
      next_tile();
      v8 = gload8(false);
      k8b = gload8(true);
    } else {
      tload(true, flip);
      next_tile();
      if (kQSeparate) tload(false, flip);
      tload(true, flip ^ 1);
    }
  }
  const uint32_t prow0 = own_stage ? own_row(0) : 0;
  bf16x8 qop[1][D / 16];
  auto first8 = [&]() {
    lstore8(s_k + flip * TILE, true, k8); lstore8(s_v + flip * TILE, false, v8); lstore8(s_k + (flip ^ 1) * TILE, true, k8b);
    next_tile();
    k8 = gload8(true);
    v8 = gload8(false);
  };
  if (KV8 && kQSeparate && ntiles > 0) first8();
  // (Q and K(0), which the first scores take; what was asked for after them may be on its way)
  if (ntiles == 0 || KV8) all_landed();
  else asm volatile("s_waitcnt vmcnt(%0)" ::"i"((kQSeparate ? 2 : 1) * CPW) : "memory");
  __syncthreads();
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) qop[0][ks] = T::read_k(q_place + wave_u * 32 * D, rdo, 0, ks);
  if (!kQSeparate) {
    __syncthreads();                             // the V tiles' place is free
    if (!KV8 && ntiles > 0) tload(false, flip);
    if (KV8 && ntiles > 0) { first8(); __syncthreads(); }
  }

  // ---- the loop: step t makes S(t+1) = K(t+1).Q^T beside the exponentials of S(t), then O += V(t).P(t).  K(t+2) and V(t+1) (FP8: one tile further, into
  // registers) are on their way meanwhile, into the places of K(t) and V(t-1), which everybody had read when the workgroup met in the step before.
  if (ntiles > 0) {
    float rs = 0.f;                              // sum of the tile before
    bf16x8 pop[KT / 16];
    auto raise_to = [&](float mx) __attribute__((always_inline)) {       // O and the sum go with the reference, once it is exceeded by more than kLazy
      if (__any(mx > m_run + T::kLazy)) {
        const float m_new = fmaxf(m_run, mx), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
        for (int db = 0; db < D / 32; db++)
#pragma unroll
          for (int i = 0; i < 16; i++) o_acc[db][0][i] *= alpha;
        l_run *= alpha;
        m_run = m_new;
      }
    };
    auto meet = [&]() __attribute__((always_inline)) {
      if (KV8) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    bf16x8 head[T::PF];
    auto step = [&](auto slot_c, f32x16 (&s_in)[KT / 32][1], f32x16 (&s_out)[KT / 32][1]) {
      constexpr int slot = decltype(slot_c)::value;
      l_run += rs;
      raise_to(T::colmax(s_in) * cp);
      next_tile();
      T::template fused<HEAD>([&](int j) __attribute__((always_inline)) {
        const int i = j / T::SPREAD;
        if (j % T::SPREAD || i >= 2 * CPW) return;
        if (KV8) {
          if (i < CPW) {
            lstore8_piece(s_k + slot * TILE, true, k8.r[i], i);              // K(t+2) over K(t)
            k8.r[i] = gload8_piece(true, i);                                 // K(t+3)
          } else {
            lstore8_piece(s_v + (slot ^ 1) * TILE, false, v8.r[i - CPW], i - CPW);       // V(t+1)
            v8.r[i - CPW] = gload8_piece(false, i - CPW);                    // V(t+2)
          }
        } else if (i < CPW) {
          tload_chunk(true, slot, i);                                        // K(t+2) over K(t)
        } else {
          tload_chunk(false, slot ^ 1, i - CPW);                             // V(t+1) over V(t-1)
        }
      }, meet, head, slot * TILE, (slot ^ 1) * TILE, (2 + slot) * TILE, qop, s_in, s_out, o_acc, m_run, cp, rs, pop, rdo);
    };
    f32x16 s_a[KT / 32][1], s_b[KT / 32][1];
    T::qk(flip * TILE, qop, s_a, rdo);
    meet();                                      // K(1) and V(0) are there
    if (ntiles > 1) {
#pragma unroll
      for (int i = 0; i < HEAD; i++) head[i] = T::read_k((flip ^ 1) * TILE, rdo, i % 2, i / 2);
    }
    // (an odd step goes first, so that the loop runs whole pairs and the last tile is in s_a and slot 0)
    int t = 0;
    if (flip) {
      step(std::integral_constant<int, 1>(), s_a, s_b);
#pragma unroll
      for (int sub = 0; sub < KT / 32; sub++) s_a[sub][0] = s_b[sub][0];
      t = 1;
    }
    for (; t < tl; t += 2) {
      step(std::integral_constant<int, 0>(), s_a, s_b);
      step(std::integral_constant<int, 1>(), s_b, s_a);
    }
    // the last tile, the only one that can be partial
    l_run += rs;
    if (own_stage) uload(true, prow0, Ru);       // (where K tiles were, or Q)
    const int tok0 = seg0 + tl * KT;
    if (tok0 + KT > seg1) {
#pragma unroll
      for (int sub = 0; sub < KT / 32; sub++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
          const int kv = tok0 + sub * 32 + 8 * (i / 4) + 4 * G + (i % 4);
          s_a[sub][0][i] = kv >= seg1 ? -INFINITY : s_a[sub][0][i];
        }
    }
    raise_to(T::colmax(s_a) * cp);
    T::finish(2 * TILE, s_a, o_acc, m_run, cp, rs, rdo);
    l_run += rs;
    if (KV8) {                                   // prompt loop -> true units
#pragma unroll
      for (int db = 0; db < D / 32; db++)
#pragma unroll
        for (int i = 0; i < 16; i++) o_acc[db][0][i] *= c.v_scale;
    }
  }
  __syncthreads();                               // every wave is done with the tiles

  // ---- the beams' own tokens: 32 rows in LDS at a time, this wave's alone, of which a column keeps its own beam's
  if (own_stage) {
    if (ntiles == 0) uload(true, prow0, Ru);
    uint32_t row_off = prow0;
    for (int pass = 0; pass * UR < Ru; pass++) {
      const int used = Ru - pass * UR;           // (V: whole halves of 16 rows, whose probabilities are 0 past the last one)
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");            // (K is there, and the pass before has read V)
      uload(false, row_off, min(UR, (used + 15) & ~15));
      const int base = pass * UR - my_lo;
      const unsigned rows = my_lo >= 0 ? (unsigned)c.u : 0u;
      f32x16 su;
#pragma unroll
      for (int i = 0; i < 16; i++) su[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ks++) su = __builtin_amdgcn_mfma_f32_32x32x16_bf16(T::read_k(own_k, rdo, 0, ks), qop[0][ks], su, 0, 0, 0);
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; i++) {
        su[i] = (unsigned)(base + 8 * (i / 4) + 4 * G + (i % 4)) < rows ? su[i] : -INFINITY;
        mx = fmaxf(mx, su[i]);
      }
      mx = halves_max(mx) * c.c;
      const float m_new = fmaxf(m_run, mx);      // (-inf while the column has seen no key at all)
      const float scale = mx > m_run ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
      m_run = m_new;
#pragma unroll
      for (int db = 0; db < D / 32; db++)
#pragma unroll
        for (int i = 0; i < 16; i++) o_acc[db][0][i] *= scale;
      const float ref = m_run > -INFINITY ? m_run : 0.f;
      float pr[16], rsum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; i++) {
        pr[i] = __builtin_amdgcn_exp2f(fmaf(su[i], c.c, -ref));
        rsum += pr[i];
      }
      l_run = l_run * scale + rsum;
      bf16x8 pu[UR / 16];
#pragma unroll
      for (int t = 0; t < UR / 16; t++)
#pragma unroll
        for (int e = 0; e < 8; e++) pu[t][e] = (__bf16)pr[8 * t + e];
      if (used > UR) { row_off = own_row(pass + 1); uload(true, row_off, used - UR); }       // (K has been read)
      all_landed();
#pragma unroll
      for (int t = 0; t < UR / 16; t++) {
        if (t > 0 && used <= 16 * t) break;
#pragma unroll
        for (int db = 0; db < D / 32; db++)
          o_acc[db][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(T::read_v(own_v, rdo, t, db), pu[t], o_acc[db][0], 0, 0, 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");                 // the mini-tiles are rewritten by the next pass
    }
  }

  // ---- normalised rows, or this segment's partials
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  const LateArgs late = late_args();
  const size_t head_wg = ((size_t)bu * (unsigned)late->W + (unsigned)beam_wg) * (unsigned)late->Hq + kvh * (unsigned)late->g;
  if (!late->part_o) {
    // The wave's 32 rows go through its own slice of LDS, so that memory sees whole rows
    uint16_t* s_o = smem + own_k;
    const float inv = l_tot > 0.f ? 1.0f / l_tot : 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; db++)
#pragma unroll
      for (int q4 = 0; q4 < 4; q4++) {
        const f32x2 a = {o_acc[db][0][4 * q4] * inv, o_acc[db][0][4 * q4 + 1] * inv};
        const f32x2 bb = {o_acc[db][0][4 * q4 + 2] * inv, o_acc[db][0][4 * q4 + 3] * inv};
        const bf16x2 ha = __builtin_convertvector(a, bf16x2), hb = __builtin_convertvector(bb, bf16x2);
        uint2 st;
        st.x = __builtin_bit_cast(uint32_t, ha);
        st.y = __builtin_bit_cast(uint32_t, hb);
        *(uint2*)(&s_o[n32 * D + ((4 * db + q4) ^ (n32 & (PPR - 1))) * 8 + 4 * G]) = st;
      }
    uint16_t* out_b = late->out + head_wg * D;
#pragma unroll
    for (int i = 0; i < 32 * PPR / 64; i++) {
      const int p = lane + 64 * i, rl = p / PPR, piece = p % PPR, rr = row_w + rl, beam = small_div(rr, c.rcp_g);
      const uint4 v = *(const uint4*)(&s_o[rl * D + (piece ^ (rl & (PPR - 1))) * 8]);
      if (rr < M) *(uint4*)(out_b + (uint32_t)(((beam - beam_wg) * late->Hq + (rr - beam * late->g)) * D + piece * 8)) = v;
    }
    if (late->lse && G == 0 && qrow >= 0)
      late->lse[((size_t)bu * (unsigned)late->W + (unsigned)beam_q) * (unsigned)late->Hq + kvh * (unsigned)late->g + (unsigned)(qrow - beam_q * late->g)] =
          l_tot > 0.f ? (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2 : -INFINITY;
  } else {
    // unnormalised O and (maximum, sum) as the lanes hold them: every store is a run of whole lines
    const int left = min(32, M - row_w);
    const size_t unit = SHARED ? (size_t)(unsigned)sp * (unsigned)late->Hkv + kvh
                               : (size_t)(unsigned)late->part0.ns * (unsigned)late->Hkv * (unsigned)late->B + ((size_t)bu * (unsigned)ns + (unsigned)sp) * (unsigned)late->Hkv + kvh;
    const size_t row_p = unit * (unsigned)M + (unsigned)row_w;
    if (qrow >= 0) {
      f32x4* part = (f32x4*)(late->part_o + row_p * D) + G * left + n32;
#pragma unroll
      for (int e = 0; e < D / 8; e++) {
        const f32x4 v = {o_acc[e / 4][0][4 * (e % 4)], o_acc[e / 4][0][4 * (e % 4) + 1], o_acc[e / 4][0][4 * (e % 4) + 2], o_acc[e / 4][0][4 * (e % 4) + 3]};
        part[2 * e * left] = v;
      }
      if (G == 0) {
        const f32x2 ml = {l_tot > 0.f ? m_run : -INFINITY, l_tot};
        *(f32x2*)(late->part_ml + (row_p + n32) * 2) = ml;
      }
    }
  }
}

// Up to 32 rows of a (request, KV head) pair: 32 rows of a workgroup of 128 would be all there is, and what counts is how soon the keys arrive.  Every wavefront
// holds the rows and takes every fourth 32 tokens of the segment through places of its own in LDS: K's next 32 are asked for as soon as the scores
// are made, V's as soon as its products are, and nobody waits for anybody until the four (maximum, sum, O) are joined in LDS.  The beams' own tokens are the
// list's last tiles.  Bound: memory; two workgroups of four wavefronts to a CU have up to 128 KB of loads on their way.
constexpr int paged_few_lds_bytes(int d) { return (4 * 2 * 32 + 32) * d * 2; }      // a K and a V place per wavefront, and Q
constexpr int paged_mix_lds_bytes(int d) { return paged_lds_bytes(d, 128) > paged_few_lds_bytes(d) ? paged_lds_bytes(d, 128) : paged_few_lds_bytes(d); }

template <int D, bool KV8>
__device__ __forceinline__ void few_rows(const PagedCtx& c, const unsigned id) {
  using T = AttnTile<D, 1>;
  constexpr int PPR = D / 8, RPC = 1024 / (D * 2), FT = 32, PLACE = FT * D, NLD = FT / RPC;      // NLD: loads of a place
  constexpr int EB = KV8 ? 1 : 2;
  extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];
  const int tid = (int)threadIdx.x, wave = tid >> 6, lane = tid & 63, G = lane >> 5, n32 = lane & 31;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const unsigned place = id >> 3, nth = div_by(place, (unsigned)c.part1.MB, c.part1.inv_mb);
  const int group = (int)(nth * 8 + (id & 7u)), mbi = (int)(place - nth * (unsigned)c.part1.MB), ns = c.part1.ns, M = c.part1.M;
  if (group >= c.part1.groups) return;
  const unsigned gq = div_by((unsigned)group, (unsigned)ns, c.part1.inv_ns);
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

  const int L = __builtin_amdgcn_readfirstlane(c.max_L == 0 ? 0 : min(max(c.lens[bu], 0), c.max_L));
  const int front = c.own_prefix, keys = front + L;
  int chunk = (int)div_by((unsigned)keys + (unsigned)ns - 1u, (unsigned)ns, c.part1.inv_ns);
  chunk = (chunk + KT - 1) / KT * KT;
  const int seg0 = min(keys, sp * chunk), seg1 = min(keys, seg0 + chunk);
  const int nt = (seg1 - seg0 + FT - 1) / FT;
  const bool own_stage = c.u > 0 && sp == (max(0, keys - (ns - 1) * chunk) < chunk ? ns - 1 : 0);
  const int qrow = row_w + n32 < M ? row_w + n32 : -1;
  const int beam_q = small_div(max(qrow, 0), c.rcp_g);
  const int Ru = own_stage ? (__builtin_amdgcn_readfirstlane(small_div(min(row_w + 31, M - 1), c.rcp_g)) - beam0 + 1) * c.u : 0;
  const int my_lo = (beam_q - beam0) * c.u;
  const int total = nt + (Ru + FT - 1) / FT;

  // ---- page numbers: lane i has that of page window + i of the list
  const int mask = (1 << c.shift) - 1, last_tok = seg1 - 1, last_chunk = last_tok & ~(RPC - 1), last_page = last_tok >> c.shift;
  auto numbers_from = [&](int first) {
    const int p = min(first + lane, max(last_page, 0)), q = p - (front >> c.shift);
    int number = 0;
    if (nt > 0) number = q < 0 ? c.prefix_pages[p] : c.table[(size_t)bu * (unsigned)c.max_pages + (unsigned)q];
    return (unsigned)number < (unsigned)c.n_pages ? number : 0;
  };
  int window = seg0 >> c.shift, numbers = numbers_from(window);
  const uint32_t tok_bytes = (uint32_t)c.Hkv * D * EB, own_bytes = (uint32_t)c.Hkv * D * 2;
  const char* k_base = c.kp + (size_t)kvh * D * EB;
  const char* v_base = c.vp + (size_t)kvh * D * EB;
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
  const LateArgs late = late_args();
  const float inv = late->part_o ? 1.f : l > 0.f ? 1.0f / l : 0.f;
  const size_t row = ((size_t)bu * (unsigned)late->W + (unsigned)beam_q) * (unsigned)late->Hq + kvh * (unsigned)late->g + (unsigned)(qrow - beam_q * late->g);
  const int left = min(32, M - row_w);
  const size_t row_p = ((size_t)(unsigned)late->part0.ns * (unsigned)late->Hkv * (unsigned)late->B + ((size_t)bu * (unsigned)ns + (unsigned)sp) * (unsigned)late->Hkv + kvh) * (unsigned)M + (unsigned)row_w;
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

// All rows by blocks of 128 or 256; all by blocks of 32; the prefix by blocks of 128 of all requests' rows, which are dealt first, and each request's list by blocks of 32.
template <int D, int NWAVES, bool KV8>
__global__ void __launch_bounds__(NWAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) k_paged_attn(PagedCtx c) {
  tile_rows<D, NWAVES, KV8, false>(c, blockIdx.x);
}
template <int D, bool KV8>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, D == 64 ? 4 : 2))) k_paged_few(PagedCtx c) {
  few_rows<D, KV8>(c, blockIdx.x);
}
template <int D, bool KV8>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) k_paged_mix(PagedCtx c) {
  if (blockIdx.x < c.grid0) tile_rows<D, 4, KV8, true>(c, blockIdx.x);
  else few_rows<D, KV8>(c, blockIdx.x - c.grid0);
}

// Joins a row's partials: those of part 0, whose rows are all requests' in one, then those of part 1.  A lane takes four columns of a row; eight rows of eight
// neighbouring lanes are a line.  Four segments are requested together.
template <int D>
__global__ void __launch_bounds__(256) k_paged_join(PagedCtx c) {
  constexpr int RPW = 1024 / D;
  static_assert(RPW % 8 == 0 && 32 % RPW == 0, "whole lines of one block");
  const unsigned M = (unsigned)c.part1.M, per_pair = (M + RPW - 1) / RPW, pair = blockIdx.x / per_pair;
  const unsigned b = pair / (unsigned)c.Hkv, kvh = pair - b * (unsigned)c.Hkv;
  const int t = (int)threadIdx.x, piece = (t >> 3) % (D / 4);
  const unsigned r = (blockIdx.x - pair * per_pair) * RPW + (unsigned)((t & 7) + 8 * (t / (2 * D)));
  if (r >= M) return;
  const int ns0 = c.part0.ns, ns = ns0 + c.part1.ns;
  const unsigned M0 = (unsigned)c.B * M, r0 = b * M + r;
  auto row_of = [&](int s) {
    return s < ns0 ? ((size_t)(unsigned)s * (unsigned)c.Hkv + kvh) * M0 + r0
                   : (size_t)(unsigned)ns0 * (unsigned)c.Hkv * M0 + (((size_t)b * (unsigned)c.part1.ns + (unsigned)(s - ns0)) * (unsigned)c.Hkv + kvh) * M + r;
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

// The launch: rows of a workgroup of part 1 (32, 128, 256), whether the prefix is met by all requests' rows together (ns[0] > 0; then 32), and segments of the keys.
struct PagedPlan { int rows, ns[2]; };
PagedPlan plan_paged(const gr_attn_paged_params* p) {
  PagedPlan plan;
  const int64_t g = p->Hq / p->Hkv, M = p->W * g, all = p->B * M;
  auto blocks = [](int64_t rows, int mwg) { return (rows + mwg - 1) / mwg; };
  // packed, the prefix is met by so many blocks of 128 rows instead of so many
  const bool pack = p->prefix_L > 0 && p->B > 1 && all < ((int64_t)1 << 22) && blocks(all, 128) * 2 <= p->B * blocks(M, 128);
  const int64_t units256 = (int64_t)p->B * p->Hkv * blocks(M, 256);
  plan.rows = pack || M <= 32 ? 32 : M > 128 && units256 >= 256 ? 256 : 128;
  // segments for about `wanted` workgroups, none under `least` tokens; and no more pages in one than have room
  auto segments = [&](int64_t wanted, int64_t units, int64_t tokens, int64_t least) {
    const int64_t most = tokens / least, want = (wanted + units / 2) / units, room = (tokens + (int64_t)kSegPages * p->page_size - 1) / ((int64_t)kSegPages * p->page_size);
    int64_t n = want < most ? want : most;
    n = n < 1 ? 1 : n > 16 ? 16 : n;
    return (int)(n < room ? room : n);
  };
  plan.ns[0] = pack ? segments(256, p->Hkv * blocks(all, 128), p->prefix_L, 4 * KT) : 0;
  plan.ns[1] = segments(512, (int64_t)p->B * p->Hkv * blocks(M, plan.rows), (pack ? 0 : (int64_t)p->prefix_L) + p->max_L, 4 * KT);
  return plan;
}

size_t paged_workspace(const gr_attn_paged_params* p, const PagedPlan& plan) {
  const int n = plan.ns[0] + plan.ns[1];
  if (n == 1) return 0;
  const size_t rows = (size_t)p->B * p->W * p->Hq * n;
  return gr_align256(rows * p->d * 4) + gr_align256(rows * 8);
}

bool shapes_ok(const gr_attn_paged_params* p) {
  return p->B > 0 && p->W > 0 && p->Hq > 0 && p->Hkv > 0 && p->d > 0 && p->Hq % p->Hkv == 0 && p->page_size > 0 && p->prefix_L >= 0 && p->max_L >= 0;
}

}  // namespace

extern "C" size_t gr_beam_attn_paged_workspace_bytes(const gr_attn_paged_params* p) {
  if (!p || !shapes_ok(p)) return 0;
  return paged_workspace(p, plan_paged(p));
}

extern "C" gr_status gr_beam_attn_paged(const gr_attn_paged_params* p, void* workspace, size_t workspace_bytes, void* stream_) {
  const hipStream_t stream = (hipStream_t)stream_;
  if (!p || !shapes_ok(p)) return GR_ERR_INVALID_ARG;
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
  if ((int64_t)p->n_pages * p->page_size >= ((int64_t)1 << 31) || (int64_t)p->prefix_L + p->max_L >= ((int64_t)1 << 31) - 1024) return GR_ERR_UNSUPPORTED;
  if ((int64_t)p->Hkv * p->d > 65536 || p->W * g >= ((int64_t)1 << 22)) return GR_ERR_UNSUPPORTED;          // row numbers go through small_div, whose bound is 2^22
  if ((int64_t)p->W * p->Hq * p->d >= ((int64_t)1 << 31) || (int64_t)p->W * p->ND * p->Hkv * p->d >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;

  const PagedPlan plan = plan_paged(p);
  PagedCtx c;
  c.B = p->B; c.W = p->W; c.Hq = p->Hq; c.Hkv = p->Hkv; c.g = (int)g; c.ND = p->ND; c.u = p->u;
  c.prefix = p->prefix_L; c.own_prefix = plan.ns[0] ? 0 : p->prefix_L;
  c.max_L = p->max_L; c.max_pages = p->max_pages; c.n_pages = p->n_pages; c.shift = __builtin_ctz((unsigned)p->page_size);
  c.inv_hkv = div_inv((uint32_t)p->Hkv);
  c.rcp_g = 1.0f / (float)g; c.rcp_u = 1.0f / (float)(p->u > 1 ? p->u : 1);
  c.c = p->sm_scale * kLog2e; c.k_scale = kv8 ? p->k_scale : 1.f; c.v_scale = kv8 ? p->v_scale : 1.f;
  c.q = (const uint16_t*)p->q; c.kp = (const char*)p->k_pages; c.vp = (const char*)p->v_pages;
  c.prefix_pages = p->prefix_pages; c.table = p->block_table; c.lens = p->seq_lens;
  c.ku = (const uint16_t*)p->k_unshared; c.vu = (const uint16_t*)p->v_unshared; c.slot = p->slot;
  c.out = (uint16_t*)p->out; c.lse = p->lse_out; c.part_o = nullptr; c.part_ml = nullptr;
  int64_t grid = 0;
  for (int k = 0; k < 2; k++) {
    const int64_t M = k == 0 ? p->B * p->W * g : p->W * g, pairs = (k == 0 ? 1 : (int64_t)p->B) * p->Hkv;
    const int64_t rows = k == 0 ? 128 : plan.rows, MB = (M + rows - 1) / rows, groups = pairs * plan.ns[k], wgs = (groups + 7) / 8 * 8 * MB;
    if (groups >= ((int64_t)1 << 31) || grid + wgs >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
    if (k == 0) c.grid0 = (unsigned)wgs;
    grid += wgs;
    PagedPart& pt = k == 0 ? c.part0 : c.part1;
    pt.M = plan.ns[k] ? (int)M : 0; pt.MB = plan.ns[k] ? (int)MB : 1; pt.ns = plan.ns[k]; pt.groups = (int)groups;
    pt.inv_mb = div_inv((uint32_t)pt.MB); pt.inv_ns = div_inv((uint32_t)(pt.ns ? pt.ns : 1));
  }
  if (const size_t need = paged_workspace(p, plan)) {
    if (!workspace || ((uintptr_t)workspace & 255)) return GR_ERR_INVALID_ARG;
    if (workspace_bytes < need) return GR_ERR_WORKSPACE_TOO_SMALL;
    const size_t rows = (size_t)p->B * p->W * p->Hq * (plan.ns[0] + plan.ns[1]);
    c.part_o = (float*)workspace;
    c.part_ml = (float*)((char*)workspace + gr_align256(rows * p->d * 4));
  }
#define GR_LAUNCH(LDS, THREADS, ...)                                                                                       \
  do {                                                                                                                     \
    const size_t lds = LDS;                                                                                                \
    if (const gr_status st = gr_allow_lds<__VA_ARGS__>(lds)) return st;                                                    \
    hipLaunchKernelGGL((__VA_ARGS__), dim3((unsigned)grid), dim3(THREADS), lds, stream, c);                                \
  } while (0)
#define GR_LAUNCH_ROWS(DD, K8)                                                                                             \
  do {                                                                                                                     \
    if (plan.ns[0]) GR_LAUNCH(paged_mix_lds_bytes(DD), 256, k_paged_mix<DD, K8>);                                          \
    else if (plan.rows == 32) GR_LAUNCH(paged_few_lds_bytes(DD), 256, k_paged_few<DD, K8>);                                \
    else if (plan.rows == 128) GR_LAUNCH(paged_lds_bytes(DD, 128), 256, k_paged_attn<DD, 4, K8>);                          \
    else GR_LAUNCH(paged_lds_bytes(DD, 256), 512, k_paged_attn<DD, 8, K8>);                                                \
  } while (0)
  if (p->d == 128) { if (kv8) GR_LAUNCH_ROWS(128, true); else GR_LAUNCH_ROWS(128, false); }
  else { if (kv8) GR_LAUNCH_ROWS(64, true); else GR_LAUNCH_ROWS(64, false); }
#undef GR_LAUNCH_ROWS
#undef GR_LAUNCH
  if (c.part_o) {
    const int rpw = 1024 / p->d;
    const int64_t join = (int64_t)p->B * p->Hkv * ((c.part1.M + rpw - 1) / rpw);
    if (join >= ((int64_t)1 << 31)) return GR_ERR_UNSUPPORTED;
    if (p->d == 128) hipLaunchKernelGGL((k_paged_join<128>), dim3((unsigned)join), dim3(256), 0, stream, c);
    else hipLaunchKernelGGL((k_paged_join<64>), dim3((unsigned)join), dim3(256), 0, stream, c);
  }
  GR_HIP_TRY(hipGetLastError());
  return GR_OK;
}
