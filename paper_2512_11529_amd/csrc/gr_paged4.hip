// gr_beam_attn_paged over pages in FP4: E2M1 codes under a power of two for every 32 values of a token's head.
//
// A code times its scale has two bits of significand: it is a bf16 value exactly, so the products are those of bf16 matrix instructions over the widened values, and no
// scale is left over.  v_cvt_scalef32_pk_bf16_fp4 makes two of them at a time.
//   - K never meets LDS.  Lane (token t, quarter h) of a wavefront takes the quarter of its token's head that lies in one piece, 16 or 8 bytes under one scale.  The sum over the
//     head's elements may be made in any order, so a matrix instruction's k-th step takes the eight codes of each quarter's k-th word, and Q is held in the same order.
//   - V has to be transposed: its operand holds eight tokens of one element.  It is widened into LDS rows and read from there with ds_read_b64_tr_b16.
#define GR_ROWS_FP4
#include "gr_paged.hpp"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// 16 * NB rows of a (request, KV head) pair against a segment of its keys.  The wavefronts hold the same rows and take 32 tokens each in turn; nobody waits for
// anybody until their (maximum, sum, O) are joined in LDS.
// Bound: memory (17/32 byte an element).  us: 64 requests of 14208 tokens x 1 beam, 32 and 8 heads of 128, 170-175 (5.7 TB/s; a plain read of 1 GiB reaches 6.3), 32 of 12001-16384 x 2, whose 256
// workgroups end with the longest list, 94 (5.2); the same loads without anything done to what they bring 87.  Vector instructions (160 for a tile of one block) keep the SIMDs busy 37 % of that time.
// Tried: the operands of V kept in order behind scheduling barriers 96.4 instead of 93.9; two tiles on their way instead of one 96-104; 128 registers for four wavefronts to a SIMD, with spills, 100-159; V asked for ahead of K 102; the powers of K and V in one load,
// spread by ds_bpermute, 95 (and 3 % more where the loads are not waited for); 48 rows a wavefront, for many rows, 482 against 495 with 32.
template <int D>
struct Fp4 {
  static constexpr int FT = 32;                    // tokens of a tile: two halves of 16
  static constexpr int NV = D / 4;                 // values of a lane's piece of a token
  static constexpr int NW = NV / 8;                // words of codes of a piece
  static constexpr int KS = D / 32;                // steps of 32 elements
  static constexpr int DB = D / 16;
  static constexpr int PLACE = FT * D;             // elements of a wavefront's V tile
  typedef uint32_t words __attribute__((ext_vector_type(NW)));
  // 16-byte pieces of a V row stand permuted, piece p of row r in slot p ^ swz(r): the eight rows that 32 lanes read 32 bytes each of are then in different banks
  static __device__ __forceinline__ int swz(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
};
constexpr int fp4_few_lds_bytes(int d, int nb, int waves) { return waves * (32 * d * 2 + 16 * nb * 8); }

template <int D, int NB, int WAVES, int ARG>
__device__ __forceinline__ void few_rows4(const AttnCtx& c, const unsigned id) {
  using F = Fp4<D>;
  constexpr int FT = F::FT, NV = F::NV, NW = F::NW, KS = F::KS, DB = F::DB, ROWS = 16 * NB;
  extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];
  const int tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 4, n16 = lane & 15;
  const unsigned place = id >> 3, nth = div_by(place, (unsigned)c.MB, c.inv_mb);
  const int group = (int)(nth * 8 + (id & 7u)), mbi = (int)(place - nth * (unsigned)c.MB), ns = c.nsplit, M = c.M;
  if (group >= c.n_groups) return;
  const unsigned gq = div_by((unsigned)group, (unsigned)ns, c.inv_split);
  const int sp = group - (int)gq * ns;
  const unsigned bu = div_by(gq, (unsigned)c.Hkv, c.inv_hkv), kvh = gq - bu * (unsigned)c.Hkv;
  const int row_w = mbi * ROWS, beam0 = __builtin_amdgcn_readfirstlane(small_div(row_w, c.rcp_g));

  // ---- page numbers: lane i has that of page window + i of the list, and `ahead` that of the 64th after it
  const int most_pages = (c.front + c.max_L + (1 << c.shift) - 1) >> c.shift;
  auto entries_from = [&](int first) { return most_pages > 0 ? page_entry(c, bu, first + lane, most_pages - 1) : 0; };
  auto checked = [&](int entry) { return (unsigned)entry < (unsigned)c.n_pages ? entry : 0; };
  int window = 0, numbers = sp == 0 ? entries_from(0) : 0;   // (checked when they are needed: the loads are waited for there)
  const int keys = c.front + __builtin_amdgcn_readfirstlane(paged_length(c, (int)bu));

  // ---- Q: lane (row n16, quarter h) has the elements of K's quarter, in K's order
  bf16x8 q[NB][KS];
  int qrow[NB], beam_q[NB];
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    const int r = row_w + 16 * nb + n16, rc = min(r, M - 1);
    beam_q[nb] = small_div(rc, c.rcp_g);
    qrow[nb] = r < M ? r : -1;
    const uint16_t* from = c.q + (((size_t)bu * (unsigned)c.W + (unsigned)beam_q[nb]) * (unsigned)c.Hq + kvh * (unsigned)c.g + (unsigned)(rc - beam_q[nb] * c.g)) * D + h * NV;
#pragma unroll
    for (int s = 0; s < KS; s++) q[nb][s] = *(const bf16x8*)(from + 8 * s);
  }

  int chunk = (int)div_by((unsigned)keys + (unsigned)ns - 1u, (unsigned)ns, c.inv_split);
  chunk = (chunk + KT - 1) / KT * KT;
  const int seg0 = min(keys, sp * chunk), seg1 = min(keys, seg0 + chunk);
  const int nt = (seg1 - seg0 + FT - 1) / FT;
  const bool own_stage = c.u > 0 && sp == (max(0, keys - (ns - 1) * chunk) < chunk ? ns - 1 : 0);
  const int Ru = own_stage ? (__builtin_amdgcn_readfirstlane(small_div(min(row_w + ROWS - 1, M - 1), c.rcp_g)) - beam0 + 1) * c.u : 0;
  const int n_own = (Ru + FT - 1) / FT;
  if (sp > 0) { window = seg0 >> c.shift; numbers = entries_from(window); }
  int ahead = entries_from(window + 64);
  numbers = checked(numbers);

  // ---- a tile's codes and powers in registers: halves of 16 tokens, each of which lies in one page
  struct Codes { typename F::words w[2]; uint32_t power[2]; };
  const uint32_t ps = 1u << c.shift, codes = gr_fp4_codes(ps, D), record = gr_fp4_record(ps, D);
  const uint8_t* k_head = (const uint8_t*)c.ks + (size_t)kvh * record;
  const uint8_t* v_head = (const uint8_t*)c.vs + (size_t)kvh * record;
  const uint32_t page_bytes = record * (unsigned)c.Hkv;
  const uint32_t k_off = (uint32_t)(n16 * (D / 2) + h * (NV / 2)), kp_off = (uint32_t)(n16 * (D / 32) + h * NV / 32);
  const int vr = lane >> 2, vb = lane & 3;                   // V: lane (token vr, quarter vb)
  const uint32_t v_off = (uint32_t)(lane * (NV / 2)), vp_off = (uint32_t)(vr * (D / 32) + vb * NV / 32);
  size_t page_at[2];                                         // of the tile asked for last
  uint32_t in_at[2];
  auto locate = [&](int j) {
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int tok = seg0 + j * FT + 16 * i, p = tok >> c.shift;
      if (p - window >= 64) {                                // (wave-uniform; both halves of a tile are in one window)
        window += 64;
        numbers = checked(ahead);
        ahead = entries_from(window + 64);
      }
      page_at[i] = (size_t)(unsigned)__builtin_amdgcn_readlane(numbers, p - window) * page_bytes;
      in_at[i] = (uint32_t)tok & (ps - 1);
    }
  };
  auto load = [&](const uint8_t* head, uint32_t off, uint32_t power_off) {
    Codes t;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const uint8_t* page = head + page_at[i];
      t.w[i] = *(const typename F::words*)(page + in_at[i] * (D / 2) + off);
      t.power[i] = *(page + codes + in_at[i] * (D / 32) + power_off);
    }
    return t;
  };

  f32x4 o[DB][NB];
  float m_run[NB], l_run[NB];
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    m_run[nb] = -INFINITY; l_run[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; db++) o[db][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  uint16_t* mine = smem + wave * F::PLACE;
  const int lds_v = (int)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)mine;
  int w_at[NW / 2], r_at;                                    // byte addresses of the lane's writes (two pieces each) and reads, of the first half
#pragma unroll
  for (int i = 0; i < NW / 2; i++) w_at[i] = lds_v + vr * (D * 2) + (((NW * vb + 2 * i) ^ F::swz(vr)) << 4);
  {
    const int row = 4 * h + (n16 >> 2);
    r_at = lds_v + row * (D * 2) + (F::swz(row) << 4) + ((n16 & 3) << 3);       // (32 elements on: another 32 bytes, in the swizzle's order)
  }
  typedef u32x4 __attribute__((address_space(3))) * lds_u32x4;
  typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
  auto put_v = [&](int i, int piece, u32x4 x) { *(lds_u32x4)(uintptr_t)(uint32_t)(w_at[piece / 2] + 16 * D * 2 * i + 16 * (piece & 1)) = x; };

  auto read_v = [&](int db) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(uint32_t)(r_at ^ (32 * db)));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(uint32_t)((r_at ^ (32 * db)) + 16 * D * 2));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // rows [lo, lo + n) of the tile are seen by column nb
  auto mask = [&](f32x4 (&s)[2][NB], int nb, int lo, unsigned n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int e = 0; e < 4; e++) s[i][nb][e] = (unsigned)(16 * i + 4 * h + e - lo) < n ? s[i][nb][e] : -INFINITY;
  };
  // The tile's scores to probabilities and onto O; V is in LDS, whose first operands are on their way meanwhile and the others PF matrix instructions' time.
  auto softmax_pv = [&](f32x4 (&s)[2][NB]) __attribute__((always_inline)) {
    constexpr int PF = NB == 1 ? 2 : 3;                      // (read where they are needed: 8 requests of 2000-4000 x 8 beams 18.2 us, 16.9; 16 of 3000 x 16 25.9, 24.4)
    bf16x8 p[NB], v[DB];
#pragma unroll
    for (int db = 0; db < PF; db++) v[db] = read_v(db);
#pragma unroll
    for (int nb = 0; nb < NB; nb++) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) mx = fmaxf(mx, s[i][nb][e]);
      mx *= c.c;
      // (a column's reference rises when a score is more than 8 above it: probabilities of up to 2^8, as in gr_beam_attn)
      if (__builtin_expect(__any(mx > m_run[nb] + AttnTile<D, 1>::kLazy), 0)) {
        float top = fmaxf(mx, __shfl_xor(mx, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = top > m_run[nb] ? top : m_run[nb];
        const float scale = top > m_run[nb] ? __builtin_amdgcn_exp2f(m_run[nb] - m_new) : 1.f;
        l_run[nb] *= scale;
        m_run[nb] = m_new;
#pragma unroll
        for (int db = 0; db < DB; db++)
#pragma unroll
          for (int e = 0; e < 4; e++) o[db][nb][e] *= scale;
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; nb++) {
      const float ref = m_run[nb] > -INFINITY ? m_run[nb] : 0.f;
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[i][nb][e], c.c, -ref));
          l_run[nb] += x;
          p[nb][4 * i + e] = (__bf16)x;
        }
    }
#pragma unroll
    for (int db = 0; db < DB; db++) {
      if (db + PF < DB) v[db + PF] = read_v(db + PF);
#pragma unroll
      for (int nb = 0; nb < NB; nb++) o[db][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[db], p[nb], o[db][nb], 0, 0, 0);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (LDS serves a wavefront in order: the next tile's V goes where this one's was)
  };

  // ---- the beams' own tokens, while the first tile is on its way
  const uint32_t own_bytes = (uint32_t)c.Hkv * D * 2;
  const char* ku_b = (const char*)(c.ku + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  const char* vu_b = (const char*)(c.vu + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  auto own_tokens = [&]() __attribute__((always_inline)) {
  for (int oj = wave; oj < n_own; oj += WAVES) {
    uint32_t off[2];                                         // of row 16 i + n16 of the tile
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int rho = oj * FT + 16 * i + n16;
      int bl, tok;
      divmod_small(rho < Ru ? rho : 0, c.u, c.rcp_u, &bl, &tok);
      int prow = (beam0 + bl) * c.ND + tok;
      if (c.slot) {                                          // (an entry outside the block falls back to the beam's own row)
        const int sl = c.slot[(size_t)bu * (unsigned)(c.W * c.ND) + (unsigned)prow];
        prow = (unsigned)sl < (unsigned)(c.W * c.ND) ? sl : prow;
      }
      off[i] = (uint32_t)prow * own_bytes;
    }
    f32x4 s[2][NB];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const char* vrow = vu_b + (uint32_t)__shfl((int)off[i], vr, 64) + vb * NW * 16;
      u32x4 v[NW];
#pragma unroll
      for (int w = 0; w < NW; w++) v[w] = *(const u32x4*)(vrow + w * 16);
#pragma unroll
      for (int w = 0; w < NW; w++) put_v(i, w, v[w]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < 2; i++) {
      bf16x8 k[KS];
#pragma unroll
      for (int st = 0; st < KS; st++) k[st] = *(const bf16x8*)(ku_b + off[i] + h * NV * 2 + 16 * st);
#pragma unroll
      for (int nb = 0; nb < NB; nb++) {
        s[i][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; st++) s[i][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[st], q[nb][st], s[i][nb], 0, 0, 0);
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; nb++) mask(s, nb, (beam_q[nb] - beam0) * c.u - oj * FT, qrow[nb] >= 0 ? (unsigned)c.u : 0u);
    softmax_pv(s);
  }
  };

  // ---- the list: a tile's K is asked for when the one before has been multiplied, its V when that one is in LDS
  int j = (wave + WAVES - (n_own & (WAVES - 1))) & (WAVES - 1);                      // (the wavefronts behind those with own tokens begin)
  Codes k, v;
  if (j < nt) {
    locate(j);
    k = load(k_head, k_off, kp_off);
    v = load(v_head, v_off, vp_off);
  }
  own_tokens();
  auto tile = [&](auto last) __attribute__((always_inline)) {
    constexpr bool LAST = decltype(last)::value;             // of this wavefront: the only one that may be partial, and none is asked for
    const int left = LAST ? seg1 - (seg0 + j * FT) : FT;
    f32x4 s[2][NB];
#pragma unroll
    for (int i = 0; i < 2; i++) {
#pragma unroll
      for (int nb = 0; nb < NB; nb++) s[i][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; st++) {
        const bf16x8 x = __builtin_bit_cast(bf16x8, fp4_values8(k.w[i][st], k.power[i]));
#pragma unroll
        for (int nb = 0; nb < NB; nb++) s[i][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[nb][st], s[i][nb], 0, 0, 0);
      }
    }
    if (!LAST) {
      locate(j + WAVES);
      k = load(k_head, k_off, kp_off);
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {
      // (rows behind the list hold anything, and must not be infinite times 0)
      const uint32_t power = !LAST || 16 * i + vr < left ? v.power[i] : 127u;
#pragma unroll
      for (int w = 0; w < NW; w++) put_v(i, w, __builtin_bit_cast(u32x4, fp4_values8(v.w[i][w], power)));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (!LAST) v = load(v_head, v_off, vp_off);
    if (LAST && left < FT) {
#pragma unroll
      for (int nb = 0; nb < NB; nb++) mask(s, nb, 0, (unsigned)left);
    }
    softmax_pv(s);
  };
  if (j < nt) {
    for (; j + WAVES < nt; j += WAVES) tile(std::false_type());
    tile(std::true_type());
  }

  // ---- the wavefronts' parts join in LDS, 16 rows at a time; then every one has columns of its own to write
  f32x2* s_ml = (f32x2*)(smem + WAVES * F::PLACE);
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    float l = l_run[nb] + __shfl_xor(l_run[nb], 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (h == 0) s_ml[(wave * NB + nb) * 16 + n16] = f32x2{l > 0.f ? m_run[nb] : -INFINITY, l};
  }
  const LateArgs late = late_args() + ARG;
#pragma unroll
  for (int nb = 0; nb < NB; nb++) {
    if (nb > 0) __syncthreads();
    f32x4* to = (f32x4*)mine + lane;
#pragma unroll
    for (int db = 0; db < DB; db++) to[64 * db] = o[db][nb];
    __syncthreads();
    if (qrow[nb] < 0) continue;
    float top = -INFINITY, l = 0.f, a[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; w++) top = fmaxf(top, s_ml[(w * NB + nb) * 16 + n16].x);
#pragma unroll
    for (int w = 0; w < WAVES; w++) {
      const f32x2 ml = s_ml[(w * NB + nb) * 16 + n16];
      a[w] = ml.x > -INFINITY ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
      l += ml.y * a[w];
    }
    const float inv = late->part_o ? 1.f : l > 0.f ? 1.0f / l : 0.f;
    const size_t row = ((size_t)bu * (unsigned)late->W + (unsigned)beam_q[nb]) * (unsigned)late->Hq + kvh * (unsigned)late->g + (unsigned)(qrow[nb] - beam_q[nb] * late->g);
    const int left = min(32, M - (row_w & ~31)), r32 = (row_w & 31) + 16 * nb + n16;
    const size_t row_p = (((size_t)bu * (unsigned)ns + (unsigned)sp) * (unsigned)late->Hkv + kvh) * (unsigned)M + (unsigned)(row_w & ~31);
#pragma unroll
    for (int k = 0; k < (DB + WAVES - 1) / WAVES; k++) {
      const int db = wave + k * WAVES;
      if (DB < WAVES && db >= DB) break;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; w++) {
        const f32x4 y = *((const f32x4*)(smem + w * F::PLACE) + 64 * db + lane);
#pragma unroll
        for (int e = 0; e < 4; e++) x[e] += y[e] * a[w];
      }
      if (late->part_o) {
        *((f32x4*)(late->part_o + row_p * D) + (4 * db + h) * left + r32) = x;
      } else {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; e++) y[e] = (__bf16)(x[e] * inv);
        *(bf16x4*)(late->out + row * D + 16 * db + 4 * h) = y;
      }
    }
    if (wave == 0 && h == 0) {
      if (late->part_o) *(f32x2*)(late->part_ml + (row_p + (unsigned)r32) * 2) = f32x2{top, l};
      else if (late->lse) late->lse[row] = l > 0.f ? (top + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    }
  }
}

template <int D, int NB, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(2))) k_fp4_few(AttnCtx c) {
  few_rows4<D, NB, WAVES, 0>(c, blockIdx.x);
}

// Blocks of 128 and 256 rows: gr_beam_attn's body, bound as it is by the issue rate of matrix instructions, softmax and LDS reads: 32 requests of 512-3700 tokens x 256 beams behind 256, 32 and 8
// heads of 128, 309-328 us from card to card (1.01-1.08 PFLOP/s; bf16 pages 313-324); heads of 64 201 (0.83).  By blocks of 32 rows whose wavefronts share out the keys 495; with the powers looked at where they are asked for 333.
template <int D, int NWAVES, int KS, bool FIND>
__global__ void __launch_bounds__(NWAVES * 64 * KS) __attribute__((amdgpu_waves_per_eu(2, 2))) k_fp4_attn(AttnCtx c) {
  constexpr int NCB = 1;
  constexpr bool CAUSAL = false, PAGED = true, KV8 = true, WHOLE = true;
#include "gr_attn_rows.inc"
}


// A packed prefix by blocks of 128 rows of all requests, which are dealt first (arguments c), and each request's list by blocks of 16 or 32 (arguments few).  64 requests of 16-600 tokens x 4
// beams behind 4096 common ones 30 us, and 6 for the join, 32-34 among others (in blocks of 16 rows over the whole lists 46): 16 tiles a workgroup, one to a CU.
constexpr int fp4_mix_lds_bytes(int d, int nb) { return attn_lds_bytes(d, 128, 1) > fp4_few_lds_bytes(d, nb, 4) ? attn_lds_bytes(d, 128, 1) : fp4_few_lds_bytes(d, nb, 4); }
template <int D, int NB>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) k_fp4_mix(AttnCtx c, AttnCtx few, unsigned blocks0) {
  if (blockIdx.x >= blocks0) {
    few_rows4<D, NB, 4, 1>(few, blockIdx.x - blocks0);
    return;
  }
  constexpr int NCB = 1, NWAVES = 4, KS = 1;
  constexpr bool CAUSAL = false, FIND = false, PAGED = true, KV8 = true, WHOLE = true;
#include "gr_attn_rows.inc"
}

}  // namespace

gr_status gr_paged_fp4(const gr_attn_paged_params* p, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return run_paged(p, workspace, workspace_bytes, stream, [&](const PagedPlan& plan, const AttnCtx& c0, const AttnCtx& c, unsigned grid, unsigned blocks0) -> gr_status {
    auto few = [&](auto dim, auto blocks) -> gr_status {
      constexpr int D = decltype(dim)::value, NB = decltype(blocks)::value;
      if (plan.ns[0] > 0) return launch<k_fp4_mix<D, NB>>(fp4_mix_lds_bytes(D, NB), 256, grid, stream, c0, c, blocks0);
      if (plan.ks == 2) return launch<k_fp4_few<D, NB, 8>>(fp4_few_lds_bytes(D, NB, 8), 512, grid, stream, c);
      return launch<k_fp4_few<D, NB, 4>>(fp4_few_lds_bytes(D, NB, 4), 256, grid, stream, c);
    };
    auto rows = [&](auto dim) -> gr_status {
      constexpr int D = decltype(dim)::value;
      if (plan.rows == 16) return few(dim, std::integral_constant<int, 1>());
      if (plan.rows == 32) return few(dim, std::integral_constant<int, 2>());
      if (plan.ks == 2) return launch<k_fp4_attn<D, 4, 2, false>>(attn_lds_bytes(D, 128, 2), 512, grid, stream, c);
      if (plan.rows == 128) {
        if (plan.find) return launch<k_fp4_attn<D, 4, 1, true>>(attn_lds_bytes(D, 128, 1), 256, grid, stream, c);
        return launch<k_fp4_attn<D, 4, 1, false>>(attn_lds_bytes(D, 128, 1), 256, grid, stream, c);
      }
      if (plan.find) return launch<k_fp4_attn<D, 8, 1, true>>(attn_lds_bytes(D, 256, 1), 512, grid, stream, c);
      return launch<k_fp4_attn<D, 8, 1, false>>(attn_lds_bytes(D, 256, 1), 512, grid, stream, c);
    };
    return p->d == 128 ? rows(std::integral_constant<int, 128>()) : rows(std::integral_constant<int, 64>());
  });
}
