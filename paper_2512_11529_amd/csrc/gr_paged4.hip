// gr_beam_attn_paged over pages in FP4: E2M1 codes under a power of two for every 32 values of a token's head.
//
// A code times its scale has two bits of significand: it is a bf16 value exactly, so the products are those of bf16 matrix instructions over the widened values, and no
// scale is left over.  v_cvt_scalef32_pk_bf16_fp4 makes two of them at a time.
//   - K never meets LDS.  Lane (token t, quarter h) of a wavefront takes the quarter of its token's head that lies in one piece, 16 or 8 bytes under one scale.  The sum over the
//     head's elements may be made in any order, so a matrix instruction's k-th step takes the eight codes of each quarter's k-th word, and Q is held in the same order.
//   - V has to be transposed: its operand holds eight tokens of one element.  It is widened into LDS rows and read from there with ds_read_b64_tr_b16.
#include "gr_paged.hpp"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// 16 * NB rows of a (request, KV head) pair against a segment of its keys.  The four wavefronts hold the same rows and take every fourth 32 tokens each; nobody waits for
// anybody until their (maximum, sum, O) are joined in LDS.
// Bound: memory (17/32 byte an element).
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
constexpr int fp4_few_lds_bytes(int d, int nb) { return 4 * 32 * d * 2 + 4 * 16 * nb * 8; }

template <int D, int NB, int ARG>
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
  auto numbers_from = [&](int first) { return most_pages > 0 ? page_number(c, bu, first + lane, most_pages - 1) : 0; };
  int window = 0, numbers = sp == 0 ? numbers_from(0) : 0;
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
  if (sp > 0) { window = seg0 >> c.shift; numbers = numbers_from(window); }
  int ahead = numbers_from(window + 64);

  // ---- a tile of codes in registers
  struct Tile { typename F::words k[2], v[2]; uint32_t ks[2], vs[2]; };
  const uint32_t ps = 1u << c.shift, codes = gr_fp4_codes(ps, D), record = gr_fp4_record(ps, D);
  const uint8_t* k_head = (const uint8_t*)c.ks + (size_t)kvh * record;
  const uint8_t* v_head = (const uint8_t*)c.vs + (size_t)kvh * record;
  const size_t page_bytes = (size_t)record * (unsigned)c.Hkv;
  const uint32_t k_off = (uint32_t)(n16 * (D / 2) + h * (NV / 2)), ks_off = (uint32_t)(n16 * (D / 32) + h * NV / 32);
  const int vr = lane >> 2, vb = lane & 3;                   // V: lane (token vr, quarter vb)
  const uint32_t v_off = (uint32_t)(lane * (NV / 2)), vs_off = (uint32_t)(vr * (D / 32) + vb * NV / 32);
  auto load = [&](int j) {
    Tile t;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int tok = seg0 + j * FT + 16 * i, p = tok >> c.shift;
      if (p - window >= 64) {                                // (wave-uniform; both halves of a tile are in one window)
        window += 64;
        numbers = ahead;
        ahead = numbers_from(window + 64);
      }
      const size_t at = (size_t)(unsigned)__builtin_amdgcn_readlane(numbers, p - window) * page_bytes;
      const uint32_t in = (uint32_t)tok & (ps - 1);
      const uint8_t* kp = k_head + at + in * (D / 2);
      const uint8_t* vp = v_head + at + in * (D / 2);
      const uint8_t* kq = k_head + at + codes + in * (D / 32);
      const uint8_t* vq = v_head + at + codes + in * (D / 32);
      t.k[i] = *(const typename F::words*)(kp + k_off);
      t.ks[i] = kq[ks_off];
      t.v[i] = *(const typename F::words*)(vp + v_off);
      t.vs[i] = vq[vs_off];
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
  int w_at[NW / 2], r_at[DB];                                // byte addresses of the lane's writes (two pieces each) and reads, of the first half
#pragma unroll
  for (int i = 0; i < NW / 2; i++) w_at[i] = lds_v + vr * (D * 2) + (((NW * vb + 2 * i) ^ F::swz(vr)) << 4);
  {
    const int row = 4 * h + (n16 >> 2);
#pragma unroll
    for (int db = 0; db < DB; db++) r_at[db] = lds_v + row * (D * 2) + (((2 * db) ^ F::swz(row)) << 4) + ((n16 & 3) << 3);
  }
  typedef u32x4 __attribute__((address_space(3))) * lds_u32x4;
  typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
  auto put_v = [&](int i, int piece, u32x4 x) { *(lds_u32x4)(uintptr_t)(uint32_t)(w_at[piece / 2] + 16 * D * 2 * i + 16 * (piece & 1)) = x; };

  // The tile's scores to probabilities and onto O, once V is in LDS.  rows [lo, lo + n) of the tile are seen by the column.
  auto softmax_pv = [&](f32x4 (&s)[2][NB], const int (&lo)[NB], const unsigned (&n)[NB], bool all, auto&& bring_v) __attribute__((always_inline)) {
    bf16x8 p[NB];
#pragma unroll
    for (int nb = 0; nb < NB; nb++) {
      if (!all) {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[i][nb][e] = (unsigned)(16 * i + 4 * h + e - lo[nb]) < n[nb] ? s[i][nb][e] : -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) mx = fmaxf(mx, s[i][nb][e]);
      mx *= c.c;
      // (a column's reference rises when a score is more than 8 above it: probabilities of up to 2^8, as in gr_beam_attn)
      if (__any(mx > m_run[nb] + AttnTile<D, 1>::kLazy)) {
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
    bring_v();
#pragma unroll
    for (int db = 0; db < DB; db++) {
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(uint32_t)r_at[db]);
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(uint32_t)(r_at[db] + 16 * D * 2));
      const bf16x8 v = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int nb = 0; nb < NB; nb++) o[db][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[nb], o[db][nb], 0, 0, 0);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (LDS serves a wavefront in order: the next tile's V goes where this one's was)
  };

  // ---- the beams' own tokens first: their addresses need no page numbers
  const uint32_t own_bytes = (uint32_t)c.Hkv * D * 2;
  const char* ku_b = (const char*)(c.ku + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  const char* vu_b = (const char*)(c.vu + ((size_t)bu * (unsigned)(c.W * c.ND) * (unsigned)c.Hkv + kvh) * D);
  for (int oj = wave; oj < n_own; oj += 4) {
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
    u32x4 v[2][NW];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      bf16x8 k[KS];
#pragma unroll
      for (int st = 0; st < KS; st++) k[st] = *(const bf16x8*)(ku_b + off[i] + h * NV * 2 + 16 * st);
      const char* vrow = vu_b + (uint32_t)__shfl((int)off[i], vr, 64);
#pragma unroll
      for (int w = 0; w < NW; w++) v[i][w] = *(const u32x4*)(vrow + (vb * NW + w) * 16);
#pragma unroll
      for (int nb = 0; nb < NB; nb++) {
        s[i][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; st++) s[i][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[st], q[nb][st], s[i][nb], 0, 0, 0);
      }
    }
    int lo[NB];
    unsigned n[NB];
#pragma unroll
    for (int nb = 0; nb < NB; nb++) { lo[nb] = (beam_q[nb] - beam0) * c.u - oj * FT; n[nb] = qrow[nb] >= 0 ? (unsigned)c.u : 0u; }
    softmax_pv(s, lo, n, false, [&] {
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int w = 0; w < NW; w++) put_v(i, w, v[i][w]);
    });
  }

  // ---- the list: the next tile is on its way while one is taken
  const int first = (wave + 4 - (n_own & 3)) & 3;            // (the wavefronts behind those with own tokens begin)
  Tile t;
  if (first < nt) t = load(first);
  for (int j = first; j < nt; j += 4) {
    Tile now = t;
    if (j + 4 < nt) t = load(j + 4);
    const int left = seg1 - (seg0 + j * FT);
    const bool all = left >= FT;
    if (!all) {                                              // rows behind the list hold anything: V's must not be infinite times 0
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const bool there = 16 * i + vr < left;
        now.vs[i] = there ? now.vs[i] : 127u;
      }
    }
    f32x4 s[2][NB];
#pragma unroll
    for (int i = 0; i < 2; i++) {
#pragma unroll
      for (int nb = 0; nb < NB; nb++) s[i][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; st++) {
        const bf16x8 k = __builtin_bit_cast(bf16x8, fp4_values8(now.k[i][st], now.ks[i]));
#pragma unroll
        for (int nb = 0; nb < NB; nb++) s[i][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[nb][st], s[i][nb], 0, 0, 0);
      }
    }
    int lo[NB];
    unsigned n[NB];
#pragma unroll
    for (int nb = 0; nb < NB; nb++) { lo[nb] = 0; n[nb] = (unsigned)left; }
    softmax_pv(s, lo, n, all, [&] {
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int w = 0; w < NW; w++) put_v(i, w, __builtin_bit_cast(u32x4, fp4_values8(now.v[i][w], now.vs[i])));
    });
  }

  // ---- the four wavefronts' parts join in LDS, 16 rows at a time; then every one has columns of its own to write
  f32x2* s_ml = (f32x2*)(smem + 4 * F::PLACE);
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
    float top = -INFINITY, l = 0.f, a[4];
#pragma unroll
    for (int w = 0; w < 4; w++) top = fmaxf(top, s_ml[(w * NB + nb) * 16 + n16].x);
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const f32x2 ml = s_ml[(w * NB + nb) * 16 + n16];
      a[w] = ml.x > -INFINITY ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
      l += ml.y * a[w];
    }
    const float inv = late->part_o ? 1.f : l > 0.f ? 1.0f / l : 0.f;
    const size_t row = ((size_t)bu * (unsigned)late->W + (unsigned)beam_q[nb]) * (unsigned)late->Hq + kvh * (unsigned)late->g + (unsigned)(qrow[nb] - beam_q[nb] * late->g);
    const int left = min(32, M - (row_w & ~31)), r32 = (row_w & 31) + 16 * nb + n16;
    const size_t row_p = (((size_t)bu * (unsigned)ns + (unsigned)sp) * (unsigned)late->Hkv + kvh) * (unsigned)M + (unsigned)(row_w & ~31);
#pragma unroll
    for (int k = 0; k < DB / 4; k++) {
      const int db = wave * (DB / 4) + k;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; w++) {
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

template <int D, int NB>
__global__ void __launch_bounds__(256) k_fp4_few(AttnCtx c) {
  few_rows4<D, NB, 0>(c, blockIdx.x);
}

}  // namespace

gr_status gr_paged_fp4(const gr_attn_paged_params* p, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return run_paged(p, workspace, workspace_bytes, stream, [&](const PagedPlan& plan, const AttnCtx&, const AttnCtx& c, unsigned grid, unsigned) -> gr_status {
    auto few = [&](auto dim) -> gr_status {
      constexpr int D = decltype(dim)::value;
      if (plan.rows == 16) return launch<k_fp4_few<D, 1>>(fp4_few_lds_bytes(D, 1), 256, grid, stream, c);
      return launch<k_fp4_few<D, 2>>(fp4_few_lds_bytes(D, 2), 256, grid, stream, c);
    };
    return p->d == 128 ? few(std::integral_constant<int, 128>()) : few(std::integral_constant<int, 64>());
  });
}
