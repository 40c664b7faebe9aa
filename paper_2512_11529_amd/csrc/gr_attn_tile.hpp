// Building blocks of the attention kernels (gfx950): the matrix-core tile of K, Q and V in LDS, its softmax, and index arithmetic.  Not part of the ABI.
#pragma once
#include "gr_internal.hpp"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int KT = 64;        // kv tokens per LDS tile

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// n / d and n % d for 0 <= n < 2^22 and a small runtime divisor, through a float reciprocal and one
// correction step (a handful of instructions where the generic 32-bit division takes dozens).
__device__ __forceinline__ void divmod_small(int n, int d, float rcp_d, int* q, int* r) {
  int qq = (int)((float)n * rcp_d);
  int rr = n - qq * d;
  if (rr >= d) { qq++; rr -= d; }
  if (rr < 0) { qq--; rr += d; }
  *q = qq; *r = rr;
}

// n / d for any n, with inv = (2^32 - 1) / d rounded down from the host: the product's high word is n / d or one less.  (In scalar registers; the generic
// division by a number from memory is three times as long, and a unit starts with four of them.)
constexpr uint32_t div_inv(uint32_t d) { return 0xffffffffu / d; }
__device__ __forceinline__ unsigned div_by(unsigned n, unsigned d, uint32_t inv) {
  const unsigned q = __umulhi(n, inv);
  return q + (n - q * d >= d ? 1u : 0u);
}
// r / g for 0 <= r < 2^22, with rcp = 1 / g rounded to nearest: (r + 1/2) / g is at least 1/(2g) from a whole number, and two roundings move it by less
// than (r + 1/2) / g * 2^-23 (1 + 2^-25) < 1/(2g).
__device__ __forceinline__ int small_div(int r, float rcp) { return (int)fmaf((float)r, rcp, 0.5f * rcp); }

// The larger of a value and the other half's (of lane ^ 32).
__device__ __forceinline__ float halves_max(float v) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// Per-tile building blocks.  A tile is KT = 64 prompt tokens; S^T of a tile is [64 kv x 32*NCB q]
// = 2 sub-tiles x NCB column blocks of 32x32 fp32 accumulators.
template <int D, int NCB>
struct AttnTile {
  // Prompt tiles arrive by direct global->LDS loads: a wave-level load writes 1 KiB of consecutive LDS (lane l -> bytes
  // 16 l ..), so tile rows cannot be padded.  Instead the 16-byte pieces of a row are stored permuted (piece p of row r
  // sits in slot p ^ swz(r); the lane that fills slot s fetches piece s ^ swz(r) from memory), chosen so that the
  // operand reads below hit every bank group once:
  //   K (ds_read_b128, 16 lanes = 16 consecutive rows, same piece): swz = r & 15 (256-byte rows) or (r >> 1) & 7 (128-byte rows);
  //   V (ds_read_b64_tr_b16, 32 lanes = 4 consecutive rows x 4 pieces):  swz = 4 (r & 3)  or  4 ((r >> 1) & 1).
  static constexpr int PPRW = D / 8;                                       // 16-byte pieces per row
  static __device__ __forceinline__ int swz_k(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  static __device__ __forceinline__ int swz_v(int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }
  // Per-lane LDS addresses of the operand reads of a tile at the start of LDS, fixed for the whole kernel: what tile slot, slab and
  // block add to them is known at compile time and goes into the instructions.
  struct Rd { int k[D / 16]; int v[D / 32]; };
  static __device__ __forceinline__ Rd make_rd(int lane, int lds_base) {
    const int G = lane >> 5, n32 = lane & 31;
    Rd r;
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) r.k[ks] = lds_base + 2 * (n32 * D + ((2 * ks + G) ^ swz_k(n32)) * 8);
    const int vrow = 4 * G + ((lane & 15) >> 2);
#pragma unroll
    for (int db = 0; db < D / 32; db++)
      r.v[db] = lds_base + 2 * (vrow * D + ((4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz_v(vrow)) * 8 + 4 * (lane & 1));
    return r;
  }
  // K operand of 32 tokens `sub` and 16 dimensions `ks`; V^T operand of 16 tokens `slab` and 32 dimensions `db`
  static __device__ __forceinline__ bf16x8 read_k(int tile, const Rd& r, int sub, int ks) {         // `tile`: element offset in LDS
    typedef const u32x4 __attribute__((address_space(3))) * lds_u32x4;
    return __builtin_bit_cast(bf16x8, *(lds_u32x4)(uintptr_t)(uint32_t)(r.k[ks] + 2 * (tile + sub * 32 * D)));
  }
  static __device__ __forceinline__ bf16x8 read_v(int tile, const Rd& r, int slab, int db) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
    const int at = r.v[db] + 2 * (tile + slab * 16 * D);
    s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(uint32_t)at);
    s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(uint32_t)(at + 2 * 8 * D));
    s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, both);
  }
  // S^T = K . Q^T from the K tile in LDS (A operand) and Q in registers (B operand)
  static __device__ __forceinline__ void qk(int sk, const bf16x8 (&qop)[NCB][D / 16], f32x16 (&s)[KT / 32][NCB],
                                            const Rd& rdo) {
#pragma unroll
    for (int sub = 0; sub < KT / 32; sub++)
#pragma unroll
      for (int cb = 0; cb < NCB; cb++)
#pragma unroll
        for (int i = 0; i < 16; i++) s[sub][cb][i] = 0.f;
    // operand reads run PF steps ahead of the MFMAs that consume them
    constexpr int N = (KT / 32) * (D / 16), PF = 4;
    bf16x8 a[N];
#pragma unroll
    for (int i = 0; i < PF; i++) a[i] = read_k(sk, rdo, i % 2, i / 2);
#pragma unroll
    for (int i = 0; i < N; i++) {
      if (i + PF < N) a[i + PF] = read_k(sk, rdo, (i + PF) % 2, (i + PF) / 2);
#pragma unroll
      for (int cb = 0; cb < NCB; cb++) s[i % 2][cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], qop[cb][i / 2], s[i % 2][cb], 0, 0, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, PF, 0);
#pragma unroll
    for (int i = 0; i < N - PF; i++) {
      __builtin_amdgcn_sched_group_barrier(0x008, NCB, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PF * NCB, 0);
  }

  // Per-lane maximum of a tile's scores for the lane's query column (both halves of the column).
  static __device__ __forceinline__ float colmax(const f32x16 (&s)[KT / 32][NCB]) {
    float mx = -INFINITY;
#pragma unroll
    for (int sub = 0; sub < KT / 32; sub++)
#pragma unroll
      for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[sub][0][i]), s[sub][0][i + 1]);
    return halves_max(mx);
  }

  // One steady-state tile with the matrix and vector pipes kept busy together.  The wave issues, in this order,
  // the MFMAs of S(t+1) = K(t+1).Q^T and then those of O += V(t).P(t); between consecutive MFMAs it
  // exponentiates a fixed share of tile t's scores (their reference m2 is already decided), so that
  // the 32 quarter-rate exponentials per lane run in the shadow of the 32 MFMAs instead of after them.  P(t)'s quarters are
  // complete when the PV MFMAs come to them.  Instruction order is pinned chunk by chunk.
  // Measured at 32 x 4096 tokens x 256 beams, two wavefronts per SIMD: 507 us with the exponentials staged over three chunks, 515
  // with each finished in one; 8 x 2048 x 128 (one wavefront per SIMD, 1.1 us a tile): 40.1 against 41.4 us.  Operand reads 5 or 6
  // MFMAs ahead: no change.
  static constexpr int NQK = (KT / 32) * (D / 16), NPV = (KT / 16) * (D / 32), NMF = NQK + NPV;
  // All 32 exponentials are issued after this many MFMAs: as late as the last quarter of the probabilities, packed two chunks later, allows.  us with NPV / 2
  // and with this: 32 x 4096 x 256 beams 477.9, 472.6; 64 ragged requests of 512-8192 853, 845; 8 causal prompts of 1024-8192 1184, 1173.
  static constexpr int EXP_BY = NQK + NPV * 11 / 16;
  static constexpr int exps_after(int j) {                // exponentials finished once MFMA j's chunk has been issued
    const int t = (32 * (j + 1) + EXP_BY - 1) / EXP_BY;
    return j < 0 ? 0 : (t > 32 ? 32 : t);
  }
  // The workgroup meets before the tile's last HEAD MFMAs (0: after all), whose operands are in registers by then: loads for the tile after have landed, everybody has
  // read K(t+1) and V(t), and the next tile's first HEAD operands are read beside those MFMAs.  With the meeting between two tiles every wave of
  // the CU asked LDS for its first operands at once, with nothing to compute meanwhile: 8 causal prompts of 1024-8192 tokens 1210 -> 1189 us, 4 x 16384
  // x 512 beams in FP8 456.7 -> 452.7, 64 ragged requests of 512-8192 x 256 864 -> 853.  (4 MFMAs: 1189, 450, 860, but 32 x 4096 x 256 478 instead of
  // 476; 1: 1199, 456, 859.)
  // `between` is called in every chunk: the loads of tiles ahead are issued there, one every second MFMA (head size 64: every one).  Issued
  // together at the start of a tile they held all waves up while the CU's address unit worked them off: 32 x 4096 x 256 beams 486 -> 472 us, the 64
  // ragged requests 873 -> 849, 16 x 2000 x 200 beams of head size 64 21.4 -> 20.5.
  static constexpr int PF = 4;                           // operand reads run PF MFMAs ahead
  static constexpr int SPREAD = D == 128 ? 2 : 1;
  template <int HEAD, class F, class G>
  static __device__ __forceinline__ void fused(F&& between, G&& meet, bf16x8 (&head)[PF], int sk_after, int sk_next, int sv_cur, const bf16x8 (&qop)[NCB][D / 16],
                                               const f32x16 (&s_cur)[KT / 32][NCB], f32x16 (&s_next)[KT / 32][NCB],
                                               f32x16 (&o)[D / 32][NCB], float m2, float c, float& rs, bf16x8 (&pop)[KT / 16], const Rd& rdo) {
    static_assert(NCB == 1, "one column block per wave");
    auto rdk = [&](int i) { return read_k(sk_next, rdo, i % 2, i / 2); };
    auto rdv = [&](int i) { return read_v(sv_cur, rdo, i / (D / 32), i % (D / 32)); };
    bf16x8 a[NMF];
    float p[32], arg[32];                                   // (a few of each are alive at a time)
    rs = 0.f;
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PF; i++) a[i] = i < HEAD ? head[i < HEAD ? i : 0] : rdk(i);
#pragma unroll
    for (int e = 0; e < exps_after(0); e++) arg[e] = fmaf(s_cur[e / 16][0][e % 16], c, -m2);
#pragma unroll
    for (int j = 0; j < NMF; j++) {
      if (j == NMF - HEAD) meet();
      if (j + PF < NMF) a[j + PF] = (j + PF < NQK) ? rdk(j + PF) : rdv(j + PF - NQK);
      else if (j >= NMF - HEAD) head[j + HEAD - NMF] = read_k(sk_after, rdo, (j + HEAD - NMF) % 2, (j + HEAD - NMF) / 2);
      if (j < NQK) {
        s_next[j % 2][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[j], qop[0][j / 2], j < 2 ? zero : s_next[j % 2][0], 0, 0, 0);
      } else {
        const int i = j - NQK;
        o[i % (D / 32)][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[j], pop[i / (D / 32)], o[i % (D / 32)][0], 0, 0, 0);
      }
      between(j);
      // the exponentials' arguments, the exponentials and their sums and packing are three stages, one chunk apart, so that none
      // waits for the one before
#pragma unroll
      for (int e = exps_after(j - 2); e < exps_after(j - 1); e++) rs += p[e];
#pragma unroll
      for (int e = exps_after(j - 1); e < exps_after(j); e++) p[e] = __builtin_amdgcn_exp2f(arg[e]);
#pragma unroll
      for (int e = exps_after(j); e < exps_after(j + 1); e++) arg[e] = fmaf(s_cur[e / 16][0][e % 16], c, -m2);
#pragma unroll
      for (int e = exps_after(j - 2); e < exps_after(j - 1); e++) {
        if (e % 8 == 7) {
          bf16x8 pk;
#pragma unroll
          for (int k = 0; k < 8; k += 2) {
            f32x2 two = {p[e - 7 + k], p[e - 7 + k + 1]};
            bf16x2 h = __builtin_convertvector(two, bf16x2);
            pk[k] = h[0];
            pk[k + 1] = h[1];
          }
          pop[e / 8] = pk;
        }
      }
      asm volatile("" : "+v"(rs));                           // the running sum is due here, not at the end of the tile
      __builtin_amdgcn_sched_barrier(0);
    }
    if (HEAD == 0) meet();
  }

  // A segment's first and last tile are searched for the columns' maxima before their probabilities are made, the tiles between only from where a
  // wavefront meets scores that rise: 16 vector instructions a tile and an exchange between lanes, in a loop bound by what it issues
  // beside the MFMAs.  Worth 3 %: 32 x 4096 tokens x 256 beams 509 -> 495 us, 4 x 16384 x 512 in FP8 467 -> 454, 4 causal prompts of 3000 278 -> 268.
  // The reference is the first tile's maximum.  Where a lane's half of a column of a later tile sums to more than kRaise = 2^kLazy, which no
  // column does without a score kLazy - 5 bits above its reference, the column gets a higher reference after that tile, a power of two
  // for which this sum lies between 1 and 2, and the wavefront searches from there on: the reference becomes the maximum before a tile's
  // probabilities are made, once it is exceeded by more than kLazy.  us with the search in every tile, with it from the first rise, and with
  // neither, but columns that rose by 48 bits in a tile computed again: 32 x 4096 x 256 beams 509, 495, 492, and with scores of eight times
  // the width that N(0,1) queries and keys give 535, 542, 860; 4 causal prompts of 3000 278, 268, 268 and 297, 302, 495.
  //   Precision, in the one tile of the rise: the best token's probability, which may be nearly all of the sum, is not 1 as with the true
  // maximum; O has it rounded to bf16 and the sum has not.  What the rounding changed of the tile's sum is kept and O scaled by it at the end.
  //   Range: O may have overflowed there although the result does not.  A wavefront that met a rise looks through its O at the end, and where
  // it finds that, or where a sum passed kTooHigh, it computes its columns again (k_beam_attn's `redo`).
  //   A wavefront whose first tile has a score above kWide searches from the start: the scores will rise, perhaps beyond kTooHigh.  N(0,1) queries
  // and keys stay below 10 there.  Without it, scores 32 times as wide were computed twice: 32 x 4096 x 256 825 -> 542 us, 4 causal prompts
  // of 3000 421 -> 300, 4 x 16384 x 512 in FP8 1147 -> 468; N(0,1) inputs within 1 %.
  static constexpr float kLazy = 8.0f, kRaise = 256.0f, kTooHigh = 0x1p100f, kWide = 16.0f;

  // The segment's last tile, which no scores follow: O += V . P with the exponentials of the next 16 tokens between the MFMAs of the present
  // ones.  V^T operand: d = 32*db + (lane%32), k slot e <-> token 16*s + 8*(e/4) + 4*G + e%4.
  static __device__ __forceinline__ void finish(int sv, const f32x16 (&s)[KT / 32][NCB], f32x16 (&o)[D / 32][NCB], float m2, float c, float& rs, const Rd& rdo) {
    static_assert(NCB == 1, "one column block per wave");
    constexpr int DB = D / 32, N = NPV, PF = 4, EPC = 8 / DB;
    auto rdv = [&](int i) { return read_v(sv, rdo, i / DB, i % DB); };
    bf16x8 a[N], pop[KT / 16];
    float p[32];
    rs = 0.f;
    auto exps = [&](int e0, int n) {
#pragma unroll
      for (int e = e0; e < e0 + n; e++) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(s[e / 16][0][e % 16], c, -m2));
        rs += p[e];
      }
    };
    auto pack = [&](int t) {
#pragma unroll
      for (int k = 0; k < 8; k += 2) {
        const f32x2 two = {p[8 * t + k], p[8 * t + k + 1]};
        const bf16x2 h = __builtin_convertvector(two, bf16x2);
        pop[t][k] = h[0];
        pop[t][k + 1] = h[1];
      }
    };
#pragma unroll
    for (int i = 0; i < PF; i++) a[i] = rdv(i);
    exps(0, 8);
    pack(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int t = i / DB, k = i % DB;
      if (i + PF < N) a[i + PF] = rdv(i + PF);
      o[k][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], pop[t], o[k][0], 0, 0, 0);
      if (t + 1 < KT / 16) {
        exps(8 * (t + 1) + EPC * k, EPC);
        if (k == DB - 1) pack(t + 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

}  // namespace
