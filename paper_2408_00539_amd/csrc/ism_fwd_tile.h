// Device parts of the forward kernels (ism_fwd.hip, ism_fwd_window.hip): tiles,
// masks, the online softmax and the pipelined step.
#pragma once

#include "ism_common.h"
#include "ism_kernels.h"

namespace ism {

namespace {

constexpr int kBN = 64;  // keys per tile
constexpr int kQW = 32;  // query rows per wave
// Four-wave workgroups, two (three at d = 64) to a CU, so that one's prologue
// and last steps run beside another's products. Eight-wave workgroups stage
// each K/V tile for twice the columns, half the transfers per product, but are
// alone on their CU. Four waves against eight (us): packed, 32/8 heads, 8 x 3000
// 560, 570; 4 x 9000 2243, 2257; 3 x 12000 2945, 2941; 2 x 16384 3625, 3614; but 4
// ragged up to 16384 5662, 6101; 6 up to 12000 3501, 3851; 16/4 heads, d 64, 2 x
// 16384 1095, 1143. Cached, 32/8 heads, new rows: 64 over 40 x 2000 keys 126, 135;
// 2048 over 4 x 16384 2096, 2086; 1000 over 4000 93, 115. (Eight would win where
// equal dialogues of 129 to 256 columns leave no second round: 40 over 40 x
// 2000 111, 103; 40 over 20 x 8000 206, 178.)
constexpr int NWV = 4;
// Waves per SIMD, which bounds registers: d = 64 fits a third wave (4 x 8000
// tokens, 16 heads: 420 -> 398 us; not the paged cache, which would spill).
// With a window (forward of 8 ragged up to 3000, 32/8 heads, window 512 188 us with
// two waves, 154 with three; but cached, 300 ragged rows over 8 x 3000 keys, 16
// heads, window 1000 36.7 and 38.3: that spills at three).
constexpr int fwd_occupancy(int d, bool paged, bool window_cache) {
  return d == 64 && !paged && !window_cache ? 3 : 2;
}

// K and V tiles of 64 keys, row-major, unpadded rows of D bf16 with the
// swz<D>() chunk swizzle, double-buffered; filled by direct global->LDS
// transfers. K is read as MFMA rows (ds_read_b128), V through transposing
// reads (ds_read_b64_tr_b16) as the V^T operand.
template <int D>
struct FwdSmem {
  bf16_t k[2][kBN * D];
  bf16_t v[2][kBN * D];
};

// S^T[key][row] = K Q^T for one 64-key tile: two 32-key blocks, D/16 steps.
template <int D>
__device__ __forceinline__ void tile_scores(const char *kl, const SwzOffsets<D> &so,
                                            const bf16x8 (&qf)[D / 16], f32x16 (&s)[2]) {
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const bf16x8 kf = *(const bf16x8 *)(kl + kb * 32 * D * 2 + so.rowk[ks]);
      s[kb] = mfma32x32x16(kf, qf[ks], ks == 0 ? f32x16{} : s[kb]);
    }
}

// Keys past the row's bound lim get score -inf.
__device__ __forceinline__ void tile_mask(f32x16 (&s)[2], int c0, int hf, int lim) {
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = c0 + kb * 32 + (r >> 2) * 8 + hf * 4 + (r & 3);
      if (key > lim) s[kb][r] = -INFINITY;
    }
}

// Windowed attention: so do keys between the sinks (below send) and the row's
// window, which starts at lo.
__device__ __forceinline__ void tile_mask_window(f32x16 (&s)[2], int c0, int hf, int lim, int lo,
                                                 int send) {
  // (key - lo as an unsigned number is below the window's width for its keys)
  const int at = c0 + hf * 4 - lo, sinks = min(send, lim + 1) - c0 - hf * 4;
  const uint32_t width = (uint32_t)max(lim - lo + 1, 0);
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int k = kb * 32 + (r >> 2) * 8 + (r & 3);
      if ((uint32_t)(at + k) >= width && k >= sinks) s[kb][r] = -INFINITY;
    }
}

// Row max of a tile, combined over the lane pair that holds the row.
__device__ __forceinline__ float tile_max(const f32x16 (&s)[2]) {
  float x[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int r = 0; r < 16; r += 2) x[r & 3] = vmax(x[r & 3], vmax(s[kb][r], s[kb][r + 1]));
  return pair_max(vmax(vmax(x[0], x[2]), vmax(x[1], x[3])));
}

// The reference max in log2 units. SPLIT: a row that has seen no key yet (an
// answer row whose keys end before the chunk) has m = -inf and keeps l = 0.
template <bool SPLIT>
__device__ __forceinline__ float log2_max(float m, float sl2) {
  return SPLIT && m == -INFINITY ? 0.f : m * sl2;
}

// Lazy online-softmax update: the reference max is only raised when a row's
// tile max exceeds it by more than tau (2^8 in probability units); exact
// either way since numerator and denominator share the reference max.
template <bool SPLIT, int NDB>
__device__ __forceinline__ void raise_max(float mt, float sl2, float tau, float &m_run,
                                          float &l_run, f32x16 (&oacc)[NDB]) {
  if (__builtin_amdgcn_ballot_w64(mt > m_run + tau) != 0) {
    const float mnew = vmax(m_run, mt);
    const float alpha = SPLIT && mnew == -INFINITY ? 1.f : fast_exp2((m_run - mnew) * sl2);
    m_run = mnew;
    l_run *= alpha;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
  }
}

// One pipelined step in a fixed instruction order: the D/8 products of
// S(t+1) = K(t+1) Q^T (its two 32-key blocks alternating), then the D/8
// products of O^T += V(t)^T P(t)^T (64-key chunks outermost), so that
// consecutive products always use different accumulators. Each product is
// followed by the LDS read of the operand LA = 2 products ahead (K rows, then
// transposed V; a third operand in flight measured ~1 % slower, one only
// ~7 % slower) and by its share of the vector work: during
// the S products the exponentials, row sums and bf16 packing of tile t,
// during the P V products the row max of S(t+1). The order is pinned with
// scheduling barriers so that the matrix core and the vector ALU of a wave
// are busy at the same time. P enters the second product rounded to bf16 (o is
// off by 0.0020 to 0.0023 of its norm, by its own rounding alone 0.0017): as two
// bf16 summands it would take half as many products again, where the matrix core
// is the bound. Returns the fp32 row sum of P(t); mt receives
// the (unmasked) row max of S(t+1). With LAST (a wave's last tile) there is
// no S(t+1): the exponentials run alone, then the P V products.
// With PRIO the wave raises its issue priority for the first half (the S
// products and the exponentials, the vector-heavy half) and drops it for the
// P V products, so that of the two waves on a SIMD the one in its
// exponentials issues first and the other one's products fill the matrix
// core around it (about 2 % faster on the packed forward; steps whose
// transfers all start at the step start measured ~1 % slower with it).
template <int D, bool LAST, bool PRIO, class Hook>
__device__ __forceinline__ float step_block(const char *kl, const char *vl,
                                            const SwzOffsets<D> &so, const bf16x8 (&qf)[D / 16],
                                            const f32x16 (&cur)[2], f32x16 (&nxt)[2],
                                            f32x16 (&oacc)[D / 32], float sl2, float moff,
                                            float &mt, Hook &&hook) {
  constexpr int NKS = D / 16, NDB = D / 32;
  constexpr int NS = 2 * NKS, NP = 4 * NDB, N = NS + NP, LA = 2;
  constexpr int PPS = 16 / NS;  // probability pairs per S product
  constexpr int MPP = 32 / NP;  // max elements per P V product
  auto read = [&](int n) -> bf16x8 {
    if (n < NS) {
      const int kb = n & 1, ks = n >> 1;
      return *(const bf16x8 *)(kl + kb * 32 * D * 2 + so.rowk[ks]);
    }
    const int j = n - NS, kc = j / NDB, db = j % NDB;
    const uint32_t o = ((kc >> 1) * 32 + 16 * (kc & 1)) * D * 2;
    return tr_operand_at(vl, o + so.trk[db][0], o + so.trk[db][1]);
  };
  constexpr int F = LAST ? NS : 0;  // first product that runs
  bf16x8 op[N];
#pragma unroll
  for (int n = F; n < F + LA; ++n) op[n] = read(n);
  u32x4 w[2][2];
  float sum[2] = {0.f, 0.f}, mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (PRIO && n == 0) __builtin_amdgcn_s_setprio(1);
    if (PRIO && n == NS) __builtin_amdgcn_s_setprio(0);
    if (n < NS) {
      if (!LAST) {
        const int kb = n & 1, ks = n >> 1;
        nxt[kb] = mfma32x32x16(op[n], qf[ks], ks == 0 ? f32x16{} : nxt[kb]);
      }
    } else {
      const int j = n - NS, kc = j / NDB, db = j % NDB;
      oacc[db] = mfma32x32x16(op[n], __builtin_bit_cast(bf16x8, w[kc >> 1][kc & 1]), oacc[db]);
    }
    hook(n);  // n is a constant once the loop is unrolled
    if (n >= F && n + LA < N) op[n + LA] = read(n + LA);
    if (n < NS) {
#pragma unroll
      for (int c = 0; c < PPS; ++c) {
        const int i = n * PPS + c, kb = i >> 3, bt = (i >> 2) & 1, u = i & 3;
        f32x2 p;
        p[0] = fast_exp2(fmaf(cur[kb][8 * bt + 2 * u], sl2, -moff));
        p[1] = fast_exp2(fmaf(cur[kb][8 * bt + 2 * u + 1], sl2, -moff));
        sum[i & 1] += p[0] + p[1];
        w[kb][bt][u] = cvt_bf16x2(p);
        asm volatile("" : "+v"(sum[i & 1]));  // keep the add in this slot
      }
    } else if (!LAST) {
#pragma unroll
      for (int c = 0; c < MPP; c += 2) {
        const int e = (n - NS) * MPP + c, m = (e >> 1) & 1;
        mx[m] = vmax(mx[m], vmax(nxt[e >> 4][e & 15], nxt[e >> 4][(e & 15) + 1]));
        asm volatile("" : "+v"(mx[m]));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  mt = LAST ? -INFINITY : pair_max(vmax(mx[0], mx[1]));
  return sum[0] + sum[1];
}

inline int gcd_int(int x, int y) {
  while (y) { const int t = x % y; x = y; y = t; }
  return x;
}

}  // namespace

}  // namespace ism
