// Windowed forward over packed dialogues (training / prefill): the forward
// kernel of ism_fwd.hip for key ranges of a few tiles. A workgroup's prologue
// (lengths, bounds, the first tiles' and queries' latency, the first scores)
// costs about five of its steps, so a workgroup here runs one column tile after
// another, and starts the next one's transfers and query loads at the last step
// of the current one, where K's buffers and the query registers are free.
// Bounds as in the forward kernel: MFMA, at 4 d FLOP per visible pair.
#include "ism_fwd_tile.h"

namespace ism {

namespace {

// A column tile: 128 (row, head) columns of `1 << lf` query heads from head0 on.
struct WinItem {
  int b, s, e, head0, c0;
  int64_t kv;  // element offset of its KV head's first key
};
// Its keys by their index in the workgroup's list (WinList), from the dialogue's
// first key s on: the workgroup's last, and the least and greatest bound of the
// wave's rows.
struct WinBounds {
  WinList wl;
  int key_hi, wave_lo, wave_hi;
};

// Work order: the column tiles of dialogue b and head set h are slots
// [first(b) + h n_b, + n_b) with n_b >= their number (at most one more, left
// out), first(b) = hsets (floor(128ths of columns before b) + b); XCD x takes a
// contiguous eighth of the slots, its workgroups every stride-th, so that the
// tiles that run at once share their keys in the XCD's L2 and every workgroup
// gets the same number of slots (to one).
template <int D>
__global__ void __launch_bounds__(NWV * 64)
__attribute__((amdgpu_waves_per_eu(fwd_occupancy(D, false, false),
                                   fwd_occupancy(D, false, false))))
fwd_window_kernel(FwdArgs a, int lf, int per_xcd, int slots) {
  constexpr int NDB = D / 32, NKS = D / 16;
  __shared__ FwdSmem<D> sm;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  const int hsets = a.hq >> lf, kv_group = a.hq / a.hkv;
  const int64_t rs = a.kv_row_stride;
  const float sl2 = a.scale * kLog2e, tau = 8.f / sl2;

  // the slots of this workgroup, and the next tile among them
  int slot = (int)(blockIdx.x & 7) * per_xcd;
  const int slot_end = min(slot + per_xcd, slots), stride = (int)gridDim.x >> 3;
  slot += (int)blockIdx.x >> 3;
  auto tiles_before = [&](int cu, int b) __attribute__((always_inline)) {
    return (int)(((int64_t)cu << lf) / (NWV * kQW)) + b;
  };
  auto next_item = [&](WinItem &x) __attribute__((always_inline)) {
    for (; slot < slot_end; slot += stride) {
      // (slots past the last dialogue's: tokens that belong to none)
      while (x.b + 1 < a.batch && hsets * tiles_before(x.e, x.b + 1) <= slot) {
        ++x.b;
        x.s = x.e;
        x.e = a.cu_q[x.b + 1];
      }
      const int t0 = tiles_before(x.s, x.b), n = tiles_before(x.e, x.b + 1) - t0;
      const int r = slot - hsets * t0, h = __builtin_amdgcn_readfirstlane(r / n);
      if (h >= hsets) break;
      x.c0 = __builtin_amdgcn_readfirstlane((r - h * n) * (NWV * kQW));
      x.head0 = h << lf;
      x.kv = (int64_t)x.s * rs + (int64_t)(x.head0 / kv_group) * a.kv_head_stride;
      if (x.c0 < (x.e - x.s) << lf) {
        slot += stride;
        return true;
      }
    }
    return false;
  };
  auto row_of = [&](const WinItem &x, int col) __attribute__((always_inline)) {
    return x.s + (min(col, ((x.e - x.s) << lf) - 1) >> lf);
  };
  auto bounds_of = [&](const WinItem &x) __attribute__((always_inline)) {
    WinBounds w;
    w.wl = win_uniform(win_list<1>(x.c0 >> lf, a.window, a.sinks, x.e - 1 - x.s));
    const int wc0 = x.c0 + wave * kQW;
    const bool active = wc0 < (x.e - x.s) << lf;
    const int last = row_of(x, x.c0 + NWV * kQW - 1), r0 = row_of(x, wc0),
              r1 = row_of(x, wc0 + kQW - 1);
    w.key_hi = __builtin_amdgcn_readfirstlane(a.lim[last] - w.wl.shift);
    w.wave_lo = __builtin_amdgcn_readfirstlane(a.lim[r0] - w.wl.shift);
    w.wave_hi = __builtin_amdgcn_readfirstlane(active ? a.lim[r1] - w.wl.shift : x.s - 1);
    return w;
  };

  WinItem it{};
  if (slot >= slot_end) return;
  // the dialogue of the first slot: 64 of those left at a time
  for (int left = a.batch; left > 1;) {
    const int step = (left + 63) >> 6, b = min(it.b + lane * step, a.batch - 1);
    const bool at = lane * step < left && hsets * tiles_before(a.cu_q[b], b) <= slot;
    const int i = __builtin_popcountll(__builtin_amdgcn_ballot_w64(at)) - 1;
    it.b += i * step;
    left = min(step, left - i * step);
  }
  it.s = a.cu_q[it.b];
  it.e = a.cu_q[it.b + 1];
  if (!next_item(it)) return;
  // (the first transfers start before the bounds: keys past them are masked)
  WinBounds bd;
  bd.wl = win_uniform(win_list<1>(it.c0 >> lf, a.window, a.sinks, it.e - 1 - it.s));
  bd.key_hi = it.e - 1 - bd.wl.shift;

  DmaTile<D, kBN, NWV> dma;
  dma.init(tid, rs);
  SwzOffsets<D> so;
  so.init(lane);
  // tile t of K (V), whose keys from index `end` on do not exist
  auto tile_off = [&](const WinItem &x, const WinBounds &w, int t)
                      __attribute__((always_inline)) {
    const int o = t * kBN;
    return x.kv + (int64_t)(o + (o >= a.sinks ? w.wl.shift : 0)) * rs;
  };
  auto issue = [&](const WinItem &x, const WinBounds &w, bool v, int t, bf16_t *lds)
                   __attribute__((always_inline)) {
    const bf16_t *base = (const bf16_t *)(v ? a.v : a.k);
    const int o = t * kBN, nvalid = w.key_hi - x.s - o + 1;
    const int64_t off = tile_off(x, w, t);
    const bool mixed = win_mixed<kBN>(w.wl, a.sinks, o);
    if (D == 128 && mixed && nvalid >= kBN)  // (at d = 64 it spills)
      dma.issue_two(base + off, base + off + (int64_t)w.wl.shift * rs, a.sinks - o, lds);
    else if (mixed)
      dma.issue_list(base + off, base + off + (int64_t)w.wl.shift * rs, rs, a.sinks - o,
                     w.wl.lo - o, nvalid, lds);
    else
      dma.issue(uniform_ptr(base + off), rs, nvalid, lds);
  };
  // K(0) and K(1) of an item, and V(0)
  auto issue_k = [&](const WinItem &x, const WinBounds &w) __attribute__((always_inline)) {
#pragma unroll 1
    for (int t = 0; t < 2 && x.s + t * kBN <= w.key_hi; ++t) issue(x, w, false, t, sm.k[t]);
  };
  bf16x8 qf[NKS];
  int lim_r;  // the bound of this lane's row
  auto load_rows = [&](const WinItem &x) __attribute__((always_inline)) {
    const int col = min(x.c0 + wave * kQW + l32, ((x.e - x.s) << lf) - 1);
    const int row = x.s + (col >> lf), head = x.head0 + (col & ((1 << lf) - 1));
    const bf16_t *qp = (const bf16_t *)a.q + ((int64_t)row * a.hq + head) * D + hf * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = *(const bf16x8 *)(qp + ks * 16);
    lim_r = a.lim[row];
  };
  issue_k(it, bd);
  issue(it, bd, true, 0, sm.v[0]);
  load_rows(it);
  bd = bounds_of(it);

  bool late_v = false;  // V(0) may still be on its way
  wait_loads();         // Q, the bounds and the first tiles
  __syncthreads();
  for (;;) {
    const int crow = row_of(it, it.c0 + wave * kQW + l32);
    lim_r -= bd.wl.shift;
    const int lo_r = crow - a.window + 1 - bd.wl.shift, send = it.s + a.sinks;
    const int lo_last = row_of(it, it.c0 + wave * kQW + kQW - 1) - a.window + 1 - bd.wl.shift;
    const int ntiles = (bd.key_hi - it.s) / kBN + 1;
    const int nw = bd.wave_hi >= it.s ? (bd.wave_hi - it.s) / kBN + 1 : 0;

    f32x16 oacc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f;
    auto mask_tile = [&](f32x16 (&x)[2], int c0) __attribute__((always_inline)) {
      if (c0 + kBN - 1 <= bd.wave_lo && (c0 >= lo_last || c0 + kBN <= send)) return false;
      tile_mask_window(x, c0, hf, lim_r, lo_r, send);
      return true;
    };
    f32x16 sa[2], sb[2];
    if (nw > 0) {
      tile_scores<D>((const char *)sm.k[0], so, qf, sa);
      mask_tile(sa, it.s);
      raise_max<true>(tile_max(sa), sl2, tau, m_run, l_run, oacc);
    }
    WinItem nx = it;
    const bool more = next_item(nx);
    WinBounds nb = bd;
    if (more) nb = bounds_of(nx);
    if (late_v) wait_vmem();
    lds_barrier();  // every wave is done with K(0); V(0) is there

    // (tiles behind the sinks, which MODE 0 is for)
    const int64_t tile_elems = (int64_t)kBN * rs, off0 = it.kv + (int64_t)bd.wl.shift * rs;
    const bf16_t *kt = uniform_ptr((const bf16_t *)a.k + off0);
    const bf16_t *vt = uniform_ptr((const bf16_t *)a.v + off0);

    // Step t, as in the forward kernel (MODE 0: full tiles, spread; MODE 1: at
    // once; MODE 2: the last tile, beside which the next item starts).
    auto step = [&](f32x16 (&cur)[2], f32x16 (&nxt)[2], int t, auto modec) {
      constexpr int MODE = decltype(modec)::value;
      constexpr bool LAST = MODE == 2;
      constexpr int NI = decltype(dma)::NI;
      const int c0 = it.s + t * kBN;
      if (MODE == 1 || (MODE == 0 && t >= nw)) {
#pragma unroll 1
        for (int i = t + 2 < ntiles ? 0 : 1; i < 2; ++i)
          issue(it, bd, i, t + 2 - i, i ? sm.v[(t + 1) & 1] : sm.k[t & 1]);
      }
      if (LAST && more) {
        issue_k(nx, nb);
        if (t & 1) issue(nx, nb, true, 0, sm.v[0]);
        load_rows(nx);
      }
      const char *kl = (const char *)sm.k[(t + 1) & 1];
      const char *vl = (const char *)sm.v[t & 1];
      const bf16_t *ksrc = kt + 2 * tile_elems, *vsrc = vt + tile_elems;
      auto hook = [&](int n) __attribute__((always_inline)) {
        if (MODE == 0 && n % 3 == 0 && n / 3 < 2 * NI) {
          if (n / 3 < NI) dma.issue_one(ksrc, n / 3, sm.k[t & 1]);
          else dma.issue_one(vsrc, n / 3 - NI, sm.v[(t + 1) & 1]);
        }
      };
      if (t < nw) {
        float mt;
        l_run += step_block<D, LAST, true>(kl, vl, so, qf, cur, nxt, oacc, sl2,
                                           log2_max<true>(m_run, sl2), mt, hook);
        if (!LAST && t + 1 < nw) {
          if (mask_tile(nxt, c0 + kBN)) mt = tile_max(nxt);
          raise_max<true>(mt, sl2, tau, m_run, l_run, oacc);
        }
      }
      if (!LAST) {
        kt += tile_elems;
        vt += tile_elems;
        wait_vmem();
        __syncthreads();
      }
    };
    int t = 0;
    // (none spread if a mixed tile comes after the first)
    if ((bd.wl.shift == 0 && bd.wl.lo <= a.sinks) || kBN >= max(a.sinks, bd.wl.lo)) {
      const int nfull = max((bd.key_hi - it.s + 1) / kBN - 2, 0) & ~1;
      for (; t < nfull; t += 2) {
        step(sa, sb, t, std::integral_constant<int, 0>{});
        step(sb, sa, t + 1, std::integral_constant<int, 0>{});
      }
    }
    for (; t + 1 < ntiles; t += 2) {
      step(sa, sb, t, std::integral_constant<int, 1>{});
      if (t + 2 < ntiles) step(sb, sa, t + 1, std::integral_constant<int, 1>{});
    }
    // (one instance of the last step: a second one cost 98 spilled registers)
    if ((ntiles - 1) & 1) {
      sa[0] = sb[0];
      sa[1] = sb[1];
    }
    step(sa, sb, ntiles - 1, std::integral_constant<int, 2>{});

    if (more) {
      wait_loads();  // the next item's first tiles, queries and bounds
      __syncthreads();
      late_v = ((ntiles - 1) & 1) == 0;
      if (late_v) issue(nx, nb, true, 0, sm.v[0]);
    }
    const float lt = pair_sum(l_run);
    const int ocol = it.c0 + wave * kQW + l32;
    if (ocol < (it.e - it.s) << lf) {
      const int row = it.s + (ocol >> lf), head = it.head0 + (ocol & ((1 << lf) - 1));
      const float inv = 1.f / lt;
      bf16_t *op = (bf16_t *)a.o + ((int64_t)row * a.hq + head) * D + hf * 8;
#pragma unroll
      for (int db = 0; db < NDB; ++db) store_bf16_col(op + db * 32, oacc[db], inv);
      if (a.lse && hf == 0)
        a.lse[(int64_t)head * a.total_q + row] = m_run * a.scale + logf(lt);
    }
    if (!more) return;
    it = nx;
    bd = nb;
  }
}

template <int D>
hipError_t launch_t(const FwdArgs &a, hipStream_t stream) {
  const int fold = gcd_int(a.hq / a.hkv, NWV);
  const int lf = fold == 4 ? 2 : fold == 2 ? 1 : 0;
  const int64_t slots =
      (int64_t)(a.hq / fold) * (((int64_t)a.total_q << lf) / (NWV * kQW) + a.batch);
  if (slots > 0x7fffffff) return hipErrorInvalidValue;
  const int per_xcd = (int)((slots + 7) / 8);
  // the workgroups that the chip holds at once (two or three to a CU)
  const int most = 32 * fwd_occupancy(D, false, false);
  const int wgs = per_xcd < most ? per_xcd : most;
  hipLaunchKernelGGL(fwd_window_kernel<D>, dim3((unsigned)wgs * 8), dim3(NWV * 64), 0, stream, a,
                     lf, per_xcd, (int)slots);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fwd_window(const FwdArgs &a, int d, hipStream_t stream) {
  if (d == 128) return launch_t<128>(a, stream);
  if (d == 64) return launch_t<64>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace ism
