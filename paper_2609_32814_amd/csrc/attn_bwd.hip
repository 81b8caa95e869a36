// Gradient of causal attention over a pack of sequences.  With the scores
// s_pu = scale_ij <Q_p, K_u> over the groups of F(i, j) (i, j the types of the
// two positions), P = exp(s - lse) and delta_p = <dO_p, O_p>:
//   dP_pu = <dO_p, V_u>          dS_pu = scale_ij P_pu (dP_pu - delta_p)
//   dQ_p = sum_u dS_pu K_u       dK_u = sum_p dS_pu Q_p      (groups of F(i, j))
//   dV_u = sum_p P_pu dO_p
// Scores and dP are computed again from the rows in both of the two launches,
// seven products where one pass with dQ summed by atomics takes five: every
// element of a gradient then has one owner and one order of summation.
//
// attn_dq_kernel: a workgroup owns 128 queries of one type, 32 per wavefront,
// and walks the keys like the forward: S^T = K Q^T and dP^T = V dO^T with the
// rows of K and V from LDS and the wave's rows of Q and dO in registers, so
// that a lane holds 16 keys of one query, then dQ^T += K^T dS^T with dS^T as
// it lies in the registers and K^T by transposing reads of the same tile.  It
// also leaves delta for the second launch.
//
// attn_dkv_kernel: a workgroup owns 128 keys of one type, 32 per wavefront,
// and walks the queries from its first key on, for every query head of its
// key/value head in turn: S = Q K^T and dP = dO V^T with the rows of Q and dO
// from LDS and those of K and V in registers, dV^T += dO^T P and
// dK^T += Q^T dS.  With few keys the heads are dealt to several workgroups, and
// attn_dkv_join_kernel adds their fp32 sums.
//
// P and dS enter their products rounded to bf16 (at most 2^-8 of each term,
// like the operands themselves); everything else is fp32.
//
// Measured: one sequence of 8192, all features: dQ 830 us for 64 heads of 64
// (990 TFLOP/s), 805 for 32 of 128 (1020); dK and dV 1105 (995) and 1105 (995),
// bound by the products (a large library product reaches 1183).  24576 tokens
// in 17 sequences, 12 heads of 64, star law, q = 4: 300 to 330 + 365 to 395 us;
// 8192 tokens in 6, 32 heads of 128 on 8, q = 2: 345 to 375 + 505 to 545.  1500
// tokens: 21 + 21 us, a prologue of about 8 us and up to 8 steps of 1 us, each a
// chain of reads, products and exponentials that few wavefronts cannot hide.
#include <type_traits>

#include "attn_common.hpp"
#include "attn_walk.hpp"

namespace starq {

namespace {

// For a row that is not there: -inf for its negated log-sum-exp, so that its
// probabilities are zero, and zero for its delta
__device__ __attribute__((aligned(256))) float g_attn_no_side[2] = {-INFINITY, 0.f};

// NG groups of four wavefronts take the steps of the walk in turn, each with a
// ring of its own; their sums meet at the end.
template <int DH, int NG, int NB>
__global__ __launch_bounds__(NG * kItemThreads, DH == 64 && NG == 1 ? 4 : 2) void attn_dq_kernel(const AttnBwdParams p) {
  constexpr int NCH = DH / 32, KS = DH / 16, TILE = tile_bytes<DH>(), NC = 2 * copies_per_step<DH>();
  extern __shared__ __attribute__((aligned(16))) char rings[];  // [group][stage][K, V]
  __shared__ ItemLds<NG> it_s;

  if (!pack_matches(p.pack, p.T, p.n_seq, p.q)) return;
  if (blockIdx.x >= static_cast<unsigned>(p.q_wgs)) {
    pack_clear_rows(p.pack, p.T, blockIdx.x - p.q_wgs, p.clear_rest, p.dQ, p.gdtype, p.n_heads * DH);
    return;
  }
  int h;
  int32_t k;
  if (!pack_item(p.pack, p.n_heads, h, k)) return;
  const int32_t* rec = p.pack.recs_q + static_cast<int64_t>(k) * pack_rec_ints(p.q);
  const int64_t seq0 = rec[0];
  const int32_t nvalid = rec[3] >> 16;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6) % kItemWaves, g = uniform(threadIdx.x >> 6) / kItemWaves;
  const int lr = lane & 31, lh = lane >> 5;
  const int hk = h / (p.n_heads / p.n_kv);
  const int64_t ldq = static_cast<int64_t>(p.n_heads) * DH, ldk = static_cast<int64_t>(p.n_kv) * DH;
  const uint16_t* Kg = static_cast<const uint16_t*>(p.K) + seq0 * ldk + hk * DH;
  const uint16_t* Vg = static_cast<const uint16_t*>(p.V) + seq0 * ldk + hk * DH;
  const uint32_t ldk16 = static_cast<uint32_t>(ldk >> 3);
  const int row0 = wave * 32;
  const int32_t my = row0 + lr < nvalid ? p.pack.perm[rec[2] + row0 + lr] : -1;
  setup_item(it_s, rec, p.law, p.q, DH);
  __syncthreads();

  char* tiles = rings + g * ring_bytes<DH>();
  Walk<NG> wx(&it_s, p.q, 1, g), wp = wx, wc = wx;  // the group's steps h, h + 5, h + 2
  const int32_t trips = wx.trips();
  Copies<DH> cp;
  auto ring = [&](int32_t step) { return it_s.ring[g][step & (kPosSlots - 1)]; };
  auto ask = [&](int32_t step) {
    if (wave == 0) ask_positions(wp, p.pack.perm, ring(step), lane);
    wp.next();
  };
  auto copy = [&](int st) {
    cp.issue(Kg, Vg, ldk16, wc.cells, tiles + st * 2 * TILE, wave, lane);
    wc.next();
  };
  for (int x = 0; x < 4; ++x) ask(x);
  // the wave's rows of Q and dO as operands, delta and lse (asked for before
  // the first copies, used behind them)
  const int m = DH / p.q;
  const Blocks<DH, NB> bl(rec[3] & 0xffff, m);
  uint4 qf[KS], df[KS];
  uint4 of[2 * KS];  // O: 8 values in the first half of each pair, or fp32 in both
  const int64_t qrow = (seq0 + max(my, 0)) * ldq + h * DH;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int fr = 16 * ks + 8 * lh;
    qf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Q) + qrow + 16 * bl.turned(ks) + 8 * lh);
    df[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.dO) + qrow + fr);
  }
  if (p.odtype == 0) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint4* o = reinterpret_cast<const uint4*>(static_cast<const float*>(p.O) + qrow + 16 * ks + 8 * lh);
      of[2 * ks] = o[0];
      of[2 * ks + 1] = o[1];
    }
  } else {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      of[2 * ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.O) + qrow + 16 * ks + 8 * lh);
      of[2 * ks + 1] = make_uint4(0, 0, 0, 0);
    }
  }
  const int64_t at = static_cast<int64_t>(h) * p.T + seq0 + max(my, 0);
  float lse2 = p.lse[at];
  // positions ascend along the block: the first and last of the wave's rows
  const int32_t tv = min(32, nvalid - row0);
  const int32_t tfirst = tv > 0 ? uniform(my) : kNoPos;
  const int32_t tlast = tv > 0 ? __builtin_amdgcn_readlane(my, tv - 1) : -1;
  wait_vm<0>();
  landed(qf, my >= 0);
  landed(df, my >= 0);
  landed(of, my >= 0);
  landed(lse2);
  lse2 = my >= 0 ? lse2 * kLog2e : 0.f;
  Ends now, then;
  auto start = [&] {
    __syncthreads();
    cp.take(ring(0), wave, lane);
    copy(0);
    cp.take(ring(1), wave, lane);
    ask(4);
    copy(1);
    cp.take(ring(2), wave, lane);
    now.take(ring(0));
    then.take(ring(1));
    now.settle();
    then.settle();
  };
  start();

  float delta = 0.f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const uint32_t d[4] = {df[ks].x, df[ks].y, df[ks].z, df[ks].w};
    const uint4 u = of[2 * ks], v = of[2 * ks + 1];
    const uint32_t o[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float o0 = p.odtype == 0 ? __uint_as_float(o[2 * e]) : bf16_to_f32(o[e] & 0xffffu);
      const float o1 = p.odtype == 0 ? __uint_as_float(o[2 * e + 1]) : bf16_to_f32(o[e] >> 16);
      delta += bf16_to_f32(d[e] & 0xffffu) * o0 + bf16_to_f32(d[e] >> 16) * o1;
    }
  }
  delta = sum_xor32(delta);
  if (my >= 0 && lh == 0) {  // for the other launch
    p.side[at] = -lse2;
    p.side[at + static_cast<int64_t>(p.n_heads) * p.T] = -delta;
  }
  f32x16_t acc[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) acc[c] = f32x16_t{};
  TileLane<DH> tl(lane);

  // stage st: the tile of step `step`
  const std::true_type yes;
  const std::false_type no;
  auto body = [&](auto care, int st, int32_t step) {
    if (wave == 0) wait_vm<NC + 1>();
    else wait_vm<NC>();
    __syncthreads();
    ask(step + 5);
    copy((st + 2) % kStages);
    cp.take(ring(step + 3), wave, lane);
    Ends after;
    after.take(ring(step + 2));
    if (now.first <= tlast) {
      const char* Kt = tiles + st * 2 * TILE;
      tl.renew();
      f32x16_t sc{}, dp{};
      const int j = wx.template block<DH, NB>(bl, m);
      tl.template add_rows<NB>(sc, Kt, qf, bl, j);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) dp = mfma(tl.row(Kt + TILE, ks), df[ks], dp);
      // keys behind a query (rows past a type's end have position kNoPos)
      if (now.last > tfirst) {
        const int32_t* kps = ring(step);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int4 kq = *reinterpret_cast<const int4*>(kps + 8 * a + 4 * lh);
          const int32_t k4[4] = {kq.x, kq.y, kq.z, kq.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (k4[e] > my) {
              sc[4 * a + e] = -INFINITY;
              if (care) dp[4 * a + e] = delta;
            }
        }
      }
      // dS = scale P (dP - delta): the scale goes into the exponent
      const float scale2 = wx.scale * kLog2e, base = lse2 - wx.lg;
      float ds[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) ds[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale2, -base)) * (dp[e] - delta);
      const uint4 pf[2] = {pack8(ds), pack8(ds + 8)};
      if (care) tl.add_odd(acc, Kt, pf, bl.own * NB / 2);
      else tl.template add_transposed_kept<NB>(acc, Kt, pf, bl, j);
    }
    wx.next();
    now = then;
    after.settle();
    then = after;
  };

  for (int32_t n = 0; n < trips; n += 3) {
    body(no, 0, n);
    if (n + 1 == trips) break;
    body(no, 1, n + 1);
    if (n + 2 == trips) break;
    body(no, 2, n + 2);
  }
  wait_vm<0>();
  if (__syncthreads_or(odd(acc))) {
    wx = wp = wc = Walk<NG>(&it_s, p.q, 1, g);
    for (int x = 0; x < 4; ++x) ask(x);
    wait_vm<0>();
    start();
#pragma unroll
    for (int c = 0; c < NCH; ++c) acc[c] = f32x16_t{};
#pragma unroll 1
    for (int32_t n = 0; n < trips; ++n) body(yes, n % kStages, n);
    wait_vm<0>();
  }
  if constexpr (NG == 2) {
    if (!join_groups<NCH>(acc, rings, g, wave, lane)) return;
  }
  if (my >= 0) store_row<DH>(p.dQ, p.gdtype, qrow, acc, lh, bl.own * NB / 2);
}

template <int DH, int NG, int NB>
__global__ __launch_bounds__(NG * kItemThreads, NG == 1 ? 3 : 2) void attn_dkv_kernel(const AttnBwdParams p) {
  constexpr int NCH = DH / 32, KS = DH / 16, TILE = tile_bytes<DH>(), NC = 2 * copies_per_step<DH>();
  extern __shared__ __attribute__((aligned(16))) char rings[];  // [group][stage][Q, dO]
  __shared__ ItemLds<NG> it_s;
  __shared__ __attribute__((aligned(16))) float side_all[NG][kStages][64];  // 32 times -lse (base 2), 32 times -delta

  if (!pack_matches(p.pack, p.T, p.n_seq, p.q)) return;
  if (blockIdx.x >= static_cast<unsigned>(p.k_wgs)) {
    pack_clear_rows(p.pack, p.T, blockIdx.x - p.k_wgs, p.clear_rest, p.dK, p.gdtype, p.n_kv * DH);
    pack_clear_rows(p.pack, p.T, blockIdx.x - p.k_wgs, p.clear_rest, p.dV, p.gdtype, p.n_kv * DH);
    return;
  }
  int share;
  int32_t k;
  if (!pack_item(p.pack, p.n_kv * p.parts, share, k)) return;
  // the query heads of this item: h0 .. h0 + rep - 1, of key/value head hk
  const int hk = share / p.parts, part = share % p.parts, rep = p.n_heads / p.n_kv / p.parts, h0 = share * rep;
  const int32_t* rec = p.pack.recs_k + static_cast<int64_t>(k) * pack_rec_ints(p.q);
  const int64_t seq0 = rec[0];
  const int32_t nvalid = rec[3] >> 16;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6) % kItemWaves, g = uniform(threadIdx.x >> 6) / kItemWaves;
  const int lr = lane & 31, lh = lane >> 5;
  const int64_t ldq = static_cast<int64_t>(p.n_heads) * DH, ldk = static_cast<int64_t>(p.n_kv) * DH;
  const uint16_t* Qg = static_cast<const uint16_t*>(p.Q) + seq0 * ldq + static_cast<int64_t>(h0) * DH;
  const uint16_t* Dg = static_cast<const uint16_t*>(p.dO) + seq0 * ldq + static_cast<int64_t>(h0) * DH;
  const uint32_t ldq16 = static_cast<uint32_t>(ldq >> 3);
  const int row0 = wave * 32;
  const int32_t my = row0 + lr < nvalid ? p.pack.perm[rec[2] + row0 + lr] : -1;
  setup_item(it_s, rec, p.law, p.q, DH);
  __syncthreads();

  char* tiles = rings + g * ring_bytes<DH>();
  float(*side_s)[64] = side_all[g];
  Walk<NG> wx(&it_s, p.q, rep, g), wp = wx, wc = wx;  // the group's steps h, h + 5, h + 2
  const int32_t trips = wx.trips();
  Copies<DH> cp;
  int32_t side_pos = kNoPos;
  auto ring = [&](int32_t step) { return it_s.ring[g][step & (kPosSlots - 1)]; };
  auto ask = [&](int32_t step) {
    if (wave == 0) ask_positions(wp, p.pack.perm, ring(step), lane);
    wp.next();
  };
  auto take = [&](int32_t step) {
    cp.take(ring(step), wave, lane);
    side_pos = ring(step)[lr];
  };
  // rows, and by wavefront 1 their log-sum-exps and deltas
  const float* side0 = p.side + static_cast<int64_t>(h0) * p.T + seq0;
  const float* no_side = g_attn_no_side;
  asm volatile("" : "+s"(no_side));
  auto copy = [&](int st) {
    if (wave == 1) {
      int half = lane;
      asm volatile("" : "+v"(half));  // (worth no register between the steps)
      half >>= 5;
      const float* row = side0 + static_cast<int64_t>(wc.hh) * p.T;
      const float* at = row + (half ? static_cast<int64_t>(p.n_heads) * p.T : 0) + side_pos;
      dma4(side_pos != kNoPos ? at : no_side + half, lds_addr(side_s[st]));
    }
    cp.issue(Qg + wc.hh * DH, Dg + wc.hh * DH, ldq16, wc.cells, tiles + st * 2 * TILE, wave, lane);
    wc.next();
  };
  for (int x = 0; x < 4; ++x) ask(x);
  const int m = DH / p.q;
  const Blocks<DH, NB> bl(rec[3] & 0xffff, m);
  uint4 kf[KS], vf[KS];
  auto krow = [&] {  // (worth no registers between its uses)
    int32_t r = max(my, 0);
    asm volatile("" : "+v"(r));
    return (seq0 + r) * ldk + hk * DH;
  };
  auto operands = [&](int64_t row) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.K) + row + 16 * bl.turned(ks) + 8 * lh);
      vf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.V) + row + 16 * ks + 8 * lh);
    }
  };
  operands(krow());
  // positions ascend along the block: the first and last of the wave's rows
  const int32_t tv = min(32, nvalid - row0);
  const int32_t tfirst = tv > 0 ? uniform(my) : kNoPos;
  const int32_t tlast = tv > 0 ? __builtin_amdgcn_readlane(my, tv - 1) : -1;
  wait_vm<0>();
  landed(kf, my >= 0);
  landed(vf, my >= 0);
  Ends now, then;
  auto start = [&] {
    __syncthreads();
    take(0);
    copy(0);
    take(1);
    ask(4);
    copy(1);
    take(2);
    now.take(ring(0));
    then.take(ring(1));
    now.settle();
    then.settle();
  };
  start();

  // dk is kept in units of the walked type's scale
  f32x16_t dk[NCH], dv[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) dk[c] = dv[c] = f32x16_t{};
  float unit = wx.scale;
  TileLane<DH> tl(lane);

  const std::true_type yes;
  const std::false_type no;
  auto body = [&](auto care, int st, int32_t step) {
    if (wave < 2) wait_vm<NC + 1>();
    else wait_vm<NC>();
    __syncthreads();
    ask(step + 5);
    copy((st + 2) % kStages);
    take(step + 3);
    Ends after;
    after.take(ring(step + 2));
    // positions ascend within a type: a step whose last row lies before the
    // wave's first key is of no use (kNoPos: the type ends in this step)
    if (now.last >= tfirst && tv > 0) {
      const char* Qt = tiles + st * 2 * TILE;
      tl.renew();
      if (wx.scale != unit) {
        const float f = unit * __builtin_amdgcn_rcpf(wx.scale);
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) dk[c][e] *= f;
        unit = wx.scale;
      }
      f32x16_t sc{}, dp;
#pragma unroll
      for (int a = 0; a < 4; ++a) {  // dP - delta: the sum starts from -delta
        const float4 de = *reinterpret_cast<const float4*>(&side_s[st][32 + 8 * a + 4 * lh]);
        dp[4 * a] = de.x, dp[4 * a + 1] = de.y, dp[4 * a + 2] = de.z, dp[4 * a + 3] = de.w;
      }
      const int j = wx.template block<DH, NB>(bl, m);
      tl.template add_rows<NB>(sc, Qt, kf, bl, j);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) dp = mfma(tl.row(Qt + TILE, ks), vf[ks], dp);
      if (now.first < tlast) {  // queries before a key
        const int32_t* qps = ring(step);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int4 qq = *reinterpret_cast<const int4*>(qps + 8 * a + 4 * lh);
          if (qq.x < my) sc[4 * a + 0] = -INFINITY;
          if (qq.y < my) sc[4 * a + 1] = -INFINITY;
          if (qq.z < my) sc[4 * a + 2] = -INFINITY;
          if (qq.w < my) sc[4 * a + 3] = -INFINITY;
        }
      }
      const float scale2 = wx.scale * kLog2e;
      float pe[16], ds[16];
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const float4 ls = *reinterpret_cast<const float4*>(&side_s[st][8 * a + 4 * lh]);
        const float l4[4] = {ls.x, ls.y, ls.z, ls.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pe[4 * a + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * a + e], scale2, l4[e]));
          ds[4 * a + e] = pe[4 * a + e] * dp[4 * a + e];
        }
      }
      if (care && now.first < tlast) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (sc[e] == -INFINITY) pe[e] = ds[e] = 0.f;
      }
      const uint4 pf[2] = {pack8(pe), pack8(pe + 8)}, sf[2] = {pack8(ds), pack8(ds + 8)};
      if (care) {
        tl.add_odd(dv, Qt + TILE, pf);
        tl.add_odd(dk, Qt, sf, bl.own * NB / 2);
      } else {
        tl.add_transposed(dv, Qt + TILE, pf);
        tl.template add_transposed_kept<NB>(dk, Qt, sf, bl, j);
      }
    }
    wx.next();
    now = then;
    after.settle();
    then = after;
  };

  for (int32_t n = 0; n < trips; n += 3) {
    body(no, 0, n);
    if (n + 1 == trips) break;
    body(no, 1, n + 1);
    if (n + 2 == trips) break;
    body(no, 2, n + 2);
  }
  wait_vm<0>();
  if (__syncthreads_or(odd(dk) || odd(dv))) {
    wx = wp = wc = Walk<NG>(&it_s, p.q, rep, g);
    for (int x = 0; x < 4; ++x) ask(x);
    operands(krow());  // (held for this they would cost the first walk registers)
    wait_vm<0>();
    landed(kf, my >= 0);
    landed(vf, my >= 0);
    start();
#pragma unroll
    for (int c = 0; c < NCH; ++c) dk[c] = dv[c] = f32x16_t{};
    unit = wx.scale;
#pragma unroll 1
    for (int32_t n = 0; n < trips; ++n) body(yes, n % kStages, n);
    wait_vm<0>();
  }
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[c][e] *= unit;
  if constexpr (NG == 2) {
    join_groups<NCH>(dk, rings, g, wave, lane);
    if (!join_groups<NCH>(dv, rings, g, wave, lane)) return;
  }
  if (my >= 0) {
    const int64_t row = krow();
    if (p.parts == 1) {
      store_row<DH>(p.dK, p.gdtype, row, dk, lh, bl.own * NB / 2);
      store_row<DH>(p.dV, p.gdtype, row, dv, lh);
    } else {
      store_row<DH>(p.part, 0, row + part * p.T * ldk, dk, lh, bl.own * NB / 2);
      store_row<DH>(p.part, 0, row + (p.parts + part) * p.T * ldk, dv, lh);
    }
  }
}

// The parts of dK (blockIdx.y 0) and dV added up, in order, for the rows that
// are tokens; four values a thread.
__global__ __launch_bounds__(kItemThreads) void attn_dkv_join_kernel(const AttnBwdParams p) {
  if (!pack_matches(p.pack, p.T, p.n_seq, p.q)) return;
  const int32_t width4 = p.n_kv * p.head_dim / 4;
  const int64_t all4 = static_cast<int64_t>(p.T) * width4, x = static_cast<int64_t>(blockIdx.x) * kItemThreads + threadIdx.x;
  if (x >= all4 || p.pack.mark[x / width4] != 1) return;
  const float4* from = reinterpret_cast<const float4*>(p.part) + blockIdx.y * p.parts * all4 + x;
  float4 s = from[0];
  for (int k = 1; k < p.parts; ++k) {
    const float4 v = from[k * all4];
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  void* out = blockIdx.y ? p.dV : p.dK;
  if (p.gdtype == 0) static_cast<float4*>(out)[x] = s;
  else static_cast<uint2*>(out)[x] = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
}

template <int DH, int NG, int NB>
hipError_t launch_dq(const AttnBwdParams& p, hipStream_t stream) {
  static std::atomic<unsigned long long> set{0};
  const auto fn = attn_dq_kernel<DH, NG, NB>;
  constexpr int smem = NG * ring_bytes<DH>();
  const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(fn), set, smem);
  if (e != hipSuccess) return e;
  const unsigned grid = static_cast<unsigned>(p.q_wgs + pack_clear_wgs(p.T));
  hipLaunchKernelGGL(fn, dim3(grid), dim3(NG * kItemThreads), smem, stream, p);
  return hipGetLastError();
}

template <int DH, int NG, int NB>
hipError_t launch_dkv(const AttnBwdParams& p, hipStream_t stream) {
  static std::atomic<unsigned long long> set{0};
  const auto fn = attn_dkv_kernel<DH, NG, NB>;
  constexpr int smem = NG * ring_bytes<DH>();
  const hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(fn), set, smem);
  if (e != hipSuccess) return e;
  const unsigned grid = static_cast<unsigned>(p.k_wgs + pack_clear_wgs(p.T));
  hipLaunchKernelGGL(fn, dim3(grid), dim3(NG * kItemThreads), smem, stream, p);
  return hipGetLastError();
}

hipError_t choose_dq(const AttnBwdParams& p, hipStream_t stream) {
  const int m = p.head_dim / p.q;
  switch (p.head_dim) {
    case 64:
      if (pack_few(p.q_wgs, p.cus)) return launch_dq<64, 2, 0>(p, stream);
      return blocks_fit<1>(p.law, p.q, m) ? launch_dq<64, 1, 1>(p, stream) : launch_dq<64, 1, 0>(p, stream);
    case 128:
      if (blocks_fit<2>(p.law, p.q, m)) return launch_dq<128, 1, 2>(p, stream);
      return blocks_fit<1>(p.law, p.q, m) ? launch_dq<128, 1, 1>(p, stream) : launch_dq<128, 1, 0>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

// Head width 128: two groups always (the registers hold two wavefronts a SIMD
// either way, and the longest walk is half as long), and all features (with
// blocks of 32, 32 heads on 8, 8192 positions, q = 4: 538 us for 519, some
// operands no longer fit the registers).
hipError_t choose_dkv(const AttnBwdParams& p, hipStream_t stream) {
  switch (p.head_dim) {
    case 64:
      if (pack_few(p.k_wgs, p.cus)) return launch_dkv<64, 2, 0>(p, stream);
      return blocks_fit<1>(p.law, p.q, 64 / p.q) ? launch_dkv<64, 1, 1>(p, stream) : launch_dkv<64, 1, 0>(p, stream);
    case 128: return launch_dkv<128, 2, 0>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_attn_packed_bwd(const AttnBwdParams& p, hipStream_t stream) {
  hipError_t e = choose_dq(p, stream);
  if (e == hipSuccess) e = choose_dkv(p, stream);
  if (e != hipSuccess || p.parts == 1) return e;
  const int64_t threads = static_cast<int64_t>(p.T) * p.n_kv * p.head_dim / 4;
  const unsigned grid = static_cast<unsigned>((threads + kItemThreads - 1) / kItemThreads);
  hipLaunchKernelGGL(attn_dkv_join_kernel, dim3(grid, 2), dim3(kItemThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace starq
