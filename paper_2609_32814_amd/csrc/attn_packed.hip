// Causal attention over a pack of sequences, forward (Alg. attention-training,
// the score and aggregation steps, per sequence).
//
// A workgroup owns 128 queries of one type of one sequence, 32 per wavefront,
// and walks the keys of every type up to its last query in steps of 32 (see
// attn_walk.hpp; the key rows come with zeros in the place of the features
// that F(i, j) leaves out).  Per step:
//   S^T = K Q^T, the key rows from LDS, the wave's queries in registers: a
//       lane ends with 16 keys of one query;
//   the causal mask where a key may lie behind a query, the running maximum
//       and sum (fp32, base 2; a lane shares its query with lane l ^ 32);
//   O^T += V^T P^T: P^T rounded to bf16 as it lies in the registers (the
//       products take no wider operand; 2^-8 of each term), V^T by transposing
//       reads.
// NG groups of wavefronts share the steps of one walk where there are few
// work items; their states meet at the end.
//
// 32 queries a wavefront let every row read from LDS serve 32 queries and leave
// room for 4 wavefronts a SIMD at width 64 (3 at 128), which hide each other's
// exponentials behind products; with steps of 64 keys there are 3, and nothing
// is won (269 us for 266, 24576 tokens, 12 heads of 64, q = 4).
// Measured: one sequence of 8192, all features, 64 heads of 64 in 641 us (858
// TFLOP/s), 32 of 128 in 560 (982); the exponentials, conversions and sums of
// 16 scores a lane bound the first (105 vector instructions a step, the VALU
// busy 71 % of the time), the products the second.  24576 tokens in 17
// sequences, 12 heads of 64, star law, q = 4: 223 us in a long run, 250 to 274 in
// short ones, by the same vector work beside fewer products (VALU busy 64 % of
// the time, MFMA 22 %).  211 tokens in 3 sequences: 10 us, a launch and a
// chain of dependent reads (plan, record, positions, rows), not bytes.
#include <cfloat>
#include <type_traits>

#include "attn_common.hpp"
#include "attn_walk.hpp"

namespace starq {

namespace {

template <int DH, int NG, int NB>
__global__ __launch_bounds__(NG * kItemThreads, NG == 2 ? 2 : DH == 64 ? 4 : 3) void attn_packed_fwd_kernel(const AttnParams p) {
  constexpr int NCH = DH / 32, KS = DH / 16, TILE = tile_bytes<DH>(), NC = 2 * copies_per_step<DH>();
  extern __shared__ __attribute__((aligned(16))) char rings[];  // [group][stage][K, V]
  __shared__ ItemLds<NG> it_s;
  __shared__ float state_s[kItemWaves][64][2];

  if (!pack_matches(p.pack, p.S, p.B, p.q)) return;
  if (blockIdx.x >= static_cast<unsigned>(p.main_wgs)) {
    pack_clear_rows(p.pack, p.S, blockIdx.x - p.main_wgs, p.clear_rest, p.O, p.odtype, p.n_heads * DH, p.lse, p.n_heads);
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
  const int m = DH / p.q;
  const Blocks<DH, NB> bl(rec[3] & 0xffff, m);
  uint4 qf[KS];
  const int64_t qrow = (seq0 + max(my, 0)) * ldq + h * DH;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Q) + qrow + 16 * bl.turned(ks) + 8 * lh);
  // positions ascend along the block: the first and last of the wave's rows
  const int32_t tv = min(32, nvalid - row0);
  const int32_t tfirst = tv > 0 ? uniform(my) : kNoPos;
  const int32_t tlast = tv > 0 ? __builtin_amdgcn_readlane(my, tv - 1) : -1;
  wait_vm<0>();
  landed(qf, my >= 0);
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

  f32x16_t acc[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) acc[c] = f32x16_t{};
  // base 2; the maximum starts below every score, and finite (-inf - -inf is
  // no number); the sum is over this lane's keys
  float run_max = -FLT_MAX, run_sum = 0.f;
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
      if (DH == 128) tl.renew();  // (at 64 there is room for the addresses)
      f32x16_t sc{};
      tl.template add_rows<NB>(sc, Kt, qf, bl, wx.template block<DH, NB>(bl, m));
      // keys behind a query (rows past a type's end have position kNoPos)
      if (now.last > tfirst) {
        const int32_t* kps = ring(step);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int4 kq = *reinterpret_cast<const int4*>(kps + 8 * a + 4 * lh);
          if (kq.x > my) sc[4 * a + 0] = -INFINITY;
          if (kq.y > my) sc[4 * a + 1] = -INFINITY;
          if (kq.z > my) sc[4 * a + 2] = -INFINITY;
          if (kq.w > my) sc[4 * a + 3] = -INFINITY;
        }
      }
      float top = sc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, sc[e]);
      // the running maximum moves only by more than 8 at a time: until then
      // probabilities stay below 2^8
      const float scale2 = wx.scale * kLog2e;
      if (__ballot(__builtin_fmaf(top, scale2, -8.f) > run_max) != 0) {
        top = max_xor32(top) * scale2;  // (both lanes of a query move alike)
        const bool need = top > run_max + 8.f;
        const float corr = need ? __builtin_amdgcn_exp2f(run_max - top) : 1.f;
        if (need) run_max = top;
        run_sum *= corr;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[c][e] *= corr;
      }
      float pe[16], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        pe[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale2, -run_max));
        sum += pe[e];
      }
      run_sum += sum;
      const uint4 pf[2] = {pack8(pe), pack8(pe + 8)};
      if (care) tl.add_odd(acc, Kt + TILE, pf);
      else tl.add_transposed(acc, Kt + TILE, pf);
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
    run_max = -FLT_MAX, run_sum = 0.f;
#pragma unroll 1
    for (int32_t n = 0; n < trips; ++n) body(yes, n % kStages, n);
    wait_vm<0>();
  }
  run_sum = sum_xor32(run_sum);
  if constexpr (NG == 2) {  // both groups in units of the larger maximum
    if (g == 1) {
      state_s[wave][lane][0] = run_max;
      state_s[wave][lane][1] = run_sum;
    }
    __syncthreads();
    const float m1 = state_s[wave][lane][0], l1 = state_s[wave][lane][1];
    __syncthreads();
    if (g == 0) state_s[wave][lane][0] = run_max;
    __syncthreads();
    const float mx = fmaxf(state_s[wave][lane][0], m1);
    const float corr = __builtin_amdgcn_exp2f(run_max - mx);
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] *= corr;
    run_sum = run_sum * corr + l1 * __builtin_amdgcn_exp2f(m1 - mx);  // (of use in the first group)
    run_max = mx;
    if (!join_groups<NCH>(acc, rings, g, wave, lane)) return;
  }
  if (my >= 0) {
    const float inv = 1.f / run_sum;  // (a query is its own key: no sum is empty)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] *= inv;
    store_row<DH>(p.O, p.odtype, qrow, acc, lh);
    if (p.lse && lh == 0)
      p.lse[static_cast<int64_t>(h) * p.S + seq0 + my] = (run_max + __log2f(run_sum)) * 0.6931471805599453f;
  }
}

template <int DH, int NG, int NB>
hipError_t launch(const AttnParams& p, hipStream_t stream) {
  static std::atomic<unsigned long long> set{0};
  const auto fn = attn_packed_fwd_kernel<DH, NG, NB>;
  constexpr int smem = NG * ring_bytes<DH>();
  hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(fn), set, smem);
  if (e != hipSuccess) return e;
  const unsigned grid = static_cast<unsigned>(p.main_wgs + pack_clear_wgs(p.S));
  hipLaunchKernelGGL(fn, dim3(grid), dim3(NG * kItemThreads), smem, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_packed_fwd(const AttnParams& p, hipStream_t stream) {
  const int m = p.head_dim / p.q;
  switch (p.head_dim) {
    case 64:
      if (pack_few(p.main_wgs, p.cus)) return launch<64, 2, 0>(p, stream);
      return blocks_fit<1>(p.law, p.q, m) ? launch<64, 1, 1>(p, stream) : launch<64, 1, 0>(p, stream);
    case 128:
      if (blocks_fit<2>(p.law, p.q, m)) return launch<128, 1, 2>(p, stream);
      return blocks_fit<1>(p.law, p.q, m) ? launch<128, 1, 1>(p, stream) : launch<128, 1, 0>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace starq
