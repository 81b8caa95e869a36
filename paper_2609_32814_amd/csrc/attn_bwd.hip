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
// dK^T += Q^T dS.
//
// P and dS enter their products rounded to bf16 (at most 2^-9 of each term,
// like the operands themselves); everything else is fp32.
#include "attn_common.hpp"

namespace starq {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kStep = 64;  // rows walked per step
constexpr int32_t kNoPos = 0x7fffffff;

// Chunk c (16 bytes) of row r of a tile sits at chunk c ^ swz(r).  Two kinds of
// reads cover all 64 banks: one chunk of 16 rows in 16 lanes (the row operands)
// and 4 chunks of 4 rows in 32 lanes (the transposing reads).
template <int DH>
__device__ __forceinline__ int swz(int r) {
  return DH == 64 ? 4 * ((r >> 1) & 1) + ((r >> 2) & 3) : 4 * (r & 3) + ((r >> 2) & 3);
}

template <int DH>
constexpr int tile_bytes() { return kStep * DH * 2; }
template <int DH>
constexpr int smem_bytes() { return 2 * 2 * tile_bytes<DH>(); }  // two stages of two tiles

__device__ __forceinline__ f32x16_t mfma(uint4 a, uint4 b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Per walked type: what its pairs with the block's type select and their scale.
struct TypeTab {
  uint32_t rot;    // selected 8-feature cells, the block's own group first
  uint32_t cells;  // the same in the order of the features
  float scale;
};

// The walk of a work item: per type a range of the pack's permutation, in
// steps of 64 rows; `heads` times over.
struct Walk {
  const int32_t* off;    // LDS: first perm index per type
  const int32_t* cnt;    // LDS: rows per type
  const int32_t* perm;
  int q, heads;
  int hh, j;
  int32_t c;
  __device__ __forceinline__ int32_t rows(int t) const { return __builtin_amdgcn_readfirstlane(cnt[t]); }
  __device__ __forceinline__ void settle() {
    while (hh < heads && c * kStep >= rows(j)) {
      c = 0;
      if (++j == q) {
        j = 0;
        ++hh;
      }
    }
  }
  __device__ __forceinline__ void next() {
    ++c;
    settle();
  }
  __device__ __forceinline__ bool done() const { return hh >= heads; }
  // position of row `lane` of the step, or kNoPos
  __device__ __forceinline__ int32_t pos(int lane) const {
    if (done()) return kNoPos;
    const int32_t r = c * kStep + lane;
    return r < rows(j) ? perm[__builtin_amdgcn_readfirstlane(off[j]) + r] : kNoPos;
  }
};

// Copies the rows of one step (lane `row` of kp holds the position of row
// `row`) of two [T][heads][DH] arrays into a stage.
template <int DH>
__device__ __forceinline__ void copy_rows(const uint16_t* A, const uint16_t* B, uint32_t stride16, int32_t kp, char* stage,
                                          int wave, int lane) {
  constexpr int CPR = DH / 8, RPC = 64 / CPR;
#pragma unroll
  for (int k = 0; k < kStep / RPC / kWaves; ++k) {
    const int cp = wave + kWaves * k;
    const int row = cp * RPC + lane / CPR, c = lane % CPR;
    const int32_t pos = __shfl(kp, row);
    const bool ok = pos != kNoPos;
    const uint64_t at = (static_cast<uint64_t>(static_cast<uint32_t>(pos)) * stride16) << 4;
    const int f = 8 * (c ^ swz<DH>(row));
    dma16(ok ? reinterpret_cast<const char*>(A + f) + at : reinterpret_cast<const char*>(g_attn_zero), lds_addr(stage + cp * 1024));
    dma16(ok ? reinterpret_cast<const char*>(B + f) + at : reinterpret_cast<const char*>(g_attn_zero),
          lds_addr(stage + tile_bytes<DH>() + cp * 1024));
  }
}

// The transposed operand of 16 rows from 16 kk on: lane l gets feature
// 32 c + l % 32 of rows 16 kk + 4 (l / 32) + 0..3 and of the 4 rows 8 behind.
template <int DH>
__device__ __forceinline__ uint4 read_transposed(const char* tile, int kk, int c, int lane) {
  const int g = lane >> 4, rr = (lane & 15) >> 2, qq = lane & 3;
  const int row = 16 * kk + 4 * (g >> 1) + rr;
  const int f = 32 * c + 16 * (g & 1) + 4 * qq;
  const int sub = ((f >> 2) & 1) * 8;
  const char* a0 = tile + row * DH * 2 + (((f >> 3) ^ swz<DH>(row)) << 4) + sub;
  const char* a1 = tile + (row + 8) * DH * 2 + (((f >> 3) ^ swz<DH>(row + 8)) << 4) + sub;
  const uint2 w0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((STARQ_LDS v4i16_t*)(a0)));
  const uint2 w1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((STARQ_LDS v4i16_t*)(a1)));
  return make_uint4(w0.x, w0.y, w1.x, w1.y);
}

// Rows of a transposed product's result: acc[c][4 a + e] is feature
// 32 c + 8 a + 4 (l / 32) + e of the lane's row.
template <int DH>
__device__ __forceinline__ void store_row(void* out, int dtype, int64_t at, const f32x16_t* acc, int lh) {
#pragma unroll
  for (int c = 0; c < DH / 32; ++c)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int f = 32 * c + 8 * a + 4 * lh;
      const float v0 = acc[c][4 * a], v1 = acc[c][4 * a + 1], v2 = acc[c][4 * a + 2], v3 = acc[c][4 * a + 3];
      if (dtype == 0)
        *reinterpret_cast<float4*>(static_cast<float*>(out) + at + f) = make_float4(v0, v1, v2, v3);
      else
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at + f) = make_uint2(pack_bf16(v0, v1), pack_bf16(v2, v3));
    }
}

// acc += (rows of `tile`)^T x ops over the features that `cells` selects.
template <int DH, bool ALL>
__device__ __forceinline__ void add_transposed(f32x16_t* acc, const char* tile, const uint4* ops, uint32_t cells, int lane) {
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) {
    if (!ALL && !((cells >> (4 * c)) & 15u)) continue;
    const bool mine = ALL || ((cells >> (4 * c + ((lane & 31) >> 3))) & 1u);
#pragma unroll
    for (int kk = 0; kk < kStep / 16; ++kk) {
      uint4 a = read_transposed<DH>(tile, kk, c, lane);
      if (!mine) a = make_uint4(0, 0, 0, 0);
      acc[c] = mfma(a, ops[kk], acc[c]);
    }
  }
}

// What both kernels set up from their record.
struct ItemLds {
  int32_t pos[kAttnBlockRows];
  int32_t off[kAttnMaxQ], cnt[kAttnMaxQ];
  TypeTab tab[kAttnMaxQ];
};

__device__ __forceinline__ void setup_item(ItemLds& s, const AttnBwdParams& p, const int32_t* rec, int own) {
  const int q = p.q, m = p.head_dim / q, cpg = m / 8;
  const int32_t b0 = rec[2], n = rec[3] >> 16;
  if (threadIdx.x < kAttnBlockRows) s.pos[threadIdx.x] = static_cast<int32_t>(threadIdx.x) < n ? p.pack.perm[b0 + threadIdx.x] : -1;
  if (threadIdx.x < static_cast<unsigned>(q)) {
    const int j = threadIdx.x;
    s.off[j] = rec[4 + j];
    s.cnt[j] = rec[4 + q + j];
    const uint32_t fm = attn_fmask(p.law, q, own, j);  // symmetric in the two types
    TypeTab t{0, 0, __builtin_amdgcn_rsqf(static_cast<float>(__popc(fm) * m))};
    for (int a = 0; a < q; ++a) {
      if ((fm >> a) & 1u) t.cells |= ((1u << cpg) - 1u) << (a * cpg);
      if ((fm >> ((a + own) % q)) & 1u) t.rot |= ((1u << cpg) - 1u) << (a * cpg);
    }
    s.tab[j] = t;
  }
}

template <int DH, bool M8>
__global__ __launch_bounds__(kThreads) void attn_dq_kernel(const AttnBwdParams p) {
  constexpr int NCH = DH / 32, KS = DH / 16, ROWB = DH * 2, TILE = tile_bytes<DH>();
  constexpr uint32_t kAll = DH == 64 ? 0xffu : 0xffffu;
  extern __shared__ __attribute__((aligned(16))) char tiles[];  // [stage][K, V]
  __shared__ ItemLds it_s;
  __shared__ int32_t kpos_s[2][kStep];

  if (!pack_matches(p.pack, p.T, p.n_seq, p.q)) return;
  if (blockIdx.x >= static_cast<unsigned>(p.q_wgs)) {
    pack_clear_rows(p.pack, p.T, blockIdx.x - p.q_wgs, p.clear_rest, p.dQ, p.gdtype, p.n_heads * DH);
    return;
  }
  int h;
  int32_t k;
  if (!pack_item(p.pack, p.n_heads, h, k)) return;
  const int q = p.q, m = DH / q;
  const int32_t* rec = p.pack.recs_q + static_cast<int64_t>(k) * pack_rec_ints(q);
  const int64_t seq0 = rec[0];
  const int own = rec[3] & 0xffff;
  const int32_t nvalid = rec[3] >> 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int hk = h / (p.n_heads / p.n_kv);
  const int64_t ldq = static_cast<int64_t>(p.n_heads) * DH, ldk = static_cast<int64_t>(p.n_kv) * DH;
  const uint16_t* Kg = static_cast<const uint16_t*>(p.K) + seq0 * ldk + hk * DH;
  const uint16_t* Vg = static_cast<const uint16_t*>(p.V) + seq0 * ldk + hk * DH;
  const uint32_t ldk16 = static_cast<uint32_t>(ldk >> 3);
  setup_item(it_s, p, rec, own);
  __syncthreads();

  const int row0 = wave * 32;
  const int32_t tv = min(32, nvalid - row0);
  const int32_t tfirst = tv > 0 ? __builtin_amdgcn_readfirstlane(it_s.pos[row0]) : kNoPos;
  const int32_t tlast = tv > 0 ? __builtin_amdgcn_readfirstlane(it_s.pos[row0 + tv - 1]) : -1;
  const int32_t my = it_s.pos[row0 + lr];

  Walk cur{it_s.off, it_s.cnt, p.pack.perm, q, 1, 0, 0, 0};
  cur.settle();
  Walk nxt = cur;
  nxt.next();
  int32_t kp = cur.pos(lane), kp_nxt = nxt.pos(lane);
  copy_rows<DH>(Kg, Vg, ldk16, kp, tiles, wave, lane);
  if (wave == 0) kpos_s[0][lane] = kp;

  // the wave's rows of Q (own group first) and dO as operands, delta and lse
  uint4 qf[KS], df[KS];
  int koff[KS], voff[KS];
  float delta = 0.f, lse2 = 0.f;
  const int64_t qrow = (seq0 + max(my, 0)) * ldq + h * DH;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int fr = 16 * ks + 8 * lh;
    const int fphys = ((fr / m + own) % q) * m + fr % m;
    koff[ks] = lr * ROWB + (((fphys >> 3) ^ swz<DH>(lr)) << 4);
    voff[ks] = lr * ROWB + (((fr >> 3) ^ swz<DH>(lr)) << 4);
    qf[ks] = df[ks] = make_uint4(0, 0, 0, 0);
    if (my >= 0) {
      qf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Q) + qrow + fphys);
      df[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.dO) + qrow + fr);
      const uint32_t w[4] = {df[ks].x, df[ks].y, df[ks].z, df[ks].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        delta += bf16_to_f32(w[e] & 0xffffu) * load_in(p.O, p.odtype, qrow + fr + 2 * e) +
                 bf16_to_f32(w[e] >> 16) * load_in(p.O, p.odtype, qrow + fr + 2 * e + 1);
    }
  }
  delta = sum_xor32(delta);
  if (my >= 0) {
    const int64_t at = static_cast<int64_t>(h) * p.T + seq0 + my;
    lse2 = p.lse[at] * kLog2e;
    if (lh == 0) p.delta[at] = delta;
  }

  f32x16_t acc[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) acc[c] = f32x16_t{};

  for (int stage = 0; !cur.done(); stage ^= 1) {
    wait_vm_all();
    __syncthreads();
    Walk nn = nxt;
    if (!nxt.done()) {
      nn.next();
      if (wave == 0) kpos_s[stage ^ 1][lane] = kp_nxt;
      copy_rows<DH>(Kg, Vg, ldk16, kp_nxt, tiles + (stage ^ 1) * 2 * TILE, wave, lane);
      kp_nxt = nn.pos(lane);
    }
    const char* Kt = tiles + stage * 2 * TILE;
    const char* Vt = Kt + TILE;
    const int32_t* kps = kpos_s[stage];
    const uint32_t rot = __builtin_amdgcn_readfirstlane(it_s.tab[cur.j].rot);
    const uint32_t cells = __builtin_amdgcn_readfirstlane(it_s.tab[cur.j].cells);
    const float scale = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(it_s.tab[cur.j].scale)));
    const float scale2 = scale * kLog2e;
    const int32_t kf0 = __builtin_amdgcn_readfirstlane(kps[0]);
    const int32_t kl[2] = {__builtin_amdgcn_readfirstlane(kps[31]), __builtin_amdgcn_readfirstlane(kps[63])};
    if (kf0 <= tlast) {
      uint4 pf[4];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x16_t sc{}, dp{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          if (ks > 0 && !((rot >> (2 * ks)) & 3u)) continue;
          uint4 kf = *reinterpret_cast<const uint4*>(Kt + 32 * t * ROWB + koff[ks]);
          if constexpr (M8) {
            if (!((rot >> (2 * ks + lh)) & 1u)) kf = make_uint4(0, 0, 0, 0);
          }
          sc = mfma(kf, qf[ks], sc);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mfma(*reinterpret_cast<const uint4*>(Vt + 32 * t * ROWB + voff[ks]), df[ks], dp);
        // keys behind a query (rows past a type's end have position kNoPos)
        if (kl[t] > tfirst) {
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int4 kq = *reinterpret_cast<const int4*>(kps + 32 * t + 8 * a + 4 * lh);
            if (kq.x > my) sc[4 * a + 0] = -INFINITY, dp[4 * a + 0] = 0.f;
            if (kq.y > my) sc[4 * a + 1] = -INFINITY, dp[4 * a + 1] = 0.f;
            if (kq.z > my) sc[4 * a + 2] = -INFINITY, dp[4 * a + 2] = 0.f;
            if (kq.w > my) sc[4 * a + 3] = -INFINITY, dp[4 * a + 3] = 0.f;
          }
        }
        float ds[16];
#pragma unroll
        for (int e = 0; e < 16; ++e)
          ds[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale2, -lse2)) * ((dp[e] - delta) * scale);
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2)
          pf[2 * t + k2] = make_uint4(pack_bf16(ds[8 * k2 + 0], ds[8 * k2 + 1]), pack_bf16(ds[8 * k2 + 2], ds[8 * k2 + 3]),
                                      pack_bf16(ds[8 * k2 + 4], ds[8 * k2 + 5]), pack_bf16(ds[8 * k2 + 6], ds[8 * k2 + 7]));
      }
      if (cells == kAll) add_transposed<DH, true>(acc, Kt, pf, cells, lane);
      else add_transposed<DH, false>(acc, Kt, pf, cells, lane);
    }
    cur = nxt;
    nxt = nn;
  }
  if (my >= 0) store_row<DH>(p.dQ, p.gdtype, (seq0 + my) * ldq + h * DH, acc, lh);
}

template <int DH, bool M8>
__global__ __launch_bounds__(kThreads) void attn_dkv_kernel(const AttnBwdParams p) {
  constexpr int NCH = DH / 32, KS = DH / 16, ROWB = DH * 2, TILE = tile_bytes<DH>();
  constexpr uint32_t kAll = DH == 64 ? 0xffu : 0xffffu;
  extern __shared__ __attribute__((aligned(16))) char tiles[];  // [stage][Q, dO]
  __shared__ ItemLds it_s;
  __shared__ int32_t qpos_s[2][kStep];
  __shared__ float side_s[2][2][kStep];  // [stage][lse (base 2), delta]

  if (!pack_matches(p.pack, p.T, p.n_seq, p.q)) return;
  if (blockIdx.x >= static_cast<unsigned>(p.k_wgs)) {
    pack_clear_rows(p.pack, p.T, blockIdx.x - p.k_wgs, p.clear_rest, p.dK, p.gdtype, p.n_kv * DH);
    pack_clear_rows(p.pack, p.T, blockIdx.x - p.k_wgs, p.clear_rest, p.dV, p.gdtype, p.n_kv * DH);
    return;
  }
  int hk;
  int32_t k;
  if (!pack_item(p.pack, p.n_kv, hk, k)) return;
  const int q = p.q, m = DH / q, rep = p.n_heads / p.n_kv;
  const int32_t* rec = p.pack.recs_k + static_cast<int64_t>(k) * pack_rec_ints(q);
  const int64_t seq0 = rec[0];
  const int own = rec[3] & 0xffff;
  const int32_t nvalid = rec[3] >> 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int64_t ldq = static_cast<int64_t>(p.n_heads) * DH, ldk = static_cast<int64_t>(p.n_kv) * DH;
  const uint16_t* Qg = static_cast<const uint16_t*>(p.Q) + seq0 * ldq + hk * rep * DH;
  const uint16_t* Dg = static_cast<const uint16_t*>(p.dO) + seq0 * ldq + hk * rep * DH;
  const uint32_t ldq16 = static_cast<uint32_t>(ldq >> 3);
  setup_item(it_s, p, rec, own);
  __syncthreads();

  const int row0 = wave * 32;
  const int32_t tv = min(32, nvalid - row0);
  const int32_t tfirst = tv > 0 ? __builtin_amdgcn_readfirstlane(it_s.pos[row0]) : kNoPos;
  const int32_t tlast = tv > 0 ? __builtin_amdgcn_readfirstlane(it_s.pos[row0 + tv - 1]) : -1;
  const int32_t my = it_s.pos[row0 + lr];

  Walk cur{it_s.off, it_s.cnt, p.pack.perm, q, rep, 0, 0, 0};
  cur.settle();
  Walk nxt = cur;
  nxt.next();
  int32_t qp = cur.pos(lane), qp_nxt = nxt.pos(lane);
  // wave 0 brings the rows' log-sum-exps, wave 1 their deltas; a row past the
  // type's end gets +inf, so that its probabilities are zero
  auto load_side = [&](const Walk& w, int32_t pos) -> float {
    if (pos == kNoPos) return wave == 0 ? INFINITY : 0.f;
    const int64_t at = static_cast<int64_t>(hk * rep + w.hh) * p.T + seq0 + pos;
    return wave == 0 ? p.lse[at] * kLog2e : p.delta[at];
  };
  float side = 0.f;
  copy_rows<DH>(Qg, Dg, ldq16, qp, tiles, wave, lane);
  if (wave == 0) qpos_s[0][lane] = qp;
  if (wave < 2) side = load_side(cur, qp);

  uint4 kf[KS], vf[KS];
  int qoff[KS], doff[KS];
  const int64_t krow = (seq0 + max(my, 0)) * ldk + hk * DH;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int fr = 16 * ks + 8 * lh;
    const int fphys = ((fr / m + own) % q) * m + fr % m;
    qoff[ks] = lr * ROWB + (((fphys >> 3) ^ swz<DH>(lr)) << 4);
    doff[ks] = lr * ROWB + (((fr >> 3) ^ swz<DH>(lr)) << 4);
    kf[ks] = vf[ks] = make_uint4(0, 0, 0, 0);
    if (my >= 0) {
      kf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.K) + krow + fphys);
      vf[ks] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.V) + krow + fr);
    }
  }

  f32x16_t dk[NCH], dv[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) dk[c] = dv[c] = f32x16_t{};

  for (int stage = 0; !cur.done(); stage ^= 1) {
    wait_vm_all();
    if (wave < 2) side_s[stage][wave][lane] = side;
    __syncthreads();
    Walk nn = nxt;
    if (!nxt.done()) {
      nn.next();
      if (wave == 0) qpos_s[stage ^ 1][lane] = qp_nxt;
      copy_rows<DH>(Qg + nxt.hh * DH, Dg + nxt.hh * DH, ldq16, qp_nxt, tiles + (stage ^ 1) * 2 * TILE, wave, lane);
      if (wave < 2) side = load_side(nxt, qp_nxt);
      qp_nxt = nn.pos(lane);
    }
    const char* Qt = tiles + stage * 2 * TILE;
    const char* Dt = Qt + TILE;
    const int32_t* qps = qpos_s[stage];
    const uint32_t rot = __builtin_amdgcn_readfirstlane(it_s.tab[cur.j].rot);
    const uint32_t cells = __builtin_amdgcn_readfirstlane(it_s.tab[cur.j].cells);
    const float scale = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(it_s.tab[cur.j].scale)));
    const float scale2 = scale * kLog2e;
    const int32_t ql = __builtin_amdgcn_readfirstlane(qps[63]);
    const int32_t qf0[2] = {__builtin_amdgcn_readfirstlane(qps[0]), __builtin_amdgcn_readfirstlane(qps[32])};
    if (ql >= tfirst && tv > 0) {
      uint4 pf[4], sf[4];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x16_t sc{}, dp{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          if (ks > 0 && !((rot >> (2 * ks)) & 3u)) continue;
          uint4 a = *reinterpret_cast<const uint4*>(Qt + 32 * t * ROWB + qoff[ks]);
          if constexpr (M8) {
            if (!((rot >> (2 * ks + lh)) & 1u)) a = make_uint4(0, 0, 0, 0);
          }
          sc = mfma(a, kf[ks], sc);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mfma(*reinterpret_cast<const uint4*>(Dt + 32 * t * ROWB + doff[ks]), vf[ks], dp);
        // queries before a key
        if (qf0[t] < tlast) {
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int4 qq = *reinterpret_cast<const int4*>(qps + 32 * t + 8 * a + 4 * lh);
            if (qq.x < my) sc[4 * a + 0] = -INFINITY;
            if (qq.y < my) sc[4 * a + 1] = -INFINITY;
            if (qq.z < my) sc[4 * a + 2] = -INFINITY;
            if (qq.w < my) sc[4 * a + 3] = -INFINITY;
          }
        }
        float pe[16], ds[16];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const float4 ls = *reinterpret_cast<const float4*>(&side_s[stage][0][32 * t + 8 * a + 4 * lh]);
          const float4 de = *reinterpret_cast<const float4*>(&side_s[stage][1][32 * t + 8 * a + 4 * lh]);
          const float l4[4] = {ls.x, ls.y, ls.z, ls.w}, d4[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pe[4 * a + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * a + e], scale2, -l4[e]));
            ds[4 * a + e] = pe[4 * a + e] * ((dp[4 * a + e] - d4[e]) * scale);
          }
        }
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          const int o = 8 * k2;
          pf[2 * t + k2] = make_uint4(pack_bf16(pe[o + 0], pe[o + 1]), pack_bf16(pe[o + 2], pe[o + 3]),
                                      pack_bf16(pe[o + 4], pe[o + 5]), pack_bf16(pe[o + 6], pe[o + 7]));
          sf[2 * t + k2] = make_uint4(pack_bf16(ds[o + 0], ds[o + 1]), pack_bf16(ds[o + 2], ds[o + 3]),
                                      pack_bf16(ds[o + 4], ds[o + 5]), pack_bf16(ds[o + 6], ds[o + 7]));
        }
      }
      add_transposed<DH, true>(dv, Dt, pf, kAll, lane);
      if (cells == kAll) add_transposed<DH, true>(dk, Qt, sf, cells, lane);
      else add_transposed<DH, false>(dk, Qt, sf, cells, lane);
    }
    cur = nxt;
    nxt = nn;
  }
  if (my >= 0) {
    store_row<DH>(p.dK, p.gdtype, krow, dk, lh);
    store_row<DH>(p.dV, p.gdtype, krow, dv, lh);
  }
}

template <int DH, bool M8>
hipError_t launch_dh(const AttnBwdParams& p, hipStream_t stream) {
  static std::atomic<unsigned long long> set_q{0}, set_k{0};
  constexpr int smem = smem_bytes<DH>();
  hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(attn_dq_kernel<DH, M8>), set_q, smem);
  if (e != hipSuccess) return e;
  e = ensure_lds_limit(reinterpret_cast<const void*>(attn_dkv_kernel<DH, M8>), set_k, smem);
  if (e != hipSuccess) return e;
  const unsigned clear = static_cast<unsigned>(pack_clear_wgs(p.T));
  hipLaunchKernelGGL((attn_dq_kernel<DH, M8>), dim3(p.q_wgs + clear), dim3(kThreads), smem, stream, p);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attn_dkv_kernel<DH, M8>), dim3(p.k_wgs + clear), dim3(kThreads), smem, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_packed_bwd(const AttnBwdParams& p, hipStream_t stream) {
  const bool m8 = p.head_dim / p.q == 8;
  switch (p.head_dim) {
    case 64: return m8 ? launch_dh<64, true>(p, stream) : launch_dh<64, false>(p, stream);
    case 128: return m8 ? launch_dh<128, true>(p, stream) : launch_dh<128, false>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace starq
