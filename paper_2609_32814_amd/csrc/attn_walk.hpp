// The walk of a pack's work item (see PackView in kernels.hpp): rows of two
// [T][heads][DH] arrays, type by type, 32 rows a step, brought into a ring
// of three LDS tiles of either array by direct copies two steps ahead of their
// use.
//
// A group of four wavefronts goes through step h like this (the kernels' loop
// body h):
//   wait until the copies of step h have landed, barrier;
//   ask for the positions of step h + 5 (wavefront 0), copy the rows of
//   step h + 2, whose positions each lane took from the ring a body ago;
//   take those of step h + 3 (asked for two bodies ago) and the first and
//   last position of step h + 2;
//   compute with the tile of step h.
// The barrier of body h says that every wavefront is through with body h - 1,
// whose tile (h - 1) mod 3 = (h + 2) mod 3 the new copies overwrite.  The
// copies into LDS are counted by hand: a body leaves what the body before it
// asked for in flight at its wait.  Other loads in between are safe, since a
// wait for the same count then waits for more, but the compiler, which does
// not see the copies, waits behind its own until nothing is in flight.  It has
// some where the registers do not hold all: in the first walk, dQ at width 64
// with feature blocks brings a quarter of Q's operands back from scratch in
// steps whose type lies in the second block from the own one (8 registers), and
// dK/dV does so in masked steps (with one group at width 64, and at 128).
#pragma once

#include "attn_common.hpp"

namespace starq {

namespace {

constexpr int kStep = 32;
constexpr int kStages = 3;    // tiles of either array
constexpr int kPosSlots = 8;  // steps whose positions are held
constexpr int32_t kNoPos = 0x7fffffff;
constexpr int kItemWaves = 4;  // per group
constexpr int kItemThreads = 64 * kItemWaves;

__device__ __attribute__((aligned(256))) int32_t g_attn_no_pos[64] = {
    kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos,
    kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos, kNoPos};

__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// Chunk c (16 bytes) of row r of a tile sits at chunk c ^ swz(r).  Two kinds of
// reads cover all 64 banks: one chunk of 16 rows in 16 lanes (row operands)
// and 4 chunks of 4 rows in 32 lanes (transposing reads).
template <int DH>
__device__ __forceinline__ int swz(int r) {
  return DH == 64 ? 4 * ((r >> 1) & 1) + ((r >> 2) & 3) : 4 * (r & 3) + ((r >> 2) & 3);
}
template <int DH>
constexpr int tile_bytes() { return kStep * DH * 2; }
template <int DH>
constexpr int ring_bytes() { return kStages * 2 * tile_bytes<DH>(); }

__device__ __forceinline__ f32x16_t mfma(uint4 a, uint4 b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint4 pack8(const float* v) {
  return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// Of a pair of types the star law keeps two groups.  NB > 0: features in blocks
// of 16 NB, each holding whole groups or lying in one, so that a pair keeps at
// most two blocks, the item's own and the walked type's, and the products can
// leave the others out; blocks are counted from the item's own one on (the
// walked block is picked by uniform branches around its products, its rows
// by their address).  NB = 0: all features, zeros where a pair keeps none.
template <int DH, int NB>
struct Blocks {
  static constexpr int KS = DH / 16, N = NB > 0 ? KS / NB : 1;
  int own;  // block of the item's type
  __device__ __forceinline__ Blocks(int type, int m) : own(NB > 0 ? type * m / (16 * (NB > 0 ? NB : 1)) : 0) {}
  // turn-th 16 features from the own block on
  __device__ __forceinline__ int turned(int ks) const { return NB > 0 ? ((own * NB) + ks) % KS : ks; }
};
// From four groups on (with two, every pair of unlike types keeps all features,
// and no block of half of them is built).  us with blocks and without:
//   24576 tokens in 17 sequences, 12 heads of 64
//     q = 4  forward 246 / 257  dQ 331 / 330 (299 / 309)  dK and dV 398 / 418
//     q = 8          301 / 321     348 / 362                        435 / 468
//   8192 in 6, 32 heads of 128 on 8
//     q = 4  forward 234 / 249  dQ 348 / 390
//     q = 8          266 / 303     404 / 446
template <int NB>
inline bool blocks_fit(int law, int q, int m) {
  return law == 0 && q >= 4 && (m >= 32 ? NB == 2 : NB == 1);
}

// What a work item's walk needs per type.
template <int NG>
struct ItemLds {
  int32_t ring[NG][kPosSlots][64];         // per group: positions of the walked rows (the first 32), kNoPos past a type's end
  int32_t off[kAttnMaxQ], cnt[kAttnMaxQ];  // the walked range of the pack's permutation
  uint32_t cells[kAttnMaxQ];               // 8-feature cells that its pairs with the item's type keep
  float scale[kAttnMaxQ], lg[kAttnMaxQ];   // their scale and its logarithm (base 2)
};

template <int NG>
__device__ __forceinline__ void setup_item(ItemLds<NG>& s, const int32_t* rec, int law, int q, int head_dim) {
  const int m = head_dim / q, cpg = m / 8, own = rec[3] & 0xffff;
  if (threadIdx.x < static_cast<unsigned>(q)) {
    const int j = threadIdx.x;
    s.off[j] = rec[4 + j];
    s.cnt[j] = rec[4 + q + j];
    const uint32_t fm = attn_fmask(law, q, own, j);  // symmetric in the two types
    uint32_t cells = 0;
    for (int a = 0; a < q; ++a)
      if ((fm >> a) & 1u) cells |= ((1u << cpg) - 1u) << (a * cpg);
    s.cells[j] = cells;
    s.scale[j] = __builtin_amdgcn_rsqf(static_cast<float>(__popc(fm) * m));
    s.lg[j] = -0.5f * __log2f(static_cast<float>(__popc(fm) * m));
  }
}

// A place in the walk: type j, rows c .. c + 31 of its range, for the hh-th of
// `heads` rounds.  The same in every lane.  Of NG groups, group g takes steps
// g, g + NG, ...
template <int NG>
struct Walk {
  const ItemLds<NG>* s;
  int q, heads, hh, j;
  int32_t c, rows, base;
  uint32_t cells;
  float scale, lg;
  __device__ __forceinline__ void take_type() {
    rows = uniform(s->cnt[j]);
    base = uniform(s->off[j]);
    cells = uniform(s->cells[j]);
    scale = __uint_as_float(uniform(__float_as_uint(s->scale[j])));
    lg = __uint_as_float(uniform(__float_as_uint(s->lg[j])));
  }
  __device__ __forceinline__ void settle() {
    while (hh < heads && c >= rows) {
      c = 0;
      if (++j == q) {
        j = 0;
        ++hh;
      }
      take_type();
    }
  }
  __device__ __forceinline__ Walk(const ItemLds<NG>* s_, int q_, int heads_, int g) : s(s_), q(q_), heads(heads_), hh(0), j(0), c(0) {
    take_type();
    settle();
    for (int x = 0; x < g; ++x) step();
  }
  __device__ __forceinline__ void step() {
    if (hh < heads) {
      c += kStep;
      settle();
    }
  }
  __device__ __forceinline__ void next() {
#pragma unroll
    for (int x = 0; x < NG; ++x) step();
  }
  __device__ __forceinline__ bool done() const { return hh >= heads; }
  // the walked type's block, counted from the item's own
  template <int DH, int NB>
  __device__ __forceinline__ int block(const Blocks<DH, NB>& bl, int m) const {
    return NB > 0 ? (j * m / (16 * (NB > 0 ? NB : 1)) - bl.own + Blocks<DH, NB>::N) % Blocks<DH, NB>::N : 0;
  }
  // steps of the first group, which has the most (a group that is done goes
  // on with empty ones)
  __device__ __forceinline__ int32_t trips() const {
    int32_t n = 0;
    for (int t = 0; t < q; ++t) n += (uniform(s->cnt[t]) + kStep - 1) / kStep;
    return (n * heads + NG - 1) / NG;
  }
};

// Wavefront 0: the positions of a step into a slot of the ring.
template <int NG>
__device__ __forceinline__ void ask_positions(const Walk<NG>& w, const int32_t* perm, int32_t* slot, int lane) {
  const int32_t r = w.c + (lane & (kStep - 1));
  dma4(!w.done() && r < w.rows ? perm + w.base + r : g_attn_no_pos, lds_addr(slot));
}

// Copies per wavefront and array in a step.
template <int DH>
constexpr int copies_per_step() { return tile_bytes<DH>() / 1024 / kItemWaves; }

// The copies of a step: of A only the cells in `cells` (zeros stand for the
// others, so products over all features keep just the selected ones), of B
// whole rows; zero rows for kNoPos.  Offsets are counted in 16 bytes: 24 bits
// of position times 24 of stride, below 2^32 (the host sees to it).
template <int DH>
struct Copies {
  static constexpr int CPR = DH / 8, RPC = 64 / CPR, N = copies_per_step<DH>();
  int32_t pos[N];
  uint64_t zero;  // (kept in registers: reading the address of a global is a load)
  __device__ __forceinline__ Copies() : zero(reinterpret_cast<uint64_t>(g_attn_zero)) { asm volatile("" : "+s"(zero)); }
  __device__ __forceinline__ static int row(int k, int wave, int lane) { return (wave + kItemWaves * k) * RPC + lane / CPR; }
  __device__ __forceinline__ void take(const int32_t* slot, int wave, int lane) {
#pragma unroll
    for (int k = 0; k < N; ++k) pos[k] = slot[row(k, wave, lane)];
  }
  __device__ __forceinline__ void issue(const uint16_t* A, const uint16_t* B, uint32_t stride16, uint32_t cells, char* stage,
                                        int wave, int lane) const {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int r = row(k, wave, lane), c = (lane % CPR) ^ swz<DH>(r);
      const uint64_t at = static_cast<uint64_t>(static_cast<uint32_t>(__umul24(pos[k], stride16)) + static_cast<uint32_t>(c)) << 4;
      const bool ok = pos[k] != kNoPos, kept = ok & (((cells >> c) & 1u) != 0);
      const uint64_t a = kept ? reinterpret_cast<uint64_t>(A) + at : zero, b = ok ? reinterpret_cast<uint64_t>(B) + at : zero;
      char* to = stage + (wave + kItemWaves * k) * 1024;
      dma16(reinterpret_cast<const void*>(a), lds_addr(to));
      dma16(reinterpret_cast<const void*>(b), lds_addr(to + tile_bytes<DH>()));
    }
  }
};

// First and last position of a step, as a lane reads them and the same in all.
struct Ends {
  int32_t first, last;
  __device__ __forceinline__ void take(const int32_t* slot) {
    first = slot[0];
    last = slot[kStep - 1];
  }
  __device__ __forceinline__ void settle() {
    first = uniform(first);
    last = uniform(last);
  }
};

template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// Loads of the prologue that the loop uses are waited for here, before the
// first copies: the compiler, which does not see the copies, would otherwise
// wait in every round of the loop until nothing is in flight.
template <int N>
__device__ __forceinline__ void landed(uint4 (&x)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) asm volatile("" : "+v"(x[k].x), "+v"(x[k].y), "+v"(x[k].z), "+v"(x[k].w));
}
// (rows that are not there: loaded from another, zeroed here)
template <int N>
__device__ __forceinline__ void landed(uint4 (&x)[N], bool there) {
  landed(x);
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = there ? x[k] : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void landed(float& x) { asm volatile("" : "+v"(x)); }

// A lane's addresses in a tile.  Row operand ks (features 16 ks + 8 (l / 32)
// + 0..7 of row l % 32) sits at rows ^ 32 ks.  For the transposed operands lane
// l addresses 4 features of rows 4 (l / 32) + (l % 16) / 4 (+ 8, + 16 kk) and
// receives feature 32 c + l % 32 of rows 16 kk + 4 (l / 32) + 0..3 and of the
// 4 rows 8 behind: the order in which a 32 x 32 product leaves its rows in a
// lane.  They sit at cols ^ 64 c, 8 rows further on with one more bit turned.
template <int DH>
struct TileLane {
  uint32_t rows, cols;
  __device__ __forceinline__ explicit TileLane(int lane) {
    const int r = lane & 31;
    rows = r * DH * 2 + (((lane >> 5) ^ swz<DH>(r)) << 4);
    const int g = lane >> 4, row = 4 * (g >> 1) + ((lane & 15) >> 2), qq = lane & 3;
    cols = row * DH * 2 + (((2 * (g & 1) + (qq >> 1)) ^ swz<DH>(row)) << 4) + (qq & 1) * 8;
  }
  // Keeps the addresses derived from these two from being held over a loop: a
  // turned bit is one instruction, the registers are short.
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(rows), "+v"(cols)); }
  __device__ __forceinline__ uint4 row(const char* tile, int ks) const {
    return *reinterpret_cast<const uint4*>(tile + (rows ^ (ks << 5)));
  }
  __device__ __forceinline__ uint4 transposed(const char* tile, int kk, int c) const {
    const char* a0 = tile + 16 * kk * DH * 2 + (cols ^ (c << 6));
    const char* a1 = tile + (16 * kk + 8) * DH * 2 + (cols ^ (c << 6) ^ 32);
    const uint2 w0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((STARQ_LDS v4i16_t*)(a0)));
    const uint2 w1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((STARQ_LDS v4i16_t*)(a1)));
    return make_uint4(w0.x, w0.y, w1.x, w1.y);
  }
  // sum += rows of `tile` x ops, ops counted from the own block on; j: the
  // walked type's block, counted likewise
  template <int NB>
  __device__ __forceinline__ void add_rows(f32x16_t& sum, const char* tile, const uint4* ops, const Blocks<DH, NB>& bl, int j) const {
    constexpr int N = Blocks<DH, NB>::N, B = NB > 0 ? NB : DH / 16;
#pragma unroll
    for (int x = 0; x < B; ++x) sum = mfma(row(tile, bl.turned(x)), ops[x], sum);
    if constexpr (NB > 0) {
      uint4 f[B];
#pragma unroll
      for (int x = 0; x < B; ++x) f[x] = row(tile, bl.turned(j * NB + x));
#pragma unroll
      for (int r = 1; r < N; ++r)
        if (j == r) {
#pragma unroll
          for (int x = 0; x < B; ++x) sum = mfma(f[x], ops[r * NB + x], sum);
        }
    }
  }
  // acc += (rows of `tile`)^T x ops of the blocks that a pair keeps, in chunks
  // of 32 features counted from the own block's on
  template <int NB>
  __device__ __forceinline__ void add_transposed_kept(f32x16_t* acc, const char* tile, const uint4* ops, const Blocks<DH, NB>& bl,
                                                      int j) const {
    if constexpr (NB == 0) {
      add_transposed(acc, tile, ops);
    } else {
      constexpr int NCH = DH / 32;
      const int c0 = bl.own * NB / 2, c1 = bl.turned(j * NB) / 2, r1 = (c1 - c0 + NCH) % NCH;
#pragma unroll
      for (int kk = 0; kk < kStep / 16; ++kk) acc[0] = mfma(transposed(tile, kk, c0), ops[kk], acc[0]);
      uint4 f[kStep / 16];
#pragma unroll
      for (int kk = 0; kk < kStep / 16; ++kk) f[kk] = transposed(tile, kk, c1);
#pragma unroll
      for (int r = 1; r < NCH; ++r)
        if (r1 == r) {
#pragma unroll
          for (int kk = 0; kk < kStep / 16; ++kk) acc[r] = mfma(f[kk], ops[kk], acc[r]);
        }
    }
  }
  // acc += (rows of `tile`)^T x ops, ops[kk] the operand of rows 16 kk and on
  __device__ __forceinline__ void add_transposed(f32x16_t* acc, const char* tile, const uint4* ops) const {
#pragma unroll
    for (int kk = 0; kk < kStep / 16; ++kk)
#pragma unroll
      for (int c = 0; c < DH / 32; ++c) acc[c] = mfma(transposed(tile, kk, c), ops[kk], acc[c]);
  }
  // Masked places enter the products above with weight zero, and zero times an
  // infinity is no number.  The same sums in parts: of the finite values, and
  // for each feature whether an infinity (or a value that is no number: both
  // signs) meets a weight.  first: the chunk that acc[0] is of
  __device__ __forceinline__ void add_odd(f32x16_t* acc, const char* tile, const uint4* ops, int first = 0) const {
    // (rare, so in the order that takes the fewest registers)
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) {
      const int chunk = (c + first) % (DH / 32);
#pragma unroll
      for (int kk = 0; kk < kStep / 16; ++kk) {
        acc[c] = mfma(picked(transposed(tile, kk, chunk), 0), ops[kk], acc[c]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int sign = 1; sign >= -1; sign -= 2) {
        f32x16_t met{};
#pragma unroll
        for (int kk = 0; kk < kStep / 16; ++kk) {
          const uint4 w = ops[kk];
          met = mfma(picked(transposed(tile, kk, chunk), sign),
                     make_uint4(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu, w.z & 0x7fff7fffu, w.w & 0x7fff7fffu), met);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[c][e] += met[e] > 0.f ? sign * __builtin_inff() : 0.f;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // which 0: the finite ones of 8 bf16 values, zeros for others; which 1 or -1:
  // ones where there is an infinity of that sign or no number
  __device__ __forceinline__ static uint32_t picked(uint32_t x, int which) {
    uint32_t r = 0;
#pragma unroll
    for (int half = 0; half < 32; half += 16) {
      const uint32_t v = (x >> half) & 0xffffu;
      const bool there = (v & 0x7f80u) == 0x7f80u;
      r |= (which == 0 ? (there ? 0u : v) : there && v != (which > 0 ? 0xff80u : 0x7f80u) ? 0x3f80u : 0u) << half;
    }
    return r;
  }
  __device__ __forceinline__ static uint4 picked(uint4 x, int which) {
    return make_uint4(picked(x.x, which), picked(x.y, which), picked(x.z, which), picked(x.w, which));
  }
};

// Whether any of a wavefront's sums is not finite: if so its workgroup walks a
// second time (`care`), one step's code for all three stages, with add_odd and
// with nothing left of masked places.  The loop that everyone runs stays as it
// is: testing the tiles that hold masked places there, or two ways to add in
// it, cost 4 to 22 % (the registers are full); so placed it costs 0 to 3 %.
template <int N>
__device__ __forceinline__ bool odd(const f32x16_t (&acc)[N]) {
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) s = __builtin_fmaf(acc[c][e], 0.f, s);
  return s != 0.f;  // zero, or no number
}

// The second group's sums added to the first's, through LDS where the rings
// were.  True in the first group.
template <int NCH>
__device__ __forceinline__ bool join_groups(f32x16_t* acc, char* rings, int g, int wave, int lane) {
  float* sum = reinterpret_cast<float*>(rings) + wave * NCH * 16 * 64 + lane;
  __syncthreads();
  if (g == 1) {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[(16 * c + e) * 64] = acc[c][e];
  }
  __syncthreads();
  if (g == 0) {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] += sum[(16 * c + e) * 64];
  }
  return g == 0;
}

// Rows of a transposed product's result: acc[c][4 a + e] is feature
// 32 c + 8 a + 4 (l / 32) + e of the lane's row.
// (first: the chunk that acc[0] is of)
template <int DH>
__device__ __forceinline__ void store_row(void* out, int dtype, int64_t at, const f32x16_t* acc, int lh, int first = 0) {
#pragma unroll
  for (int c = 0; c < DH / 32; ++c)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int f = 32 * ((c + first) % (DH / 32)) + 8 * a + 4 * lh;
      const float v0 = acc[c][4 * a], v1 = acc[c][4 * a + 1], v2 = acc[c][4 * a + 2], v3 = acc[c][4 * a + 3];
      if (dtype == 0)
        *reinterpret_cast<float4*>(static_cast<float*>(out) + at + f) = make_float4(v0, v1, v2, v3);
      else
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at + f) = make_uint2(pack_bf16(v0, v1), pack_bf16(v2, v3));
    }
}

}  // namespace

}  // namespace starq
