// Attention on the tensor cores: tcgen05 products with scores, weights and sums in tensor memory.
//
//   S = Q K^T (128 queries x BN keys, fp32), t = scale S (capped, biased, masked), P = 2^(t - m) rounded to bf16,
//   O += P V;  m: the row's running maximum, l: the row's running sum of the unrounded weights;  y = O / l
//
// One persistent CTA per SM takes work items of up to 256 queries of one head: two tiles of 128, each with a warpgroup whose
// thread owns a row (no shuffles) and with a thread that issues its products, so that one tile's exponentials run beside the
// other's products. Warp 8 loads: Q once an item, K and V tiles through one ring of TMA stages that both tiles read (128-byte
// swizzle, columns beyond head_dim zero-filled by the tensor map); A of the second product (P) comes from tensor memory, V is read
// along its rows as an MN-major operand.
// Tensor memory, 512 columns: S0 S1, P0 P1 (half as wide), O0 O1. P stands beside S, so that the next scores are computed while a
// warpgroup still takes exponentials; that asks for 2 (3/2 BN + D) columns: 128 keys to a tile up to D = 64, 96 up to D = 96, 80 up
// to 128 (P over S with 128 keys there, measured: 8192 tokens causal with distance bias, 16 heads of 128: 342 us).
// Where an item of 128 queries is all there is (CUT), the warpgroups take its key tiles in turn and the first joins their sums.
// A warp beside them decodes the work items ahead of everybody (a dozen divisions and the sequences' offsets), through a small
// ring in shared memory.
//
// The maximum that the weights refer to moves only when a row's own maximum has outgrown it by 2^8: until then the sums stay
// as they are (fp32 and bf16 have the range), and O is rescaled a few times an item instead of once a tile.
//
// A tile that reaches behind the sequence's keys holds other sequences' rows, or nobody's: their scores are masked whatever they
// are, and their V rows are overwritten with zeros before the product, since 0 * NaN would be NaN.
#include <cuda.h>
#include <cuda_bf16.h>

#include "attn.cuh"
#include "gemm_device.cuh"

namespace dp {

constexpr int kTcTile = 128;                      // queries of a tile
constexpr int kTcBlock = kTcTile * 128;           // bytes of 128 rows x 64 columns
constexpr int kTcThreads = 384;                   // two warpgroups; loads, an issuing warp for each tile, work items
// Registers a thread: 384 threads are launched with 168; the third warpgroup gives up what the first two take on:
// 2 * 128 * 208 + 128 * 88 = 384 * 168.
constexpr int kTcRegsLaunch = 168, kTcRegsSoftmax = 208, kTcRegsRest = 88;
static_assert(256 * kTcRegsSoftmax + 128 * kTcRegsRest == kTcThreads * kTcRegsLaunch, "register split");
constexpr float kTcRise = 8.0f;                   // log2 units by which a row's maximum may outgrow the reference

constexpr int kTcOrderBytes = 784;                // of a TcOrder, a multiple of 16

// Tiles for vectors of up to 16 KS elements.
template <int KS>
struct TcForm {
  static constexpr int BN = KS <= 4 ? 128 : KS <= 6 ? 96 : 80;  // keys of a tile
  static constexpr int D = 16 * KS, NBLK = (D + 63) / 64;
  static constexpr int kQBytes = NBLK * kTcBlock, kKvBlock = BN * 128, kKvBytes = NBLK * kKvBlock;
  static constexpr int NS = NBLK == 1 ? 8 : BN == 96 ? 6 : 7;  // ring stages
  static constexpr uint32_t kS = 0, kP = 2 * BN, kO = 3 * BN;  // columns
  static_assert(BN % 16 == 0 && kO + 2 * D <= 512, "tensor memory");
  // (after the tiles: rows' maxima and sums, the ring of items, the sequences' order, barriers, turns, tensor memory's address, the abort flag)
  static constexpr size_t kSmem = 1024 + 2 * kQBytes + NS * kKvBytes + 1024 + 4 * 48 + kTcOrderBytes + (2 * NS + 14 + 2 * 4) * 8 + 48;
  static_assert(kSmem <= 232448, "shared memory");
};

struct AttnTcSched {
  int32_t rows;        // queries of a work item: 128 or 256
  int32_t cut;         // whether its two warpgroups share the keys of 128 queries
  int32_t tiles;       // items of the longest sequence
  int32_t items;       // tiles * heads * sequences
  int32_t group;       // (sequence, head) pairs whose items are taken together, longest ones first
  int64_t budget;      // cycles that a wait may take
  int32_t skip;        // test hook (dp_debug_skip_stage_load): copy of a CTA's first item that is left out, or -1
  int32_t sorted;      // sequences by their keys instead, and no items that are not there (up to kTcSorted packed sequences)
};

// mbar_wait with a limit that goes by the call: a warp of one tile of queries may wait for the other tile's whole item, and the
// item ring for a few of them, so the limit grows with the keys.
__device__ __forceinline__ bool tc_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int64_t budget) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  uint32_t polls = 0;
  while (!mbar_try_wait(bar, parity)) {
    if ((++polls & 63u) == 0) {
      if (*abort_flag) return false;
      if (clock64() - t0 > budget) {
        *abort_flag = 1;
        return false;
      }
    }
  }
  return true;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, int c0, int c1, int c2, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], A bf16 pairs in 32-bit columns. Issued by one thread.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// This warp's 32 lanes, 32 (16) consecutive 32-bit columns: thread t <-> lane t.
__device__ __forceinline__ void tmem_ld_x32(uint32_t a, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
      "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
        "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
        "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(a)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_x16(uint32_t a, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(a)
      : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t a, const uint32_t* u) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(a),
      "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]),
      "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_x8(uint32_t a, const uint32_t* u) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(a), "r"(u[0]), "r"(u[1]),
               "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// MN-major operand (the contraction's index is the row): 64 columns a row of 128 bytes with the 128-byte swizzle, groups of 8 rows
// 1024 bytes apart (stride), further 64 columns `lead` bytes apart.
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t saddr, uint32_t lead) {
  uint64_t d = smem_desc_sw128(saddr) & ~(0x3FFFull << 16);
  return d | static_cast<uint64_t>(lead >> 4) << 16;
}
constexpr uint32_t kIdescBMn = 1u << 16;  // instruction descriptor: B is MN-major

// The weights 2^(s scale - sub) of N scores, their sum and their bf16 pairs. The special-function unit takes 16 values a clock and SM,
// for 96 scores of two warps to an SM quarter 1536 clocks of the 1640 that this takes. (A share of the powers by a cubic on the FMA
// pipe, measured: 1360 clocks at two of eight pairs; in the kernel, where the warps take turns, nothing.)
template <int N>
__device__ __forceinline__ float tc_weights(const float (&s)[N], float scale, float sub, uint32_t (&w)[N / 2]) {
  const uint64_t scale2 = f32x2_pack(scale, scale), sub2 = f32x2_pack(-sub, -sub);
  uint64_t sum[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    float lo, hi;
    f32x2_unpack(f32x2_fma(f32x2_pack(s[2 * i], s[2 * i + 1]), scale2, sub2), lo, hi);
    lo = ex2(lo);
    hi = ex2(hi);
    sum[i & 1] = f32x2_add(sum[i & 1], f32x2_pack(lo, hi));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(hi), "f"(lo));
  }
  float u, v;
  f32x2_unpack(f32x2_add(sum[0], sum[1]), u, v);
  return u + v;
}

// tanh(s k) in place of N scores: up to 3/4 by an odd polynomial fitted for the least relative error (7.2e-7), without the
// special-function unit, beyond by two operations of it. Which one is decided score by score, so that a result does not depend on the
// scores beside it (other sequences' queries and keys may be among them); a warp whose scores are all small, as capped scores of real
// models are, takes polynomials only. (8 x 1024 tokens, 16 heads of 64, most scores beyond: 137 us with one form for a warp's 32 rows, 153 so; within
// the range 98 and 99.)
template <int N>
__device__ __forceinline__ void tc_tanh(float (&s)[N], float two_log2e_k, float k) {
  float top[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < N; i += 2) top[(i >> 1) & 3] = fmaxf(fmaxf(top[(i >> 1) & 3], fabsf(s[i])), fabsf(s[i + 1]));
  const float big = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * k;
  const uint64_t k2 = f32x2_pack(k, k);
  auto polynomial = [&](float a, float b, float& lo, float& hi) {
    const uint64_t c3 = f32x2_pack(0.01310583670f, 0.01310583670f), c2 = f32x2_pack(-0.05027795583f, -0.05027795583f);
    const uint64_t c1 = f32x2_pack(0.13268236816f, 0.13268236816f), c0 = f32x2_pack(-0.33329668641f, -0.33329668641f);
    const uint64_t u = f32x2_mul(f32x2_pack(a, b), k2), z = f32x2_mul(u, u);
    uint64_t y = f32x2_fma(z, c3, c2);
    y = f32x2_fma(y, z, c1);
    y = f32x2_fma(y, z, c0);
    f32x2_unpack(f32x2_fma(f32x2_mul(y, z), u, u), lo, hi);
  };
  if (__all_sync(0xFFFFFFFFu, big <= 0.75f)) {
#pragma unroll
    for (int i = 0; i < N; i += 2) polynomial(s[i], s[i + 1], s[i], s[i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float lo, hi;
      polynomial(s[i], s[i + 1], lo, hi);
      s[i] = fabsf(s[i]) * k <= 0.75f ? lo : capped(1.0f, s[i] * two_log2e_k);
      s[i + 1] = fabsf(s[i + 1]) * k <= 0.75f ? hi : capped(1.0f, s[i + 1] * two_log2e_k);
    }
  }
}

// s scale - slope |pos - key| for N keys from key0 on; d = pos - key0, `side`: +1 if no key that counts lies behind pos, -1 if none
// lies before it, 0 otherwise (the same for the whole warp).
template <int N>
__device__ __forceinline__ void tc_bias(float (&s)[N], float scale, float slope, int d, int side) {
  if (side != 0) {
    const float a = side > 0 ? slope : -slope, base = -a * static_cast<float>(d);  // + a (key - pos)
    const uint64_t scale2 = f32x2_pack(scale, scale), step2 = f32x2_pack(2.0f * a, 2.0f * a);
#pragma unroll
    for (int g = 0; g < N; g += 16) {
      const float first = fmaf(a, static_cast<float>(g), base);
      uint64_t y = f32x2_pack(first, first + a);
#pragma unroll
      for (int i = g; i < g + 16; i += 2) {
        f32x2_unpack(f32x2_fma(f32x2_pack(s[i], s[i + 1]), scale2, y), s[i], s[i + 1]);
        y = f32x2_add(y, step2);
      }
    }
  } else {
    const float d0 = static_cast<float>(d);
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = fmaf(-slope, fabsf(d0 - i), s[i] * scale);
  }
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// 32 rows (one a lane) x 32 bf16 columns from registers to memory: lanes change their 16-byte pieces in fours, so that a store
// writes 64 bytes of eight rows instead of 16 bytes of 32. row0: the warp's first row, of `live` ones.
__device__ __forceinline__ void tc_store_32(uint16_t* y, int64_t ld, int row0, int live, int cols, const uint32_t (&w)[16]) {
  const int lane = threadIdx.x & 31;
  uint32_t e[4][4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) e[c][i] = w[4 * c + i];
#pragma unroll
  for (int b = 1; b <= 2; b <<= 1)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c & b) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // the lane without the bit gives its piece c | b for the other's piece c
        const bool up = lane & b;
        const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, up ? e[c][i] : e[c | b][i], b);
        if (up) e[c][i] = got;
        else e[c | b][i] = got;
      }
    }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int row = row0 + (lane & 28) + k;
    if (row < live && (lane & 3) * 8 < cols) st_global_v4(y + row * ld + (lane & 3) * 8, e[k]);
  }
}

// A work item: the sequence, its queries' first row in it, and the key tiles that either tile of queries has to see.
struct __align__(16) TcItem {
  AttnSeq s;
  int head, row0;    // row0 < 0: no more items
  int n0, n1;        // key tiles of the two tiles of queries, or (cut) of the two warpgroups
  int live0, live1;  // queries in them
  __device__ __forceinline__ int n(bool cut) const { return cut ? n0 + n1 : max(n0, n1); }
};
constexpr int kTcSorted = 64;
constexpr int kTcSlots = 4;      // of the ring of items
constexpr int kTcItemReaders = 11;  // loads, two issuing threads, eight warps
template <int BN>
__device__ __forceinline__ bool tc_item(const AttnParams& p, const AttnTcSched& c, int seq, int head, int tile, TcItem& r) {
  r.head = head;
  r.s = attn_seq(p, seq);
  r.row0 = tile * c.rows;
  if (r.row0 >= r.s.nq) return false;
  r.live0 = min(r.s.nq - r.row0, kTcTile);
  r.live1 = c.rows > kTcTile ? min(max(r.s.nq - r.row0 - kTcTile, 0), kTcTile) : 0;
  r.n0 = (attn_keys(p, r.s, r.row0 + r.live0 - 1) + BN - 1) / BN;
  if (c.cut) {
    r.n1 = r.n0 / 2;
    r.n0 -= r.n1;
    return true;
  }
  r.n1 = r.live1 > 0 ? (attn_keys(p, r.s, r.row0 + kTcTile + r.live1 - 1) + BN - 1) / BN : 0;
  return true;
}
// Sequences in the order of their keys, most first, for packed ones of unlike lengths: order[rank] the sequence and its items per head,
// start[rank] the items before it. By one warp.
struct TcOrder {
  int seq[kTcSorted], tiles[kTcSorted], start[kTcSorted + 1];
};
static_assert(sizeof(TcOrder) <= kTcOrderBytes, "sequences' order");
__device__ __forceinline__ void tc_sort(const AttnParams& p, const AttnTcSched& c, TcOrder& o) {
  const int lane = threadIdx.x & 31;
  int keys[2], tiles[2], rank[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    keys[i] = -1;
    tiles[i] = 0;
    if (lane + 32 * i < p.n_seq) {
      const AttnSeq s = attn_seq(p, lane + 32 * i);
      keys[i] = s.nk;
      tiles[i] = (s.nq + c.rows - 1) / c.rows;
    }
  }
  for (int k = 0; k < kTcSorted; ++k) {
    const int other = __shfl_sync(0xFFFFFFFFu, k < 32 ? keys[0] : keys[1], k & 31);
#pragma unroll
    for (int i = 0; i < 2; ++i) rank[i] += other > keys[i] || (other == keys[i] && k < lane + 32 * i);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    o.seq[rank[i]] = lane + 32 * i;
    o.tiles[rank[i]] = tiles[i];
  }
  __syncwarp();
  int before = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int mine = o.tiles[lane + 32 * i] * p.H;
    int sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, sum, d);
      if (lane >= d) sum += x;
    }
    o.start[lane + 32 * i] = before + sum - mine;
    before += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  if (lane == 0) o.start[kTcSorted] = before;
  __syncwarp();
}
// Item i in the order without a sort: pairs in groups; within a group the last rows, which see the most keys under a causal mask, come
// first. The sequence.
__device__ __forceinline__ int tc_place(const AttnParams& p, const AttnTcSched& c, int i, int& head, int& tile) {
  const int pairs = p.H * p.n_seq, g = i / (c.group * c.tiles), in = i - g * c.group * c.tiles;
  const int size = min(c.group, pairs - g * c.group), from_last = in / size;
  const int pair = g * c.group + in - from_last * size, seq = pair / p.H;
  head = pair - seq * p.H;
  tile = c.tiles - 1 - from_last;
  return seq;
}
// The next item of this CTA: rounds of gridDim.x items, every other one backwards, so that the long items that come first
// even out. `rank`: where the last one was found. False: there is none. By a whole warp: where packed sequences are shorter than
// max_q most items may not be there, and the lanes look through 32 rounds at a time (256 sequences of 200 tokens, 16 heads of 72,
// causal, max_q = 8192: 395 us by one thread, 201 so).
template <int BN>
__device__ __forceinline__ bool tc_next(const AttnParams& p, const AttnTcSched& c, const TcOrder& o, int& round, int& rank, TcItem& it) {
  const int items = c.sorted ? o.start[kTcSorted] : c.items;
  auto at = [&](int r) {
    return static_cast<int64_t>(r) * gridDim.x + ((r & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
  };
  for (;;) {
    if (static_cast<int64_t>(round) * gridDim.x >= items) return false;
    const int64_t here = at(round++);
    int head, tile;
    if (here >= items) continue;
    const int i = static_cast<int>(here);
    if (c.sorted) {  // (items of later rounds stand behind those of earlier ones)
      while (o.start[rank + 1] <= i) ++rank;
      const int in = i - o.start[rank];
      tile = in / p.H;
      if (tc_item<BN>(p, c, o.seq[rank], in - tile * p.H, tile, it)) return true;
      continue;
    }
    const int seq = tc_place(p, c, i, head, tile);
    if (tc_item<BN>(p, c, seq, head, tile, it)) return true;
    for (;; round += 32) {
      if (static_cast<int64_t>(round) * gridDim.x >= items) return false;
      const int64_t mine = at(round + static_cast<int>(threadIdx.x & 31));
      bool there = false;
      if (mine < items) {
        const int s = tc_place(p, c, static_cast<int>(mine), head, tile);
        there = static_cast<int64_t>(tile) * c.rows < attn_seq(p, s).nq;
      }
      if (const uint32_t some = __ballot_sync(0xFFFFFFFFu, there); some != 0) {
        round += __ffs(some) - 1;
        break;
      }
    }
  }
}

// CUT: items of one tile of queries, whose key tiles the warpgroups take in turn (even ones, odd ones); their sums are joined at the end.
template <int KS, bool CAP, bool BIAS, bool CUT>
__global__ void __launch_bounds__(kTcThreads, 1)
attn_tc_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
               const __grid_constant__ CUtensorMap tv, const AttnParams p, const AttnTcSched c) {
  using F = TcForm<KS>;
  constexpr int BN = F::BN, NS = F::NS, NBLK = F::NBLK;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                    // [2][NBLK][128 rows][128 bytes]
  uint8_t* sKV = sQ + 2 * F::kQBytes;    // [NS][NBLK][BN rows][128 bytes]
  float2* half = reinterpret_cast<float2*>(sKV + NS * F::kKvBytes);  // [128]
  TcItem* slots = reinterpret_cast<TcItem*>(half + kTcTile);
  TcOrder* order = reinterpret_cast<TcOrder*>(slots + kTcSlots);
  uint64_t* full = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(order) + kTcOrderBytes);
  uint64_t* empty = full + NS;
  uint64_t* item_full = empty + NS;
  uint64_t* item_empty = item_full + kTcSlots;
  uint64_t* q_full = item_empty + kTcSlots;  // [2]
  uint64_t* q_empty = q_full + 2;            // [2]
  uint64_t* s_full = q_empty + 2;  // [2] scores are there
  uint64_t* s_read = s_full + 2;   // [2] and in the warpgroup's registers
  uint64_t* p_full = s_read + 2;   // [2] weights are there
  uint64_t* pv_done = p_full + 2;  // [2] and their product has ended
  uint64_t* half_full = pv_done + 2;     // the second warpgroup's half of the keys is summed
  uint64_t* half_read = half_full + 1;   // and in the first one's registers
  volatile uint32_t* turns = reinterpret_cast<uint32_t*>(half_read + 1);  // [8] tiles whose exponentials a warp has taken
  uint32_t* tmem_slot = const_cast<uint32_t*>(turns) + 8;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 2);
    }
    for (int i = 0; i < kTcSlots; ++i) {
      mbar_init(&item_full[i], 1);
      mbar_init(&item_empty[i], kTcItemReaders);
    }
    for (int i = 0; i < 8; ++i) turns[i] = 0;
    for (int t = 0; t < 2; ++t) {
      mbar_init(&q_full[t], 1);
      mbar_init(&q_empty[t], 1);
      mbar_init(&s_full[t], 1);
      mbar_init(&s_read[t], 4);
      mbar_init(&p_full[t], 4);
      mbar_init(&pv_done[t], 1);
    }
    mbar_init(half_full, 4);
    mbar_init(half_read, 4);
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tq);
    tma_prefetch_desc(&tk);
    tma_prefetch_desc(&tv);
  }
  if (warp == 8) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  // The next item from the ring; `leader`: the thread that gives the slot back once all that read it with this one have.
  Ring item_at;
  auto next_item = [&](TcItem& it, bool warp_wide) {
    bool ok = tc_wait(&item_full[item_at.s], item_at.ph, abort_flag, c.budget);
    if (warp_wide) ok = __all_sync(0xFFFFFFFFu, ok);
    if (!ok) {
      it.row0 = -1;
      return false;
    }
    it = slots[item_at.s];
    if (warp_wide) __syncwarp();
    if (!warp_wide || lane == 0) mbar_arrive(&item_empty[item_at.s]);
    item_at.next(kTcSlots);
    return true;
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcRegsRest));
    if (warp == 8 && elect_one()) {
      // ================= loads =================
      Ring st;
      bool ok = true;
      uint32_t items[2] = {0, 0};
      int skip = c.skip;
      TcItem it;
      const uint32_t group = p.H / p.KV;
      auto load_q = [&](int t) {
        if (!(ok = tc_wait(&q_empty[t], (items[t] & 1) ^ 1u, abort_flag, c.budget))) return;
        ++items[t];
        mbar_arrive_expect_tx(&q_full[t], F::kQBytes);
#pragma unroll
        for (int b = 0; b < NBLK; ++b)
          tma_load_3d(smem_u32(sQ) + t * F::kQBytes + b * kTcBlock, &tq, b * 64, it.head, it.s.q0 + it.row0 + (CUT ? 0 : t * kTcTile), &q_full[t]);
      };
      while (ok && (ok = next_item(it, false)) && it.row0 >= 0) {
        const int n = it.n(CUT);
        if (it.n0 > 0) load_q(0);
        const int kvh = it.head / group;
        for (int j = 0; j < 2 * n && ok; ++j) {  // K, V, K, V, ..
          if (!(ok = tc_wait(&empty[st.s], st.ph ^ 1u, abort_flag, c.budget))) break;
          if (j == skip) {  // (nothing is issued for this stage, and nobody completes its barrier)
            st.next(NS);
            continue;
          }
          mbar_arrive_expect_tx(&full[st.s], F::kKvBytes);
#pragma unroll
          for (int b = 0; b < NBLK; ++b)
            tma_load_3d(smem_u32(sKV) + st.s * F::kKvBytes + b * F::kKvBlock, (j & 1) ? &tv : &tk, b * 64, kvh,
                        it.s.k0 + (j >> 1) * BN, &full[st.s]);
          st.next(NS);
          if (j == 0 && it.n1 > 0) load_q(1);
        }
        skip = -1;
      }
      if (!ok) producer_drain();
    } else if (warp == 11) {
      // ================= work items =================
      int round = 0, rank = 0;
      if (c.sorted) tc_sort(p, c, *order);
      TcItem it;
      bool ok = true, more = true;
      while (ok && more) {
        more = tc_next<BN>(p, c, *order, round, rank, it);
        if (!more) it.row0 = -1;
        if (lane == 0) {
          ok = tc_wait(&item_empty[item_at.s], item_at.ph ^ 1u, abort_flag, c.budget);
          if (ok) {
            slots[item_at.s] = it;
            mbar_arrive(&item_full[item_at.s]);
          }
        }
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
        item_at.next(kTcSlots);
      }
    } else if ((warp == 9 || warp == 10) && elect_one()) {
      // ================= products of tile t =================
      const int t = warp - 9;
      constexpr uint32_t idesc_s = idesc_bf16(kTcTile, BN), idesc_o = idesc_bf16(kTcTile, F::D) | kIdescBMn;
      const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ) + t * F::kQBytes), k_desc = smem_desc_sw128(smem_u32(sKV));
      const uint64_t v_desc = smem_desc_sw128_mn(smem_u32(sKV), F::kKvBlock);
      const uint32_t d_s = tmem + F::kS + t * BN, d_p = tmem + F::kP + t * (BN / 2), d_o = tmem + F::kO + t * F::D;
      bool ok = true, ahead = false;  // ahead: the next item's first scores are issued
      uint32_t n_s = 0, n_p = 0, items = 0;  // scores, weights, items so far
      // Scores of the key tile in stage k into S, which the warpgroup has read.
      auto scores = [&](const Ring& k) {
        if (n_s > 0 && !(ok = tc_wait(&s_read[t], (n_s - 1) & 1, abort_flag, c.budget))) return;
        if (!(ok = tc_wait(&full[k.s], k.ph, abort_flag, c.budget))) return;
        tc_fence_after();
        const uint64_t kd = k_desc + static_cast<uint64_t>(k.s * (F::kKvBytes >> 4));
#pragma unroll
        for (int i = 0; i < KS; ++i)
          mma_bf16_ss(d_s, q_desc + (i >> 2) * (kTcBlock >> 4) + (i & 3) * 2, kd + (i >> 2) * (F::kKvBlock >> 4) + (i & 3) * 2,
                      idesc_s, i != 0);
        mma_commit(&s_full[t]);
        mma_commit(&empty[k.s]);
        ++n_s;
      };
      auto first_scores = [&](const Ring& k, int n) {  // of an item with n key tiles for this tile
        if (!(ok = tc_wait(&q_full[t], items & 1, abort_flag, c.budget))) return;
        ++items;
        scores(k);
        if (ok && n == 1) mma_commit(&q_empty[t]);
      };
      Ring st;  // K of the item's first tile
      auto pass_on = [&](int stages) {  // the other tile's
        for (int j = 0; j < stages && ok; ++j) {
          if (!(ok = tc_wait(&full[st.s], st.ph, abort_flag, c.budget))) break;
          mbar_arrive(&empty[st.s]);
          st.next(NS);
        }
      };
      TcItem nxt;
      ok = next_item(nxt, false);
      while (ok && nxt.row0 >= 0) {
        const int n_all = nxt.n(CUT), n = t ? nxt.n1 : nxt.n0;
        if (!(ok = next_item(nxt, false))) break;
        const int n_next = nxt.row0 >= 0 ? (t ? nxt.n1 : nxt.n0) : 0;
        if (n > 0) {
          if (CUT && t == 1) pass_on(2);
          if (!ahead && ok) first_scores(st, n);
          ahead = false;
          st.next(NS);
          for (int j = 0; j < n && ok; ++j) {
            const Ring v = st;
            st.next(NS);
            auto next_scores = [&]() {
              scores(st);
              if (ok && j + 2 == n) mma_commit(&q_empty[t]);
            };
            if (CUT && j + 1 < n) pass_on(2);
            if (ok && j + 1 < n) next_scores();
            if (!ok || !(ok = tc_wait(&p_full[t], n_p & 1, abort_flag, c.budget)) || !(ok = tc_wait(&full[v.s], v.ph, abort_flag, c.budget))) break;
            ++n_p;
            tc_fence_after();
            const uint64_t vd = v_desc + static_cast<uint64_t>(v.s * (F::kKvBytes >> 4));
            const uint32_t add = j != 0;
            mma_bf16_ts(d_o, d_p, vd, idesc_o, add);
#pragma unroll
            for (int i = 1; i < BN / 16; ++i) mma_bf16_ts(d_o, d_p + i * 8, vd + i * 128, idesc_o, 1u);
            mma_commit(&pv_done[t]);
            mma_commit(&empty[v.s]);
            if (j + 1 < n) {
              st.next(NS);
            } else if (!CUT && n == n_all && n_next > 0) {  // the next item's first scores while this one's output is written
              first_scores(st, n_next);
              ahead = true;
            }
          }
        }
        // the rest of the item's tiles is the other tile's: passed on as they come
        pass_on(2 * (n_all - (CUT && n > 0 ? 2 * n - 1 + t : n)));
      }
      // Products still in flight get a bounded time to end, before tensor memory is given back under them; so do copies in flight where the
      // loads' thread is already done.
      if (!ok) producer_drain();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTcRegsSoftmax));
    // ================= softmax: warpgroup t, thread <-> row =================
    const int t = warp >> 2;
    const int row = threadIdx.x & 127;
    const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t a_s = lanes + F::kS + t * BN, a_p = lanes + F::kP + t * (BN / 2), a_o = lanes + F::kO + t * F::D;
    Ring st;
    bool ok = true;
    uint32_t n_s = 0, others = 0, joins = 0;  // tiles so far, the other warpgroup's up to this item, items joined
    TcItem it;
    while (ok && (ok = next_item(it, true)) && it.row0 >= 0) {
      const int n_all = it.n(CUT), n = t ? it.n1 : it.n0, live = t ? it.live1 : it.live0;
      const int pos = it.row0 + (CUT ? 0 : t * kTcTile) + row + it.s.behind;  // of this thread's query
      // keys below this bound are visible
      const int bound = p.causal ? min(it.s.nk, max(pos + 1, it.s.prefix)) : it.s.nk;
      const float slope = BIAS ? ld_global_f32(p.slopes + it.head) * kLog2e : 0.0f;
      const float scale = BIAS ? 1.0f : CAP ? p.cap : p.scale;
      float m = -INFINITY, l = 0.0f;
      for (int j = 0; j < n_all; ++j) {
        st.next(NS);  // (K)
        const Ring v = st;
        st.next(NS);
        if (CUT ? (j & 1) != t : j >= n) continue;
        const int own = CUT ? j >> 1 : j;
        ok = tc_wait(&s_full[t], n_s & 1, abort_flag, c.budget);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        tc_fence_after();
        float s[BN];
#pragma unroll
        for (int i = 0; i < BN / 32; ++i) tmem_ld_x32(a_s + i * 32, s + i * 32);
        if constexpr (BN % 32 != 0) tmem_ld_x16(a_s + BN / 32 * 32, s + BN / 32 * 32);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_read[t]);
        const int left = bound - j * BN;  // visible keys of this tile
        if constexpr (CAP) tc_tanh(s, p.scale_by_cap, p.scale_by_cap * (0.5f / kLog2e));
        if constexpr (BIAS) {
          const int d = pos - lane - j * BN;  // of the warp's first row
          const int side = d >= BN - 1 || (p.causal && j * BN >= it.s.prefix) ? 1 : d + 31 <= 0 ? -1 : 0;
          tc_bias(s, CAP ? p.cap : p.scale, slope, d + lane, side);
        }
        if (__any_sync(0xFFFFFFFFu, left < BN)) {
#pragma unroll
          for (int g = 0; g < BN; g += 16)
            if (__any_sync(0xFFFFFFFFu, left < g + 16)) {
#pragma unroll
              for (int i = g; i < g + 16; ++i) s[i] = i < left ? s[i] : -INFINITY;
            }
        }
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int i = 4; i < BN - 4; i += 2) mx[(i >> 1) & 3] = max3(mx[(i >> 1) & 3], s[i], s[i + 1]);
        const float top = fmaxf(max3(max3(mx[0], mx[1], s[BN - 4]), mx[2], s[BN - 3]), max3(mx[3], s[BN - 2], s[BN - 1])) * scale;
        // P and O are this warpgroup's once the product before has ended
        auto product_before = [&]() {
          if (n_s == 0) return true;
          ok = tc_wait(&pv_done[t], (n_s - 1) & 1, abort_flag, c.budget);
          ok = __all_sync(0xFFFFFFFFu, ok);
          tc_fence_after();
          return ok;
        };
        if (own == 0) {
          m = top;
        } else if (__any_sync(0xFFFFFFFFu, top > m + kTcRise)) {
          if (!product_before()) break;
          // Only rows whose own maximum has: the warp's others may be queries of another sequence, or nobody's. (8192 tokens causal with distance
          // bias, whose maxima rise with the keys: 364 us with all rows of the warp at once, 370 so.)
          const float to_m = top > m + kTcRise ? top : m, f = to_m == -INFINITY ? 1.0f : ex2(m - to_m);
          m = to_m;
          l *= f;
#pragma unroll 1
          for (int k = 0; k < F::D; k += 16) {
            float o[16];
            tmem_ld_x16(a_o + k, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= f;
            tmem_st_x16(a_o + k, reinterpret_cast<const uint32_t*>(o));
          }
        }
        const float sub = m == -INFINITY ? 0.0f : m;
        // The two warps of an SM quarter take turns at the exponentials: both at once would be no faster, and apart one's stand
        // beside the other's loads, scans and waits (32 x 1024 tokens, 16 heads of 72: 250 us without turns, 237 with). A
        // bounded wait: what it orders is time, not data.
        const uint32_t until = others + min(own + t, t ? it.n0 : it.n1);
        for (int i = 0; i < 64 && turns[warp ^ 4] < until; ++i) {
        }
        uint32_t w[BN / 2];
        l += tc_weights(s, scale, sub, w);
        if (!(l < 0.0f)) turns[warp] = n_s + 1;  // (never negative: the store waits for the sum)
        if (!product_before()) break;
        if (CUT && t == 1 && own == 0 && joins > 0) {  // (the last item's sums are read: this product overwrites them)
          ok = tc_wait(half_read, (joins - 1) & 1, abort_flag, c.budget);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) break;
          tc_fence_after();
        }
        ++n_s;
#pragma unroll
        for (int k = 0; k < BN / 32; ++k) tmem_st_x16(a_p + k * 16, w + k * 16);
        if constexpr (BN % 32 != 0) tmem_st_x8(a_p + BN / 32 * 16, w + BN / 32 * 16);
        const int keys_here = it.s.nk - j * BN;
        if (keys_here < BN) {  // V rows behind the sequence: zeros
          ok = tc_wait(&full[v.s], v.ph, abort_flag, c.budget);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) break;
          uint8_t* vt = sKV + v.s * F::kKvBytes + keys_here * 128;
#pragma unroll
          for (int b = 0; b < NBLK; ++b)
            for (int i = row; i < (BN - keys_here) * 8; i += 128)
              *reinterpret_cast<uint4*>(vt + b * F::kKvBlock + i * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[t]);
      }
      if (!ok) break;
      others += t ? it.n0 : it.n1;
      if (CUT && t == 1 && n > 0) {
        ok = tc_wait(&pv_done[1], (n_s - 1) & 1, abort_flag, c.budget);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        tc_fence_after();
        half[row] = make_float2(m, l);
        ++joins;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(half_full);
      }
      if (live == 0) continue;
      float mine = 1.0f, other = 0.0f;  // shares of the two halves of the keys
      const bool join = CUT && it.n1 > 0;
      if (join) {
        ok = tc_wait(half_full, joins & 1, abort_flag, c.budget);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        ++joins;
        tc_fence_after();
        const float2 h = half[row];
        const float top = fmaxf(m, h.x), sub = top == -INFINITY ? 0.0f : top;
        mine = ex2(m - sub);
        other = ex2(h.x - sub);
        l = fmaf(l, mine, h.y * other);
      }
      const float inv = l != 0.0f ? __fdiv_rn(1.0f, l) : 0.0f;  // (no key in sight: O is zero too)
      uint16_t* yt = p.y + static_cast<int64_t>(it.s.q0 + it.row0 + t * kTcTile) * p.ldy + it.head * p.y_hs;
      float o[(F::D + 31) / 32 * 32];
      if (n > 0) {
        ok = tc_wait(&pv_done[t], (n_s - 1) & 1, abort_flag, c.budget);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < F::D; k += 16) tmem_ld_x16(a_o + k, o + k);
        tmem_ld_wait();
        if (join) {
#pragma unroll
          for (int k = 0; k < F::D; k += 16) {
            float h[16];
            tmem_ld_x16(lanes + F::kO + F::D + k, h);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[k + i] = fmaf(o[k + i], mine, h[i] * other);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(half_read);
        }
        tc_fence_before();  // (the next item's products write O behind this thread's next arrival on p_full)
      } else {
#pragma unroll
        for (int k = 0; k < F::D; ++k) o[k] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < F::D; k += 32) {
        if (k >= p.D) break;
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float a = k + 2 * i < F::D ? o[k + 2 * i] * inv : 0.0f, b = k + 2 * i < F::D ? o[k + 2 * i + 1] * inv : 0.0f;
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(b), "f"(a));
        }
        tc_store_32(yt + k, p.ldy, (warp & 3) * 32, live, p.D - k, w);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (threadIdx.x == 0 && *abort_flag && p.status != nullptr) atomicExch(p.status, DP_ERR_TIMEOUT);
}

// ---- host side -------------------------------------------------------------------------------------
template <int KS, bool CAP, bool BIAS>
static cudaError_t tc_init() {
  cudaError_t e = cudaFuncSetAttribute(attn_tc_kernel<KS, CAP, BIAS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(TcForm<KS>::kSmem));
  return e != cudaSuccess ? e
                          : cudaFuncSetAttribute(attn_tc_kernel<KS, CAP, BIAS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 static_cast<int>(TcForm<KS>::kSmem));
}
template <int KS>
static int tc_init_ks() {
  DP_CUDA_OK((tc_init<KS, false, false>()));
  DP_CUDA_OK((tc_init<KS, false, true>()));
  DP_CUDA_OK((tc_init<KS, true, false>()));
  DP_CUDA_OK((tc_init<KS, true, true>()));
  return DP_OK;
}
int attn_tc_init_device() {
  int st = tc_init_ks<4>();
  if (st == DP_OK) st = tc_init_ks<5>();
  if (st == DP_OK) st = tc_init_ks<6>();
  if (st == DP_OK) st = tc_init_ks<8>();
  return st;
}

template <int KS, bool CUT>
static int launch_tc(const AttnParams& p, const AttnTcSched& c, unsigned ctas, cudaStream_t stream, bool pdl) {
  using F = TcForm<KS>;
  CUtensorMap tq, tk, tv;
  int st = gemm_encode_heads(&tq, p.q, p.D, p.H, p.Mq, p.q_hs, p.ldq, kTcTile);
  if (st == DP_OK) st = gemm_encode_heads(&tk, p.k, p.D, p.KV, p.Mk, p.k_hs, p.ldk, F::BN);
  if (st == DP_OK) st = gemm_encode_heads(&tv, p.v, p.D, p.KV, p.Mk, p.v_hs, p.ldv, F::BN);
  if (st != DP_OK) return st;
  const dim3 grid(ctas), block(kTcThreads);
  const bool cap = p.cap != 0.0f, bias = p.slopes != nullptr;
  const cudaError_t e =
      cap && bias ? launch(attn_tc_kernel<KS, true, true, CUT>, grid, block, F::kSmem, stream, pdl, tq, tk, tv, p, c)
      : cap       ? launch(attn_tc_kernel<KS, true, false, CUT>, grid, block, F::kSmem, stream, pdl, tq, tk, tv, p, c)
      : bias      ? launch(attn_tc_kernel<KS, false, true, CUT>, grid, block, F::kSmem, stream, pdl, tq, tk, tv, p, c)
                  : launch(attn_tc_kernel<KS, false, false, CUT>, grid, block, F::kSmem, stream, pdl, tq, tk, tv, p, c);
  if (e != cudaSuccess) return fail(DP_ERR_CUDA, "attention launch failed: %s", cudaGetErrorString(e));
  return DP_OK;
}
template <bool CUT>
static int launch_tc_width(const AttnParams& p, const AttnTcSched& c, unsigned ctas, cudaStream_t stream, bool pdl) {
  return p.D <= 64   ? launch_tc<4, CUT>(p, c, ctas, stream, pdl)
         : p.D <= 80 ? launch_tc<5, CUT>(p, c, ctas, stream, pdl)
         : p.D <= 96 ? launch_tc<6, CUT>(p, c, ctas, stream, pdl)
                     : launch_tc<8, CUT>(p, c, ctas, stream, pdl);
}

int launch_attn_tc(const AttnParams& p, cudaStream_t stream, bool pdl) {
  const int sms = num_sms() > 0 ? num_sms() : 148;
  const int64_t pairs = static_cast<int64_t>(p.H) * p.n_seq;
  AttnTcSched c;
  // Items of 256 queries share K and V between two tiles and hide one's products behind the other's exponentials; of 128, whose
  // keys the warpgroups share, where that many more SMs get work.
  c.rows = 2 * kTcTile;
  if (attn_product((static_cast<int64_t>(p.max_q) + 255) / 256, pairs) <= sms / 2 || p.max_q <= kTcTile) c.rows = kTcTile;
  // From 385 keys on the second warpgroup, idle otherwise, takes every other tile of the keys of 128 queries (one sequence of 256 queries, 16 heads
  // of 72, over 256 / 512 / 1000 / 4096 keys: 9.1 / 12.1 / 17.3 / 50.4 us -> 9.2 / 11.6 / 15.3 / 39.9; 64 of 96, over 96 / 200 / 512: 21.1 / 41.4 / 62.7
  // -> 23.9 / 43.1 / 58.4).
  c.cut = c.rows == kTcTile && p.max_k > 384;
  const int64_t tiles = (static_cast<int64_t>(p.max_q) + c.rows - 1) / c.rows;
  if (attn_product(tiles, pairs) > 0x7FFFFFFF) return fail(DP_ERR_SHAPE, "attention: %lld tiles of queries", (long long)attn_product(tiles, pairs));
  c.tiles = static_cast<int32_t>(tiles);
  c.items = static_cast<int32_t>(tiles * pairs);
  // Of equal sequences without a mask all items are alike and a pair's stand together, for its K and V in L2; else 64 pairs, so that
  // what is there of a tile is a run of items (256 sequences of 200 tokens, 16 heads of 72, max_q = 1024: a pair's together 340 us,
  // 64 pairs 186).
  // Packed sequences are taken longest first, and only items that are there: 16 documents of 1 to 1500 tokens.
  c.sorted = !p.causal && p.q_start != nullptr && p.n_seq <= kTcSorted;
  const int64_t group = p.causal || p.q_start != nullptr ? 64 : 1;
  c.group = static_cast<int32_t>(group < pairs ? group : pairs);
  const unsigned ctas = static_cast<unsigned>(c.items < sms ? c.items : sms);
  c.skip = take_debug_skip();
  // Six items of the most keys there can be, at 8192 cycles a tile (2500 or so are usual), and the items that may not be there,
  // 4096 cycles (800) to 32 of them, on top of the library's usual limit.
  c.budget = kWaitBudgetCycles + 6 * 8192 * (p.Mk / 80 + 1) + 4096 * (c.items / (32ll * ctas) + 1);
  return c.cut ? launch_tc_width<true>(p, c, ctas, stream, pdl) : launch_tc_width<false>(p, c, ctas, stream, pdl);
}

}  // namespace dp
