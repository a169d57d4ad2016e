// Attention on the tensor cores: tcgen05 products with scores, weights and sums in tensor memory.
//
//   S = Q K^T (128 queries x 128 keys, fp32), t = scale S (capped, biased, masked), P = 2^(t - m) rounded to bf16 in place of S,
//   O += P V;  m: the row's running maximum, l: the row's running sum of the unrounded weights;  y = O / l
//
// One persistent CTA per SM takes work items of up to 256 queries of one head: two tiles of 128, each with a warpgroup whose
// thread owns a row (no shuffles), so that one warpgroup's exponentials run beside the other's products. Warp 8 loads: Q once
// an item, K and V tiles through one ring of TMA stages (128-byte swizzle, columns beyond head_dim zero-filled by the tensor
// map); warp 9 issues the products, A of the second one (P) from tensor memory, V read along its rows as an MN-major operand.
// Tensor memory: S0 S1 (128 columns each, P in the first 64 of them), O0 O1 (128 each).
//
// The maximum that the weights refer to moves only when a row's own maximum has outgrown it by 2^8: until then the sums stay
// as they are (fp32 and bf16 have the range), and O is rescaled a few times an item instead of once a tile. A rescale needs no
// barrier of its own: the products run in issue order, so S of a tile being there says that the product before it has ended.
//
// A tile that reaches behind the sequence's keys holds other sequences' rows, or nobody's: their scores are masked whatever they
// are, and their V rows are overwritten with zeros before the product, since 0 * NaN would be NaN.
#include <cuda.h>
#include <cuda_bf16.h>

#include "attn.cuh"
#include "gemm_device.cuh"

namespace dp {

constexpr int kTcTile = 128;                      // queries and keys of a tile
constexpr int kTcBlock = kTcTile * 128;           // bytes of 128 rows x 64 columns
constexpr int kTcThreads = 320;
constexpr float kTcRise = 8.0f;                   // log2 units by which a row's maximum may outgrow the reference
__host__ __device__ constexpr int tc_stages(int nblk) { return nblk == 1 ? 8 : 5; }

struct AttnTcSched {
  int32_t rows;        // queries of a work item: 128 or 256
  int32_t tiles;       // items of the longest sequence
  int32_t items;       // tiles * heads * sequences
  int32_t group;       // (sequence, head) pairs whose items are taken together, longest ones first
};

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
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// MN-major operand (the contraction's index is the row): 64 columns a row of 128 bytes with the 128-byte swizzle, groups of 8 rows
// 1024 bytes apart (stride), further 64 columns `lead` bytes apart.
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t saddr, uint32_t lead) {
  uint64_t d = smem_desc_sw128(saddr) & ~(0x3FFFull << 16);
  return d | static_cast<uint64_t>(lead >> 4) << 16;
}
constexpr uint32_t kIdescBMn = 1u << 16;  // instruction descriptor: B is MN-major

// A work item: the sequence, its queries' first row in it, and the key tiles that either tile of queries has to see.
struct TcItem {
  AttnSeq s;
  int head, kvh, row0;
  int n[2];  // key tiles of the two tiles of queries
  int live[2];  // queries in them
  bool valid;
  __device__ __forceinline__ int tiles() const { return max(n[0], n[1]); }
};
__device__ __forceinline__ TcItem tc_item(const AttnParams& p, const AttnTcSched& c, int item) {
  TcItem r;
  // pairs in groups; within a group the last rows, which see the most keys under a causal mask, come first
  const int pairs = p.H * p.n_seq;
  const int g = item / (c.group * c.tiles), in = item - g * c.group * c.tiles;
  const int size = min(c.group, pairs - g * c.group);
  const int tile = c.tiles - 1 - in / size, pair = g * c.group + in % size;
  const int seq = pair / p.H;
  r.head = pair - seq * p.H;
  r.kvh = r.head / (p.H / p.KV);
  r.s = attn_seq(p, seq);
  r.row0 = tile * c.rows;
  r.valid = r.row0 < r.s.nq;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int first = r.row0 + t * kTcTile;
    r.live[t] = t * kTcTile < c.rows ? min(max(r.s.nq - first, 0), kTcTile) : 0;
    r.n[t] = r.live[t] > 0 ? (attn_keys(p, r.s, first + r.live[t] - 1) + kTcTile - 1) / kTcTile : 0;
  }
  return r;
}
// The i-th item of this CTA: rounds of gridDim.x items, every other one backwards, so that the long items that come first
// even out. False: there is none.
__device__ __forceinline__ bool tc_next(const AttnParams& p, const AttnTcSched& c, int& round, TcItem& it) {
  for (;; ++round) {
    const int64_t base = static_cast<int64_t>(round) * gridDim.x;
    if (base >= c.items) return false;
    const int64_t i = base + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    if (i >= c.items) continue;
    it = tc_item(p, c, static_cast<int>(i));
    if (it.valid) {
      ++round;
      return true;
    }
  }
}

template <bool CAP, bool BIAS>
__global__ void __launch_bounds__(kTcThreads, 1)
attn_tc_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
               const __grid_constant__ CUtensorMap tv, const AttnParams p, const AttnTcSched c, const int nblk) {
  extern __shared__ uint8_t smem_raw[];
  const int NS = tc_stages(nblk), tile_bytes = nblk * kTcBlock;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                   // [2][nblk][128 rows][128 bytes]
  uint8_t* sKV = sQ + 2 * tile_bytes;   // [NS][nblk][128 rows][128 bytes]
  uint64_t* full = reinterpret_cast<uint64_t*>(sKV + NS * tile_bytes);
  uint64_t* empty = full + NS;
  uint64_t* q_full = empty + NS;
  uint64_t* q_empty = q_full + 1;
  uint64_t* s_full = q_empty + 1;  // [2]
  uint64_t* p_full = s_full + 2;   // [2]
  uint64_t* o_full = p_full + 2;   // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_full + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&s_full[t], 1);
      mbar_init(&p_full[t], 4);
      mbar_init(&o_full[t], 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tq);
    tma_prefetch_desc(&tk);
    tma_prefetch_desc(&tv);
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  if (warp == 8) {
    if (elect_one()) {
      // ================= loads =================
      Ring st;
      bool ok = true;
      int round = 0, n_items = 0;
      TcItem it;
      auto load = [&](const CUtensorMap* map, int head, int row) {
        if (!(ok = mbar_spin_wait(&empty[st.s], st.ph ^ 1u, abort_flag))) return;
        mbar_arrive_expect_tx(&full[st.s], tile_bytes);
        for (int b = 0; b < nblk; ++b)
          tma_load_3d(smem_u32(sKV) + st.s * tile_bytes + b * kTcBlock, map, b * 64, head, row, &full[st.s]);
        st.next(NS);
      };
      while (ok && tc_next(p, c, round, it)) {
        const int n = it.tiles();
        if (n == 0) continue;
        if (!(ok = mbar_spin_wait(q_empty, (n_items & 1) ^ 1u, abort_flag))) break;
        const int q_tiles = it.n[1] > 0 ? 2 : 1;
        mbar_arrive_expect_tx(q_full, q_tiles * tile_bytes);
        for (int t = 0; t < q_tiles; ++t)
          for (int b = 0; b < nblk; ++b)
            tma_load_3d(smem_u32(sQ) + t * tile_bytes + b * kTcBlock, &tq, b * 64, it.head, it.s.q0 + it.row0 + t * kTcTile, q_full);
        ++n_items;
        for (int j = 0; j < n && ok; ++j) {
          load(&tk, it.kvh, it.s.k0 + j * kTcTile);
          if (ok) load(&tv, it.kvh, it.s.k0 + j * kTcTile);
        }
      }
      if (!ok) producer_drain();
    }
  } else if (warp == 9) {
    if (elect_one()) {
      // ================= products =================
      const int ks = (p.D + 15) / 16;
      const uint32_t idesc_s = idesc_bf16(kTcTile, kTcTile), idesc_o = idesc_bf16(kTcTile, ks * 16) | kIdescBMn;
      const uint64_t q_desc = smem_desc_sw128(smem_u32(sQ)), k_desc = smem_desc_sw128(smem_u32(sKV));
      const uint64_t v_desc = smem_desc_sw128_mn(smem_u32(sKV), kTcBlock);
      Ring st;  // the next tile of the ring to be used
      bool ok = true;
      int round = 0, n_items = 0;
      uint32_t p_ph[2] = {0, 0};
      TcItem cur, nxt;
      auto scores = [&](int t, int stage) {
#pragma unroll 1
        for (int k = 0; k < ks; ++k) {
          const uint64_t at = static_cast<uint64_t>((k >> 2) * (kTcBlock >> 4) + (k & 3) * 2);
          mma_bf16_ss(tmem + t * 128, q_desc + static_cast<uint64_t>(t * (tile_bytes >> 4)) + at,
                      k_desc + static_cast<uint64_t>(stage * (tile_bytes >> 4)) + at, idesc_s, k != 0);
        }
        mma_commit(&s_full[t]);
      };
      // first scores of an item, for tile t; K's stage is st
      bool have = tc_next(p, c, round, nxt);
      bool first_in = false;  // nxt's Q and first K are there
      auto enter = [&]() {    // waits for nxt's Q and first K tile
        if (first_in) return true;
        ok = mbar_spin_wait(q_full, n_items & 1, abort_flag) && mbar_spin_wait(&full[st.s], st.ph, abort_flag);
        tc_fence_after();
        ++n_items;
        first_in = true;
        return ok;
      };
      auto first_done = [&]() {  // both tiles' first scores are issued
        mma_commit(&empty[st.s]);
        st.next(NS);
        if (nxt.tiles() == 1) mma_commit(q_empty);
      };
      bool pending = have;  // nxt's first scores are still to be issued
      while (ok && have) {
        cur = nxt;
        const int n = cur.tiles();
        if (pending && n > 0) {
          if (!enter()) break;
          for (int t = 0; t < 2; ++t)
            if (cur.n[t] > 0) scores(t, st.s);
          first_done();
        }
        have = tc_next(p, c, round, nxt);
        first_in = false;
        pending = true;
        for (int j = 0; j < n && ok; ++j) {
          const Ring v = st;
          st.next(NS);  // (the next K tile: of this item, or the next item's first)
          const bool last = j + 1 == n;
          const bool more = !last || (have && nxt.tiles() > 0);
          bool v_in = false, k_in = false;
          for (int t = 0; t < 2 && ok; ++t) {
            if (j < cur.n[t]) {
              if (!(ok = mbar_spin_wait(&p_full[t], p_ph[t], abort_flag))) break;
              p_ph[t] ^= 1u;
              if (!v_in && !(ok = mbar_spin_wait(&full[v.s], v.ph, abort_flag))) break;
              v_in = true;
              tc_fence_after();
#pragma unroll 1
              for (int k = 0; k < kTcTile / 16; ++k)
                mma_bf16_ts(tmem + 256 + t * 128, tmem + t * 128 + k * 8,
                            v_desc + static_cast<uint64_t>(v.s * (tile_bytes >> 4) + k * 128), idesc_o, (j | k) != 0);
              if (j + 1 == cur.n[t]) mma_commit(&o_full[t]);
            }
            if (t == 1) mma_commit(&empty[v.s]);
            if (last) {  // the next item's first scores, while this one's last weights are under way
              if (more && nxt.n[t] > 0) {
                if (!enter()) break;
                scores(t, st.s);
              }
            } else if (j + 1 < cur.n[t]) {
              if (!k_in && !(ok = mbar_spin_wait(&full[st.s], st.ph, abort_flag))) break;
              k_in = true;
              tc_fence_after();
              scores(t, st.s);
            }
          }
          if (!ok) break;
          if (last) {
            if (more) {
              first_done();
              pending = false;
            }
          } else {
            mma_commit(&empty[st.s]);
            st.next(NS);
            if (j + 2 == n) mma_commit(q_empty);
          }
        }
      }
    }
  } else {
    // ================= softmax: warpgroup t, thread <-> row =================
    const int t = warp >> 2;
    const int row = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + t * 128, to = tmem + lanes + 256 + t * 128;
    Ring st;
    bool ok = true;
    int round = 0;
    uint32_t s_ph = 0, o_ph = 0;
    TcItem it;
    float s[128];
    while (ok && tc_next(p, c, round, it)) {
      const int n_all = it.tiles(), n = it.n[t];
      const int q = it.row0 + t * kTcTile + row;  // this thread's query
      const int pos = q + it.s.behind;
      // keys below this bound are visible
      const int bound = p.causal ? min(it.s.nk, max(pos + 1, it.s.prefix)) : it.s.nk;
      const float slope = BIAS ? ld_global_f32(p.slopes + it.head) * kLog2e : 0.0f;
      const float scale = CAP || BIAS ? 1.0f : p.scale;
      float m = -INFINITY, l = 0.0f;
      for (int j = 0; j < n_all; ++j) {
        st.next(NS);  // (K)
        const Ring v = st;
        st.next(NS);
        if (j >= n) continue;
        ok = mbar_wait(&s_full[t], s_ph, abort_flag);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        s_ph ^= 1u;
        tc_fence_after();
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld_x32(ts + i * 32, s + i * 32);
        tmem_ld_wait();
        const int left = bound - j * kTcTile;  // visible keys of this tile
        if constexpr (CAP) {
#pragma unroll
          for (int i = 0; i < 128; ++i) s[i] = capped(p.cap, s[i] * p.scale_by_cap);
        } else if constexpr (BIAS) {
#pragma unroll
          for (int i = 0; i < 128; ++i) s[i] *= p.scale;
        }
        if constexpr (BIAS) {
          const float d0 = static_cast<float>(pos - j * kTcTile);
#pragma unroll
          for (int i = 0; i < 128; ++i) s[i] = fmaf(-slope, fabsf(d0 - i), s[i]);
        }
        if (__any_sync(0xFFFFFFFFu, left < kTcTile)) {
#pragma unroll
          for (int i = 0; i < 128; ++i) s[i] = i < left ? s[i] : -INFINITY;
        }
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int i = 4; i < 128; ++i) mx[i & 3] = fmaxf(mx[i & 3], s[i]);
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
        if (j == 0) {
          m = top;
        } else if (__any_sync(0xFFFFFFFFu, top > m + kTcRise)) {
          const float to_m = fmaxf(m, top), f = to_m == -INFINITY ? 1.0f : ex2(m - to_m);
          m = to_m;
          l *= f;
#pragma unroll 1
          for (int k = 0; k < p.D; k += 16) {
            float o[16];
            tmem_ld_x16(to + k, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= f;
            tmem_st_x16(to + k, reinterpret_cast<const uint32_t*>(o));
          }
        }
        const float sub = m == -INFINITY ? 0.0f : m;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float a = ex2(fmaf(s[k * 32 + 2 * i], scale, -sub)), b = ex2(fmaf(s[k * 32 + 2 * i + 1], scale, -sub));
            sum[(2 * i) & 3] += a;
            sum[(2 * i + 1) & 3] += b;
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(b), "f"(a));
          }
          tmem_st_x16(ts + k * 16, w);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        const int keys_here = it.s.nk - j * kTcTile;
        if (keys_here < kTcTile) {  // V rows behind the sequence: zeros
          ok = mbar_wait(&full[v.s], v.ph, abort_flag);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) break;
          uint8_t* vt = sKV + v.s * tile_bytes + row * 128;
          if (row >= keys_here)
            for (int b = 0; b < nblk; ++b)
#pragma unroll
              for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(vt + b * kTcBlock + i * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[t]);
      }
      if (!ok) break;
      if (n > 0) {
        ok = mbar_wait(&o_full[t], o_ph, abort_flag);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        o_ph ^= 1u;
        tc_fence_after();
      }
      const bool live = row < it.live[t];
      const float inv = l != 0.0f ? __fdiv_rn(1.0f, l) : 0.0f;  // (no key in sight: O is zero too)
      uint16_t* yr = p.y + static_cast<int64_t>(it.s.q0 + q) * p.ldy + it.head * p.y_hs;
      if (it.live[t] > 0) {
#pragma unroll 1
        for (int k = 0; k < p.D; k += 16) {
          float o[16];
          if (n > 0) {
            tmem_ld_x16(to + k, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = 0.0f;
          }
          uint32_t w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float a = o[2 * i] * inv, b = o[2 * i + 1] * inv;
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(b), "f"(a));
          }
          if (live) {
            st_global_v4(yr + k, reinterpret_cast<const uint32_t(&)[4]>(w[0]));
            if (k + 8 < p.D) st_global_v4(yr + k + 8, reinterpret_cast<const uint32_t(&)[4]>(w[4]));
          }
        }
        tc_fence_before();  // (the next item's products write O behind this thread's next arrival on p_full)
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (threadIdx.x == 0 && *abort_flag && p.status != nullptr) atomicExch(p.status, DP_ERR_TIMEOUT);
}

// ---- host side -------------------------------------------------------------------------------------
static size_t tc_smem_bytes(int nblk) {
  return 1024 + static_cast<size_t>(2 + tc_stages(nblk)) * nblk * kTcBlock + (2 * tc_stages(nblk) + 8) * 8 + 16;
}
template <bool CAP, bool BIAS>
static cudaError_t tc_init() {
  const size_t a = tc_smem_bytes(1), b = tc_smem_bytes(2);
  return cudaFuncSetAttribute(attn_tc_kernel<CAP, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(a > b ? a : b));
}
int attn_tc_init_device() {
  DP_CUDA_OK((tc_init<false, false>()));
  DP_CUDA_OK((tc_init<false, true>()));
  DP_CUDA_OK((tc_init<true, false>()));
  DP_CUDA_OK((tc_init<true, true>()));
  return DP_OK;
}

int launch_attn_tc(const AttnParams& p, cudaStream_t stream, bool pdl) {
  const int nblk = (p.D + 63) / 64;
  CUtensorMap tq, tk, tv;
  int st = gemm_encode_heads(&tq, p.q, p.D, p.H, p.Mq, p.q_hs, p.ldq, kTcTile);
  if (st == DP_OK) st = gemm_encode_heads(&tk, p.k, p.D, p.KV, p.Mk, p.k_hs, p.ldk, kTcTile);
  if (st == DP_OK) st = gemm_encode_heads(&tv, p.v, p.D, p.KV, p.Mk, p.v_hs, p.ldv, kTcTile);
  if (st != DP_OK) return st;
  const int sms = num_sms() > 0 ? num_sms() : 148;
  const int64_t pairs = static_cast<int64_t>(p.H) * p.n_seq;
  AttnTcSched c;
  // Items of 256 queries share K and V between two tiles and hide one's products behind the other's exponentials; of 128 where
  // that many more SMs get work.
  c.rows = 2 * kTcTile;
  if ((static_cast<int64_t>(p.max_q) + 255) / 256 * pairs * 2 <= sms || p.max_q <= kTcTile) c.rows = kTcTile;
  const int64_t tiles = (static_cast<int64_t>(p.max_q) + c.rows - 1) / c.rows;
  if (tiles * pairs > 0x7FFFFFFF) return fail(DP_ERR_SHAPE, "attention: %lld tiles of queries", (long long)(tiles * pairs));
  c.tiles = static_cast<int32_t>(tiles);
  c.items = static_cast<int32_t>(tiles * pairs);
  // Without a mask all items are alike and a pair's stand together, for its K and V in L2; with one, 64 pairs.
  const int64_t group = p.causal ? 64 : 1;
  c.group = static_cast<int32_t>(group < pairs ? group : pairs);
  const dim3 grid(static_cast<unsigned>(c.items < sms ? c.items : sms)), block(kTcThreads);
  const size_t smem = tc_smem_bytes(nblk);
  cudaError_t e;
  if (p.cap != 0.0f && p.slopes != nullptr) e = launch(attn_tc_kernel<true, true>, grid, block, smem, stream, pdl, tq, tk, tv, p, c, nblk);
  else if (p.cap != 0.0f) e = launch(attn_tc_kernel<true, false>, grid, block, smem, stream, pdl, tq, tk, tv, p, c, nblk);
  else if (p.slopes != nullptr) e = launch(attn_tc_kernel<false, true>, grid, block, smem, stream, pdl, tq, tk, tv, p, c, nblk);
  else e = launch(attn_tc_kernel<false, false>, grid, block, smem, stream, pdl, tq, tk, tv, p, c, nblk);
  if (e != cudaSuccess) return fail(DP_ERR_CUDA, "attention launch failed: %s", cudaGetErrorString(e));
  return DP_OK;
}

}  // namespace dp
