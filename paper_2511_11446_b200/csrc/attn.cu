// Attention of few queries, mma.sync tiles of 16, one pass over the keys with a running maximum and sum; and of any number of
// them (attn_rows_kernel: shapes that the tcgen05 kernel would fill badly, and its counterpart in tests).
//
//   t_ij = scale q_i . k_j, capped by a tanh, less slope |pos(i) - j|;   y_i = sum_j softmax_j(t_ij) v_j
//
// A row is a (query, head) pair: the heads / kv_heads heads that read one key head stand beside each other, so keys and values
// are read once for all of them. Few rows make this a stream of K and V (one query, 16 heads of 72: 4 operations a byte), so what
// counts is bytes in flight: in attn_few_kernel every warp walks a part of the keys of its own, 16 or 32 at a time through a private ring
// of cp.async stages without a barrier between warps, and the keys of a sequence are cut over the CTAs of a cluster too, whose
// partial sums (m, l, O) meet in distributed shared memory: one launch, no scratch memory.
#include <cuda_bf16.h>

#include "attn.cuh"
#include "dp_internal.h"

namespace dp {

constexpr int kAtThreads = 128, kAtKeys = 64;
constexpr int kAtMaxSplits = kAttnMaxSplits;  // CTAs of a cluster
// Keys of a stage of a warp's ring, and stages: two CTAs to an SM. Small stages cost more arithmetic a key, so they are taken only where they
// overlap what else would wait (8 sequences of 8192 keys, 4 key heads of 128, one query: 32.9 us by one stage of 32, 28.2 by three of 16; seven
// queries, two blocks of rows: 44.4 / 45.3).
__host__ __device__ constexpr int few_keys(int dp, int mb) { return dp > 96 && mb == 1 ? 16 : 32; }
__host__ __device__ constexpr int few_stages(int dp, int mb) { return dp <= 96 ? 2 : mb == 1 ? 3 : 1; }

// Bytes between the rows of a tile in shared memory: an odd number of 16-byte units, so that the eight rows of a matrix that
// ldmatrix fetches lie in different banks.
__host__ __device__ constexpr int at_row_bytes(int dp) { return (dp * 2 / 16) % 2 ? dp * 2 : dp * 2 + 16; }
__host__ __device__ constexpr int at_stage_bytes(int dp) { return 2 * kAtKeys * at_row_bytes(dp); }
constexpr int kAtStages = 3;

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool ok) {  // !ok: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm_x4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void ld_cluster_f32x2(uint32_t a, float& x, float& y) {
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x), "=f"(y) : "r"(a) : "memory");
}

struct AtRows {
  int pos[2];          // of fragment rows lane / 4 and lane / 4 + 8
  int bound[2];        // keys below it are visible
  float slope[2];
};
// What both kernels do with a fragment of 16 rows x 8 N keys of scores: scaled, capped, biased, masked, in log2 units; the rows'
// new maxima (of the four lanes that share a row) into mx. tile_end: behind the fragment's last key.
template <int N>
__device__ __forceinline__ void at_scores(const AttnParams& p, const AtRows& w, int key0, int tile_end, float (&sc)[N][4],
                                          float (&mx)[2]) {
  if (p.cap != 0.0f) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[n][i] = capped(p.cap, sc[n][i] * p.scale_by_cap);
  } else {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[n][i] *= p.scale;
  }
  if (p.slopes != nullptr) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sc[n][i] = fmaf(-w.slope[i >> 1], fabsf(static_cast<float>(w.pos[i >> 1] - (key0 + n * 8 + (i & 1)))), sc[n][i]);
  }
  if (__any_sync(0xFFFFFFFFu, tile_end > min(w.bound[0], w.bound[1]))) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (key0 + n * 8 + (i & 1) >= w.bound[i >> 1]) sc[n][i] = -INFINITY;
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) mx[i >> 1] = fmaxf(mx[i >> 1], sc[n][i]);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xFFFFFFFFu, mx[e], 1));
    mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xFFFFFFFFu, mx[e], 2));
  }
}
// Where a CTA's rows lie (a query's `group` heads side by side): its first row is head `head0` of the group of query `tok0`, `left` rows
// are there. (32-bit divisions row by row: 64-bit ones took 0.4 us of a small call's 6.2.)
struct AtPlace {
  int tok0, head0, left, group, kvh;
  __device__ __forceinline__ int tok(int row) const { return tok0 + (head0 + row) / group; }
  __device__ __forceinline__ int head(int row) const { return kvh * group + (head0 + row) % group; }
};
// Rows row0 .. row0 + 15 of the CTA: their places and query fragments.
template <int KS>
__device__ __forceinline__ void at_rows(const AttnParams& p, const AttnSeq& s, const AtPlace& at, int row0, AtRows& w,
                                        uint32_t (&qf)[KS][4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int row = row0 + (lane >> 2) + 8 * e;
    const bool live = row < at.left;
    const int tok = live ? at.tok(row) : 0, head = live ? at.head(row) : at.kvh * at.group;
    w.pos[e] = tok + s.behind;
    w.bound[e] = p.causal ? min(s.nk, max(w.pos[e] + 1, s.prefix)) : s.nk;
    if (!live) w.bound[e] = 0x7FFFFFFF;  // (nobody's row: nothing to be masked)
    w.slope[e] = p.slopes != nullptr ? ld_global_f32(p.slopes + head) * kLog2e : 0.0f;
    const uint16_t* qr = p.q + static_cast<int64_t>(s.q0 + tok) * p.ldq + head * p.q_hs;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int col = k * 16 + c * 8 + (lane & 3) * 2;
        qf[k][2 * c + e] = live && col < p.D ? static_cast<uint32_t>(ld_global_s32(reinterpret_cast<const int32_t*>(qr + col))) : 0u;
      }
  }
}
__device__ __forceinline__ uint16_t* at_out(const AttnParams& p, const AttnSeq& s, const AtPlace& at, int row) {
  return p.y + static_cast<int64_t>(s.q0 + at.tok(row)) * p.ldy + at.head(row) * p.y_hs;
}

// 16 MB rows by every one of W warps, each with keys of its own. grid.x = splits * row_blocks * KV * n_seq, clusters of `splits` along x;
// row_blocks: blocks of 16 MB rows of the longest sequence.
template <int DP, int MB, int W>
__global__ void __launch_bounds__(32 * W)
attn_few_kernel(const AttnParams p, const int splits, const int row_blocks) {
  constexpr int ROWS = 16 * MB, RB = at_row_bytes(DP), KS = DP / 16, NB = DP / 8, OW = DP + 4;
  constexpr int STAGE = 2 * few_keys(DP, MB) * RB;
  constexpr int kFewKeys = few_keys(DP, MB), kFewStages = few_stages(DP, MB);
  extern __shared__ __align__(128) uint8_t at_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_launch_dependents();
  const int split = blockIdx.x % splits;
  int u = blockIdx.x / splits;
  const int block = u % row_blocks;
  u /= row_blocks;
  const int kvh = u % p.KV, group = p.H / p.KV;
  uint8_t* ring = at_smem + warp * kFewStages * STAGE;
  if (p.D < DP)  // the columns of padding between D and DP are zero throughout
    for (int i = lane; i < kFewStages * 2 * kFewKeys * (DP - p.D) / 8; i += 32) {
      const int r = i / ((DP - p.D) / 8), c = i % ((DP - p.D) / 8);
      *reinterpret_cast<uint4*>(ring + r * RB + p.D * 2 + c * 16) = make_uint4(0, 0, 0, 0);
    }
  pdl_wait();
  const AttnSeq s = attn_seq(p, u / p.KV);
  const int tok0 = block * ROWS / group;
  const int64_t all = static_cast<int64_t>(s.nq) * group - block * ROWS;
  if (all <= 0) return;  // (the whole cluster)
  const int rows = static_cast<int>(min(all, static_cast<int64_t>(ROWS)));
  const AtPlace at{tok0, block * ROWS - tok0 * group, rows, group, kvh};
  const int keys = attn_keys(p, s, at.tok(rows - 1));
  const int n = (keys + kFewKeys - 1) / kFewKeys, parts = splits * W, part_at = split * W + warp;
  const int begin = static_cast<int>(static_cast<int64_t>(n) * part_at / parts), end = static_cast<int>(static_cast<int64_t>(n) * (part_at + 1) / parts);
  const uint16_t* kp = p.k + static_cast<int64_t>(s.k0) * p.ldk + kvh * p.k_hs;
  const uint16_t* vp = p.v + static_cast<int64_t>(s.k0) * p.ldv + kvh * p.v_hs;
  const int vecs = p.D / 8;
  const uint32_t ring0 = smem_u32(ring);
  // The tile's 16-byte pieces in the order of memory, one a lane: a warp's request then covers few lines. (Two lanes to a key and
  // 32 bytes at a time needs less arithmetic and is slower, 49 us against 37: every request touches 16 lines.) A piece's successor
  // is 32 pieces on: dr rows and dc pieces, one row more where those pass the row's end.
  const int r_first = lane / vecs, c_first = lane % vecs, dr = 32 / vecs, dc = 32 % vecs;
  const int64_t k_on = dr * p.ldk + dc * 8, k_wrap = k_on + p.ldk - vecs * 8, v_on = dr * p.ldv + dc * 8, v_wrap = v_on + p.ldv - vecs * 8;
  const int dst_on = dr * RB + dc * 16, dst_wrap = dst_on + RB - vecs * 16;
  auto load = [&](int t) {
    uint32_t dst = ring0 + ((t - begin) % kFewStages) * STAGE + r_first * RB + c_first * 16;
    const int64_t row = static_cast<int64_t>(t) * kFewKeys + r_first;
    const uint16_t *ks = kp + row * p.ldk + c_first * 8, *vs = vp + row * p.ldv + c_first * 8;
    int c = c_first, r = r_first;
    const int left = keys - t * kFewKeys;  // keys of this tile
    // rows behind the sequence belong to others: zeros in their place (and the first key's address, which exists)
#pragma unroll 2
    for (int i = 0; i < (vecs * kFewKeys + 31) / 32; ++i) {
      if (kFewKeys % 32 != 0 && r >= kFewKeys) break;
      const bool ok = r < left;
      cp_async_16(dst, ok ? ks : kp, ok);
      cp_async_16(dst + kFewKeys * RB, ok ? vs : vp, ok);
      c += dc;
      const bool wrap = c >= vecs;
      c -= wrap ? vecs : 0;
      r += dr + wrap;
      dst += wrap ? dst_wrap : dst_on;
      ks += wrap ? k_wrap : k_on;
      vs += wrap ? v_wrap : v_on;
    }
  };
#pragma unroll
  for (int i = 0; i < kFewStages; ++i) {
    if (begin + i < end) load(begin + i);
    cp_async_commit();
  }
  AtRows w[MB];
  uint32_t qf[MB][KS][4];
  float o[MB][NB][4], m[MB][2], l[MB][2];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    at_rows<KS>(p, s, at, 16 * b, w[b], qf[b]);
#pragma unroll
    for (int k = 0; k < NB; ++k) o[b][k][0] = o[b][k][1] = o[b][k][2] = o[b][k][3] = 0.0f;
    m[b][0] = m[b][1] = -INFINITY;
    l[b][0] = l[b][1] = 0.0f;
  }
  const int blocks = rows > 16 ? MB : 1;
  for (int t = begin; t < end; ++t) {
    cp_async_wait<kFewStages - 1>();
    __syncwarp();
    const uint32_t kt = ring0 + ((t - begin) % kFewStages) * STAGE, vt = kt + kFewKeys * RB;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      if (b >= blocks) break;
      float sc[kFewKeys / 8][4];
#pragma unroll
      for (int i = 0; i < kFewKeys / 8; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.0f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int n2 = 0; n2 < kFewKeys / 16; ++n2) {
          uint32_t f[4];
          ldsm_x4(kt + (n2 * 16 + (lane & 7) + (lane & 16) / 2) * RB + k * 32 + (lane & 8) * 2, f);
          mma_16816(sc[2 * n2], qf[b][k], f[0], f[1]);
          mma_16816(sc[2 * n2 + 1], qf[b][k], f[2], f[3]);
        }
      float mx[2] = {m[b][0], m[b][1]}, sub[2];
      at_scores(p, w[b], t * kFewKeys + (lane & 3) * 2, (t + 1) * kFewKeys, sc, mx);
      if (__any_sync(0xFFFFFFFFu, mx[0] != m[b][0] || mx[1] != m[b][1])) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float alpha = ex2(m[b][e] - (mx[e] == -INFINITY ? 0.0f : mx[e]));
          m[b][e] = mx[e];
          l[b][e] *= alpha;
#pragma unroll
          for (int k = 0; k < NB; ++k) {
            o[b][k][2 * e] *= alpha;
            o[b][k][2 * e + 1] *= alpha;
          }
        }
      }
      sub[0] = mx[0] == -INFINITY ? 0.0f : mx[0];  // (no key in sight so far)
      sub[1] = mx[1] == -INFINITY ? 0.0f : mx[1];
      // P rounded to bf16 (the operand's type; relative to the largest weight of the row, half a step is 2^-9)
#pragma unroll
      for (int n2 = 0; n2 < kFewKeys / 16; ++n2) {
        uint32_t pf[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float(&x)[4] = sc[2 * n2 + h];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = ex2(x[i] - sub[i >> 1]);
            l[b][i >> 1] += x[i];
          }
          pf[2 * h] = pack_bf16(x[0], x[1]);
          pf[2 * h + 1] = pack_bf16(x[2], x[3]);
        }
#pragma unroll
        for (int d2 = 0; d2 < DP / 16; ++d2) {
          uint32_t f[4];
          ldsm_x4_t(vt + (n2 * 16 + (lane & 15)) * RB + d2 * 32 + (lane & 16), f);
          mma_16816(o[b][2 * d2], pf, f[0], f[1]);
          mma_16816(o[b][2 * d2 + 1], pf, f[2], f[3]);
        }
      }
    }
    __syncwarp();  // (all lanes have read the stage)
    if (t + kFewStages < end) load(t + kFewStages);
    cp_async_commit();
  }
  cp_async_wait<0>();
  __syncthreads();  // ---- join: the CTA's warps, then the cluster's CTAs ----
  float* part = reinterpret_cast<float*>(at_smem);  // [W][ROWS][OW]: O, then m and l
  float* joined = part + W * ROWS * OW;             // [ROWS][OW]
#pragma unroll
  for (int b = 0; b < MB; ++b) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      l[b][e] += __shfl_xor_sync(0xFFFFFFFFu, l[b][e], 1);
      l[b][e] += __shfl_xor_sync(0xFFFFFFFFu, l[b][e], 2);
      float* mine = part + static_cast<size_t>(warp * ROWS + 16 * b + (lane >> 2) + 8 * e) * OW;
#pragma unroll
      for (int k = 0; k < NB; ++k) *reinterpret_cast<float2*>(mine + k * 8 + (lane & 3) * 2) = make_float2(o[b][k][2 * e], o[b][k][2 * e + 1]);
      if ((lane & 3) == 0) *reinterpret_cast<float2*>(mine + DP) = make_float2(m[b][e], l[b][e]);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * (DP / 4); i += 32 * W) {
    const int r = i / (DP / 4), c = i % (DP / 4);
    float mm = -INFINITY, ll = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < W; ++k) mm = fmaxf(mm, part[(k * ROWS + r) * OW + DP]);
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float* pr = part + (k * ROWS + r) * OW;
      const float f = mm == -INFINITY ? 0.0f : ex2(pr[DP] - mm);
      ll = fmaf(pr[DP + 1], f, ll);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(pr[4 * c + j], f, acc[j]);
    }
    if (splits == 1) {
      const float inv = ll != 0.0f ? __fdiv_rn(1.0f, ll) : 0.0f;  // (no key in sight: O is zero too)
      if (4 * c < p.D)
        *reinterpret_cast<uint2*>(at_out(p, s, at, r) + 4 * c) =
            make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
    } else {
      *reinterpret_cast<float4*>(joined + r * OW + 4 * c) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      if (c == 0) *reinterpret_cast<float2*>(joined + r * OW + DP) = make_float2(mm, ll);
    }
  }
  if (splits == 1) return;
  __syncwarp();
  cluster_sync();
  for (int i = threadIdx.x + 32 * W * split; i < rows * (DP / 2); i += 32 * W * splits) {
    const int r = i / (DP / 2), c = i % (DP / 2);
    if (2 * c >= p.D) continue;
    float pm[kAtMaxSplits], pl[kAtMaxSplits], a0[kAtMaxSplits], a1[kAtMaxSplits], mm = -INFINITY;
#pragma unroll
    for (int k = 0; k < kAtMaxSplits; ++k) {  // (all on their way at once)
      if (k >= splits) break;
      const uint32_t from = map_to_cta(joined + r * OW, k);
      ld_cluster_f32x2(from + DP * 4, pm[k], pl[k]);
      ld_cluster_f32x2(from + 8 * c, a0[k], a1[k]);
    }
#pragma unroll
    for (int k = 0; k < kAtMaxSplits; ++k)
      if (k < splits) mm = fmaxf(mm, pm[k]);
    float ll = 0.0f, x0 = 0.0f, x1 = 0.0f;
#pragma unroll
    for (int k = 0; k < kAtMaxSplits; ++k)
      if (k < splits) {
        const float f = mm == -INFINITY ? 0.0f : ex2(pm[k] - mm);
        ll = fmaf(pl[k], f, ll);
        x0 = fmaf(a0[k], f, x0);
        x1 = fmaf(a1[k], f, x1);
      }
    const float inv = ll != 0.0f ? __fdiv_rn(1.0f, ll) : 0.0f;
    *reinterpret_cast<uint32_t*>(at_out(p, s, at, r) + 2 * c) = pack_bf16(x0 * inv, x1 * inv);
  }
  __syncwarp();
  cluster_sync();  // nobody leaves while its partial sums are read
}

// 64 rows by four warps of 16, which share 64-key tiles. grid.x = (row tiles of the longest sequence) * KV * n_seq.
template <int DP>
__global__ void __launch_bounds__(kAtThreads)
attn_rows_kernel(const AttnParams p, const int tiles) {
  constexpr int ROWS = 64, RB = at_row_bytes(DP), KS = DP / 16, NB = DP / 8;
  extern __shared__ __align__(128) uint8_t at_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_launch_dependents();
  int u = blockIdx.x;
  const int tile = u % tiles;
  u /= tiles;
  const int kvh = u % p.KV, group = p.H / p.KV;
  if (p.D < DP)  // the columns of padding between D and DP are zero throughout
    for (int i = threadIdx.x; i < kAtStages * 2 * kAtKeys * (DP - p.D) / 8; i += kAtThreads) {
      const int r = i / ((DP - p.D) / 8), c = i % ((DP - p.D) / 8);
      *reinterpret_cast<uint4*>(at_smem + r * RB + p.D * 2 + c * 16) = make_uint4(0, 0, 0, 0);
    }
  pdl_wait();
  const AttnSeq s = attn_seq(p, u / p.KV);
  const int64_t rows = static_cast<int64_t>(s.nq) * group;
  const int64_t row0 = static_cast<int64_t>(tile) * ROWS;
  if (row0 >= rows) return;
  const int tok0 = static_cast<int>(row0 / group);
  const AtPlace at{tok0, static_cast<int>(row0 - static_cast<int64_t>(tok0) * group), static_cast<int>(min(rows - row0, static_cast<int64_t>(ROWS))), group, kvh};
  const int keys = attn_keys(p, s, at.tok(at.left - 1));
  const int n_tiles = (keys + kAtKeys - 1) / kAtKeys;
  const uint16_t* kp = p.k + static_cast<int64_t>(s.k0) * p.ldk + kvh * p.k_hs;
  const uint16_t* vp = p.v + static_cast<int64_t>(s.k0) * p.ldv + kvh * p.v_hs;
  const int vecs = p.D / 8;
  const uint32_t smem0 = smem_u32(at_smem);
  auto load = [&](int t) {
    const uint32_t dst = smem0 + (t % kAtStages) * at_stage_bytes(DP);
    for (int i = threadIdx.x; i < kAtKeys * vecs; i += kAtThreads) {
      const int r = i / vecs, c = i - r * vecs;
      const int64_t key = static_cast<int64_t>(t) * kAtKeys + r;
      const bool ok = key < keys;  // rows behind the sequence belong to others: zeros in their place
      const int64_t kk = ok ? key : 0;
      cp_async_16(dst + r * RB + c * 16, kp + kk * p.ldk + c * 8, ok);
      cp_async_16(dst + (kAtKeys + r) * RB + c * 16, vp + kk * p.ldv + c * 8, ok);
    }
  };
#pragma unroll
  for (int i = 0; i < kAtStages - 1; ++i) {
    if (i < n_tiles) load(i);
    cp_async_commit();
  }
  AtRows w;
  uint32_t qf[KS][4];
  at_rows<KS>(p, s, at, warp * 16, w, qf);
  float o[NB][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int k = 0; k < NB; ++k) o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.0f;
  for (int t = 0; t < n_tiles; ++t) {
    cp_async_wait<kAtStages - 2>();
    __syncthreads();
    if (t + kAtStages - 1 < n_tiles) load(t + kAtStages - 1);
    cp_async_commit();
    const uint32_t kt = smem0 + (t % kAtStages) * at_stage_bytes(DP), vt = kt + kAtKeys * RB;
    float sc[kAtKeys / 8][4];
#pragma unroll
    for (int i = 0; i < kAtKeys / 8; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.0f;
    // S = Q K^T: a 16 x 16 matrix of K holds the fragments of two 8-key blocks
#pragma unroll
    for (int n2 = 0; n2 < kAtKeys / 16; ++n2)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t f[4];
        ldsm_x4(kt + (n2 * 16 + (lane & 7) + (lane & 16) / 2) * RB + k * 32 + (lane & 8) * 2, f);
        mma_16816(sc[2 * n2], qf[k], f[0], f[1]);
        mma_16816(sc[2 * n2 + 1], qf[k], f[2], f[3]);
      }
    float mx[2] = {m[0], m[1]}, sub[2];
    at_scores(p, w, t * kAtKeys + (lane & 3) * 2, (t + 1) * kAtKeys, sc, mx);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      sub[e] = mx[e] == -INFINITY ? 0.0f : mx[e];  // (no key in sight so far)
      const float alpha = ex2(m[e] - sub[e]);
      m[e] = mx[e];
      l[e] *= alpha;
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        o[k][2 * e] *= alpha;
        o[k][2 * e + 1] *= alpha;
      }
    }
#pragma unroll
    for (int n2 = 0; n2 < kAtKeys / 16; ++n2) {
      uint32_t pf[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float(&x)[4] = sc[2 * n2 + h];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = ex2(x[i] - sub[i >> 1]);
          l[i >> 1] += x[i];
        }
        pf[2 * h] = pack_bf16(x[0], x[1]);
        pf[2 * h + 1] = pack_bf16(x[2], x[3]);
      }
#pragma unroll
      for (int d2 = 0; d2 < DP / 16; ++d2) {
        uint32_t f[4];
        ldsm_x4_t(vt + (n2 * 16 + (lane & 15)) * RB + d2 * 32 + (lane & 16), f);
        mma_16816(o[2 * d2], pf, f[0], f[1]);
        mma_16816(o[2 * d2 + 1], pf, f[2], f[3]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 1);
    l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 2);
    const int row = warp * 16 + (lane >> 2) + 8 * e;
    if (row >= at.left) continue;
    uint16_t* yr = at_out(p, s, at, row);
    const float inv = l[e] != 0.0f ? __fdiv_rn(1.0f, l[e]) : 0.0f;  // (no key in sight: O is zero too)
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int col = k * 8 + (lane & 3) * 2;
      if (col < p.D) *reinterpret_cast<uint32_t*>(yr + col) = pack_bf16(o[k][2 * e] * inv, o[k][2 * e + 1] * inv);
    }
  }
}

// ---- host side -------------------------------------------------------------------------------------
template <int DP>
constexpr size_t at_rows_smem() { return static_cast<size_t>(kAtStages) * at_stage_bytes(DP); }
template <int DP, int MB, int W>
constexpr size_t at_few_smem() {
  constexpr size_t ring = W * static_cast<size_t>(few_stages(DP, MB)) * 2 * few_keys(DP, MB) * at_row_bytes(DP);
  constexpr size_t join = (W + 1) * static_cast<size_t>(16 * MB) * (DP + 4) * 4;
  return ring > join ? ring : join;
}
constexpr int at_width(int dp) { return dp == 32 ? 0 : dp == 64 ? 1 : dp == 80 ? 2 : dp == 96 ? 3 : 4; }  // of AttnLimits
// The clusters of 1 .. 8 CTAs that the device holds at once (a cluster stays within a group of 16 to 18 SMs).
template <int DP, int MB, int W>
static cudaError_t at_few_init(AttnLimits* limits) {
  cudaError_t e = cudaFuncSetAttribute(attn_few_kernel<DP, MB, W>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(at_few_smem<DP, MB, W>()));
  for (int splits = 1; splits <= kAtMaxSplits && e == cudaSuccess; ++splits) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(splits * 1024));
    cfg.blockDim = dim3(32 * W);
    cfg.dynamicSmemBytes = at_few_smem<DP, MB, W>();
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(splits);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&limits->few[at_width(DP)][MB - 1][W == 8][splits], attn_few_kernel<DP, MB, W>, &cfg);
  }
  return e;
}
template <int DP>
static int at_init(AttnLimits* limits) {
  DP_CUDA_OK(cudaFuncSetAttribute(attn_rows_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(at_rows_smem<DP>())));
  DP_CUDA_OK((at_few_init<DP, 1, 4>(limits)));
  DP_CUDA_OK((at_few_init<DP, 2, 4>(limits)));
  DP_CUDA_OK((at_few_init<DP, 1, 8>(limits)));
  DP_CUDA_OK((at_few_init<DP, 2, 8>(limits)));
  return DP_OK;
}
int attn_init_device(AttnLimits* limits) {
  int st = at_init<32>(limits);
  if (st == DP_OK) st = at_init<64>(limits);
  if (st == DP_OK) st = at_init<80>(limits);
  if (st == DP_OK) st = at_init<96>(limits);
  if (st == DP_OK) st = at_init<128>(limits);
  return st;
}

template <int DP, int MB, int W>
static cudaError_t launch_few(const AttnParams& p, int64_t units, int row_blocks, cudaStream_t stream, bool pdl) {
  // Each unit's keys over as many CTAs, up to eight, as all run at once, and as long as a warp has a tile of keys. (Six CTAs to each of 48
  // units, for which there are SMs but no places: 3 sequences of 16 x 72, 8192 keys 39.6 us, 26.1 by five; and with three
  // to each of 80, which fit, 39.1 us, by two 51.2.)
  const int64_t tiles_of_keys = (static_cast<int64_t>(p.max_k) + 31) / 32;
  int splits = static_cast<int>(tiles_of_keys / W < kAtMaxSplits ? tiles_of_keys / W : kAtMaxSplits);
  const AttnLimits* limits = attn_limits();
  while (splits > 1 && limits != nullptr && limits->few[at_width(DP)][MB - 1][W == 8][splits] < units) --splits;
  splits = splits < 1 ? 1 : splits;
  return launch_cluster(attn_few_kernel<DP, MB, W>, dim3(static_cast<unsigned>(units * splits)), dim3(32 * W), at_few_smem<DP, MB, W>(),
                        stream, pdl, static_cast<unsigned>(splits), p, splits, row_blocks);
}
// tiles: of attn_rows_kernel; 0: attn_few_kernel.
template <int DP>
static cudaError_t launch_at(const AttnParams& p, int64_t units, int64_t tiles, int64_t rows, cudaStream_t stream, bool pdl) {
  if (tiles > 0)
    return launch(attn_rows_kernel<DP>, dim3(static_cast<unsigned>(units)), dim3(kAtThreads), at_rows_smem<DP>(), stream, pdl, p,
                  static_cast<int>(tiles));
  // CTAs of eight warps where there are only a few units (4 of 128, 8192 keys: 18.5 us by four warps, 15.4 by eight; 16 of 72: 17.5
  // and 22, since clusters of eight whole SMs are hard to place).
  const bool wide = units <= 8;
  if (rows <= 16) return wide ? launch_few<DP, 1, 8>(p, units, 1, stream, pdl) : launch_few<DP, 1, 4>(p, units, 1, stream, pdl);
  const int blocks = static_cast<int>((rows + 31) / 32);
  return wide ? launch_few<DP, 2, 8>(p, units, blocks, stream, pdl) : launch_few<DP, 2, 4>(p, units, blocks, stream, pdl);
}

static int64_t few_units(const AttnParams& p) {  // blocks of 32 rows of a key head
  return attn_product(attn_product((static_cast<int64_t>(p.max_q) * (p.H / p.KV) + 31) / 32, p.KV), p.n_seq);
}
// Whether the keys are cut over clusters, for blocks of 32 rows: always where there is one, and of more where that makes few units of long
// contexts, which would leave the tcgen05 kernel's tiles of 128 on few SMs. (From 769 keys on and up to 64 units, 40 of more than 96 columns. 16 heads of
// 72, one sequence: 128 queries = 64 units, 1024 / 4096 keys 14 / 27 us against 15 / 40 on tcgen05, 256 queries 19 / 43 against 15 / 40; 512 keys 11 and 12; heads
// of 128, 100 queries: 32 units 14 / 27 against 15 / 38, 64 units 18 / 40 against 15 / 38.)
// With a tile of keys or less there is nothing to cut: the kernel whose warps share it (256 sequences of 32, 16 heads of 72: 48 us
// against 87).
bool attn_cuts_keys(const AttnParams& p) {
  const int64_t rows = static_cast<int64_t>(p.max_q) * (p.H / p.KV);
  return p.max_k > kAtKeys && (rows <= 32 || (p.max_k > 768 && few_units(p) <= (p.D <= 96 ? 64 : 40)));
}

int launch_attn_rows(const AttnParams& p, cudaStream_t stream, bool pdl) {
  const int64_t rows = static_cast<int64_t>(p.max_q) * (p.H / p.KV);
  const bool few = attn_cuts_keys(p);
  const int64_t tiles = few ? 0 : (rows + 63) / 64, units = few ? few_units(p) : attn_product(attn_product(tiles, p.KV), p.n_seq);
  if (units > (few ? 0x7FFFFFFF / kAtMaxSplits : 0x7FFFFFFF) || tiles > 0x7FFFFFFF)
    return fail(DP_ERR_SHAPE, "attention: %lld tiles of queries", (long long)units);
  const cudaError_t e = p.D <= 32   ? launch_at<32>(p, units, tiles, rows, stream, pdl)
                        : p.D <= 64 ? launch_at<64>(p, units, tiles, rows, stream, pdl)
                        : p.D <= 80 ? launch_at<80>(p, units, tiles, rows, stream, pdl)
                        : p.D <= 96 ? launch_at<96>(p, units, tiles, rows, stream, pdl)
                                    : launch_at<128>(p, units, tiles, rows, stream, pdl);
  if (e != cudaSuccess) return fail(DP_ERR_CUDA, "attention launch failed: %s", cudaGetErrorString(e));
  return DP_OK;
}

}  // namespace dp
