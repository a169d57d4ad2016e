// Attention of few queries (and of any number, as the plain form of the kernel in attn_tc.cu): mma.sync tiles of 16 queries,
// one pass over the keys with a running maximum and sum.
//
//   t_ij = scale q_i . k_j, capped by a tanh, less slope |pos(i) - j|;   y_i = sum_j softmax_j(t_ij) v_j
//
// A row is a (query, head) pair: the heads / kv_heads heads that read one key head stand beside each other, so keys and values
// are read once for all of them. Few rows make this a stream of K and V (one query, 16 heads of 72: 4 operations a byte), so
// what counts is bytes in flight: 64-key tiles through a ring of cp.async stages, three CTAs or more to an SM, and the keys of
// a sequence cut over the CTAs of a cluster, whose partial sums (m, l, O) meet in distributed shared memory: one launch, no
// scratch memory. WR warps of a CTA stand beside each other in rows, 4 / WR split a tile's keys.
#include <cuda_bf16.h>

#include "attn.cuh"
#include "dp_internal.h"

namespace dp {

constexpr int kAtThreads = 128, kAtKeys = 64;
constexpr int kAtMaxSplits = 16;  // CTAs of a cluster

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
__device__ __forceinline__ float ld_cluster_f32(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// grid.x = splits * (row tiles of the longest sequence) * KV * n_seq, clusters of `splits` along x.
template <int DP, int WR>
__global__ void __launch_bounds__(kAtThreads)
attn_rows_kernel(const AttnParams p, const int tiles, const int splits) {
  constexpr int KW = 4 / WR, ROWS = 16 * WR, KPW = kAtKeys / KW;  // keys of a tile that a warp takes
  constexpr int RB = at_row_bytes(DP), KS = DP / 16, NB = DP / 8;
  constexpr int OW = DP + 4;  // floats between rows of a partial sum: O, then m and l
  extern __shared__ __align__(128) uint8_t at_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wr = warp / KW, wk = warp % KW;
  pdl_launch_dependents();
  int u = blockIdx.x / splits;
  const int split = blockIdx.x % splits;
  const int tile = u % tiles;
  u /= tiles;
  const int kvh = u % p.KV, seq = u / p.KV;
  const int group = p.H / p.KV;
  // the columns of padding between D and DP are zero throughout
  if (p.D < DP)
    for (int i = threadIdx.x; i < kAtStages * 2 * kAtKeys * (DP - p.D) / 8; i += kAtThreads) {
      const int r = i / ((DP - p.D) / 8), c = i % ((DP - p.D) / 8);
      *reinterpret_cast<uint4*>(at_smem + r * RB + p.D * 2 + c * 16) = make_uint4(0, 0, 0, 0);
    }
  pdl_wait();
  const AttnSeq s = attn_seq(p, seq);
  const int64_t rows = static_cast<int64_t>(s.nq) * group;
  const int64_t row0 = static_cast<int64_t>(tile) * ROWS;
  if (row0 >= rows) return;  // (the whole cluster)
  const int last = static_cast<int>(min(row0 + ROWS, rows) - 1) / group;
  const int keys = attn_keys(p, s, last);
  const int n_tiles = (keys + kAtKeys - 1) / kAtKeys;
  // this CTA's part of the key tiles
  const int t_begin = static_cast<int>(static_cast<int64_t>(n_tiles) * split / splits);
  const int t_end = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / splits);
  const uint16_t* kp = p.k + static_cast<int64_t>(s.k0) * p.ldk + kvh * p.k_hs;
  const uint16_t* vp = p.v + static_cast<int64_t>(s.k0) * p.ldv + kvh * p.v_hs;
  const int vecs = p.D / 8;
  const uint32_t smem0 = smem_u32(at_smem);
  auto load = [&](int t) {
    const int stage = (t - t_begin) % kAtStages;
    const uint32_t dst = smem0 + stage * at_stage_bytes(DP);
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
    if (t_begin + i < t_end) load(t_begin + i);
    cp_async_commit();
  }
  // ---- this warp's 16 rows: fragment rows lane / 4 and lane / 4 + 8 ----
  int tok[2], pos[2];
  float slope[2] = {0.0f, 0.0f};
  uint32_t qf[KS][4];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int64_t row = row0 + wr * 16 + (lane >> 2) + 8 * e;
    const bool live = row < rows;
    tok[e] = live ? static_cast<int>(row / group) : -1;
    const int head = kvh * group + (live ? static_cast<int>(row % group) : 0);
    pos[e] = tok[e] + s.behind;
    if (p.slopes != nullptr) slope[e] = ld_global_f32(p.slopes + head) * kLog2e;
    const uint16_t* qr = p.q + static_cast<int64_t>(s.q0 + (live ? tok[e] : 0)) * p.ldq + head * p.q_hs;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int col = k * 16 + c * 8 + (lane & 3) * 2;
        qf[k][2 * c + e] = live && col < p.D ? static_cast<uint32_t>(ld_global_s32(reinterpret_cast<const int32_t*>(qr + col))) : 0u;
      }
  }
  float o[NB][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int n = 0; n < NB; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;

  for (int t = t_begin; t < t_end; ++t) {
    cp_async_wait<kAtStages - 2>();
    __syncthreads();
    if (t + kAtStages - 1 < t_end) load(t + kAtStages - 1);
    cp_async_commit();
    const uint32_t kt = smem0 + ((t - t_begin) % kAtStages) * at_stage_bytes(DP);
    const uint32_t vt = kt + kAtKeys * RB;
    float sc[KPW / 8][4];
#pragma unroll
    for (int n = 0; n < KPW / 8; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.0f;
    // S = Q K^T: a 16 x 16 matrix of K holds the fragments of two 8-key blocks
#pragma unroll
    for (int n2 = 0; n2 < KPW / 16; ++n2)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t b[4];
        const int row = wk * KPW + n2 * 16 + (lane & 7) + (lane & 16) / 2;
        ldsm_x4(kt + row * RB + k * 32 + (lane & 8) * 2, b);
        mma_16816(sc[2 * n2], qf[k], b[0], b[1]);
        mma_16816(sc[2 * n2 + 1], qf[k], b[2], b[3]);
      }
    const int key0 = t * kAtKeys + wk * KPW + (lane & 3) * 2;
    float mx[2] = {m[0], m[1]};
#pragma unroll
    for (int n = 0; n < KPW / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = i >> 1, key = key0 + n * 8 + (i & 1);
        float x = p.cap != 0.0f ? capped(p.cap, sc[n][i] * p.scale_by_cap) : sc[n][i] * p.scale;
        if (p.slopes != nullptr) x = fmaf(-slope[e], fabsf(static_cast<float>(pos[e] - key)), x);
        if (key >= keys || (p.causal && key > pos[e] && key >= s.prefix)) x = -INFINITY;
        sc[n][i] = x;
        mx[e] = fmaxf(mx[e], x);
      }
    float alpha[2], sub[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xFFFFFFFFu, mx[e], 1));
      mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xFFFFFFFFu, mx[e], 2));
      sub[e] = mx[e] == -INFINITY ? 0.0f : mx[e];  // (no key in sight so far)
      alpha[e] = ex2(m[e] - sub[e]);
      m[e] = mx[e];
      l[e] *= alpha[e];
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      o[n][0] *= alpha[0];
      o[n][1] *= alpha[0];
      o[n][2] *= alpha[1];
      o[n][3] *= alpha[1];
    }
    // O += P V, P rounded to bf16 (the operand's type; relative to the largest weight of the row, half a step is 2^-9)
#pragma unroll
    for (int n2 = 0; n2 < KPW / 16; ++n2) {
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
        uint32_t b[4];
        const int row = wk * KPW + n2 * 16 + (lane & 15);
        ldsm_x4_t(vt + row * RB + d2 * 32 + (lane & 16), b);
        mma_16816(o[2 * d2], pf, b[0], b[1]);
        mma_16816(o[2 * d2 + 1], pf, b[2], b[3]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 1);
    l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 2);
  }
  if (KW == 1 && splits == 1) {  // nothing to join
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t row = row0 + wr * 16 + (lane >> 2) + 8 * e;
      if (row >= rows) continue;
      const int head = kvh * group + static_cast<int>(row % group);
      uint16_t* yr = p.y + static_cast<int64_t>(s.q0 + tok[e]) * p.ldy + head * p.y_hs;
      const float inv = l[e] != 0.0f ? __fdiv_rn(1.0f, l[e]) : 0.0f;  // (no key in sight: O is zero too)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int col = n * 8 + (lane & 3) * 2;
        if (col < p.D) *reinterpret_cast<uint32_t*>(yr + col) = pack_bf16(o[n][2 * e] * inv, o[n][2 * e + 1] * inv);
      }
    }
    return;
  }
  // ---- join: the warps that shared a tile's keys, then the cluster's CTAs ----
  cp_async_wait<0>();
  __syncthreads();
  float* part = reinterpret_cast<float*>(at_smem);  // [KW][ROWS][OW]
  float* joined = part + KW * ROWS * OW;            // [ROWS][OW]
  {
    float* mine = part + static_cast<size_t>(wk * ROWS + wr * 16 + (lane >> 2)) * OW;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      *reinterpret_cast<float2*>(mine + n * 8 + (lane & 3) * 2) = make_float2(o[n][0], o[n][1]);
      *reinterpret_cast<float2*>(mine + 8 * OW + n * 8 + (lane & 3) * 2) = make_float2(o[n][2], o[n][3]);
    }
    if ((lane & 3) == 0) {
      *reinterpret_cast<float2*>(mine + DP) = make_float2(m[0], l[0]);
      *reinterpret_cast<float2*>(mine + 8 * OW + DP) = make_float2(m[1], l[1]);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < ROWS * (DP / 4); i += kAtThreads) {
    const int r = i / (DP / 4), c = i % (DP / 4);
    float mm = -INFINITY, ll = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < KW; ++w) mm = fmaxf(mm, part[(w * ROWS + r) * OW + DP]);
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const float* pr = part + (w * ROWS + r) * OW;
      const float f = mm == -INFINITY ? 0.0f : ex2(pr[DP] - mm);
      ll = fmaf(pr[DP + 1], f, ll);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(pr[4 * c + j], f, acc[j]);
    }
    if (splits == 1) {
      const int64_t row = row0 + r;
      if (row < rows && 4 * c < p.D) {
        const int head = kvh * group + static_cast<int>(row % group);
        const float inv = ll != 0.0f ? __fdiv_rn(1.0f, ll) : 0.0f;
        uint16_t* yr = p.y + static_cast<int64_t>(s.q0 + static_cast<int>(row / group)) * p.ldy + head * p.y_hs;
        *reinterpret_cast<uint2*>(yr + 4 * c) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
      }
    } else {
      *reinterpret_cast<float4*>(joined + r * OW + 4 * c) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      if (c == 0) *reinterpret_cast<float2*>(joined + r * OW + DP) = make_float2(mm, ll);
    }
  }
  if (splits == 1) return;
  cluster_sync();
  for (int i = threadIdx.x + kAtThreads * split; i < ROWS * (DP / 2); i += kAtThreads * splits) {
    const int r = i / (DP / 2), c = i % (DP / 2);
    const int64_t row = row0 + r;
    if (row >= rows || 2 * c >= p.D) continue;
    float mm = -INFINITY, ll = 0.0f, a0 = 0.0f, a1 = 0.0f;
    for (int w = 0; w < splits; ++w) mm = fmaxf(mm, ld_cluster_f32(map_to_cta(joined + r * OW + DP, w)));
    if (mm != -INFINITY)
      for (int w = 0; w < splits; ++w) {
        const uint32_t from = map_to_cta(joined + r * OW, w);
        const float f = ex2(ld_cluster_f32(from + DP * 4) - mm);
        ll = fmaf(ld_cluster_f32(from + DP * 4 + 4), f, ll);
        a0 = fmaf(ld_cluster_f32(from + 8 * c), f, a0);
        a1 = fmaf(ld_cluster_f32(from + 8 * c + 4), f, a1);
      }
    const int head = kvh * group + static_cast<int>(row % group);
    const float inv = ll != 0.0f ? __fdiv_rn(1.0f, ll) : 0.0f;
    uint16_t* yr = p.y + static_cast<int64_t>(s.q0 + static_cast<int>(row / group)) * p.ldy + head * p.y_hs;
    *reinterpret_cast<uint32_t*>(yr + 2 * c) = pack_bf16(a0 * inv, a1 * inv);
  }
  cluster_sync();  // nobody leaves while its partial sums are read
}

// ---- host side -------------------------------------------------------------------------------------
template <int DP, int WR>
constexpr size_t at_smem_bytes() {
  constexpr size_t ring = static_cast<size_t>(kAtStages) * at_stage_bytes(DP);
  constexpr size_t join = static_cast<size_t>(4 / WR + 1) * 16 * WR * (DP + 4) * 4;
  return ring > join ? ring : join;
}
template <int DP, int WR>
static cudaError_t at_init() {
  cudaError_t e = cudaFuncSetAttribute(attn_rows_kernel<DP, WR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(at_smem_bytes<DP, WR>()));
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(attn_rows_kernel<DP, WR>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
}
int attn_init_device() {
  DP_CUDA_OK((at_init<32, 1>()));
  DP_CUDA_OK((at_init<64, 1>()));
  DP_CUDA_OK((at_init<80, 1>()));
  DP_CUDA_OK((at_init<96, 1>()));
  DP_CUDA_OK((at_init<128, 1>()));
  DP_CUDA_OK((at_init<32, 4>()));
  DP_CUDA_OK((at_init<64, 4>()));
  DP_CUDA_OK((at_init<80, 4>()));
  DP_CUDA_OK((at_init<96, 4>()));
  DP_CUDA_OK((at_init<128, 4>()));
  return DP_OK;
}

template <int DP, int WR>
static cudaError_t launch_at(const AttnParams& p, unsigned grid, int tiles, int splits, cudaStream_t stream, bool pdl) {
  return launch_cluster(attn_rows_kernel<DP, WR>, dim3(grid), dim3(kAtThreads), at_smem_bytes<DP, WR>(), stream, pdl,
                        static_cast<unsigned>(splits), p, tiles, splits);
}
template <int WR>
static cudaError_t launch_at_d(const AttnParams& p, unsigned grid, int tiles, int splits, cudaStream_t stream, bool pdl) {
  return p.D <= 32   ? launch_at<32, WR>(p, grid, tiles, splits, stream, pdl)
         : p.D <= 64 ? launch_at<64, WR>(p, grid, tiles, splits, stream, pdl)
         : p.D <= 80 ? launch_at<80, WR>(p, grid, tiles, splits, stream, pdl)
         : p.D <= 96 ? launch_at<96, WR>(p, grid, tiles, splits, stream, pdl)
                     : launch_at<128, WR>(p, grid, tiles, splits, stream, pdl);
}

int launch_attn_rows(const AttnParams& p, cudaStream_t stream, bool pdl) {
  const int64_t rows = static_cast<int64_t>(p.max_q) * (p.H / p.KV);
  const bool few = rows <= 16;
  const int64_t tiles = few ? 1 : (rows + 63) / 64;
  const int64_t units = tiles * p.KV * p.n_seq;
  // Keys are split until the grid fills the SMs, as long as a part has two tiles of keys or more.
  int splits = 1;
  const int64_t key_tiles = (static_cast<int64_t>(p.max_k) + kAtKeys - 1) / kAtKeys;
  while (splits < kAtMaxSplits && units * splits * 2 <= 4 * num_sms() && key_tiles >= 4 * splits) splits *= 2;
  if (units * splits > 0x7FFFFFFF || tiles > 0x7FFFFFFF)
    return fail(DP_ERR_SHAPE, "attention: %lld tiles of queries", (long long)units);
  const unsigned grid = static_cast<unsigned>(units * splits);
  const cudaError_t e = few ? launch_at_d<1>(p, grid, static_cast<int>(tiles), splits, stream, pdl)
                            : launch_at_d<4>(p, grid, static_cast<int>(tiles), splits, stream, pdl);
  if (e != cudaSuccess) return fail(DP_ERR_CUDA, "attention launch failed: %s", cudaGetErrorString(e));
  return DP_OK;
}

}  // namespace dp
