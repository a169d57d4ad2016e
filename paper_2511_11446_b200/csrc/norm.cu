// Group normalisation of channels-last feature maps, with an activation, to bf16 or straight to int8 codes for a quantized
// linear.
//
//   x [sample][row][C], G groups of C / G neighbouring channels; over the rows x C / G values of a sample's group
//     mean, var (biased);   h = (x - mean) / sqrt(var + eps) * gamma + beta;   y = act(h)
//
// In front of a U-Net block's projections the paper's method quantizes the activations like any other linear's (Eq. "daq");
// dp_group_norm_daq writes the codes in the pass that would write y.
//
// Statistics first, from one pass over x: sums of d and d^2, d = x - pivot with the group's first value as pivot, so that a
// level far above the spread does not cancel (a constant map gives var = 0 and h = beta exactly). A thread keeps 8 channels
// of every R-th row, sums in fp32 over at most a few thousand values, and a CTA leaves one pair of sums per group; the second
// kernel adds the CTAs' sums in double, in a fixed order, and makes one coefficient pair per channel of them:
//     h = (x - pivot) * a + b,   a = gamma * rstd,   b = beta - (mean - pivot) * a       (x - pivot is exact or nearly so)
#include "daq_device.cuh"

namespace dp {

constexpr int kGnThreads = 256, kGnMaxChunks = 128;

struct GnArgs {
  const uint16_t* x;
  int64_t rows, ldx;  // rows of a sample
  int32_t C, G;
  const uint16_t *gamma, *beta;  // [C] or null
  float eps;
  uint16_t* y;
  int64_t ldy;
  int8_t* q;
  int64_t ldq;
  float* s_a;
  float2* sums;  // [sample][chunk][G]
  int32_t chunks;
  int64_t chunk_rows;
};

__device__ __forceinline__ float gn_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float gn_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float gn_bf16(const uint16_t* p) {
  uint16_t v;
  asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
  return __uint_as_float(static_cast<uint32_t>(v) << 16);
}
__device__ __forceinline__ void gn_unpack(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f[2 * j] = gn_lo(w[j]);
    f[2 * j + 1] = gn_hi(w[j]);
  }
}
template <bool SILU>
__device__ __forceinline__ float gn_act(float h) {
  if constexpr (!SILU) return h;
  return __fdividef(h, 1.0f + __expf(-h));
}

// Threads of a CTA: `lanes` rows of C / 8 vectors at a time.
struct GnThread {
  int vecs, lanes, vec, lane;
  __device__ __forceinline__ explicit GnThread(int C) {
    vecs = C >> 3;
    lanes = blockDim.x / vecs;
    vec = threadIdx.x % vecs;
    lane = threadIdx.x / vecs;  // == lanes: idle
  }
};

__global__ void gn_stats_kernel(const GnArgs a) {
  extern __shared__ float gn_part[];  // [2][lanes][C]
  pdl_launch_dependents();
  const GnThread t(a.C);
  const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int per = a.C / a.G;
  const int64_t r0 = chunk * a.chunk_rows, r1 = min(r0 + a.chunk_rows, a.rows);
  pdl_wait();
  const uint16_t* xs = a.x + sample * a.rows * a.ldx;
  float s[8], ss[8], pivot[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    s[j] = ss[j] = 0.0f;
    pivot[j] = gn_bf16(xs + (t.vec * 8 + j) / per * per);
  }
  if (t.lane < t.lanes) {
    const uint16_t* xp = xs + t.vec * 8;
    for (int64_t r = r0 + t.lane; r < r1; r += t.lanes) {
      uint4 v;
      ld_stream_u32x4(reinterpret_cast<const uint4*>(xp + r * a.ldx), v);
      float f[8];
      gn_unpack(v, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = f[j] - pivot[j];
        s[j] += d;
        ss[j] = fmaf(d, d, ss[j]);
      }
    }
    float* ps = gn_part + t.lane * a.C + t.vec * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      ps[j] = s[j];
      ps[t.lanes * a.C + j] = ss[j];
    }
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, ln = threadIdx.x & 31;
  for (int g = warp; g < a.G; g += blockDim.x >> 5) {
    float u = 0.0f, w = 0.0f;
    for (int i = ln; i < t.lanes * per; i += 32) {
      const int at = i / per * a.C + g * per + i % per;
      u += gn_part[at];
      w += gn_part[t.lanes * a.C + at];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      u += __shfl_xor_sync(0xFFFFFFFFu, u, o);
      w += __shfl_xor_sync(0xFFFFFFFFu, w, o);
    }
    if (ln == 0) a.sums[(static_cast<int64_t>(sample) * a.chunks + chunk) * a.G + g] = make_float2(u, w);
  }
}

// Per group: (pivot, mean - pivot, rstd) into shared memory, from all chunks' sums.
__device__ __forceinline__ void gn_groups(const GnArgs& a, int sample, float* out) {
  const int warp = threadIdx.x >> 5, ln = threadIdx.x & 31, per = a.C / a.G;
  const uint16_t* xs = a.x + sample * a.rows * a.ldx;
  for (int g = warp; g < a.G; g += blockDim.x >> 5) {
    double u = 0.0, w = 0.0;
    for (int c = ln; c < a.chunks; c += 32) {
      float2 v;
      const float2* p = a.sums + (static_cast<int64_t>(sample) * a.chunks + c) * a.G + g;
      asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p) : "memory");
      u += v.x;
      w += v.y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      u += __shfl_xor_sync(0xFFFFFFFFu, u, o);
      w += __shfl_xor_sync(0xFFFFFFFFu, w, o);
    }
    if (ln == 0) {
      const double n = static_cast<double>(a.rows) * per, mean = u / n;
      const double var = fmax(w / n - mean * mean, 0.0);
      out[3 * g] = gn_bf16(xs + g * per);
      out[3 * g + 1] = static_cast<float>(mean);
      out[3 * g + 2] = static_cast<float>(1.0 / sqrt(var + static_cast<double>(a.eps)));
    }
  }
}
// Coefficients of 8 channels.
__device__ __forceinline__ void gn_coefs(const GnArgs& a, const float* groups, int c0, float (&pv)[8], float (&ca)[8],
                                         float (&cb)[8]) {
  const int per = a.C / a.G;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float* g = groups + (c0 + j) / per * 3;
    pv[j] = g[0];
    ca[j] = (a.gamma != nullptr ? gn_bf16(a.gamma + c0 + j) : 1.0f) * g[2];
    cb[j] = fmaf(-g[1], ca[j], a.beta != nullptr ? gn_bf16(a.beta + c0 + j) : 0.0f);
  }
}

template <bool SILU>
__global__ void gn_apply_kernel(const GnArgs a) {
  extern __shared__ float gn_part[];  // [G][3]
  pdl_launch_dependents();
  const GnThread t(a.C);
  const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int64_t r0 = chunk * a.chunk_rows, r1 = min(r0 + a.chunk_rows, a.rows);
  pdl_wait();
  gn_groups(a, sample, gn_part);
  __syncthreads();
  if (t.lane >= t.lanes) return;
  float pv[8], ca[8], cb[8];
  gn_coefs(a, gn_part, t.vec * 8, pv, ca, cb);
  const uint16_t* xp = a.x + sample * a.rows * a.ldx + t.vec * 8;
  uint16_t* yp = a.y + sample * a.rows * a.ldy + t.vec * 8;
  for (int64_t r = r0 + t.lane; r < r1; r += t.lanes) {
    const uint4 v = ld_global_v4(xp + r * a.ldx);
    float f[8];
    gn_unpack(v, f);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float h0 = gn_act<SILU>(fmaf(f[2 * j] - pv[2 * j], ca[2 * j], cb[2 * j]));
      const float h1 = gn_act<SILU>(fmaf(f[2 * j + 1] - pv[2 * j + 1], ca[2 * j + 1], cb[2 * j + 1]));
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(h1), "f"(h0));
    }
    st_global_v4(yp + r * a.ldy, w);
  }
}

// The same to codes: RW warps to a row (each lane up to three vectors), the row's absmax first.
constexpr int kGnVecs = 3;
template <int RW, bool SILU>
__global__ void __launch_bounds__(kGnThreads) gn_codes_kernel(const GnArgs a) {
  constexpr int TPR = 32 * RW, ROWS = kGnThreads / TPR;
  extern __shared__ float gn_part[];  // [G][3]
  __shared__ uint32_t gn_max[2][kGnThreads / 32];
  pdl_launch_dependents();
  const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int64_t r0 = chunk * a.chunk_rows, r1 = min(r0 + a.chunk_rows, a.rows);
  const int warp = threadIdx.x >> 5, rw = threadIdx.x / TPR, lane = threadIdx.x % TPR, vecs = a.C >> 3;
  pdl_wait();
  gn_groups(a, sample, gn_part);
  __syncthreads();
  float pv[kGnVecs][8], ca[kGnVecs][8], cb[kGnVecs][8];
#pragma unroll
  for (int i = 0; i < kGnVecs; ++i)
    if (lane + TPR * i < vecs) gn_coefs(a, gn_part, (lane + TPR * i) * 8, pv[i], ca[i], cb[i]);
  const int64_t m0 = sample * a.rows;
  int it = 0;
  for (int64_t base = r0; base < r1; base += ROWS, it ^= 1) {
    const int64_t r = base + rw;
    const bool live = r < r1;
    float h[kGnVecs][8];
    uint32_t mx = 0;
    if (live) {
      const uint16_t* xr = a.x + (m0 + r) * a.ldx;
#pragma unroll
      for (int i = 0; i < kGnVecs; ++i)
        if (lane + TPR * i < vecs) {
          gn_unpack(ld_global_v4(xr + (lane + TPR * i) * 8), h[i]);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            h[i][j] = gn_act<SILU>(fmaf(h[i][j] - pv[i][j], ca[i][j], cb[i][j]));
            mx = max(mx, __float_as_uint(h[i][j]) & 0x7FFFFFFFu);
          }
        }
    }
    mx = __reduce_max_sync(0xFFFFFFFFu, mx);
    if constexpr (RW > 1) {
      if ((threadIdx.x & 31) == 0) gn_max[it][warp] = mx;
      __syncthreads();  // (two buffers: the next row's maximum is written behind the next barrier's arrival only)
#pragma unroll
      for (int w = 0; w < RW; ++w) mx = max(mx, gn_max[it][rw * RW + w]);
    }
    if (!live) continue;
    const float amax = __uint_as_float(mx);
    float sa = 0.0f, inv = 0.0f;
    if (!(amax < 7.888609052210118e-31f)) {  // 2^-100, as in dp_daq_quantize
      sa = __fdiv_rn(amax, 127.0f);
      inv = __fdiv_rn(127.0f, amax);
    }
    uint2* qr = reinterpret_cast<uint2*>(a.q + (m0 + r) * a.ldq);
#pragma unroll
    for (int i = 0; i < kGnVecs; ++i)
      if (lane + TPR * i < vecs) {
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = __float_as_uint(__fmaf_rn(h[i][j], inv, 12582912.0f));
        qr[lane + TPR * i] = make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                                        __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
      }
    if (lane == 0) a.s_a[m0 + r] = sa;
  }
}

// ---- host side -------------------------------------------------------------------------------------
static int gn_chunks(int64_t samples, int64_t rows) {
  // about four CTAs to an SM, 16 rows or more to each
  int64_t c = (148 * 4 + samples - 1) / samples;
  c = c < 1 ? 1 : c > kGnMaxChunks ? kGnMaxChunks : c;
  const int64_t most = (rows + 15) / 16;
  return static_cast<int>(c < most ? c : most < 1 ? 1 : most);
}
size_t group_norm_workspace(int64_t samples, int64_t rows, int32_t G) {
  if (samples <= 0 || rows <= 0) return 256;
  return (static_cast<size_t>(samples) * gn_chunks(samples, rows) * G * sizeof(float2) + 255) & ~static_cast<size_t>(255);
}

template <bool SILU>
static cudaError_t launch_gn_codes(const GnArgs& a, dim3 grid, size_t smem, cudaStream_t stream) {
  return a.C <= 768     ? launch(gn_codes_kernel<1, SILU>, grid, dim3(kGnThreads), smem, stream, true, a)
         : a.C <= 768 * 2 ? launch(gn_codes_kernel<2, SILU>, grid, dim3(kGnThreads), smem, stream, true, a)
         : a.C <= 768 * 4 ? launch(gn_codes_kernel<4, SILU>, grid, dim3(kGnThreads), smem, stream, true, a)
                       : launch(gn_codes_kernel<8, SILU>, grid, dim3(kGnThreads), smem, stream, true, a);
}

int launch_group_norm(const void* x, int64_t samples, int64_t rows, int32_t C, int64_t ldx, int32_t G, const void* gamma,
                      const void* beta, float eps, bool silu, void* y, int64_t ldy, int8_t* q, int64_t ldq, float* s_a,
                      void* workspace, cudaStream_t stream) {
  GnArgs a{static_cast<const uint16_t*>(x), rows, ldx, C, G, static_cast<const uint16_t*>(gamma),
           static_cast<const uint16_t*>(beta), eps, static_cast<uint16_t*>(y), ldy, q, ldq, s_a,
           static_cast<float2*>(workspace), 0, 0};
  a.chunks = gn_chunks(samples, rows);
  a.chunk_rows = (rows + a.chunks - 1) / a.chunks;
  const int vecs = C / 8, threads = vecs > kGnThreads ? (vecs + 31) / 32 * 32 : kGnThreads;
  const dim3 grid(static_cast<unsigned>(samples * a.chunks));
  const size_t stats_smem = 2 * sizeof(float) * static_cast<size_t>(threads / vecs) * C, smem = 3 * sizeof(float) * static_cast<size_t>(G);
  cudaError_t e = launch(gn_stats_kernel, grid, dim3(threads), stats_smem, stream, true, a);
  if (e == cudaSuccess) {
    if (q != nullptr) e = silu ? launch_gn_codes<true>(a, grid, smem, stream) : launch_gn_codes<false>(a, grid, smem, stream);
    else e = silu ? launch(gn_apply_kernel<true>, grid, dim3(threads), smem, stream, true, a)
                  : launch(gn_apply_kernel<false>, grid, dim3(threads), smem, stream, true, a);
  }
  if (e != cudaSuccess) return fail(DP_ERR_CUDA, "group norm launch failed: %s", cudaGetErrorString(e));
  return DP_OK;
}

}  // namespace dp
