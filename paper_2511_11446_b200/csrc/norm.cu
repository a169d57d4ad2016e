// Group normalisation of channels-last feature maps, with an activation, to bf16 or straight to int8 codes for a quantized
// linear.
//
//   x [sample][row][C], G groups of C / G neighbouring channels; over the rows x C / G values of a sample's group
//     mean, var (biased);   h = (x - mean) / sqrt(var + eps) * gamma + beta;   y = act(h)
//
// In front of a U-Net block's projections the paper's method quantizes the activations like any other linear's (Eq. "daq");
// dp_group_norm_daq writes the codes in the pass that would write y.
//
// Statistics first, as means and sums of squared deviations M2, joined like those of samples (Chan, Golub and LeVeque 1979: two have
// M2 = M2a + M2b + na nb / (na + nb) (mean_a - mean_b)^2), in a fixed order and in fp32. A thread keeps 8 channels of every `lanes`-th row; over
// runs of 24 rows it sums d and d^2, d = x - the run's first value. That value is one of the run's own, so (it - mean)^2 <= M2: neither a
// level nor an outlier cancels more than a factor of 25 in the last bits of M2. The same holds for what joins lanes, channels and
// CTAs about the first of them. (One pivot for the group loses what it is untypical by: level 100, spread 0.5, first value 0, 150 samples of 8192 x
// 320 gave rstd a tenth off.) Means are held less the group's first value, so that a constant map gives var = 0 and h = beta exactly, and
// give each channel
//     h = (x - pivot) * a + b,   a = gamma * rstd,   b = beta - (mean - pivot) * a,   pivot = mean rounded to fp32
//
// Bound by memory: 2 bytes in and 2 (or 1) out per element, if x need not be read twice from it. Two forms:
//  - maps of up to 8 x 64 KB or so a sample: one kernel, a cluster of CTAs to a sample. Each keeps its rows in shared memory while the
//    group sums meet through distributed shared memory; x is read once, and there is one launch.
//  - larger ones: a kernel of sums and one that applies them, which reads x again: from the L2 as far as it is still there, the last
//    rows first. (A few samples at a time, so that all of it is: 16 samples of 16384 x 320, 10 MB each, 140 us by two, 101 by four,
//    103 by eight, 96 all at once: each pair of launches costs more than the second read.)
#include "daq_device.cuh"

namespace dp {

constexpr int kGnMaxThreads = 640;
constexpr int kGnSumUnroll = 6, kGnUnroll = 4;                  // rows that a thread adds while as many are in flight
constexpr int kGnRun = 4 * kGnSumUnroll;                        // rows that it adds about one of them
constexpr int kGnMaxCluster = 8;               // (16, measured: 8 samples of 64 x 640 12.7 us, 6.5 with 8)
constexpr size_t kGnSmem = 113 * 1024;          // of a CTA: two to an SM, one of which reads while the other writes
// (rows in shared memory are one run a thread: more than half of kGnMaxThreads hold 16 bytes of each)
static_assert(kGnSmem / (16 * (kGnMaxThreads / 2 + 1)) < kGnRun, "rows of a thread in shared memory");

struct GnArgs {
  const uint16_t* x;
  int64_t rows, ldx;  // rows of a sample
  int32_t C, G, per;   // per: channels of a group
  uint64_t per_inv;    // ceil(2^32 / per): c / per = c * per_inv >> 32 for c < 2^16 (a division takes twenty instructions)
  const uint16_t *gamma, *beta;  // [C] or null
  float eps;
  float inv_n, inv_rows;  // 1 / values of a group, of a channel
  uint16_t* y;
  int64_t ldy;
  int8_t* q;
  int64_t ldq;
  float* s_a;
  float2* sums;  // [sample][chunk][G]: mean less the group's first value, M2
  int32_t sum_bits, join_bits;  // log2 of the threads that take a group in gn_sums, gn_groups
  int32_t chunks;      // (CTAs of the cluster in the one-kernel form)
  int64_t chunk_rows;
  int32_t out_chunks;  // of the kernel that applies them
  int64_t out_rows;
};

__device__ __forceinline__ uint32_t gn_bits(const uint16_t* p) {
  uint16_t v;
  asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float gn_bf16(const uint16_t* p) { return __uint_as_float(gn_bits(p) << 16); }
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Eight bf16 as four packed fp32 pairs.
__device__ __forceinline__ void gn_unpack(const uint4& v, uint64_t (&f)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = static_cast<uint64_t>(w[j] & 0xFFFF0000u) << 32 | static_cast<uint32_t>(w[j] << 16);
}
// act of a pair. SiLU h / (1 + e^-h): the special-function unit would be the bound at two operations an element (2 x 16 bf16 bytes
// take it as long as they take memory), so a pair shares a reciprocal: 1 / u = v / (uv). Powers end at 2^62, so that products
// stay finite: from h = -43 on the result is h 2^-62 instead of less. Both operations are good to 2^-22.
template <bool SILU>
__device__ __forceinline__ uint64_t gn_act(uint64_t h) {
  if constexpr (!SILU) return h;
  float lo, hi, u, v, r;
  f32x2_unpack(f32x2_mul(h, f32x2_pack(-1.4426950408889634f, -1.4426950408889634f)), lo, hi);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(u) : "f"(fminf(lo, 62.0f)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(v) : "f"(fminf(hi, 62.0f)));
  f32x2_unpack(f32x2_add(f32x2_pack(u, v), f32x2_pack(1.0f, 1.0f)), u, v);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(u * v));
  return f32x2_mul(h, f32x2_mul(f32x2_pack(r, r), f32x2_pack(v, u)));
}

__device__ __forceinline__ int gn_group(const GnArgs& a, int c) { return static_cast<int>(c * a.per_inv >> 32); }

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

// Mean (less the group's first value) and M2 of rows [r0, r1) of a sample (xs) by group into out[G] (shared memory or global); with KEEP
// the rows go to `rows_at` too. part: [2][lanes][C] floats of shared memory.
template <bool KEEP>
__device__ __forceinline__ void gn_sums(const GnArgs& a, const GnThread& t, const uint16_t* xs, int64_t r0, int64_t r1, float* part,
                                        uint4* rows_at, float2* out) {
  const int rows = r1 > r0 ? static_cast<int>(r1 - r0) : 0;
  const int full = rows / t.lanes, extra = rows - full * t.lanes;  // rows of a lane, lanes with one more
  const uint64_t minus1 = f32x2_pack(-1.0f, -1.0f);
  if (t.lane < t.lanes) {
    int n = full + (t.lane < extra);  // rows of this thread
    const uint16_t* xp = xs + (r0 + t.lane) * a.ldx + t.vec * 8;
    uint4* keep = rows_at + t.lane * t.vecs + t.vec;
    const int64_t step = t.lanes * a.ldx;
    const int keep_step = t.lanes * t.vecs;
    uint4 v[kGnSumUnroll];
#pragma unroll
    for (int u = 0; u < kGnSumUnroll; ++u, xp += step)
      if (u < n) v[u] = ld_global_v4(xp);
    uint4 base;  // the groups' first values
    uint32_t* bw = &base.x;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      bw[j] = gn_bits(xs + gn_group(a, t.vec * 8 + 2 * j) * a.per) | gn_bits(xs + gn_group(a, t.vec * 8 + 2 * j + 1) * a.per) << 16;
    if (n == 0) v[0] = make_uint4(0, 0, 0, 0);  // (counts for nothing)
    uint64_t s2[4], ss2[4], minus[4];
    auto begin_run = [&](const uint4& v) {
      uint64_t f[4];
      gn_unpack(v, f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        minus[j] = f32x2_mul(f[j], minus1);
        s2[j] = ss2[j] = 0;
      }
    };
    auto add = [&](const uint4& v) {
      uint64_t f[4];
      gn_unpack(v, f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t d = f32x2_add(f[j], minus[j]);
        s2[j] = f32x2_add(s2[j], d);
        ss2[j] = f32x2_fma(d, d, ss2[j]);
      }
    };
    // A run's mean and M2, joined to those of the `done` rows before it in this thread's own place of `part`; means less the run's first
    // value, then less what `next` holds: the next run's first value, or the groups'.
    ulonglong2* means = reinterpret_cast<ulonglong2*>(part + t.lane * a.C + t.vec * 8);
    ulonglong2* m2s = reinterpret_cast<ulonglong2*>(part + (t.lanes + t.lane) * a.C + t.vec * 8);
    int done = 0;
    auto end_run = [&](int run, const uint4& next) {
      const float inv = rcp_approx(static_cast<float>(max(run, 1)));
      const uint64_t inv2 = f32x2_pack(inv, inv);
      uint64_t f[4], mean[4], m2[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        mean[j] = f32x2_mul(s2[j], inv2);
        m2[j] = f32x2_fma(f32x2_mul(s2[j], minus1), mean[j], ss2[j]);
      }
      if (!KEEP && done > 0) {
        const float w = run * rcp_approx(static_cast<float>(done + run));
        const uint64_t w2 = f32x2_pack(w, w), dw2 = f32x2_pack(done * w, done * w);
        const ulonglong2 mo[2] = {means[0], means[1]}, qo[2] = {m2s[0], m2s[1]};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t old = j & 1 ? mo[j >> 1].y : mo[j >> 1].x, d = f32x2_fma(old, minus1, mean[j]);
          mean[j] = f32x2_fma(d, w2, old);
          m2[j] = f32x2_fma(f32x2_mul(d, d), dw2, f32x2_add(j & 1 ? qo[j >> 1].y : qo[j >> 1].x, m2[j]));
        }
      }
      gn_unpack(next, f);
#pragma unroll
      for (int j = 0; j < 4; ++j) mean[j] = f32x2_fma(f32x2_add(f[j], minus[j]), minus1, mean[j]);
      means[0] = make_ulonglong2(mean[0], mean[1]);
      means[1] = make_ulonglong2(mean[2], mean[3]);
      m2s[0] = make_ulonglong2(m2[0], m2[1]);
      m2s[1] = make_ulonglong2(m2[2], m2[3]);
      done += run;
    };
    begin_run(v[0]);
    int run = 0;
    // the next rows are on their way while these are added
    for (; n > 0; n -= kGnSumUnroll) {
      uint4 nx[kGnSumUnroll];
#pragma unroll
      for (int u = 0; u < kGnSumUnroll; ++u, xp += step)
        if (u + kGnSumUnroll < n) nx[u] = ld_global_v4(xp);
#pragma unroll
      for (int u = 0; u < kGnSumUnroll; ++u)
        if (u < n) {
          if constexpr (KEEP) keep[u * keep_step] = v[u];
          add(v[u]);
        }
      if constexpr (KEEP) keep += kGnSumUnroll * keep_step;
      run += min(n, kGnSumUnroll);
      if constexpr (!KEEP)
        if (run == kGnRun && n > kGnSumUnroll) {
          end_run(run, nx[0]);
          run = 0;
          begin_run(nx[0]);
        }
#pragma unroll
      for (int u = 0; u < kGnSumUnroll; ++u) v[u] = nx[u];
    }
    end_run(run, base);
  }
  __syncthreads();
  // Channel by channel over the lanes, in the first lane's place: blocks of 16 about their first lane's mean, whose distance from the
  // block's, squared, is at most 16 / rows of the block's M2, are summed and joined. (Two passes, the mean first: 0.3 us more.)
  const float n_lane = static_cast<float>(full), more = n_lane + 1.0f;
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
    const float *mu = part + c, *m2 = mu + t.lanes * a.C;
    float n = 0.0f, mean = 0.0f, q = 0.0f;
    for (int l0 = 0; l0 < t.lanes; l0 += 16) {
      const int l2 = min(l0 + 16, t.lanes), l1 = min(max(extra, l0), l2);
      const float ref = mu[l0 * a.C];
      float u = 0.0f, uu = 0.0f, w = 0.0f;
#pragma unroll 8
      for (int l = l0; l < l2; ++l) {
        const float d = mu[l * a.C] - ref, nd = (l < extra ? more : n_lane) * d;
        u += nd;
        uu = fmaf(nd, d, uu);
        w += m2[l * a.C];
      }
      const float nb = more * (l1 - l0) + n_lane * (l2 - l1);
      if (nb == 0.0f) break;
      const float ub = u * rcp_approx(nb), qb = w + fmaf(-u, ub, uu), d = ref + ub - mean, share = nb * rcp_approx(n + nb);
      q += fmaf(d * d, n * share, qb);
      mean = n > 0.0f ? fmaf(d, share, mean) : d;
      n += nb;
    }
    part[c] = mean;
    part[t.lanes * a.C + c] = q;
  }
  __syncthreads();
  // Then group by group by 2^bits threads. Up to 48 channels about the first one's mean; of more it may be too far from the others: the
  // mean first.
  const int bits = a.sum_bits, threads = 1 << bits, at_once = blockDim.x >> bits, in = threadIdx.x & (threads - 1);
  const float n_rows = static_cast<float>(rows), inv_per = rcp_approx(static_cast<float>(a.per));
  for (int g0 = 0; g0 < a.G; g0 += at_once) {
    const int g = g0 + (threadIdx.x >> bits);
    if ((threadIdx.x & ~31) >> bits >= a.G - g0) break;  // (whole warps)
    const float *mu = part + min(g, a.G - 1) * a.per, *m2 = mu + t.lanes * a.C;
    float ref = mu[0], u = 0.0f, uu = 0.0f, w = 0.0f;
    if (a.per > 48) {
      for (int i = in; i < a.per; i += threads) u += mu[i] - ref;
      for (int o = threads >> 1; o > 0; o >>= 1) u += __shfl_xor_sync(0xFFFFFFFFu, u, o);
      ref = fmaf(u, inv_per, ref);
      u = 0.0f;
    }
    for (int i = in; i < a.per; i += threads) {
      const float d = mu[i] - ref;
      u += d;
      uu = fmaf(d, d, uu);
      w += m2[i];
    }
    for (int o = threads >> 1; o > 0; o >>= 1) {
      u += __shfl_xor_sync(0xFFFFFFFFu, u, o);
      uu += __shfl_xor_sync(0xFFFFFFFFu, uu, o);
      w += __shfl_xor_sync(0xFFFFFFFFu, w, o);
    }
    if (g < a.G && in == 0) out[g] = make_float2(fmaf(u, inv_per, ref), fmaf(n_rows, fmaf(-u, u * inv_per, uu), w));
  }
}

// Per group (pivot, mean - pivot, rstd) in shared memory, from the means and M2 of `parts` CTAs: fetch(part, group).
template <typename Fetch>
__device__ __forceinline__ void gn_groups(const GnArgs& a, const uint16_t* xs, int parts, float* out, Fetch fetch) {
  const int bits = a.join_bits;  // 2^bits threads to a group
  const int sub = 1 << bits, step = blockDim.x >> bits;
  const float chunk_rows = static_cast<float>(a.chunk_rows), n_rows = static_cast<float>(a.rows);
  for (int g0 = 0; g0 < a.G; g0 += step) {  // (the same trips for all threads: shuffles)
    const int g = g0 + (threadIdx.x >> bits), k = threadIdx.x & (sub - 1);
    const bool live = g < a.G;  // (blockDim.x is a multiple of 32)
    const float first = live && k == 0 ? gn_bf16(xs + g * a.per) : 0.0f;
    // About the first part's mean, whose distance from the group's, squared, is at most `parts` / n of M2.
    float ref = 0.0f, u = 0.0f, uu = 0.0f, w = 0.0f;
    for (int c = 0; c < parts; c += 8 * sub) {
      float2 part[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c + i * sub >= parts) break;
        part[i] = live && c + i * sub + k < parts ? fetch(c + i * sub + k, g) : make_float2(0.0f, 0.0f);
      }
      if (c == 0) ref = __shfl_sync(0xFFFFFFFFu, part[0].x, threadIdx.x & 31 & ~(sub - 1));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c + i * sub >= parts) break;
        // its rows (none behind the last part's; beyond 2^24 rounded, which shifts weights by as little)
        const float n = fminf(fmaxf(fmaf(static_cast<float>(c + i * sub + k), -chunk_rows, n_rows), 0.0f), chunk_rows);
        const float d = part[i].x - ref, nd = n * d;
        u += nd;
        uu = fmaf(nd, d, uu);
        w += part[i].y;
      }
    }
    for (int o = sub >> 1; o > 0; o >>= 1) {
      u += __shfl_xor_sync(0xFFFFFFFFu, u, o);
      uu += __shfl_xor_sync(0xFFFFFFFFu, uu, o);
      w += __shfl_xor_sync(0xFFFFFFFFu, w, o);
    }
    if (live && k == 0) {
      // (a group that holds an infinity or a NaN keeps its NaN, which fmax would drop)
      const float off = u * a.inv_rows, mean = ref + off, pivot = first + mean;
      const float var = fmaf(fmaf(-u, off, uu), a.inv_rows, w * a.inv_n), v = (var < 0.0f ? 0.0f : var) + a.eps;
      float r = rsqrtf(v);
      if (v > 1e-30f) r = fmaf(0.5f * r, fmaf(-v * r, r, 1.0f), r);  // (a step of Newton's: the last bits; none where v r^2 would underflow)
      out[3 * g] = pivot;
      // what rounding it has left out (Knuth's sum of two)
      const float back = pivot - first;
      out[3 * g + 1] = (first - (pivot - back)) + (mean - back);
      out[3 * g + 2] = r;
    }
  }
}
// Coefficients of 8 channels, in pairs; `minus`: the pivots' negatives.
struct GnCoefs {
  uint64_t minus[4], a[4], b[4];
  __device__ __forceinline__ uint64_t h(uint64_t x, int j) const { return f32x2_fma(f32x2_add(x, minus[j]), a[j], b[j]); }
};
__device__ __forceinline__ void gn_coefs(const GnArgs& a, const float* groups, int c0, const uint4& gamma, const uint4& beta, GnCoefs& k) {
  uint64_t gm[4], bt[4];
  gn_unpack(gamma, gm);
  gn_unpack(beta, bt);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float *g = groups + gn_group(a, c0 + 2 * j) * 3, *h = groups + gn_group(a, c0 + 2 * j + 1) * 3;
    k.minus[j] = f32x2_pack(-g[0], -h[0]);
    k.a[j] = f32x2_mul(gm[j], f32x2_pack(g[2], h[2]));
    k.b[j] = f32x2_fma(f32x2_pack(-g[1], -h[1]), k.a[j], bt[j]);
  }
}

// A thread's gamma and beta, on their way while the statistics are joined.
struct GnAffine {
  uint4 gamma, beta;
  __device__ __forceinline__ GnAffine(const GnArgs& a, const GnThread& t) {
    gamma = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);  // ones
    beta = make_uint4(0, 0, 0, 0);
    if (a.gamma != nullptr) {
      gamma = ld_global_v4(a.gamma + t.vec * 8);
      beta = ld_global_v4(a.beta + t.vec * 8);
    }
  }
};
__device__ __forceinline__ int gn_rows(const GnThread& t, int64_t r0, int64_t r1) {  // of this thread
  const int rows = static_cast<int>(r1 - r0);
  return t.lane < t.lanes && rows > t.lane ? (rows - t.lane + t.lanes - 1) / t.lanes : 0;
}

// bf16 output of rows [r0, r1). Source: where a row's vectors are read, by next row of the thread; the first ones fly before
// ready(), which leaves the groups' statistics.
template <bool SILU, typename Source, typename Ready>
__device__ __forceinline__ void gn_write(const GnArgs& a, const GnThread& t, const float* groups, int64_t m0, int64_t r0, int64_t r1,
                                         Source src, Ready ready) {
  int n = gn_rows(t, r0, r1);
  uint16_t* yp = a.y + (m0 + r0 + t.lane) * a.ldy + t.vec * 8;
  const int64_t step = t.lanes * a.ldy;
  src.start(r0 + t.lane, t.vec, t.lanes);
  uint4 v[kGnUnroll];
#pragma unroll
  for (int u = 0; u < kGnUnroll; ++u)
    if (u < n) v[u] = src.next();
  const GnAffine affine(a, t);
  ready();
  GnCoefs k;
  gn_coefs(a, groups, t.vec * 8, affine.gamma, affine.beta, k);
  auto put = [&](const uint4& v) {
    uint64_t f[4];
    gn_unpack(v, f);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      f32x2_unpack(gn_act<SILU>(k.h(f[j], j)), lo, hi);
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(hi), "f"(lo));
    }
    st_global_v4(yp, w);
    yp += step;
  };
  for (; n > 0; n -= kGnUnroll) {
    uint4 nx[kGnUnroll];
#pragma unroll
    for (int u = 0; u < kGnUnroll; ++u)
      if (u + kGnUnroll < n) nx[u] = src.next();
#pragma unroll
    for (int u = 0; u < kGnUnroll; ++u)
      if (u < n) put(v[u]);
#pragma unroll
    for (int u = 0; u < kGnUnroll; ++u) v[u] = nx[u];
  }
}
struct GnFromGlobal {
  const uint16_t* x;  // the sample
  int64_t ldx, step = 0;
  const uint16_t* at = nullptr;
  __device__ __forceinline__ void start(int64_t row, int vec, int rows) {
    at = x + row * ldx + vec * 8;
    step = rows * ldx;
  }
  __device__ __forceinline__ uint4 next() {
    const uint4 v = ld_global_v4(at);
    at += step;
    return v;
  }
};
struct GnFromShared {
  const uint4* x;  // rows from r0 on
  int64_t r0;
  int vecs, step = 0;
  const uint4* at = nullptr;
  __device__ __forceinline__ void start(int64_t row, int vec, int rows) {
    at = x + static_cast<int>(row - r0) * vecs + vec;
    step = rows * vecs;
  }
  __device__ __forceinline__ uint4 next() {
    const uint4 v = *at;
    at += step;
    return v;
  }
};

// Codes of rows [r0, r1), kGnUnroll x lanes rows a turn: a thread's values of its rows stay in registers while the rows' maxima meet
// in shared memory (warps first, then an atomic maximum each) and one thread a row makes scale and reciprocal of its. `scales`:
// kGnUnroll x lanes pairs of (maximum, then reciprocal) words, zero before and after.
template <bool SILU, typename Source, typename Ready>
__device__ __forceinline__ void gn_codes(const GnArgs& a, const GnThread& t, const float* groups, uint32_t* scales, int64_t m0,
                                         int64_t r0, int64_t r1, Source src, Ready ready) {
  const bool live = t.lane < t.lanes;
  const int rows = static_cast<int>(r1 - r0), turn = kGnUnroll * t.lanes;
  src.start(r0 + t.lane, t.vec, t.lanes);
  int8_t* qp = a.q + (m0 + r0 + t.lane) * a.ldq + t.vec * 8;
  const int64_t step = t.lanes * a.ldq;
  float* inverse = reinterpret_cast<float*>(scales + turn);
  for (int i = threadIdx.x; i < turn; i += blockDim.x) scales[i] = 0;
  int n = gn_rows(t, r0, r1);  // left of this thread's
  uint4 v[kGnUnroll];
#pragma unroll
  for (int u = 0; u < kGnUnroll; ++u)
    if (u < n) v[u] = src.next();
  const GnAffine affine(a, t);
  ready();
  __syncthreads();
  GnCoefs k;
  gn_coefs(a, groups, t.vec * 8, affine.gamma, affine.beta, k);
  // lanes of this warp that share a row: those with the same t.lane; up to two such groups where a row has 32 vectors or more
  const uint32_t peers = __match_any_sync(0xFFFFFFFFu, t.lane);
  const uint32_t first = __shfl_sync(0xFFFFFFFFu, peers, 0);
  const bool in_first = peers == first, two = t.vecs >= 32;
  for (int base = 0; base < rows; base += turn, n -= kGnUnroll) {
    uint64_t h[kGnUnroll][4];
#pragma unroll
    for (int u = 0; u < kGnUnroll; ++u) {
      uint32_t mx = 0;
      if (u < n) {
        gn_unpack(v[u], h[u]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          h[u][j] = gn_act<SILU>(k.h(h[u][j], j));
          mx = max(mx, max(static_cast<uint32_t>(h[u][j]) & 0x7FFFFFFFu, static_cast<uint32_t>(h[u][j] >> 32) & 0x7FFFFFFFu));
        }
        if (u + kGnUnroll < n) v[u] = src.next();
      }
      if (two) {
        const uint32_t m1 = __reduce_max_sync(0xFFFFFFFFu, in_first ? mx : 0u), m2 = __reduce_max_sync(0xFFFFFFFFu, in_first ? 0u : mx);
        if (live && (peers & ((1u << (threadIdx.x & 31)) - 1u)) == 0) atomicMax(scales + u * t.lanes + t.lane, in_first ? m1 : m2);
      } else if (live) {
        atomicMax(scales + u * t.lanes + t.lane, mx);
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < turn; i += blockDim.x) {
      const float amax = __uint_as_float(scales[i]);
      float sa = 0.0f, inv = 0.0f;
      if (!(amax < 7.888609052210118e-31f)) {  // 2^-100, as in dp_daq_quantize
        sa = __fdiv_rn(amax, 127.0f);
        inv = __fdiv_rn(127.0f, amax);
      }
      inverse[i] = inv;
      scales[i] = 0;
      if (base + i < rows) a.s_a[m0 + r0 + base + i] = sa;
    }
    __syncthreads();  // (the next turn's maxima are behind it, its reciprocals behind the next but one)
    const uint64_t magic2 = f32x2_pack(12582912.0f, 12582912.0f);
#pragma unroll
    for (int u = 0; u < kGnUnroll; ++u)
      if (u < n) {
        const float inv = inverse[u * t.lanes + t.lane];
        const uint64_t inv2 = f32x2_pack(inv, inv);
        uint32_t c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t w = f32x2_fma(h[u][j], inv2, magic2);
          c[j] = __byte_perm(static_cast<uint32_t>(w), static_cast<uint32_t>(w >> 32), 0x0040);
        }
        *reinterpret_cast<uint2*>(qp) = make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
        qp += step;
      }
  }
}

template <bool CODES, bool SILU, typename Source, typename Ready>
__device__ __forceinline__ void gn_out(const GnArgs& a, const GnThread& t, const float* groups, uint32_t* scales, int64_t m0,
                                       int64_t r0, int64_t r1, const Source& src, Ready ready) {
  if constexpr (CODES) gn_codes<SILU>(a, t, groups, scales, m0, r0, r1, src, ready);
  else gn_write<SILU>(a, t, groups, m0, r0, r1, src, ready);
}
// shared memory: the groups' (pivot, mean - pivot, rstd) and sums, gn_codes' scales; then gn_sums' part, then rows
__host__ __device__ constexpr int gn_head_floats(int G, int lanes) { return (5 * G + 1 + 2 * kGnUnroll * lanes + 3) & ~3; }
__device__ __forceinline__ uint32_t* gn_scales(const GnArgs& a) {
  extern __shared__ __align__(16) float gn_smem[];
  return reinterpret_cast<uint32_t*>(gn_smem + 5 * a.G + 1);
}

__global__ void __launch_bounds__(kGnMaxThreads) gn_stats_kernel(const GnArgs a) {
  extern __shared__ __align__(16) float gn_smem[];
  pdl_launch_dependents();
  const GnThread t(a.C);
  const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int64_t r0 = chunk * a.chunk_rows;
  pdl_wait();
  gn_sums<false>(a, t, a.x + sample * a.rows * a.ldx, r0, min(r0 + a.chunk_rows, a.rows), gn_smem, nullptr,
                 a.sums + static_cast<int64_t>(blockIdx.x) * a.G);
}

template <bool CODES, bool SILU>
__global__ void __launch_bounds__(kGnMaxThreads) gn_apply_kernel(const GnArgs a) {
  extern __shared__ __align__(16) float gn_smem[];
  pdl_launch_dependents();
  const GnThread t(a.C);
  // the last chunks first: of maps beyond the L2 they are what is left there
  const int block = gridDim.x - 1 - blockIdx.x, sample = block / a.out_chunks, chunk = block % a.out_chunks;
  const int64_t r0 = chunk * a.out_rows, m0 = sample * a.rows;
  const uint16_t* xs = a.x + m0 * a.ldx;
  pdl_wait();
  gn_out<CODES, SILU>(a, t, gn_smem, gn_scales(a), m0, r0, min(r0 + a.out_rows, a.rows), GnFromGlobal{xs, a.ldx}, [&]() {
    gn_groups(a, xs, a.chunks, gn_smem, [&](int c, int g) {
      float2 v;
      const float2* p = a.sums + (static_cast<int64_t>(sample) * a.chunks + c) * a.G + g;
      asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p) : "memory");
      return v;
    });
    __syncthreads();
  });
}

// One sample by a cluster of a.chunks CTAs, each with its rows in shared memory.
template <bool CODES, bool SILU>
__global__ void __launch_bounds__(kGnMaxThreads) gn_cluster_kernel(const GnArgs a) {
  extern __shared__ __align__(16) float gn_smem[];
  pdl_launch_dependents();
  const GnThread t(a.C);
  const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int64_t r0 = min(chunk * a.chunk_rows, a.rows), r1 = min(r0 + a.chunk_rows, a.rows), m0 = sample * a.rows;
  float* groups = gn_smem;
  float2* sums = reinterpret_cast<float2*>(gn_smem + ((3 * a.G + 1) & ~1));
  float* part = gn_smem + gn_head_floats(a.G, t.lanes);
  uint4* rows_at = reinterpret_cast<uint4*>(part + 2 * t.lanes * a.C);
  const uint16_t* xs = a.x + m0 * a.ldx;
  pdl_wait();
  gn_sums<true>(a, t, xs, r0, r1, part, rows_at, sums);
  gn_out<CODES, SILU>(a, t, groups, gn_scales(a), m0, r0, r1, GnFromShared{rows_at, r0, t.vecs}, [&]() {
    __syncwarp();
    cluster_sync();
    gn_groups(a, xs, a.chunks, groups, [&](int c, int g) {
      float2 v;
      asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(map_to_cta(sums + g, c)) : "memory");
      return v;
    });
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (this CTA has read the others' sums)
  });
  __syncwarp();
  cluster_wait();  // nobody leaves while its sums are read
}

// ---- host side -------------------------------------------------------------------------------------
static int gn_threads(int32_t C, int most = kGnMaxThreads) {  // whole rows of C / 8 vectors
  const int vecs = C / 8, rows = most / vecs;
  return ((rows < 1 ? 1 : rows) * vecs + 31) / 32 * 32;
}
static size_t gn_part_bytes(int32_t C) { return 2 * sizeof(float) * static_cast<size_t>(gn_threads(C) / (C / 8)) * C; }
static int gn_head_bytes(int32_t C, int32_t G, int threads) { return static_cast<int>(sizeof(float)) * gn_head_floats(G, threads / (C / 8)); }

// CTAs to a cluster of the one-kernel form, 0 where a sample does not fit.
static int gn_cluster(int64_t samples, int64_t rows, int32_t C, int32_t G) {
  const size_t room = kGnSmem - gn_head_bytes(C, G, gn_threads(C)) - gn_part_bytes(C);
  int cs = 1;
  while (cs <= kGnMaxCluster && static_cast<size_t>((rows + cs - 1) / cs) * C * 2 > room) cs *= 2;
  if (cs > kGnMaxCluster) return 0;
  while (cs < kGnMaxCluster && samples * cs * 2 <= 148 && rows >= 4 * cs) cs *= 2;
  return cs;
}
// CTAs to a sample of the two-kernel form, where `ctas` fill the device: 16 rows or more to each
static int gn_chunks(int64_t samples, int64_t rows, int ctas) {
  const int64_t c = ctas / samples, most = (rows + 15) / 16;
  return static_cast<int>(c < 1 ? 1 : c < most ? c : most);
}
size_t group_norm_workspace(int64_t samples, int64_t rows, int32_t C, int32_t G) {
  if (samples <= 0 || rows <= 0 || C < 8 || gn_cluster(samples, rows, C, G) != 0) return 256;
  return (static_cast<size_t>(samples) * gn_chunks(samples, rows, 148) * G * sizeof(float2) + 255) & ~static_cast<size_t>(255);
}

#define GN_PICK(KERNEL, codes, silu) \
  ((codes) ? ((silu) ? KERNEL<true, true> : KERNEL<true, false>) : ((silu) ? KERNEL<false, true> : KERNEL<false, false>))

int group_norm_init_device() {
  for (bool codes : {false, true})
    for (bool silu : {false, true})
      DP_CUDA_OK(cudaFuncSetAttribute(GN_PICK(gn_cluster_kernel, codes, silu), cudaFuncAttributeMaxDynamicSharedMemorySize, kGnSmem));
  return DP_OK;
}

int launch_group_norm(const void* x, int64_t samples, int64_t rows, int32_t C, int64_t ldx, int32_t G, const void* gamma,
                      const void* beta, float eps, bool silu, void* y, int64_t ldy, int8_t* q, int64_t ldq, float* s_a,
                      void* workspace, cudaStream_t stream) {
  GnArgs a{static_cast<const uint16_t*>(x), rows, ldx, C, G, C / G, ((1ull << 32) + C / G - 1) / (C / G), static_cast<const uint16_t*>(gamma),
           static_cast<const uint16_t*>(beta), eps, static_cast<float>(1.0 / (static_cast<double>(rows) * (C / G))), static_cast<float>(1.0 / static_cast<double>(rows)), static_cast<uint16_t*>(y), ldy, q, ldq, s_a,
           static_cast<float2*>(workspace), 0, 0, 0, 0, 0, 0};
  const bool codes = q != nullptr;
  const int threads = gn_threads(C);
  const size_t head = gn_head_bytes(C, G, threads), part = gn_part_bytes(C);
  // as many as there are, up to a warp and one to `least` channels or parts
  const auto bits = [G](int32_t of, int least, int of_threads) {
    int b = 0;
    while (b < 5 && least << b < of && (2 << b) * G <= of_threads) ++b;
    return b;
  };
  a.sum_bits = bits(C / G, 4, threads);
  cudaError_t e = cudaSuccess;
  if (const int cs = gn_cluster(samples, rows, C, G); cs != 0) {
    a.chunks = cs;
    a.chunk_rows = (rows + cs - 1) / cs;
    a.join_bits = bits(cs, 1, threads);
    e = launch_cluster(GN_PICK(gn_cluster_kernel, codes, silu), dim3(static_cast<unsigned>(samples * cs)), dim3(threads),
                       head + part + static_cast<size_t>(a.chunk_rows) * C * 2, stream, true, static_cast<unsigned>(cs), a);
  } else {
    a.chunks = gn_chunks(samples, rows, 148);
    a.chunk_rows = (rows + a.chunks - 1) / a.chunks;
    // Codes wait for their rows' maxima: two CTAs of ten warps to an SM, one of which works while the other waits (8 x 4096 x 320 with
    // SiLU 19.0 -> 18.0 us, 128 x 1400 x 320 87.6 -> 83.3; four of five warps 17.7 / 81.8, but 2 x 1023 x 640 10.2 -> 12.6). Rows of
    // more than 1280 channels leave such a CTA one at a time (8 x 256 x 1920 13.0 -> 17.2): one of twenty warps.
    const bool halves = codes && C <= 1280;
    const int out_threads = halves ? gn_threads(C, kGnMaxThreads / 2) : threads;
    a.out_chunks = halves ? gn_chunks(samples, rows, 296) : a.chunks;
    a.out_rows = (rows + a.out_chunks - 1) / a.out_chunks;
    a.join_bits = bits(a.chunks, 1, out_threads);
    e = launch(gn_stats_kernel, dim3(static_cast<unsigned>(samples * a.chunks)), dim3(threads), part, stream, true, a);
    if (e == cudaSuccess)
      e = launch(GN_PICK(gn_apply_kernel, codes, silu), dim3(static_cast<unsigned>(samples * a.out_chunks)), dim3(out_threads),
                 gn_head_bytes(C, G, out_threads), stream, true, a);
  }
  if (e != cudaSuccess) return fail(DP_ERR_CUDA, "group norm launch failed: %s", cudaGetErrorString(e));
  return DP_OK;
}

}  // namespace dp
