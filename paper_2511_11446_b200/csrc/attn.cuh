// What the two attention kernels (attn.cu, attn_tc.cu) share: the call's description on the device, the sequences' bounds,
// the scores' form.
#pragma once

#include "dp_common.cuh"

namespace dp {

struct AttnParams {
  const uint16_t *q, *k, *v;  // bf16; token t, head h at t * ld + h * hs
  uint16_t* y;
  int64_t ldq, ldk, ldv, ldy, q_hs, k_hs, v_hs, y_hs;
  int64_t Mq, Mk;
  int32_t H, KV, D;
  int32_t n_seq, max_q, max_k;
  const int32_t *q_start, *k_start, *prefix;
  const float* slopes;
  // Scores are kept in units of log2: s = q . k * scale * log2(e), and with a cap c: cap * tanh(q . k * scale / c) with
  // cap = c * log2(e). cap = 0: none.
  float scale, cap, scale_by_cap;
  int32_t causal;
  int32_t* status;
};

// a * b of numbers that are not negative, or the largest one where it does not fit: tiles, heads and sequences of a call may be up to
// 2^31 each.
static inline int64_t attn_product(int64_t a, int64_t b) { return b != 0 && a > INT64_MAX / b ? INT64_MAX : a * b; }

#ifdef __CUDACC__

constexpr float kLog2e = 1.4426950408889634f;

// A sequence's rows. Offsets that leave the buffers or go backwards are cut to what is there, so that no access leaves the
// buffers whatever they hold.
struct AttnSeq {
  int32_t q0, nq, k0, nk;
  int32_t behind;  // position among the keys of query 0: the last query stands at the last key
  int32_t prefix;
};
__device__ __forceinline__ AttnSeq attn_seq(const AttnParams& p, int s) {
  AttnSeq r;
  if (p.q_start != nullptr) {
    const int32_t Mq = static_cast<int32_t>(p.Mq), Mk = static_cast<int32_t>(p.Mk);
    r.q0 = min(max(ld_global_s32(p.q_start + s), 0), Mq);
    r.nq = min(max(ld_global_s32(p.q_start + s + 1), r.q0), Mq) - r.q0;
    r.k0 = min(max(ld_global_s32(p.k_start + s), 0), Mk);
    r.nk = min(max(ld_global_s32(p.k_start + s + 1), r.k0), Mk) - r.k0;
  } else {
    r.nq = p.max_q;
    r.nk = p.max_k;
    r.q0 = s * p.max_q;  // (n_seq * max_q <= Mq < 2^31)
    r.k0 = s * p.max_k;
  }
  r.behind = r.nk - r.nq;
  r.nq = min(r.nq, p.max_q);
  r.prefix = p.causal && p.prefix != nullptr ? ld_global_s32(p.prefix + s) : 0;
  return r;
}
// Keys that queries up to `last` can see: those below the result.
__device__ __forceinline__ int attn_keys(const AttnParams& p, const AttnSeq& s, int last) {
  return p.causal ? min(s.nk, max(max(last + s.behind + 1, s.prefix), 0)) : s.nk;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// cap * tanh(u), tanh(u) = 1 - 2 / (e^2u + 1): two operations of the special-function unit and an absolute error of a few
// 2^-24 of the cap over the whole range (e^2u = inf gives 1, 0 gives -1). The hardware's own tanh is good to 2^-11, which for a
// cap of 50 would be 0.02 in the exponent. two_u_log2e = 2 u log2(e).
__device__ __forceinline__ float capped(float cap, float two_u_log2e) {
  return fmaf(-2.0f * cap, rcp_approx(ex2(two_u_log2e) + 1.0f), cap);
}

#endif

}  // namespace dp
