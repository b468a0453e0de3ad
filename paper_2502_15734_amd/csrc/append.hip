// cc_append_attention: causal attention of the last rows of each request over its whole paged context, a few rows or one at a time.
//
// Plain form (CC_IMPL_SCALAR): one wavefront per (row, query head), one key at a time with the running maximum and sum of the softmax.
#include "device_util.h"

namespace cc {

template <typename T, int D>
__global__ __launch_bounds__(64) void append_scalar_kernel(
    const T* __restrict__ q, const int32_t* __restrict__ src_rows, const int32_t* __restrict__ q_pos, const int32_t* __restrict__ cu_q,
    int n_requests, const T* __restrict__ k_pool, const T* __restrict__ v_pool, int n_blocks, const int32_t* __restrict__ block_tab,
    const cc_segment* __restrict__ segs, const int32_t* __restrict__ req_seg_off, int hq, int hkv, InvFreq inv_freq,
    T* __restrict__ out, float* __restrict__ lse, ValueSource vs) {
  const int j = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  if (j >= cu_q[n_requests]) return;                  // (the list may be shorter than its capacity)
  int lo = 0, hi = n_requests;                        // cu_q[lo] <= j < cu_q[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu_q[mid] <= j) lo = mid; else hi = mid;
  }
  const int r = lo, p = q_pos[j], kvh = h / (hq / hkv);
  const bool own = lane < D / 2;
  float qx = 0.f, qy = 0.f;
  if (own) {
    const T* qp = q + (static_cast<size_t>(src_rows != nullptr ? src_rows[j] : j) * hq + h) * D;
    const float x = to_float(qp[lane]), y = to_float(qp[lane + D / 2]);
    float c, s;
    rot_cos_sin(p, inv_freq.f[lane], &c, &s);
    qx = x * c - y * s;
    qy = y * c + x * s;
  }
  const float scale = rsqrtf(static_cast<float>(D));
  float m = -INFINITY, z = 0.f, ox = 0.f, oy = 0.f;
  for (int s = req_seg_off[r]; s < req_seg_off[r + 1]; ++s) {
    const cc_segment ks = segs[s];
    const int n_vis = min(ks.n_tokens, p - ks.logical_start + 1);
    for (int t = 0; t < n_vis; ++t) {
      const int blk = block_tab[ks.tab_off + t / kBlock];
      if (blk < 0 || blk >= n_blocks) continue;
      const T* kp = k_pool + ((static_cast<size_t>(blk) * hkv + kvh) * kBlock + t % kBlock) * D;
      const float logit = wave_sum(own ? qx * to_float(kp[lane]) + qy * to_float(kp[lane + D / 2]) : 0.f) * scale;
      if (logit > m) {                                // (the same in all lanes)
        const float a = expf(m - logit);
        z *= a; ox *= a; oy *= a;
        m = logit;
      }
      const float e = logit == -INFINITY ? 0.f : expf(logit - m);
      z += e;
      if (own) {
        const T* vp = value_block<T>(v_pool, static_cast<const T*>(vs.v_shared), vs.n_shared_blocks, vs.v_map, blk,
                                     static_cast<size_t>(hkv) * D * kBlock) + static_cast<size_t>(kvh) * D * kBlock + t % kBlock;
        ox += e * to_float(vp[static_cast<size_t>(lane) * kBlock]);
        oy += e * to_float(vp[static_cast<size_t>(lane + D / 2) * kBlock]);
      }
    }
  }
  const float inv = z == 0.f ? 0.f : 1.f / z;         // (a row without keys: zeros, and -inf for the logarithm)
  if (own) {
    T* op = out + (static_cast<size_t>(j) * hq + h) * D;
    op[lane] = from_float<T>(ox * inv);
    op[lane + D / 2] = from_float<T>(oy * inv);
  }
  if (lse != nullptr && lane == 0) lse[static_cast<size_t>(j) * hq + h] = z == 0.f ? -INFINITY : m + logf(z);
}

size_t append_bytes(const cc_ctx*, int, int, int, int, int) { return 0; }

void launch_append_attention(const cc_ctx* ctx, const void* q, const int32_t* src_rows, const int32_t* q_pos, const int32_t* cu_q, int n_q_tot,
                             int max_q_per_req, const void* k_pool, const void* v_pool, int n_blocks, const int32_t* block_tab,
                             const cc_segment* segs, const int32_t* req_seg_off, int n_requests, int max_ctx_tokens, int max_segs_per_req,
                             void* out, float* lse, void* workspace, hipStream_t stream, const ValueSource& vs) {
  const bool bf = ctx->cfg.dtype == CC_BF16;
  const int d = ctx->cfg.head_dim, hq = ctx->cfg.n_q_heads, hkv = ctx->cfg.n_kv_heads;
#define CC_LAUNCH(T, D)                                                                                                          \
  hipLaunchKernelGGL((append_scalar_kernel<T, D>), dim3(n_q_tot, hq), dim3(64), 0, stream, static_cast<const T*>(q), src_rows, q_pos, \
                     cu_q, n_requests, static_cast<const T*>(k_pool), static_cast<const T*>(v_pool), n_blocks, block_tab, segs,      \
                     req_seg_off, hq, hkv, ctx->inv_freq, static_cast<T*>(out), lse, vs)
  if (bf && d == 128) CC_LAUNCH(bf16_t, 128);
  else if (bf) CC_LAUNCH(bf16_t, 64);
  else if (d == 128) CC_LAUNCH(float, 128);
  else CC_LAUNCH(float, 64);
#undef CC_LAUNCH
}

}  // namespace cc
