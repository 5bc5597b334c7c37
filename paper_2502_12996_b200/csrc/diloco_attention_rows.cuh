// Causal attention over packed sequences, one row at a time: a warp computes one row of out, dq, or dk and dv
// with plain fp32 arithmetic over exactly the rows it sees.  Lanes hold 32 rows of the other side for the
// products over the head dimension, and the columns of the result (lane, lane + 32, ...) for the sums.
#pragma once
#include "diloco_ops.cuh"

namespace diloco {

constexpr int kMaxHeadDim = 128;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnArgs {
  const __nv_bfloat16 *q, *k, *v, *out_in, *dout;
  __nv_bfloat16 *out, *dq, *dk, *dv;
  float *lse;   // [heads, tokens]
  float *delta; // [heads, tokens] workspace of the backward
  const int *cu;
  long long q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, do_row, do_head;
  long long dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
  int tokens, sequences, heads, kv_heads, group, head_dim;
  float scale, scale_log2; // scale, scale * log2(e)
  unsigned *status;
};

__device__ __forceinline__ float dot_row(const __nv_bfloat16 *a, const __nv_bfloat16 *b, int d) {
  float s = 0.f;
  for (int i = 0; i < d; i += 8) {
    float x[8], y[8];
    load_vec<__nv_bfloat16, 8>(a + i, x);
    load_vec<__nv_bfloat16, 8>(b + i, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x[j], y[j], s);
  }
  return s;
}

__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// acc[c] += sum over the warp's 32 rows r of weight_r * rows[r][lane + 32 c], `n` rows
__device__ __forceinline__ void add_rows(float (&acc)[4], float weight, const __nv_bfloat16 *rows, long long stride, int n, int d, int lane) {
  for (int r = 0; r < n; ++r) {
    const float w = __shfl_sync(0xffffffffu, weight, r);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int col = lane + 32 * c;
      if (col < d) acc[c] = fmaf(w, __bfloat162float(rows[r * stride + col]), acc[c]);
    }
  }
}

// out row i of head h, of the sequence that starts at `first`, and its log-sum-exp
__device__ __forceinline__ void attn_out_row(const AttnArgs &a, int i, int h, int first, int lane) {
  const int g = h / a.group, d = a.head_dim;
  const __nv_bfloat16 *q = a.q + i * a.q_row + h * a.q_head, *k = a.k + g * a.k_head, *v = a.v + g * a.v_head;
  float top = -INFINITY, total = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = first; j0 <= i; j0 += 32) {
    const int n = min(32, i - j0 + 1);
    const float z = lane < n ? dot_row(q, k + (j0 + lane) * a.k_row, d) * a.scale : -INFINITY;
    const float m = fmaxf(top, lanes_max(z));
    const float old = m == -INFINITY ? 1.f : expf(top - m); // nothing but -infinity so far: nothing to rescale
    const float p = lane >= n ? 0.f : m == -INFINITY ? 0.f : expf(z - m);
    total = total * old + lanes_sum(p);
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] *= old;
    add_rows(acc, p, v + j0 * a.v_row, a.v_row, n, d, lane);
    top = m;
  }
  __nv_bfloat16 *o = a.out + i * a.o_row + h * a.o_head;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (lane + 32 * c < d) o[lane + 32 * c] = __float2bfloat16_rn(acc[c] / total);
  if (lane == 0) a.lse[(long long)h * a.tokens + i] = top + logf(total);
}

// dq row i of head h
__device__ __forceinline__ void attn_dq_row(const AttnArgs &a, int i, int h, int first, int lane) {
  const int g = h / a.group, d = a.head_dim;
  const __nv_bfloat16 *q = a.q + i * a.q_row + h * a.q_head, *k = a.k + g * a.k_head, *v = a.v + g * a.v_head;
  const __nv_bfloat16 *dout = a.dout + i * a.do_row + h * a.do_head;
  const float lse = a.lse[(long long)h * a.tokens + i];
  const float delta = dot_row(dout, a.out_in + i * a.o_row + h * a.o_head, d);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = first; j0 <= i; j0 += 32) {
    const int n = min(32, i - j0 + 1);
    float dz = 0.f;
    if (lane < n) {
      const float p = expf(dot_row(q, k + (j0 + lane) * a.k_row, d) * a.scale - lse);
      dz = p * (dot_row(dout, v + (j0 + lane) * a.v_row, d) - delta);
    }
    add_rows(acc, dz, k + j0 * a.k_row, a.k_row, n, d, lane);
  }
  __nv_bfloat16 *o = a.dq + i * a.dq_row + h * a.dq_head;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (lane + 32 * c < d) o[lane + 32 * c] = __float2bfloat16_rn(acc[c] * a.scale);
}

// dk and dv row j of head g of k and v; `end` is one past the sequence
__device__ __forceinline__ void attn_dkv_row(const AttnArgs &a, int j, int g, int end, int lane) {
  const int d = a.head_dim;
  const __nv_bfloat16 *k = a.k + j * a.k_row + g * a.k_head, *v = a.v + j * a.v_row + g * a.v_head;
  float dk[4] = {0.f, 0.f, 0.f, 0.f}, dv[4] = {0.f, 0.f, 0.f, 0.f};
  for (int h = g * a.group; h < (g + 1) * a.group; ++h) {
    const __nv_bfloat16 *q = a.q + h * a.q_head, *dout = a.dout + h * a.do_head, *o = a.out_in + h * a.o_head;
    for (int i0 = j; i0 < end; i0 += 32) {
      const int n = min(32, end - i0);
      float p = 0.f, dz = 0.f;
      if (lane < n) {
        const long long i = i0 + lane;
        p = expf(dot_row(q + i * a.q_row, k, d) * a.scale - a.lse[(long long)h * a.tokens + i]);
        const float delta = dot_row(dout + i * a.do_row, o + i * a.o_row, d);
        dz = p * (dot_row(dout + i * a.do_row, v, d) - delta);
      }
      add_rows(dv, p, dout + i0 * a.do_row, a.do_row, n, d, lane);
      add_rows(dk, dz, q + i0 * a.q_row, a.q_row, n, d, lane);
    }
  }
  __nv_bfloat16 *ok = a.dk + j * a.dk_row + g * a.dk_head, *ov = a.dv + j * a.dv_row + g * a.dv_head;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (lane + 32 * c < d) {
      ok[lane + 32 * c] = __float2bfloat16_rn(dk[c] * a.scale);
      ov[lane + 32 * c] = __float2bfloat16_rn(dv[c]);
    }
}

} // namespace diloco
