// Distillation from a teacher's top logits (k = 1: cross-entropy) with z-loss: loss, log-sum-exp and gradient
// of every row in one kernel.
//
//   lse = log sum_v exp(x_v / T), p = softmax of the used teacher entries / T
//   loss = w (T^2 (sum_k p_k (log p_k - x_{id_k} / T) + lse) + z lse^2)          (sum_k p_k = 1)
//   dx_v = exp(x_v / T - lse) w (T + 2 z lse / T) - w T sum_{k: id_k = v} p_k
//
// A row of logits is read once and its gradient written once; memory bounds it as long as a row is not read
// twice, so one block holds a whole row in registers (16-byte accesses, RV of them a thread): maximum, sum of
// exponentials and gradient all come from that copy.  Rows that fit no block are read twice, the second time
// mostly from L2.  Rows need not start on 16 bytes (an odd vocabulary): the elements before the first and
// after the last whole access are taken one by one.  The teacher's few entries are fetched while the row's
// loads are in flight; where they touch the gradient, the thread that owns the first entry of an id writes
// that element again after the row, with the sum of all entries of the id, so nothing is added by atomics.
#include <type_traits>

#include "diloco_ops.cuh"

namespace diloco {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct DistillArgs {
  const void *logits, *ids, *teacher;
  const float *row_weight;
  float *loss, *lse;
  void *dlogits;
  long long rows, vocab, logits_stride, grad_stride;
  int k, ids64, teacher_bf16;
  float temperature, inv_t, z, grad_scale;
};

// The teacher's side of one row in shared memory.
constexpr int kMaxK = 1024;
struct Teacher {
  int id[kMaxK];   // -1: unused
  float p[kMaxK];  // t / T, then the share of the entry
  float x[kMaxK];  // the student's logit there
  float red[3][32];
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Entries of row n into shared memory (any number of threads); the caller synchronises.
template <typename T> __device__ __forceinline__ void fetch_teacher(const DistillArgs &a, long long n, const T *row, Teacher &t) {
  for (int i = threadIdx.x; i < a.k; i += blockDim.x) {
    const long long at = n * a.k + i;
    const long long id = a.ids64 ? static_cast<const long long *>(a.ids)[at] : (long long)static_cast<const int *>(a.ids)[at];
    const bool used = id >= 0 && id < a.vocab;
    t.id[i] = used ? (int)id : -1;
    float x[1] = {0.f}, q = 0.f;
    if (used) {
      load_vec<T, 1>(row + id, x);
      q = a.teacher_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(a.teacher)[at]) : static_cast<const float *>(a.teacher)[at];
    }
    t.x[i] = x[0];
    t.p[i] = q * a.inv_t;
  }
}

// One warp: t.p becomes the softmax over the used entries; returns sum_k p_k (log p_k - x_k / T), and in `any`
// whether an entry is used.
__device__ __forceinline__ float finish_teacher(const DistillArgs &a, Teacher &t, bool &any) {
  const int lane = threadIdx.x & 31;
  float top = -INFINITY, total = 0.f, kl = 0.f;
  bool mine = false;
  for (int i = lane; i < a.k; i += 32)
    if (t.id[i] >= 0) top = fmaxf(top, t.p[i]), mine = true;
  any = __any_sync(0xffffffffu, mine);
  top = warp_max(top);
  for (int i = lane; i < a.k; i += 32)
    if (t.id[i] >= 0) total += expf(t.p[i] - top);
  total = warp_sum(total);
  const float log_total = logf(total);
  for (int i = lane; i < a.k; i += 32) {
    float p = 0.f;
    if (t.id[i] >= 0) {
      const float lp = t.p[i] - top - log_total;
      p = expf(lp);
      if (p > 0.f) kl += p * (lp - t.x[i] * a.inv_t);
    }
    t.p[i] = p;
  }
  return warp_sum(kl);
}

// After the row's gradient: elements that teacher entries point at, each by the thread of its first entry.
template <typename T>
__device__ __forceinline__ void put_teacher(const DistillArgs &a, const Teacher &t, T *grad, float lse2, float coef, float wt) {
  for (int i = threadIdx.x; i < a.k; i += blockDim.x) {
    const int id = t.id[i];
    if (id < 0) continue;
    bool first = true;
    float p = 0.f;
    for (int j = 0; j < a.k; ++j)
      if (t.id[j] == id) {
        if (j < i) first = false;
        p += t.p[j];
      }
    if (!first) continue;
    const float g[1] = {ex2(fmaf(t.x[i], a.inv_t * kLog2e, -lse2)) * coef - wt * p};
    store_vec<T, 1>(grad + id, g);
  }
}

// Places of a row: `head` single elements, `body` accesses of W, `tail` single elements.
struct Span {
  int head, tail, body;
};
template <typename T, int W> __device__ __forceinline__ Span span_of(const T *row, long long vocab) {
  Span s;
  const int off = (int)((reinterpret_cast<uintptr_t>(row) / sizeof(T)) % W);
  s.head = off ? W - off : 0;
  if (s.head > vocab) s.head = (int)vocab;
  s.body = ((int)vocab - s.head) / W;
  s.tail = (int)vocab - s.head - s.body * W;
  return s;
}

// Combines the threads' (max, sum) pairs of base-2 exponentials; every thread gets both.
template <int NT> __device__ __forceinline__ void block_lse(float &m, float &s, float (*red)[32]) {
  const float wm = warp_max(m);
  s = wm == -INFINITY ? s : s * ex2(m - wm); // m = -inf: s is 0
  s = warp_sum(s);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[0][warp] = wm, red[1][warp] = s;
  __syncthreads();
  float bm = lane < NT / 32 ? red[0][lane] : -INFINITY, bs = lane < NT / 32 ? red[1][lane] : 0.f;
  const float top = warp_max(bm);
  bs = bm == -INFINITY ? 0.f : bs * ex2(bm - top);
  s = warp_sum(bs);
  m = top;
}

template <typename T, int W, int NT, int RV>
__global__ void __launch_bounds__(NT, 1) distill_resident_kernel(const DistillArgs a) {
  using Raw = typename Pack<T, W>::raw;
  __shared__ Teacher t;
  const float c = a.inv_t * kLog2e;
  for (long long n = blockIdx.x; n < a.rows; n += gridDim.x) {
    const T *row = static_cast<const T *>(a.logits) + n * a.logits_stride;
    const Span sp = span_of<T, W>(row, a.vocab);
    const T *body = row + sp.head;
    Raw raw[RV];
#pragma unroll
    for (int i = 0; i < RV; ++i) {
      const int v = i * NT + threadIdx.x;
      if (v < sp.body) raw[i] = reinterpret_cast<const Raw *>(body)[v];
    }
    // one single element for each of the first head + tail threads
    const int odd = (int)threadIdx.x < sp.head ? (int)threadIdx.x
                    : (int)threadIdx.x < sp.head + sp.tail ? sp.body * W + (int)threadIdx.x : -1;
    float single[1] = {-INFINITY};
    if (odd >= 0) load_vec<T, 1>(row + odd, single);
    fetch_teacher<T>(a, n, row, t);
    float m = single[0];
#pragma unroll
    for (int i = 0; i < RV; ++i)
      if (i * NT + (int)threadIdx.x < sp.body) {
        float v[W];
        unpack(raw[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j) m = fmaxf(m, v[j]);
      }
    m *= c;
    const float m0 = m == -INFINITY ? 0.f : m; // nothing but -infinity (or no element): every term is 0
    float s = odd >= 0 ? ex2(fmaf(single[0], c, -m0)) : 0.f;
#pragma unroll
    for (int i = 0; i < RV; ++i)
      if (i * NT + (int)threadIdx.x < sp.body) {
        float v[W];
        unpack(raw[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j) s += ex2(fmaf(v[j], c, -m0));
      }
    block_lse<NT>(m, s, t.red); // its barrier also ends the fetch of the teacher's entries
    const float lse2 = m + log2f(s), lse = lse2 * kLn2;
    const float wn = a.grad_scale * (a.row_weight ? a.row_weight[n] : 1.f);
    if (threadIdx.x < 32) {
      bool any;
      const float kl = finish_teacher(a, t, any);
      if (threadIdx.x == 0) {
        a.loss[n] = any ? wn * (a.temperature * a.temperature * (kl + lse) + a.z * lse * lse) : 0.f;
        a.lse[n] = lse;
        t.red[2][0] = any ? 1.f : 0.f;
      }
    }
    if (a.dlogits) {
      __syncthreads();
      const float wt = t.red[2][0] != 0.f ? wn * a.temperature : 0.f;
      const float coef = t.red[2][0] != 0.f ? wn * (a.temperature + 2.f * a.z * lse * a.inv_t) : 0.f;
      T *grad = static_cast<T *>(a.dlogits) + n * a.grad_stride;
#pragma unroll
      for (int i = 0; i < RV; ++i) {
        const int v = i * NT + threadIdx.x;
        if (v < sp.body) {
          float x[W];
          unpack(raw[i], x);
#pragma unroll
          for (int j = 0; j < W; ++j) x[j] = ex2(fmaf(x[j], c, -lse2)) * coef;
          store_vec<T, W>(grad + sp.head + (long long)v * W, x);
        }
      }
      if (odd >= 0) {
        single[0] = ex2(fmaf(single[0], c, -lse2)) * coef;
        store_vec<T, 1>(grad + odd, single);
      }
      __syncthreads(); // the row is written before single elements of it are written again
      if (wt != 0.f) put_teacher<T>(a, t, grad, lse2, coef, wt);
    }
    __syncthreads(); // the next row's entries
  }
}

// Rows that no block holds: two passes over memory.
constexpr int kStreamThreads = 512;
template <typename T, int W> __global__ void __launch_bounds__(kStreamThreads) distill_stream_kernel(const DistillArgs a) {
  using Raw = typename Pack<T, W>::raw;
  __shared__ Teacher t;
  const float c = a.inv_t * kLog2e;
  for (long long n = blockIdx.x; n < a.rows; n += gridDim.x) {
    const T *row = static_cast<const T *>(a.logits) + n * a.logits_stride;
    const Span sp = span_of<T, W>(row, a.vocab);
    const Raw *body = reinterpret_cast<const Raw *>(row + sp.head);
    const int odd = (int)threadIdx.x < sp.head ? (int)threadIdx.x
                    : (int)threadIdx.x < sp.head + sp.tail ? sp.body * W + (int)threadIdx.x : -1;
    float single[1] = {-INFINITY};
    if (odd >= 0) load_vec<T, 1>(row + odd, single);
    fetch_teacher<T>(a, n, row, t);
    float m = single[0] * c, s = odd >= 0 ? 1.f : 0.f;
    if (m == -INFINITY) s = 0.f; // exp(-inf) counts nothing
#pragma unroll 4
    for (int i = threadIdx.x; i < sp.body; i += kStreamThreads) {
      float v[W], top = -INFINITY;
      unpack(body[i], v);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        v[j] *= c;
        top = fmaxf(top, v[j]);
      }
      if (top > m) {
        s *= ex2(m - top); // m = -inf: s is 0
        m = top;
      }
#pragma unroll
      for (int j = 0; j < W; ++j) s += v[j] == -INFINITY ? 0.f : ex2(v[j] - m);
    }
    block_lse<kStreamThreads>(m, s, t.red);
    const float lse2 = m + log2f(s), lse = lse2 * kLn2;
    const float wn = a.grad_scale * (a.row_weight ? a.row_weight[n] : 1.f);
    if (threadIdx.x < 32) {
      bool any;
      const float kl = finish_teacher(a, t, any);
      if (threadIdx.x == 0) {
        a.loss[n] = any ? wn * (a.temperature * a.temperature * (kl + lse) + a.z * lse * lse) : 0.f;
        a.lse[n] = lse;
        t.red[2][0] = any ? 1.f : 0.f;
      }
    }
    if (a.dlogits) {
      __syncthreads();
      const float wt = t.red[2][0] != 0.f ? wn * a.temperature : 0.f;
      const float coef = t.red[2][0] != 0.f ? wn * (a.temperature + 2.f * a.z * lse * a.inv_t) : 0.f;
      T *grad = static_cast<T *>(a.dlogits) + n * a.grad_stride;
#pragma unroll 4
      for (int i = threadIdx.x; i < sp.body; i += kStreamThreads) {
        float x[W];
        unpack(body[i], x);
#pragma unroll
        for (int j = 0; j < W; ++j) x[j] = ex2(fmaf(x[j], c, -lse2)) * coef;
        store_vec<T, W>(grad + sp.head + (long long)i * W, x);
      }
      if (odd >= 0) {
        single[0] = ex2(fmaf(single[0], c, -lse2)) * coef;
        store_vec<T, 1>(grad + odd, single);
      }
      __syncthreads();
      if (wt != 0.f) put_teacher<T>(a, t, grad, lse2, coef, wt);
    }
    __syncthreads();
  }
}

int valid(const diloco_distill_t *l) {
  if (!l) return DILOCO_ERR_INVALID_ARG;
  if (l->rows < 0 || l->vocab < 1 || l->k < 1 || l->logits_stride < l->vocab) return DILOCO_ERR_INVALID_ARG;
  if (!dtype_ok(l->dtype) || !dtype_ok(l->teacher_dtype) || (l->ids_int64 != 0 && l->ids_int64 != 1)) return DILOCO_ERR_INVALID_ARG;
  if (!(l->temperature > 0.f) || !(l->temperature < INFINITY) || !(l->z_coef >= 0.f) || !(l->z_coef < INFINITY)) return DILOCO_ERR_INVALID_ARG;
  if (!(l->grad_scale > -INFINITY && l->grad_scale < INFINITY)) return DILOCO_ERR_INVALID_ARG;
  if (l->k > kMaxK || l->vocab > INT32_MAX) return DILOCO_ERR_UNSUPPORTED;
  return DILOCO_OK;
}

template <typename T, int W> void launch(const DistillArgs &a, int sms, cudaStream_t s) {
  const long long n = (a.vocab + W - 1) / W;
  auto grid = [&](int per_sm) { return (unsigned)(a.rows < (long long)sms * per_sm ? a.rows : (long long)sms * per_sm); };
  if (n <= 256) distill_resident_kernel<T, W, 128, 2><<<grid(8), 128, 0, s>>>(a);
  else if (n <= 1024) distill_resident_kernel<T, W, 256, 4><<<grid(4), 256, 0, s>>>(a);
  else if (n <= 4096) distill_resident_kernel<T, W, 512, 8><<<grid(2), 512, 0, s>>>(a);
  else if (n <= 8192) distill_resident_kernel<T, W, 1024, 8><<<grid(1), 1024, 0, s>>>(a);
  else distill_stream_kernel<T, W><<<grid(4), kStreamThreads, 0, s>>>(a);
}

template <typename T> void launch_any(const DistillArgs &a, int sms, cudaStream_t s) {
  constexpr int W = 16 / (int)sizeof(T);
  // whole accesses need the same place within 16 bytes in a row of logits and in its gradient
  const auto x = reinterpret_cast<uintptr_t>(a.logits), g = reinterpret_cast<uintptr_t>(a.dlogits);
  const bool same = !a.dlogits || ((x - g) % 16 == 0 && ((a.logits_stride - a.grad_stride) * (long long)sizeof(T)) % 16 == 0);
  if (same) launch<T, W>(a, sms, s);
  else distill_stream_kernel<T, 1><<<(unsigned)(a.rows < sms * 4ll ? a.rows : sms * 4ll), kStreamThreads, 0, s>>>(a);
}

} // namespace
} // namespace diloco

using namespace diloco;

extern "C" int diloco_distill_loss(const diloco_distill_t *l, const void *logits, const void *teacher_ids, const void *teacher_logits,
                                   const float *row_weight, float *loss, float *lse, void *dlogits, void *stream) {
  const int rc = valid(l);
  if (rc != DILOCO_OK) return rc;
  if (dlogits && l->grad_stride < l->vocab) return DILOCO_ERR_INVALID_ARG;
  if (l->rows == 0) return DILOCO_OK;
  const uintptr_t e = (uintptr_t)dtype_bytes(l->dtype);
  PointerCheck pc;
  pc.need(logits, e).need(teacher_ids, l->ids_int64 ? 8 : 4).need(teacher_logits, (uintptr_t)dtype_bytes(l->teacher_dtype));
  pc.maybe(row_weight, 4).need(loss, 4).need(lse, 4).maybe(dlogits, e);
  if (pc.rc != DILOCO_OK) return pc.rc;
  DistillArgs a = {};
  a.logits = logits, a.ids = teacher_ids, a.teacher = teacher_logits, a.row_weight = row_weight, a.loss = loss, a.lse = lse;
  a.dlogits = dlogits, a.rows = l->rows, a.vocab = l->vocab, a.logits_stride = l->logits_stride, a.grad_stride = l->grad_stride;
  a.k = l->k, a.ids64 = l->ids_int64, a.teacher_bf16 = l->teacher_dtype == DILOCO_DTYPE_BF16;
  a.temperature = l->temperature, a.inv_t = 1.f / l->temperature, a.z = l->z_coef, a.grad_scale = l->grad_scale;
  const int sms = sm_count(pc.device);
  if (l->dtype == DILOCO_DTYPE_F32) launch_any<float>(a, sms, static_cast<cudaStream_t>(stream));
  else launch_any<__nv_bfloat16>(a, sms, static_cast<cudaStream_t>(stream));
  return launched();
}
