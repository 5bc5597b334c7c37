// Causal attention over packed sequences, backward, on the fifth-generation tensor cores: one kernel for dq, one for
// dk and dv.  Each forms P and dz again from q, k and the forward's log-sum-exp:
//   P_ij = exp(z_ij - lse_i),  dz_ij = P_ij (dout_i . v_j - delta_i),  delta_i = dout_i . out_i
//   dq_i = scale sum_j dz_ij k_j;   dv_j = sum_i P_ij dout_i,  dk_j = scale sum_i dz_ij q_i  (over the heads of a group)
// Two kernels take 7 products where one takes 5, but every sum then has one owner: the rows of a block's own
// tile accumulate in tensor memory over the whole loop, and nothing is added to memory by atomics, whose order
// would change the result from call to call, nor kept in an fp32 copy of dq.
//
// Both loops keep one tile pair in flight and alternate so that the tensor cores work during the exponentials:
//   dk, dv   tensor cores: dz^T Q of the last tile, V dO^T of this one | P^T dO, K Q^T of the next
//            256 threads : P^T = exp of this tile                       | dz^T of this tile
//   dq       S of the next tile is under way (two buffers) while dz of this one is formed
// P and dz stay in tensor memory as bf16, over the columns of S and dP that the same threads have read.  Tiles
// are 128 x 128; warps 0-3 take the first 64 columns, warps 4-7 the last, one row a thread.  Rows of a partial last
// tile are zeroed in shared memory where they are summed over; a row that comes out non-finite is computed
// again over the rows it has to do with alone.
#include <type_traits>

#include "diloco_attention_tiles.cuh"

namespace diloco {
namespace {

constexpr int kBwdThreads = 384;
constexpr int kStages = 2;

template <int HD> struct BwdLayout { // two tiles of the block's own, two rings
  static constexpr int kPanels = HD / 64, kTileBytes = kPanels * kPanel;
  static constexpr int kOwn = 0, kRing = 2 * kTileBytes, kStats = kRing + 2 * kStages * kTileBytes;
  // at least half of an SM's shared memory, so that no second block waits for tensor memory
  static constexpr int kUsed = kStats + kStages * 2 * kRows * 4 + 1024, kBytes = kUsed > 120 * 1024 ? kUsed : 120 * 1024;
};

__device__ __forceinline__ void math_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// ------------------------------------------------------------------------------------- dq
struct DqBarriers {
  unsigned long long own_full, k_full[kStages], v_full[kStages], k_empty[kStages], v_empty[kStages], s_full[2], dp_full, ds_full, o_full;
  unsigned tmem;
  volatile unsigned abort;
  unsigned char bad[kRows];
  float delta[2][kRows];
};

template <int HD>
__global__ void __launch_bounds__(kBwdThreads, 1)
    attn_dq_kernel(const AttnArgs a, const __grid_constant__ HeadMap mq, const __grid_constant__ HeadMap mk, const __grid_constant__ HeadMap mv,
                   const __grid_constant__ HeadMap mdo, int split) {
  using L = BwdLayout<HD>;
  extern __shared__ unsigned char raw_smem[];
  __shared__ DqBarriers bar;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = cluster_rank(), unit = blockIdx.x / split, h = unit % a.heads, g = h / a.group;
  const Place at = place_of<false>(a, unit / a.heads, kRows);
  if (at.block < 0) {
    if (part != 0) return;
    const int r0 = at.first + (-1 - at.block) * kRows;
    for (int r = r0 + warp; r < min(r0 + kRows, at.end); r += kBwdThreads / 32) {
      for (int c = lane; c < a.head_dim; c += 32) a.dq[r * a.dq_row + h * a.dq_head + c] = __float2bfloat16_rn(0.f);
    }
    return;
  }
  const int q0 = at.first + at.block * kRows;
  if (q0 >= at.end) return;
  const int all = at.block + 1, tiles = (all - part + split - 1) / split; // this block's key tiles: part, part + split, ...
  const unsigned smem = (smem_u32(raw_smem) + 1023) & ~1023u;
  const unsigned s_q = smem + L::kOwn, s_do = s_q + L::kTileBytes, s_k = smem + L::kRing, s_v = s_k + kStages * L::kTileBytes;

  if (warp == 8) tmem_alloc(&bar.tmem, 512);
  if (threadIdx.x == 0) {
    mbar_init(&bar.own_full, 1), mbar_init(&bar.dp_full, 1), mbar_init(&bar.ds_full, 256), mbar_init(&bar.o_full, 1);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bar.k_full[i], 1), mbar_init(&bar.v_full[i], 1);
      mbar_init(&bar.k_empty[i], 1), mbar_init(&bar.v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&bar.s_full[i], 1);
    bar.abort = 0;
    fence_mbar_init();
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const unsigned tmem = bar.tmem, t_s = tmem, t_dp = tmem + 256, t_dq = tmem + 384;

  if (warp >= 8) {
    if (warp == 9 && lane == 0) {
      int issued = 0;
      if (tiles > 0) {
        mbar_expect_tx(&bar.own_full, 2 * L::kTileBytes);
        load_tile<HD>(s_q, mq, h, q0, &bar.own_full);
        load_tile<HD>(s_do, mdo, h, q0, &bar.own_full);
      }
      for (int it = 0; it < tiles; ++it) {
        const int s = it % kStages, row = at.first + (all - 1 - (it * split + part)) * kRows;
        const unsigned ph = ((it / kStages) & 1) ^ 1;
        if (!wait_or_abort(&bar.k_empty[s], ph, &bar.abort)) break;
        mbar_expect_tx(&bar.k_full[s], L::kTileBytes);
        load_tile<HD>(s_k + s * L::kTileBytes, mk, g, row, &bar.k_full[s]);
        issued = 2 * it + 1;
        if (!wait_or_abort(&bar.v_empty[s], ph, &bar.abort)) break;
        mbar_expect_tx(&bar.v_full[s], L::kTileBytes);
        load_tile<HD>(s_v + s * L::kTileBytes, mv, g, row, &bar.v_full[s]);
        issued = 2 * it + 2;
      }
      if (issued < 2 * tiles) land_copies<kStages>(issued, &bar.own_full, bar.k_full, bar.v_full);
    } else if (warp == 8 && lane == 0 && tiles > 0) {
      constexpr unsigned kk = mma_desc(128, false, false), kn = mma_desc(HD, false, true);
      bool ok = wait_or_abort(&bar.own_full, 0, &bar.abort) && wait_or_abort(&bar.k_full[0], 0, &bar.abort);
      if (ok) {
        product_ss<HD>(t_s, s_q, s_k, kk);
        mma_commit(&bar.s_full[0]);
        ok = wait_or_abort(&bar.v_full[0], 0, &bar.abort);
      }
      if (ok) {
        product_ss<HD>(t_dp, s_do, s_v, kk);
        mma_commit(&bar.dp_full);
        mma_commit(&bar.v_empty[0]);
      }
      for (int it = 0; ok && it < tiles; ++it) {
        const int s = it % kStages, sn = (it + 1) % kStages;
        const unsigned phn = ((it + 1) / kStages) & 1;
        const bool more = it + 1 < tiles;
        if (more) {
          ok = wait_or_abort(&bar.k_full[sn], phn, &bar.abort);
          if (!ok) break;
          product_ss<HD>(t_s + ((it + 1) & 1) * 128, s_q, s_k + sn * L::kTileBytes, kk);
          mma_commit(&bar.s_full[(it + 1) & 1]);
        }
        ok = wait_or_abort(&bar.ds_full, it & 1, &bar.abort);
        if (!ok) break;
        tmem_fence_after();
        product_ts(t_dq, t_dp, s_k + s * L::kTileBytes, kn, it > 0);
        mma_commit(&bar.k_empty[s]);
        if (more) {
          ok = wait_or_abort(&bar.v_full[sn], phn, &bar.abort);
          if (!ok) break;
          product_ss<HD>(t_dp, s_do, s_v + sn * L::kTileBytes, kk);
          mma_commit(&bar.dp_full);
          mma_commit(&bar.v_empty[sn]);
        } else {
          mma_commit(&bar.o_full);
        }
      }
    }
    __syncwarp();
    if (split > 1) {
      cluster_sync();
      cluster_sync();
    }
  } else {
    const int half = warp >> 2, r = threadIdx.x & 127, i = q0 + r;
    const bool mine = i < at.end;
    const unsigned lanes = (unsigned)(warp & 3) << 21;
    // delta: each half of the row's threads sums half of the columns
    float delta = 0.f;
    if (mine) {
      const __nv_bfloat16 *x = a.dout + (long long)i * a.do_row + h * a.do_head, *y = a.out_in + (long long)i * a.o_row + h * a.o_head;
#pragma unroll
      for (int c = 0; c < HD / 2; c += 8) {
        const int col = half * (HD / 2) + c;
        if (col < a.head_dim) {
          float u[8], v[8];
          load_vec<__nv_bfloat16, 8>(x + col, u);
          load_vec<__nv_bfloat16, 8>(y + col, v);
#pragma unroll
          for (int j = 0; j < 8; ++j) delta = fmaf(u[j], v[j], delta);
        }
      }
    }
    bar.delta[half][r] = delta;
    if (half == 0) bar.bad[r] = 0;
    math_sync();
    delta = bar.delta[0][r] + bar.delta[1][r];
    const long long stat = (long long)h * a.tokens + i;
    if (mine && half == 0 && part == 0) a.delta[stat] = delta;
    const float lse2 = mine ? a.lse[stat] * kLog2e : 0.f;
    const float c = a.scale_log2;
    bool ok = true;
    for (int it = 0; it < tiles; ++it) {
      ok = warp_wait(&bar.s_full[it & 1], (it >> 1) & 1, &bar.abort);
      if (!ok) break;
      tmem_fence_after();
      unsigned s[2][32];
#pragma unroll
      for (int u = 0; u < 2; ++u) tmem_load32(t_s + (it & 1) * 128 + half * 64 + u * 32 + lanes, s[u]);
      tmem_wait_load();
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          const float2 y = fma2(make_float2(__uint_as_float(s[u][j]), __uint_as_float(s[u][j + 1])), make_float2(c, c), make_float2(-lse2, -lse2));
          s[u][j] = __float_as_uint(ex2(y.x)), s[u][j + 1] = __float_as_uint(ex2(y.y));
        }
      const bool diagonal = it == 0 && part == 0;
      if (diagonal) { // it is the last of the sequence's tiles that this block sees
        const int valid = at.end - q0; // K rows of it inside the sequence
        if (valid < kRows) {
          ok = warp_wait(&bar.k_full[0], 0, &bar.abort);
          if (!ok) break;
          if (r >= valid) zero_row<HD>(s_k, r, half);
          fence_async_smem();
        }
      }
      ok = warp_wait(&bar.dp_full, it & 1, &bar.abort);
      if (!ok) break;
      tmem_fence_after();
      auto slopes = [&](auto masked) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          unsigned d[32], x[8];
          tmem_load32(t_dp + half * 64 + u * 32 + lanes, d);
          tmem_wait_load();
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float2 y = add2(make_float2(__uint_as_float(d[j]), __uint_as_float(d[j + 1])), make_float2(-delta, -delta));
            y = mul2(make_float2(__uint_as_float(s[u][j]), __uint_as_float(s[u][j + 1])), y);
            if (decltype(masked)::value) {
              if (half * 64 + u * 32 + j > r) y.x = 0.f;
              if (half * 64 + u * 32 + j + 1 > r) y.y = 0.f;
            }
            x[j / 2 % 8] = bf16_pair(y.x, y.y);
            if (j % 16 == 14) tmem_store8(t_dp + half * 64 + u * 16 + j / 16 * 8 + lanes, x);
          }
        }
      };
      if (diagonal) slopes(std::true_type{});
      else slopes(std::false_type{});
      tmem_wait_store();
      tmem_fence_before();
      mbar_arrive(&bar.ds_full);
    }
    if (ok && tiles > 0) ok = warp_wait(&bar.o_full, 0, &bar.abort);
    tmem_fence_after();
    if (split == 1) {
      if (ok) {
        const bool fine = put_row<HD / 2>(t_dq + lanes, a.dq + (long long)i * a.dq_row + h * a.dq_head, half * (HD / 2), a.head_dim, a.scale, mine);
        if (mine && !fine) bar.bad[r] = 1;
      }
    } else if (ok) {
      // every operand has been read: the tiles' place takes this block's sums
      if (tiles > 0) stage_row<HD / 2>(t_dq + lanes + half * (HD / 2), smem + half * (HD / 2) * kRows * 4, r);
      else
        for (int c = half * (HD / 8); c < (half + 1) * (HD / 8); ++c)
          asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(smem + (c * kRows + r) * 16), "r"(0) : "memory");
    }
    if (split == 1) {
      math_sync(); // both halves are written before a row is written again
    } else {
      cluster_sync(); // all blocks' sums are staged
      // eight columns at a time, dealt to the cluster's blocks and both halves
      if (mine && !bar.abort)
        for (int c = (part * 2 + half) * 8; c < a.head_dim; c += split * 16) {
          float v[8];
          sum_staged(v, smem, split, c, r);
          if (!put8(a.dq + (long long)i * a.dq_row + h * a.dq_head + c, v, a.scale)) mark_remote(smem_u32(&bar.bad[r]));
        }
      cluster_sync(); // and read: the row is written, and marked in the first block where it is not finite
    }
    if (half == 0 && part == 0 && !bar.abort)
      for (unsigned again = __ballot_sync(0xffffffffu, bar.bad[r] != 0); again; again &= again - 1)
        attn_dq_row(a, i - lane + __ffs(again) - 1, h, at.first, lane);
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 8) {
    tmem_fence_after();
    tmem_free(tmem, 512);
  }
  if (threadIdx.x == 0 && bar.abort && a.status) atomicExch(a.status, kStatusTimeout);
}

// --------------------------------------------------------------------------------- dk and dv
struct DkvBarriers {
  unsigned long long own_full, q_full[kStages], do_full[kStages], empty[kStages], stat_full[kStages], stat_empty[kStages];
  unsigned long long s_full, dp_full, p_full, ds_full, o_full;
  unsigned tmem;
  volatile unsigned abort;
  unsigned char bad[kRows];
};

template <int HD>
__global__ void __launch_bounds__(kBwdThreads, 1)
    attn_dkv_kernel(const AttnArgs a, const __grid_constant__ HeadMap mq, const __grid_constant__ HeadMap mk, const __grid_constant__ HeadMap mv,
                    const __grid_constant__ HeadMap mdo, int split) {
  using L = BwdLayout<HD>;
  extern __shared__ unsigned char raw_smem[];
  __shared__ DkvBarriers bar;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = cluster_rank(), unit = blockIdx.x / split, g = unit % a.kv_heads;
  grid_wait(); // delta is the work of the kernel before this one
  const Place at = place_of<true>(a, unit / a.kv_heads, kRows);
  if (at.block < 0) {
    if (part != 0) return;
    const int r0 = at.first + (-1 - at.block) * kRows;
    for (int r = r0 + warp; r < min(r0 + kRows, at.end); r += kBwdThreads / 32)
      for (int c = lane; c < a.head_dim; c += 32) {
        a.dk[r * a.dk_row + g * a.dk_head + c] = __float2bfloat16_rn(0.f);
        a.dv[r * a.dv_row + g * a.dv_head + c] = __float2bfloat16_rn(0.f);
      }
    return;
  }
  const int k0 = at.first + at.block * kRows; // first key
  if (k0 >= at.end) return;
  const int per_head = (at.end - k0 + kRows - 1) / kRows, all = per_head * a.group; // query tiles
  const int tiles = (all - part + split - 1) / split;                              // this block's: part, part + split, ...
  const unsigned smem = (smem_u32(raw_smem) + 1023) & ~1023u;
  const unsigned s_k = smem + L::kOwn, s_v = s_k + L::kTileBytes, s_q = smem + L::kRing, s_do = s_q + kStages * L::kTileBytes;
  // minus log-sum-exp (times log2 e) and minus delta of a query tile's rows
  float *stats = reinterpret_cast<float *>(raw_smem + (smem - smem_u32(raw_smem)) + L::kStats);

  if (warp == 8) tmem_alloc(&bar.tmem, 512);
  if (threadIdx.x == 0) {
    mbar_init(&bar.own_full, 1), mbar_init(&bar.s_full, 1), mbar_init(&bar.dp_full, 1), mbar_init(&bar.o_full, 1);
    mbar_init(&bar.p_full, 256), mbar_init(&bar.ds_full, 256);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bar.q_full[i], 1), mbar_init(&bar.do_full[i], 1), mbar_init(&bar.empty[i], 1);
      mbar_init(&bar.stat_full[i], 32), mbar_init(&bar.stat_empty[i], 256);
    }
    bar.abort = 0;
    fence_mbar_init();
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const unsigned tmem = bar.tmem, t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = t_dv + HD;

  if (warp >= 8) {
    if (warp == 9 && lane == 0) {
      int issued = 0;
      if (tiles > 0) {
        mbar_expect_tx(&bar.own_full, 2 * L::kTileBytes);
        load_tile<HD>(s_k, mk, g, k0, &bar.own_full);
        load_tile<HD>(s_v, mv, g, k0, &bar.own_full);
      }
      for (int it = 0; it < tiles; ++it) {
        const int s = it % kStages, n = it * split + part, h = g * a.group + n / per_head, row = k0 + (n % per_head) * kRows;
        if (!wait_or_abort(&bar.empty[s], ((it / kStages) & 1) ^ 1, &bar.abort)) break;
        mbar_expect_tx(&bar.q_full[s], L::kTileBytes);
        load_tile<HD>(s_q + s * L::kTileBytes, mq, h, row, &bar.q_full[s]);
        mbar_expect_tx(&bar.do_full[s], L::kTileBytes);
        load_tile<HD>(s_do + s * L::kTileBytes, mdo, h, row, &bar.do_full[s]);
        issued = 2 * it + 2;
      }
      if (issued < 2 * tiles) land_copies<kStages>(issued, &bar.own_full, bar.q_full, bar.do_full);
    } else if (warp == 10) {
      for (int it = 0; it < tiles; ++it) {
        const int s = it % kStages, n = it * split + part, h = g * a.group + n / per_head, row = k0 + (n % per_head) * kRows;
        if (!warp_wait(&bar.stat_empty[s], ((it / kStages) & 1) ^ 1, &bar.abort)) break;
        float *to = stats + s * 2 * kRows;
#pragma unroll
        for (int u = 0; u < kRows / 32; ++u) {
          const int i = row + u * 32 + lane;
          const bool in = i < at.end;
          const long long stat = (long long)h * a.tokens + i;
          to[u * 32 + lane] = in ? -a.lse[stat] * kLog2e : 0.f;
          to[kRows + u * 32 + lane] = in ? -a.delta[stat] : 0.f;
        }
        mbar_arrive(&bar.stat_full[s]);
      }
    } else if (warp == 8 && lane == 0 && tiles > 0) {
      constexpr unsigned kk = mma_desc(128, false, false), kn = mma_desc(HD, false, true);
      bool ok = wait_or_abort(&bar.own_full, 0, &bar.abort) && wait_or_abort(&bar.q_full[0], 0, &bar.abort);
      if (ok) {
        product_ss<HD>(t_s, s_k, s_q, kk);
        mma_commit(&bar.s_full);
        ok = wait_or_abort(&bar.do_full[0], 0, &bar.abort);
      }
      if (ok) {
        product_ss<HD>(t_dp, s_v, s_do, kk);
        mma_commit(&bar.dp_full);
      }
      for (int it = 0; ok && it < tiles; ++it) {
        const int s = it % kStages, sn = (it + 1) % kStages;
        const unsigned phn = ((it + 1) / kStages) & 1;
        const bool more = it + 1 < tiles;
        ok = wait_or_abort(&bar.p_full, it & 1, &bar.abort);
        if (!ok) break;
        tmem_fence_after();
        product_ts(t_dv, t_s, s_do + s * L::kTileBytes, kn, it > 0);
        if (more) {
          ok = wait_or_abort(&bar.q_full[sn], phn, &bar.abort);
          if (!ok) break;
          product_ss<HD>(t_s, s_k, s_q + sn * L::kTileBytes, kk);
          mma_commit(&bar.s_full);
        }
        ok = wait_or_abort(&bar.ds_full, it & 1, &bar.abort);
        if (!ok) break;
        tmem_fence_after();
        product_ts(t_dk, t_dp, s_q + s * L::kTileBytes, kn, it > 0);
        mma_commit(&bar.empty[s]);
        if (more) {
          ok = wait_or_abort(&bar.do_full[sn], phn, &bar.abort);
          if (!ok) break;
          product_ss<HD>(t_dp, s_v, s_do + sn * L::kTileBytes, kk);
          mma_commit(&bar.dp_full);
        } else {
          mma_commit(&bar.o_full);
        }
      }
    }
    __syncwarp();
    if (split > 1) {
      cluster_sync();
      cluster_sync();
    }
  } else {
    const int half = warp >> 2, r = threadIdx.x & 127, j0 = k0 + r; // this thread's key, and its half of the queries
    const bool mine = j0 < at.end;
    const unsigned lanes = (unsigned)(warp & 3) << 21;
    if (half == 0) bar.bad[r] = 0;
    const float c = a.scale_log2;
    bool ok = true;
    for (int it = 0; it < tiles; ++it) {
      const int st = it % kStages, t = (it * split + part) % per_head;
      const unsigned ph = (it / kStages) & 1;
      const int valid = at.end - (k0 + t * kRows); // query rows of this tile inside the sequence
      const bool edge = t == 0 || valid < kRows;
      ok = warp_wait(&bar.s_full, it & 1, &bar.abort);
      if (!ok) break;
      tmem_fence_after();
      unsigned s[2][32];
#pragma unroll
      for (int u = 0; u < 2; ++u) tmem_load32(t_s + half * 64 + u * 32 + lanes, s[u]);
      tmem_wait_load();
      ok = warp_wait(&bar.stat_full[st], ph, &bar.abort);
      if (!ok) break;
      const float4 *lse = reinterpret_cast<const float4 *>(stats + st * 2 * kRows + half * 64);
      const float4 *delta = lse + kRows / 4;
      // query q sees this key from the diagonal on, and there are `valid` queries: masks on the edge tiles alone
      auto hidden = [&](int u, int j) {
        const int q = half * 64 + u * 32 + j;
        return (t == 0 && q < r) || q >= valid;
      };
      auto weights = [&](auto masked) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          unsigned x[8];
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const float4 m = lse[u * 8 + j / 4];
            const float2 y[2] = {fma2(make_float2(__uint_as_float(s[u][j]), __uint_as_float(s[u][j + 1])), make_float2(c, c), make_float2(m.x, m.y)),
                                 fma2(make_float2(__uint_as_float(s[u][j + 2]), __uint_as_float(s[u][j + 3])), make_float2(c, c), make_float2(m.z, m.w))};
            float p[4] = {ex2(y[0].x), ex2(y[0].y), ex2(y[1].x), ex2(y[1].y)};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (decltype(masked)::value && hidden(u, j + e)) p[e] = 0.f;
              s[u][j + e] = __float_as_uint(p[e]);
            }
            x[j / 2 % 8] = bf16_pair(p[0], p[1]), x[j / 2 % 8 + 1] = bf16_pair(p[2], p[3]);
            if (j % 16 == 12) tmem_store8(t_s + half * 64 + u * 16 + j / 16 * 8 + lanes, x);
          }
        }
      };
      if (edge) weights(std::true_type{});
      else weights(std::false_type{});
      if (valid < kRows) {
        ok = warp_wait(&bar.q_full[st], ph, &bar.abort) && warp_wait(&bar.do_full[st], ph, &bar.abort);
        if (!ok) break;
        if (r >= valid) {
          zero_row<HD>(s_q + st * L::kTileBytes, r, half);
          zero_row<HD>(s_do + st * L::kTileBytes, r, half);
        }
        fence_async_smem();
      }
      tmem_wait_store();
      tmem_fence_before();
      mbar_arrive(&bar.p_full);

      ok = warp_wait(&bar.dp_full, it & 1, &bar.abort);
      if (!ok) break;
      tmem_fence_after();
      auto slopes = [&](auto masked) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          unsigned d[32], x[8];
          tmem_load32(t_dp + half * 64 + u * 32 + lanes, d);
          tmem_wait_load();
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const float4 m = delta[u * 8 + j / 4];
            float2 y[2] = {add2(make_float2(__uint_as_float(d[j]), __uint_as_float(d[j + 1])), make_float2(m.x, m.y)),
                           add2(make_float2(__uint_as_float(d[j + 2]), __uint_as_float(d[j + 3])), make_float2(m.z, m.w))};
            y[0] = mul2(make_float2(__uint_as_float(s[u][j]), __uint_as_float(s[u][j + 1])), y[0]);
            y[1] = mul2(make_float2(__uint_as_float(s[u][j + 2]), __uint_as_float(s[u][j + 3])), y[1]);
            if (decltype(masked)::value) { // 0 * (infinity or NaN of a row that is not seen)
              if (hidden(u, j)) y[0].x = 0.f;
              if (hidden(u, j + 1)) y[0].y = 0.f;
              if (hidden(u, j + 2)) y[1].x = 0.f;
              if (hidden(u, j + 3)) y[1].y = 0.f;
            }
            x[j / 2 % 8] = bf16_pair(y[0].x, y[0].y), x[j / 2 % 8 + 1] = bf16_pair(y[1].x, y[1].y);
            if (j % 16 == 12) tmem_store8(t_dp + half * 64 + u * 16 + j / 16 * 8 + lanes, x);
          }
        }
      };
      if (edge) slopes(std::true_type{});
      else slopes(std::false_type{});
      tmem_wait_store();
      tmem_fence_before();
      mbar_arrive(&bar.ds_full);
      mbar_arrive(&bar.stat_empty[st]);
    }
    if (ok && tiles > 0) ok = warp_wait(&bar.o_full, 0, &bar.abort);
    tmem_fence_after();
    if (split == 1) {
      if (ok) {
        bool fine = put_row<HD / 2>(t_dv + lanes, a.dv + (long long)j0 * a.dv_row + g * a.dv_head, half * (HD / 2), a.head_dim, 1.f, mine);
        fine &= put_row<HD / 2>(t_dk + lanes, a.dk + (long long)j0 * a.dk_row + g * a.dk_head, half * (HD / 2), a.head_dim, a.scale, mine);
        if (mine && !fine) bar.bad[r] = 1;
      }
    } else if (ok) {
      // every operand has been read: the tiles' place takes this block's sums, dv by warps 0-3, dk by warps 4-7
      const unsigned to = smem + half * HD * kRows * 4;
      if (tiles > 0) stage_row<HD>((half ? t_dk : t_dv) + lanes, to, r);
      else
        for (int c = 0; c < HD / 4; ++c) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to + (c * kRows + r) * 16), "r"(0) : "memory");
    }
    if (split == 1) {
      math_sync(); // both halves are written before a row is written again
    } else {
      cluster_sync(); // all blocks' sums are staged
      __nv_bfloat16 *row = half ? a.dk + (long long)j0 * a.dk_row + g * a.dk_head : a.dv + (long long)j0 * a.dv_row + g * a.dv_head;
      if (mine && !bar.abort)
        for (int c = part * 8; c < a.head_dim; c += split * 8) {
          float v[8];
          sum_staged(v, smem + half * HD * kRows * 4, split, c, r);
          if (!put8(row + c, v, half ? a.scale : 1.f)) mark_remote(smem_u32(&bar.bad[r]));
        }
      cluster_sync(); // and read: the row is written, and marked in the first block where it is not finite
    }
    if (half == 0 && part == 0 && !bar.abort)
      for (unsigned again = __ballot_sync(0xffffffffu, bar.bad[r] != 0); again; again &= again - 1)
        attn_dkv_row(a, j0 - lane + __ffs(again) - 1, g, at.end, lane);
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 8) {
    tmem_fence_after();
    tmem_free(tmem, 512);
  }
  if (threadIdx.x == 0 && bar.abort && a.status) atomicExch(a.status, kStatusTimeout);
}

template <int HD> int launch(const AttnArgs &a, const HeadMap &mq, const HeadMap &mk, const HeadMap &mv, const HeadMap &mdo, cudaStream_t s) {
  constexpr int bytes = BwdLayout<HD>::kBytes;
  static OncePerDevice once;
  if (!once.get([] { return allow_smem(attn_dq_kernel<HD>, bytes) && allow_smem(attn_dkv_kernel<HD>, bytes); })) return DILOCO_ERR_CUDA;
  int dev = 0;
  cudaGetDevice(&dev);
  const int sms = sm_count(dev);
  const long long ranks = ranks_of(a, kRows);
  const int by_q = split_of(a, kRows, a.heads, 1, sms), by_k = split_of(a, kRows, a.kv_heads, a.group, sms);
  const int rc = launch_split(attn_dq_kernel<HD>, ranks * a.heads, by_q, kBwdThreads, bytes, s, false, a, mq, mk, mv, mdo, by_q);
  if (rc != DILOCO_OK) return rc;
  return launch_split(attn_dkv_kernel<HD>, ranks * a.kv_heads, by_k, kBwdThreads, bytes, s, true, a, mq, mk, mv, mdo, by_k);
}

} // namespace

int attn_backward(const AttnArgs &a, cudaStream_t s) {
  HeadMap mq, mk, mv, mdo;
  int rc = encode_heads(&mq, a.q, a.head_dim, a.heads, a.q_head, a.tokens, a.q_row, kRows);
  if (rc == DILOCO_OK) rc = encode_heads(&mk, a.k, a.head_dim, a.kv_heads, a.k_head, a.tokens, a.k_row, kRows);
  if (rc == DILOCO_OK) rc = encode_heads(&mv, a.v, a.head_dim, a.kv_heads, a.v_head, a.tokens, a.v_row, kRows);
  if (rc == DILOCO_OK) rc = encode_heads(&mdo, a.dout, a.head_dim, a.heads, a.do_head, a.tokens, a.do_row, kRows);
  if (rc != DILOCO_OK) return rc;
  return a.head_dim <= 64 ? launch<64>(a, mq, mk, mv, mdo, s) : launch<128>(a, mq, mk, mv, mdo, s);
}

} // namespace diloco
