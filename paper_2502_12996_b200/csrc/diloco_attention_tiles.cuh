// What the tensor-core attention kernels share: which rows a block has, tiles of 128 rows in shared memory and
// their products.
#pragma once
#include "diloco_attention_rows.cuh"
#include "diloco_tcgen05.cuh"

namespace diloco {

constexpr int kRows = 128, kPanel = 128 * 128; // rows of a tile, bytes of a panel of 64 columns

// Rank -> sequence and block of `rows` rows, by a whole warp; dearest blocks first, since blocks are handed out in
// order and the last ones to start decide when the kernel ends.  A sequence of n blocks has one of every cost 1 .. n
// (forward and dq: block c - 1 walks c blocks of keys; dk and dv: block n - c is seen by c blocks of queries), so the
// blocks of cost c and above number sum_b max(0, n_b - c + 1): a binary search finds a rank's cost, and its place within that cost
// its sequence.  Behind the sequences' blocks come those of the rows behind the last sequence, then empty ranks.  With
// more than 1024 sequences (short ones, whose order matters little) ranks are slots: sequence b's blocks start at
// slot cu[b] / rows + b, which has room for every partial block, and no sum is needed.  Whatever cu_seqlens holds, rows are
// inside the tensors.
struct Place {
  int first, end, block; // block < 0: block -1 - block of the rows of no sequence; first + block * rows >= end: nothing
};
template <bool FROM_END> __device__ __forceinline__ Place place_of(const AttnArgs &a, int rank, int rows) {
  const int lane = threadIdx.x & 31, B = a.sequences;
  auto start = [&](int b) { return min(max(a.cu[b], 0), a.tokens); };
  Place p;
  if (B > 1024) {
    int lo = 0, hi = B;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (start(mid) / rows + mid <= rank) lo = mid;
      else hi = mid - 1;
    }
    p.first = start(lo);
    p.end = lo == B ? a.tokens : start(lo + 1);
    p.block = rank - (p.first / rows + lo);
    if (lo == B) p.block = -1 - p.block;
    return p;
  }
  auto blocks = [&](int b) { return b < B ? max(start(b + 1) - start(b) + rows - 1, 0) / rows : 0; };
  const int n0 = blocks(lane); // the first 32 sequences stay in registers
  auto count = [&](int c) {    // blocks of cost c and above
    int n = max(0, n0 - c + 1);
    for (int b = 32; b < B; b += 32) n += max(0, blocks(b + lane) - c + 1);
    return __reduce_add_sync(0xffffffffu, n);
  };
  const int total = count(1);
  if (rank >= total) {
    p.first = start(B), p.end = a.tokens, p.block = -1 - (rank - total);
    return p;
  }
  int lo = 1, hi = a.tokens / rows + 1; // count(lo) > rank
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (count(mid) > rank) lo = mid;
    else hi = mid - 1;
  }
  int nth = rank - count(lo + 1); // which of the sequences with a block of cost `lo`
  for (int b = 0; b < B; b += 32) {
    const int n = b == 0 ? n0 : blocks(b + lane);
    const unsigned has = __ballot_sync(0xffffffffu, n >= lo);
    if (nth < __popc(has)) {
      const int at = (int)__fns(has, 0, nth + 1);
      p.first = start(b + at), p.end = start(b + at + 1);
      p.block = FROM_END ? __shfl_sync(0xffffffffu, n, at) - lo : lo - 1;
      return p;
    }
    nth -= __popc(has);
  }
  p.first = p.end = 0, p.block = 0; // not reached
  return p;
}
// Ranks that a kernel has to start for every head: all sequences' blocks, the rows behind them, and empty ones.
inline long long ranks_of(const AttnArgs &a, int rows) { return (long long)a.tokens / rows + a.sequences + 1; }

// How many blocks share one tile's loop (a cluster, 1 to 8): doubled while the tiles do not fill the `slots` (blocks that
// the SMs hold) and a tile of average length still leaves every block two steps.  (Clusters are dearer to start: two
// blocks a tile where 264 tiles met 148 slots took 216 us instead of 181, and clusters of two for all ragged calls, the
// short tiles' second blocks leaving at once, 168 instead of 115.)
inline int split_of(const AttnArgs &a, int rows, int heads, int steps_per_row_block, int slots) {
  const long long tiles = ((long long)a.tokens / rows + (a.sequences + 1) / 2) * heads;
  const long long steps = (long long)a.tokens / (a.sequences > 0 ? a.sequences : 1) / rows * steps_per_row_block / 2;
  int s = 1;
  while (s < 8 && tiles * s < slots && steps >= 4ll * s) s *= 2;
  return s;
}

__device__ __forceinline__ int cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return (int)r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// shared memory of block `rank` of the cluster, at the place of this block's `smem`
__device__ __forceinline__ unsigned remote(unsigned smem, int rank) {
  unsigned r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 load_remote4(unsigned at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float load_remote(unsigned at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
// An accumulator's row (this thread's lane) as fp32 into shared memory, four columns by four: [N / 4][128 rows][4].
template <int N> __device__ __forceinline__ void stage_row(unsigned tmem, unsigned smem, int r) {
#pragma unroll
  for (int i = 0; i < N; i += 32) {
    unsigned o[32];
    tmem_load32(tmem + i, o);
    tmem_wait_load();
#pragma unroll
    for (int u = 0; u < 8; ++u)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(smem + ((i / 4 + u) * kRows + r) * 16), "r"(o[u * 4]), "r"(o[u * 4 + 1]),
                   "r"(o[u * 4 + 2]), "r"(o[u * 4 + 3])
                   : "memory");
  }
}
// A row's columns c0 .. c0 + 8 of a staged accumulator, summed over the cluster's blocks in their order.
__device__ __forceinline__ void sum_staged(float (&v)[8], unsigned smem, int split, int c0, int r) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = 0.f;
  for (int b = 0; b < split; ++b) {
    const unsigned at = remote(smem + (c0 / 4 * kRows + r) * 16, b);
    const float4 x = load_remote4(at), y = load_remote4(at + kRows * 16);
    const float w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    Each<8>::add(v, v, w);
  }
}
__device__ __forceinline__ bool put8(__nv_bfloat16 *to, float (&v)[8], float factor) {
  bool fine = true;
  Each<8>::mul(v, v, factor);
#pragma unroll
  for (int j = 0; j < 8; ++j) fine &= fabsf(v[j]) < INFINITY;
  store_vec<__nv_bfloat16, 8>(to, v);
  return fine;
}

// Marks a row in the cluster's first block.
__device__ __forceinline__ void mark_remote(unsigned smem) {
  asm volatile("st.shared::cluster.u8 [%0], %1;" ::"r"(remote(smem, 0)), "r"(1) : "memory");
}

// N columns from c0 of an accumulator's row (this thread's lane) times `factor` to bf16; whether all of them are finite.
template <int N> __device__ __forceinline__ bool put_row(unsigned tmem, __nv_bfloat16 *row, int c0, int head_dim, float factor, bool mine) {
  bool fine = true;
#pragma unroll
  for (int i = 0; i < N; i += 32) {
    unsigned o[32];
    tmem_load32(tmem + c0 + i, o);
    tmem_wait_load();
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      v[j] = __uint_as_float(o[j]) * factor;
      fine &= fabsf(v[j]) < INFINITY;
    }
    if (mine) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (c0 + i + u * 8 < head_dim) {
          uint4 x;
          x.x = bf16_pair(v[u * 8], v[u * 8 + 1]), x.y = bf16_pair(v[u * 8 + 2], v[u * 8 + 3]);
          x.z = bf16_pair(v[u * 8 + 4], v[u * 8 + 5]), x.w = bf16_pair(v[u * 8 + 6], v[u * 8 + 7]);
          *reinterpret_cast<uint4 *>(row + c0 + i + u * 8) = x;
        }
    }
  }
  return fine;
}

// Launch of blocks in clusters of `split`, which may follow the kernel before it on the stream as launch_chained's do.
template <typename... KArgs, typename... Args>
int launch_split(void (*kernel)(KArgs...), long long blocks, int split, int threads, int smem, cudaStream_t s, bool chained, Args... args) {
  if (blocks * split > INT32_MAX) return DILOCO_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks * split));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = split, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = chained ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return cuda_fail(e);
  }
  count_launch();
  return DILOCO_OK;
}

// ROWS rows by boxes of BOX rows, panels of 64 columns one behind the other
template <int HD, int ROWS = kRows, int BOX = kRows>
__device__ __forceinline__ void load_tile(unsigned smem, const HeadMap &m, int head, int row, unsigned long long *bar) {
#pragma unroll
  for (int p = 0; p < HD / 64; ++p)
#pragma unroll
    for (int b = 0; b < ROWS; b += BOX) load_panel(smem + p * ROWS * 128 + b * 128, m, p * 64, head, row + b, bar);
}

// Shared memory is not given back under a copy: after a wait that gave up, the loads still in flight of a block's own
// tiles and of two rings (copy n: tile n / 2, first ring where n is even) are waited for, within the limit.
template <int STAGES>
__device__ __forceinline__ void land_copies(int issued, unsigned long long *own, unsigned long long *first, unsigned long long *second) {
  mbar_wait_bounded(own, 0, kOpWaitNs, nullptr);
  for (int n = issued - 1; n >= 0 && n >= issued - 2 * STAGES; --n) {
    const int it = n / 2, s = it % STAGES;
    mbar_wait_bounded(n & 1 ? &second[s] : &first[s], (it / STAGES) & 1, kOpWaitNs, nullptr);
  }
}

// Keeps what is computed from `x` inside its loop: descriptors of a whole loop's products do not fit the registers.
__device__ __forceinline__ unsigned opaque(unsigned x) {
  asm volatile("" : "+r"(x));
  return x;
}

// [128 rows of a] x [128 rows of b] over HD columns, both in shared memory
template <int HD> __device__ __forceinline__ void product_ss(unsigned d, unsigned a, unsigned b, unsigned idesc) {
  const unsigned long long da = tile_desc(opaque(a), kPanel), db = tile_desc(opaque(b), kPanel); // addresses in units of 16 bytes at the bottom
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
    const unsigned off = ((i / 4) * kPanel + (i % 4) * 32) / 16;
    mma_ss(d, da + off, db + off, idesc, i > 0);
  }
}
// [128 x ROWS bf16 in tensor memory: every 32 numbers in the first 16 of 32 columns] x [ROWS rows of b], summed over b's rows
template <int ROWS> __device__ __forceinline__ void product_ts(unsigned d, unsigned a, unsigned b, unsigned idesc, bool add) {
  const unsigned long long db = tile_desc(opaque(b), kPanel);
#pragma unroll
  for (int i = 0; i < ROWS / 16; ++i) mma_ts(d, a + (i / 2) * 32 + (i % 2) * 8, db + i * (2048 / 16), idesc, add || i > 0);
}

// Row r of a tile of ROWS rows in shared memory, or one of `parts` equal parts of its bytes
template <int HD, int ROWS = kRows> __device__ __forceinline__ void zero_row(unsigned tile, int r, int part = 0, int parts = 1) {
  for (int u = part; u < HD / 8; u += parts)
    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (u / 8) * ROWS * 128 + r * 128 + (u % 8) * 16), "r"(0) : "memory");
}

} // namespace diloco
