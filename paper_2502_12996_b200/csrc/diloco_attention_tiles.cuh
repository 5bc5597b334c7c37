// What the tensor-core attention kernels share: which rows a block has, tiles of 128 rows in shared memory and
// their products.
#pragma once
#include "diloco_attention_rows.cuh"
#include "diloco_tcgen05.cuh"

namespace diloco {

constexpr int kRows = 128, kPanel = 128 * 128; // rows of a tile, bytes of a panel of 64 columns

// Slot -> sequence and block of `rows` rows.  Sequence b's blocks start at slot cu[b] / rows + b: there is room for each
// sequence's last, partial block, and no prefix sum is needed; slots in between are empty.  Sequence number
// `sequences` stands for the rows behind the last one.  Whatever cu_seqlens holds, rows are inside the tensors.
struct Place {
  int first, end, block; // block < 0: block -1 - block of the rows of no sequence
};
__device__ __forceinline__ Place place_of(const AttnArgs &a, int slot, int rows) {
  auto start = [&](int b) { return min(max(a.cu[b], 0), a.tokens); };
  int lo = 0, hi = a.sequences;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start(mid) / rows + mid <= slot) lo = mid;
    else hi = mid - 1;
  }
  Place p;
  p.first = start(lo);
  p.end = lo == a.sequences ? a.tokens : start(lo + 1);
  p.block = slot - (p.first / rows + lo);
  if (lo == a.sequences) p.block = -1 - p.block;
  return p;
}

template <int HD> __device__ __forceinline__ void load_tile(unsigned smem, const HeadMap &m, int head, int row, unsigned long long *bar) {
#pragma unroll
  for (int p = 0; p < HD / 64; ++p) load_panel(smem + p * kPanel, m, p * 64, head, row, bar);
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

// [128 rows of a] x [128 rows of b] over HD columns, both in shared memory
template <int HD> __device__ __forceinline__ void product_ss(unsigned d, unsigned a, unsigned b, unsigned idesc) {
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
    const unsigned off = (i / 4) * kPanel + (i % 4) * 32;
    mma_ss(d, tile_desc(a + off, kPanel), tile_desc(b + off, kPanel), idesc, i > 0);
  }
}
// [128 x 128 bf16 in tensor memory: columns 0-63 at a, 64-127 at a + 64] x [128 rows of b], summed over b's rows
__device__ __forceinline__ void product_ts(unsigned d, unsigned a, unsigned b, unsigned idesc, bool add) {
#pragma unroll
  for (int i = 0; i < 8; ++i) mma_ts(d, a + (i / 4) * 64 + (i % 4) * 8, tile_desc(b + i * 2048, kPanel), idesc, add || i > 0);
}

// Row r of a tile in shared memory; `half` 0 / 1: one half of its bytes
template <int HD> __device__ __forceinline__ void zero_row(unsigned tile, int r, int half) {
#pragma unroll
  for (int p = 0; p < HD / 64; ++p)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + p * kPanel + r * 128 + (half * 4 + u) * 16), "r"(0) : "memory");
}

} // namespace diloco
