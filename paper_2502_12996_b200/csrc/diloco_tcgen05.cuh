// Fifth-generation tensor cores and tensor maps, as the attention kernels use them: tensor memory, shared-memory
// operand descriptors for 128-byte swizzled bf16 tiles, and waits that end.
#pragma once
#include <cuda.h>

#include "diloco_bulk.cuh"
#include "diloco_ops.cuh"

namespace diloco {

constexpr unsigned long long kOpWaitNs = 1000000000ull; // bound of one wait

// A wait that gives up raises `abort` (shared memory) so that every role of the block leaves its loop.  Each poll after
// the first looks at the clock, which also spaces them: polls without it, or with a suspension time, took issue slots from
// the arithmetic beside them (1 to 3 % of the kernels).
__device__ __forceinline__ bool wait_or_abort(unsigned long long *bar, unsigned parity, volatile unsigned *abort) {
  if (mbar_try_wait(bar, parity)) return true;
  if (mbar_wait_bounded(bar, parity, kOpWaitNs, abort)) return true;
  *abort = 1;
  return false;
}
// The same for a whole warp, with one answer for all its lanes: what follows may be warp-wide.
__device__ __forceinline__ bool warp_wait(unsigned long long *bar, unsigned parity, volatile unsigned *abort) {
  return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort));
}
__device__ __forceinline__ void mbar_arrive(unsigned long long *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ bool elect_one() {
  unsigned p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}

// Register shares of a block's warpgroups (of 4 warps).  They draw on what the block was launched with, threads x
// registers a thread: the shares of all warpgroups together must not exceed it.
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// ---------------------------------------------------------------------------- tensor memory
__device__ __forceinline__ void tmem_alloc(unsigned *where, unsigned columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(unsigned at, unsigned columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define DILOCO_R8(v, o) "=r"(v[o]), "=r"(v[o + 1]), "=r"(v[o + 2]), "=r"(v[o + 3]), "=r"(v[o + 4]), "=r"(v[o + 5]), "=r"(v[o + 6]), "=r"(v[o + 7])
#define DILOCO_I8(v, o) "r"(v[o]), "r"(v[o + 1]), "r"(v[o + 2]), "r"(v[o + 3]), "r"(v[o + 4]), "r"(v[o + 5]), "r"(v[o + 6]), "r"(v[o + 7])
// 32 (16) consecutive columns of this thread's lane
__device__ __forceinline__ void tmem_load32(unsigned at, unsigned (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
      "%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : DILOCO_R8(v, 0), DILOCO_R8(v, 8), DILOCO_R8(v, 16), DILOCO_R8(v, 24)
      : "r"(at));
}
__device__ __forceinline__ void tmem_store32(unsigned at, const unsigned (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31};" ::DILOCO_I8(v, 0), DILOCO_I8(v, 8), DILOCO_I8(v, 16), DILOCO_I8(v, 24), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_store16(unsigned at, const unsigned (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::DILOCO_I8(v, 0),
               DILOCO_I8(v, 8), "r"(at)
               : "memory");
}

__device__ __forceinline__ void tmem_store8(unsigned at, const unsigned (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::DILOCO_I8(v, 0), "r"(at) : "memory");
}

// ------------------------------------------------------------------------- matrix instructions
// kind::f16, bf16 operands, fp32 accumulator [128 lanes, N columns]
__host__ __device__ constexpr unsigned mma_desc(int n, bool a_mn_major, bool b_mn_major, bool negate_a = false) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (negate_a ? 1u << 13 : 0u) | (a_mn_major ? 1u << 15 : 0u) | (b_mn_major ? 1u << 16 : 0u) |
         ((unsigned)(n >> 3) << 17) | ((128u >> 4) << 24);
}
// Operand tiles are panels of 64 bf16 columns: [rows][128 bytes], 16-byte units of row r permuted by r mod 8 (the
// 128-byte swizzle of TMA), panels 1024-byte aligned.  Used with the columns as the product's inner dimension
// (K-major): 8-row groups 1024 bytes apart.  Used with the rows as the inner dimension (MN-major): 8-row
// groups 1024 bytes apart along it, and the next 64 columns one panel (`panel` bytes) further.
__device__ __forceinline__ unsigned long long tile_desc(unsigned smem, unsigned panel) {
  return (unsigned long long)((smem & 0x3ffff) >> 4) | ((unsigned long long)(panel >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_ss(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(unsigned d, unsigned a, unsigned long long b, unsigned idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
      : "memory");
}
// `bar` completes when everything issued so far by this thread has
__device__ __forceinline__ void mma_commit(unsigned long long *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// ----------------------------------------------------------------------------------- TMA
// A [tokens, heads, head_dim] tensor as panels of 64 columns x 128 rows of one head.  The map's axes are in order of
// their strides; `token_last`: the token axis is the outermost.  A broadcast head axis has one element.
struct HeadMap {
  CUtensorMap map;
  int token_last, head_mul;
};
__device__ __forceinline__ void load_panel(unsigned smem, const HeadMap &m, int col, int head, int row, unsigned long long *bar) {
  const int h = head * m.head_mul;
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem),
               "l"(&m.map), "r"(col), "r"(m.token_last ? h : row), "r"(m.token_last ? row : h), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void prefetch_map(const HeadMap &m) { asm volatile("prefetch.tensormap [%0];" ::"l"(&m.map) : "memory"); }

int encode_heads(HeadMap *m, const void *base, int head_dim, int heads, long long head_stride, long long tokens, long long row_stride,
                 int box_rows);

} // namespace diloco
