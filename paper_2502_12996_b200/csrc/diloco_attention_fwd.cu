// Causal attention over packed sequences, forward, on the fifth-generation tensor cores.
//
// Per head and query row i: z_ij = scale q_i . k_j, running maximum m and sum l of 2^((z - m) log2 e), out = sum_j P_ij v_j / l.
// A block holds 256 query rows of one sequence and head as two tiles of 128 rows and walks the keys in tiles of
// 128, from the diagonal down to the sequence's start:
//   warps 0-3, 4-7  softmax of tile 0 and 1, one row a thread (a tensor-memory lane): loads S, keeps m and l in
//                   registers, writes P as bf16 over S, rescales the accumulator where the maximum grew
//   warp 8          issues S = Q K^T (both from shared memory) and O += P V (P from tensor memory)
//   warp 9          TMA: Q once, K and V tiles through a ring of stages (warps 10 and 11 only complete the warpgroup)
// Tensor memory (512 columns): S0, S1 (128 each, P in their place), O0, O1.  While one tile is in its softmax the
// tensor cores work on the other.
//
// Rescaling: a row keeps its old maximum until the new one is 2^8 above it (weights up to 2^8, held in bf16 and summed in
// fp32, lose nothing), so that O is rarely read back; the statistics stay exact since l uses the same maximum.
// Tiles of a sequence that start together on both axes need a mask on the diagonal tile alone.  V rows behind the
// sequence's end are zeroed in shared memory (0 * NaN); a row that comes out non-finite all the same is computed
// again over the rows that it sees alone, so that a later token's NaN cannot reach an earlier one.
#include <type_traits>

#include "diloco_attention_tiles.cuh"

namespace diloco {
namespace {

constexpr int kFwdThreads = 384;
// launched with 168 registers a thread (64512 of a block): 2 x 128 x 208 + 128 x 88 = 64512
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;

template <int HD> struct FwdLayout {
  static constexpr int kPanels = HD / 64;
  static constexpr int kTileBytes = kPanels * kPanel;
  static constexpr int kStages = HD == 128 ? 2 : 4;
  static constexpr int kQ = 0, kK = 2 * kTileBytes, kV = kK + kStages * kTileBytes;
  static constexpr int kBytes = kV + kStages * kTileBytes + 1024; // 1024: alignment of the panels
};

struct FwdBarriers {
  unsigned long long q_full, k_full[4], v_full[4], k_empty[4], v_empty[4], s_full[2], p_full[2], o_full[2];
  unsigned tmem;
  volatile unsigned abort;
};

template <int HD>
__global__ void __launch_bounds__(kFwdThreads, 1)
    attn_forward_kernel(const AttnArgs a, const __grid_constant__ HeadMap mq, const __grid_constant__ HeadMap mk, const __grid_constant__ HeadMap mv,
                        int slots, int negate) {
  using L = FwdLayout<HD>;
  extern __shared__ unsigned char raw_smem[];
  __shared__ FwdBarriers bar;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.x % a.heads, g = h / a.group;
  const Place at = place_of(a, slots - 1 - (int)(blockIdx.x / a.heads), 2 * kRows);
  if (at.block < 0) { // rows of no sequence
    const int r0 = at.first + (-1 - at.block) * 2 * kRows;
    for (int r = r0 + warp; r < min(r0 + 2 * kRows, at.end); r += kFwdThreads / 32) {
      for (int c = lane; c < a.head_dim; c += 32) a.out[r * a.o_row + h * a.o_head + c] = __float2bfloat16_rn(0.f);
      if (lane == 0) a.lse[(long long)h * a.tokens + r] = -INFINITY;
    }
    return;
  }
  const int q0 = at.first + at.block * 2 * kRows; // first query row
  if (q0 >= at.end) return;                       // an empty slot
  const bool two = at.end - q0 > kRows;           // the second tile has rows
  const int tiles = 2 * at.block + 1 + (two ? 1 : 0);
  const unsigned smem = (smem_u32(raw_smem) + 1023) & ~1023u;

  if (warp == 8) tmem_alloc(&bar.tmem, 512);
  if (threadIdx.x == 0) {
    mbar_init(&bar.q_full, 1);
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(&bar.k_full[i], 1), mbar_init(&bar.v_full[i], 1);
      mbar_init(&bar.k_empty[i], 1), mbar_init(&bar.v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&bar.s_full[i], 1), mbar_init(&bar.p_full[i], kRows), mbar_init(&bar.o_full[i], 1);
    bar.abort = 0;
    fence_mbar_init();
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const unsigned tmem = bar.tmem;

  if (warp >= 8) {
    registers_down<kOtherRegs>();
    if (warp == 9) {
      // ------------------------------------------------------------------------------ loads
      if (lane == 0) {
        int issued = 0; // K and V tiles in flight or landed, for the give-up path
        mbar_expect_tx(&bar.q_full, (two ? 2 : 1) * L::kTileBytes);
        for (int w = 0; w < (two ? 2 : 1); ++w)
          load_tile<HD>(smem + L::kQ + w * L::kTileBytes, mq, h, q0 + w * kRows, &bar.q_full);
        for (int it = 0; it < tiles; ++it) {
          const int s = it % L::kStages, row = at.first + (tiles - 1 - it) * kRows;
          const unsigned ph = ((it / L::kStages) & 1) ^ 1;
          if (!wait_or_abort(&bar.k_empty[s], ph, &bar.abort)) break;
          mbar_expect_tx(&bar.k_full[s], L::kTileBytes);
          load_tile<HD>(smem + L::kK + s * L::kTileBytes, mk, g, row, &bar.k_full[s]);
          issued = 2 * it + 1;
          if (!wait_or_abort(&bar.v_empty[s], ph, &bar.abort)) break;
          mbar_expect_tx(&bar.v_full[s], L::kTileBytes);
          load_tile<HD>(smem + L::kV + s * L::kTileBytes, mv, g, row, &bar.v_full[s]);
          issued = 2 * it + 2;
        }
        if (issued < 2 * tiles) land_copies<L::kStages>(issued, &bar.q_full, bar.k_full, bar.v_full);
      }
    } else if (warp == 8) {
      // --------------------------------------------------------------------- matrix products
      if (lane == 0) {
        const unsigned qk_desc = mma_desc(128, false, false) | (negate ? 1u << 13 : 0u), pv_desc = mma_desc(HD, false, true);
        auto qk = [&](int w, int s) {
          product_ss<HD>(tmem + w * 128, smem + L::kQ + w * L::kTileBytes, smem + L::kK + s * L::kTileBytes, qk_desc);
          mma_commit(&bar.s_full[w]);
        };
        auto pv = [&](int w, int s, bool add) {
          const unsigned v = smem + L::kV + s * L::kTileBytes;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            mma_ts(tmem + 256 + w * HD, tmem + w * 128 + i * 8, tile_desc(v + i * 2048, kPanel), pv_desc, add || i > 0);
        };
        const int start0 = two ? 1 : 0; // tile 0 sees one key tile less
        bool ok = wait_or_abort(&bar.q_full, 0, &bar.abort) && wait_or_abort(&bar.k_full[0], 0, &bar.abort);
        if (ok) {
          qk(two ? 1 : 0, 0);
          mma_commit(&bar.k_empty[0]);
        }
        for (int it = 0; ok && it < tiles; ++it) {
          const int s = it % L::kStages, sn = (it + 1) % L::kStages;
          const unsigned ph = (it / L::kStages) & 1, phn = ((it + 1) / L::kStages) & 1;
          const bool more = it + 1 < tiles;
          for (int w = 0; ok && w < (two ? 2 : 1); ++w) {
            const int n = w == 0 ? it - start0 : it; // this tile's own count of key tiles
            if (n >= 0) {
              ok = wait_or_abort(&bar.p_full[w], n & 1, &bar.abort) && wait_or_abort(&bar.v_full[s], ph, &bar.abort);
              if (!ok) break;
              tmem_fence_after();
              pv(w, s, n > 0);
              if (!more) mma_commit(&bar.o_full[w]);
            }
            if (more) {
              ok = wait_or_abort(&bar.k_full[sn], phn, &bar.abort);
              if (!ok) break;
              qk(w, sn);
            }
          }
          if (ok) {
            mma_commit(&bar.v_empty[s]);
            if (more) mma_commit(&bar.k_empty[sn]);
          }
        }
      }
    }
  } else {
    registers_up<kSoftmaxRegs>();
    // ----------------------------------------------------------------------------- softmax
    const int w = warp >> 2, r = threadIdx.x & 127;
    if (w == 0 || two) {
      const unsigned lanes = (unsigned)(warp & 3) << 21; // this warp's 32 lanes, in bits 16 and up
      const unsigned ts = tmem + w * 128 + lanes, to = tmem + 256 + w * HD + lanes;
      const int n_tiles = 2 * at.block + 1 + w;
      const float c = fabsf(a.scale_log2);
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      for (int n = 0; n < n_tiles; ++n) {
        ok = warp_wait(&bar.s_full[w], n & 1, &bar.abort);
        if (!ok) break;
        tmem_fence_after();
        unsigned s[4][32];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_load32(ts + i * 32, s[i]);
        tmem_wait_load();
        if (n == 0) { // the diagonal tile: key j of query r only where j <= r
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (i * 32 + j > r) s[i][j] = 0xff800000u;
        }
        float top[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          top[i] = max3(__uint_as_float(s[i][0]), __uint_as_float(s[i][1]), __uint_as_float(s[i][2]));
#pragma unroll
          for (int j = 3; j < 31; j += 2) top[i] = max3(top[i], __uint_as_float(s[i][j]), __uint_as_float(s[i][j + 1]));
          top[i] = fmaxf(top[i], __uint_as_float(s[i][31]));
        }
        const float mt = fmaxf(max3(top[0], top[1], top[2]), top[3]);
        if (n == 0) m = mt;
        else {
          const bool grew = (mt - m) * c > 8.f;
          if (__any_sync(0xffffffffu, grew)) {
            const float mn = fmaxf(m, mt), f = ex2((m - mn) * c);
            m = mn;
            l *= f;
#pragma unroll
            for (int i = 0; i < HD; i += 32) {
              unsigned o[32];
              tmem_load32(to + i, o);
              tmem_wait_load();
#pragma unroll
              for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_store32(to + i, o);
            }
          }
        }
        const float2 mc = make_float2(-m * c, -m * c), cc = make_float2(c, c);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        auto weights = [&](auto masked) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            unsigned p[16];
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float2 y = fma2(make_float2(__uint_as_float(s[i][j]), __uint_as_float(s[i][j + 1])), cc, mc);
              float2 x = make_float2(ex2(y.x), ex2(y.y));
              if (decltype(masked)::value) { // scale = 0 leaves no -infinity in the masked places
                if (i * 32 + j > r) x.x = 0.f;
                if (i * 32 + j + 1 > r) x.y = 0.f;
              }
              sum[(j >> 1) & 1] = add2(sum[(j >> 1) & 1], x);
              p[j / 2] = bf16_pair(x.x, x.y);
            }
            tmem_store16(ts + i * 16, p);
          }
        };
        if (n == 0) weights(std::true_type{});
        else weights(std::false_type{});
        sum[0] = add2(sum[0], sum[1]);
        l += sum[0].x + sum[0].y;
        if (n == 0) {
          const int valid = at.end - (q0 + w * kRows); // V rows of this tile inside the sequence
          if (valid < kRows) {
            ok = warp_wait(&bar.v_full[0], 0, &bar.abort);
            if (!ok) break;
            if (r >= valid) zero_row<HD>(smem + L::kV, r, 0), zero_row<HD>(smem + L::kV, r, 1);
            fence_async_smem();
          }
        }
        tmem_wait_store();
        tmem_fence_before();
        mbar_arrive(&bar.p_full[w]);
      }
      if (ok) ok = warp_wait(&bar.o_full[w], 0, &bar.abort);
      if (ok) {
        tmem_fence_after();
        const int i = q0 + w * kRows + r;
        const bool mine = i < at.end;
        const float inv = 1.f / l;
        bool fine = true;
        __nv_bfloat16 *out = a.out + (long long)i * a.o_row + h * a.o_head;
#pragma unroll
        for (int c0 = 0; c0 < HD; c0 += 32) {
          unsigned o[32];
          tmem_load32(to + c0, o);
          tmem_wait_load();
          float v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            v[j] = __uint_as_float(o[j]) * inv;
            fine &= fabsf(v[j]) < INFINITY;
          }
          if (mine) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (c0 + u * 8 < a.head_dim) {
                uint4 x;
                x.x = bf16_pair(v[u * 8], v[u * 8 + 1]), x.y = bf16_pair(v[u * 8 + 2], v[u * 8 + 3]);
                x.z = bf16_pair(v[u * 8 + 4], v[u * 8 + 5]), x.w = bf16_pair(v[u * 8 + 6], v[u * 8 + 7]);
                *reinterpret_cast<uint4 *>(out + c0 + u * 8) = x;
              }
          }
        }
        if (mine) a.lse[(long long)h * a.tokens + i] = m * c * kLn2 + logf(l);
        __syncwarp();
        for (unsigned again = __ballot_sync(0xffffffffu, mine && !fine); again; again &= again - 1)
          attn_out_row(a, i - lane + __ffs(again) - 1, h, at.first, lane);
      }
    }
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 8) {
    tmem_fence_after();
    tmem_free(tmem, 512);
  }
  if (threadIdx.x == 0 && bar.abort && a.status) atomicExch(a.status, kStatusTimeout);
}

template <int HD> int launch(const AttnArgs &a, const HeadMap &mq, const HeadMap &mk, const HeadMap &mv, cudaStream_t s) {
  auto kernel = attn_forward_kernel<HD>;
  static OncePerDevice once;
  if (!once.get([&] { return allow_smem(kernel, FwdLayout<HD>::kBytes); })) return DILOCO_ERR_CUDA;
  const long long slots = (long long)a.tokens / (2 * kRows) + a.sequences + 1;
  if (slots * a.heads > INT32_MAX) return DILOCO_ERR_UNSUPPORTED;
  kernel<<<(unsigned)(slots * a.heads), kFwdThreads, FwdLayout<HD>::kBytes, s>>>(a, mq, mk, mv, (int)slots, a.scale < 0.f);
  return launched();
}

} // namespace

int attn_forward(const AttnArgs &a, cudaStream_t s) {
  HeadMap mq, mk, mv;
  int rc = encode_heads(&mq, a.q, a.head_dim, a.heads, a.q_head, a.tokens, a.q_row, kRows);
  if (rc == DILOCO_OK) rc = encode_heads(&mk, a.k, a.head_dim, a.kv_heads, a.k_head, a.tokens, a.k_row, kRows);
  if (rc == DILOCO_OK) rc = encode_heads(&mv, a.v, a.head_dim, a.kv_heads, a.v_head, a.tokens, a.v_row, kRows);
  if (rc != DILOCO_OK) return rc;
  return a.head_dim <= 64 ? launch<64>(a, mq, mk, mv, s) : launch<128>(a, mq, mk, mv, s);
}

} // namespace diloco
