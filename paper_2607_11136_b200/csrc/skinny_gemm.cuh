// The same products for few tokens at a time, where what counts is how fast the weights arrive and that all SMs take part.
//
// Features are the rows of the MMA and tokens its columns: a CTA takes R features (a multiple of 8) for a tile of up to NT tokens,
// and a cluster of S CTAs shares K, so that all SMs stream weights with all the bytes in flight that their rings hold.  An MMA reads 128
// rows whatever R is and takes 50 to 73 clocks; what lies behind the R rows only reaches lanes that nobody looks at.  Few features are
// therefore better covered by CTAs with many rows and a part of K each.  The partial sums meet through distributed shared memory and
// are added in the order of the ranks.
//
//   kGated   gate and up rows lie behind one another and are one MMA up to R = 64, two beyond
//   kGradX   dx = dg Wg + du Wu: features are columns of the weights, which are read as they lie (M-major operand)
//   kShrink  t = scale_a x A_a^T of one request a tile: features are the adapter's columns
//   kLora    y = x W^T + bias + t B_a^T for single tokens: the epilogue warps work out t B^T on the CUDA cores while the weights stream
//   kPacked  the same for requests of a few rows: a tile holds `slots` requests of `pad` columns (a multiple of 16) each, and an
//            adapter's second product is an MMA on the columns of its request alone -- no other request's sums meet its values
//
// Bound by HBM where the weights come from there: gated, one token of 4096 x 11264 in bf16 (185 MB) 31.4 us (5.9 TB/s), 24 tokens of 4096 x
// 16384 in e4m3 (135 MB) 23.4 us (5.8 TB/s), back to back in a graph; with 128 x 128 tiles 52 and 36.  4096 x 4096 by one CTA of 32
// features each 13.7 us (once 20.6, with a single block a stage); K shared by 2 or 4 CTAs 14.0 and 13.7.  dx of 333 tokens, 512 x 8192, with dg and
// du: 57 us by single CTAs, 25 with K shared by 4.  48 tokens with adapters of rank 16, 4096 x 4096: 141 us by tiles of a request each, 12.3 here.
#pragma once
#include "tile_gemm.cuh"

namespace xema {
namespace skinny {
using namespace sm100;

enum class Kind { kGated, kGradX, kShrink, kLora, kPacked };

constexpr int kThreads = 192;
constexpr int kSmem = 231424;                 // of the 232448 bytes that a CTA may have
constexpr int kHalfSmem = 115712;             // two CTAs an SM
constexpr int kTail = 16384;                  // rows that an MMA reads behind the last stage's; kLora: beside it the adapters' sums
constexpr int kMaxStages = 16, kMaxSplit = 4;

struct Params {
  int rows, cols, batch;          // tokens (kShrink, kPacked: of a request, of `batch`), features
  int nt, tiles, f_tiles;         // columns of the MMA; token tiles; feature tiles
  int R, split, S;                // features of a cluster, CTAs in it; split: gate and up are products of their own
  int k_blocks, per_cta;          // blocks of 128 bytes along K; of one CTA
  int k_half;                     // kGradX: of the gate's half
  int ks, stages;                 // blocks per stage, stages
  int tail, smem;                 // bytes behind the ring; of shared memory
  int act;
  const float *row_scale, *gate_scale, *up_scale;   // e4m3
  __nv_bfloat16* out;
  long long ldo, out_batch_rows;
  __nv_bfloat16* z;               // kGated: [3][rows][cols], or null
  const __nv_bfloat16 *bias, *t, *lora_b;           // kLora, kPacked
  const int* adapter;             // kShrink, kLora, kPacked
  const float* adapter_scale;     // kShrink
  int n_adapters, rank;
  int slots, pad;                 // kPacked
  int behind;                     // launched right behind the kernel that makes t, which waited for everything before it
  unsigned int* status;
};
struct Maps {
  CUtensorMap a, a2, x, t;        // weights (gate, up; kPacked: W, B) in boxes of R rows, tokens, t (kPacked)
};

__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float c) {
  c = fmaf(bf16_lo(a.x), bf16_lo(b.x), c); c = fmaf(bf16_hi(a.x), bf16_hi(b.x), c);
  c = fmaf(bf16_lo(a.y), bf16_lo(b.y), c); c = fmaf(bf16_hi(a.y), bf16_hi(b.y), c);
  c = fmaf(bf16_lo(a.z), bf16_lo(b.z), c); c = fmaf(bf16_hi(a.z), bf16_hi(b.z), c);
  c = fmaf(bf16_lo(a.w), bf16_lo(b.w), c); c = fmaf(bf16_hi(a.w), bf16_hi(b.w), c);
  return c;
}

// Eight neighbouring sums of all S CTAs of the cluster, added in the order of their ranks.
__device__ __forceinline__ void add_partials(const float* own, int S, float (&v)[8]) {
  if (S == 1) {
    *reinterpret_cast<float4*>(v) = reinterpret_cast<const float4*>(own)[0];
    *reinterpret_cast<float4*>(v + 4) = reinterpret_cast<const float4*>(own)[1];
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = 0.f;
#pragma unroll 4
  for (int s = 0; s < S; ++s) {
    const uint32_t at = mapa_shared(smem_u32(own), s);
    float u[8];
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(u[0]), "=f"(u[1]), "=f"(u[2]), "=f"(u[3]) : "r"(at));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(u[4]), "=f"(u[5]), "=f"(u[6]), "=f"(u[7]) : "r"(at + 16));
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += u[k];
  }
}
__device__ __forceinline__ void store_bf16x8(__nv_bfloat16* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ int valid_adapter(const Params& p, int b) {
  const int a = b < p.batch ? p.adapter[b] : -1;
  return a < p.n_adapters ? a : -1;
}

template <Kind KIND, bool F8, int NT>
__global__ void __launch_bounds__(kThreads, 2) skinny_kernel(const __grid_constant__ Maps maps, const Params p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr bool GATED = KIND == Kind::kGated, GRAD = KIND == Kind::kGradX, SHRINK = KIND == Kind::kShrink;
  constexpr bool LORA = KIND == Kind::kLora, PACKED = KIND == Kind::kPacked;
  constexpr int STEP = F8 ? 128 : 64;
  constexpr int TMEM_COLS = GATED ? 2 * NT : NT < 32 ? 32 : NT;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + p.smem - 512);
  uint64_t* empty = full + kMaxStages;
  uint64_t* done = empty + kMaxStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int nt = PACKED ? p.nt : NT;
  const int cluster = blockIdx.x / p.S, rank = blockIdx.x - cluster * p.S;
  const int tile = cluster / p.f_tiles, f0 = (cluster - tile * p.f_tiles) * p.R;
  // the tile's request (kPacked: first one), and its first token in it
  const int per_slab = PACKED ? (p.rows + p.pad - 1) / p.pad : (p.rows + NT - 1) / NT;
  const int slab = SHRINK || PACKED ? tile / per_slab : 0;
  const int b0 = PACKED ? slab * p.slots : slab, t0 = (tile - slab * per_slab) * (PACKED ? p.pad : NT);
  const int n_tok = PACKED ? nt : min(NT, p.rows - t0), n_feat = min(p.R, p.cols - f0);
  const int w_rows = (GATED ? 2 : 1) * p.R;
  const int block_bytes = (w_rows + nt) * 128, stage_bytes = p.ks * block_bytes;
  const int k0 = rank * p.per_cta, k_end = min(p.k_blocks, k0 + p.per_cta);
  const int n_stages = (k_end - k0 + p.ks - 1) / p.ks;
  // results in groups of eight features; this CTA finishes [first, last) of them
  const int groups = n_feat / 8, first = n_tok * groups * rank / p.S, last = n_tok * groups * (rank + 1) / p.S;
  float* sums = reinterpret_cast<float*>(smem);                                // [n_tok][w_rows]
  float* delta = reinterpret_cast<float*>(smem + p.smem - 512 - p.tail);       // kLora: [last - first][8]
  const bool aligned = (smem_u32(smem) & 1023u) == 0;

  if constexpr (SHRINK) {
    // (ahead of grid_dep_launch() below, as everywhere: the next launch reads x and W before its own wait)
    grid_dep_wait();
    if (valid_adapter(p, b0) < 0) return;      // the whole cluster
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(done, 1);
    *abort_flag = aligned ? 0u : 1u;
    fence_mbar_init();
    prefetch_tmap(&maps.a);
    prefetch_tmap(&maps.x);
    if (GATED || GRAD || PACKED) prefetch_tmap(&maps.a2);
    if (PACKED) prefetch_tmap(&maps.t);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  // as in tile_gemm.cuh: everything waits for the launch before this one, or only what needs t and the results
  const bool late = (LORA || PACKED) && p.behind;
  if (!late) {
    grid_dep_wait();
    if (threadIdx.x == 0) grid_dep_launch();
    __syncwarp();
  }

  // kPacked: lane j has slot j's adapter
  const int my_adapter = PACKED && lane < p.slots ? valid_adapter(p, b0 + lane) : -1;
  if (warp == 0) {
    // ---------------- TMA producer ----------------
    bool ok = aligned;
    int stage = 0;
    uint32_t phase = 0;
    const int adapter = SHRINK ? valid_adapter(p, b0) : 0;
    for (int s = 0; ok && s < n_stages; ++s) {
      if (!(ok = mbar_wait_warp(&empty[stage], phase ^ 1, abort_flag))) break;
      if (elect_one()) {
        const int kb = k0 + s * p.ks, n = min(p.ks, k_end - kb);
        uint8_t* st = smem + stage * stage_bytes;
        mbar_expect_tx(&full[stage], n * block_bytes);
        if constexpr (GRAD) {
          for (int u = 0; u < n; ++u) {
            const int half = kb + u >= p.k_half, k = (kb + u - half * p.k_half) * STEP;
            uint8_t* at = st + u * block_bytes;
            tma_load_3d(at, half ? &maps.a2 : &maps.a, &full[stage], f0, k, 0);
            if (p.R > 64) tma_load_3d(at + 8192, half ? &maps.a2 : &maps.a, &full[stage], f0 + 64, k, 0);
            tma_load_3d(at + w_rows * 128, &maps.x, &full[stage], k, t0, half);
          }
        } else {
          // an operand's blocks behind one another: they are neighbours in its rows
          for (int u = 0; u < n; ++u) tma_load_3d(st + u * block_bytes, &maps.a, &full[stage], (kb + u) * STEP, f0, adapter);
          if (GATED)
            for (int u = 0; u < n; ++u) tma_load_3d(st + u * block_bytes + p.R * 128, &maps.a2, &full[stage], (kb + u) * STEP, f0, 0);
          for (int u = 0; u < n; ++u) {
            uint8_t* at = st + u * block_bytes + w_rows * 128;
            if constexpr (PACKED) {
              for (int j = 0; j < p.slots; ++j) tma_load_3d(at + j * p.pad * 128, &maps.x, &full[stage], (kb + u) * STEP, t0, b0 + j);
            } else {
              tma_load_3d(at, &maps.x, &full[stage], (kb + u) * STEP, t0, b0);
            }
          }
        }
      }
      __syncwarp();
      if (++stage == p.stages) { stage = 0; phase ^= 1; }
    }
    if constexpr (PACKED) {
      if (late) grid_dep_wait();
      for (int j = rank; ok && j < p.slots; j += p.S) {
        const int a = __shfl_sync(0xffffffffu, my_adapter, j);
        for (int k = 0; a >= 0 && k < p.rank; k += 64) {
          if (!(ok = mbar_wait_warp(&empty[stage], phase ^ 1, abort_flag))) break;
          if (elect_one()) {
            uint8_t* st = smem + stage * stage_bytes;
            mbar_expect_tx(&full[stage], (p.R + p.pad) * 128);
            tma_load_3d(st, &maps.a2, &full[stage], k, f0, a);
            tma_load_3d(st + w_rows * 128, &maps.t, &full[stage], k, t0, b0 + j);
          }
          __syncwarp();
          if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
      }
    }
    if (!ok && aligned) {
      report_timeout(p.status);
      // gave up: copies under way must land before the CTA leaves
      if (lane == 0) {
        for (int s = 0; s < p.stages; ++s) {
          const int st = (stage + s) % p.stages;
          volatile uint32_t dummy = 0;
          mbar_wait_slow(&full[st], st < stage ? phase : phase ^ 1, &dummy, 100000000ll);
        }
      }
      __syncwarp();
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    const uint32_t idesc = F8 ? idesc_e4m3_f32(128, nt) : idesc_bf16_f32(128, nt, GRAD, false);
    constexpr uint64_t A_ADV = GRAD ? 2048 >> 4 : 2;           // 16 rows of 128 bytes, or 32 bytes of a row
    const uint64_t a0 = smem_desc_sw128(smem_u32(smem), GRAD ? 8192 : 16, 1024), x0 = smem_desc_sw128(smem_u32(smem), 16, 1024);
    bool ok = aligned;
    int stage = 0;
    uint32_t phase = 0;
    for (int s = 0; ok && s < n_stages; ++s) {
      if (!(ok = mbar_wait_warp(&full[stage], phase, abort_flag))) break;
      tc_fence_after();
      if (elect_one()) {
        const int n = min(p.ks, k_end - k0 - s * p.ks);
        for (int u = 0; u < n; ++u) {
          const uint64_t at = (uint64_t)((stage * stage_bytes + u * block_bytes) >> 4), a = a0 + at, b = x0 + at + (uint64_t)(w_rows * 8);
          const uint64_t a2 = a + (uint64_t)(p.R * 8);
          auto mma = [&](uint32_t d, uint64_t ad, uint64_t bd, uint32_t acc) {
            if constexpr (F8) mma_ss_f8(d, ad, bd, idesc, acc);
            else mma_ss(d, ad, bd, idesc, acc);
          };
#pragma unroll
          for (int k = 0; k < 4; ++k) mma(tmem_base, a + A_ADV * k, b + 2 * k, s > 0 || u > 0 || k > 0);
          if (GATED && p.split) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma(tmem_base + NT, a2 + 2 * k, b + 2 * k, s > 0 || u > 0 || k > 0);
          }
        }
        mma_commit(&empty[stage]);
      }
      __syncwarp();
      if (++stage == p.stages) { stage = 0; phase ^= 1; }
    }
    if constexpr (PACKED) {
      const uint32_t idesc_slot = idesc_bf16_f32(128, p.pad, false, false);
      for (int j = rank; ok && j < p.slots; j += p.S) {
        const int a = __shfl_sync(0xffffffffu, my_adapter, j);
        for (int k = 0; a >= 0 && k < p.rank; k += 64) {
          if (!(ok = mbar_wait_warp(&full[stage], phase, abort_flag))) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t at = (uint64_t)((stage * stage_bytes) >> 4);
            const int steps = min(4, (p.rank - k + 15) / 16);
            for (int i = 0; i < steps; ++i)
              mma_ss(tmem_base + j * p.pad, a0 + at + 2 * i, x0 + at + (uint64_t)(w_rows * 8) + 2 * i, idesc_slot, 1);
            mma_commit(&empty[stage]);
          }
          __syncwarp();
          if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
      }
    }
    if (ok && elect_one()) mma_commit(done);
    __syncwarp();
    if (!ok) report_timeout(p.status);
  } else {
    // ---------------- epilogue ----------------
    const int quad = warp & 3, et = threadIdx.x - 64;
    if (late) {
      grid_dep_wait();
      if (et == 0) grid_dep_launch();
      __syncwarp();
    }
    if constexpr (LORA) {
      for (int i = first + et; i < last; i += 128) {
        const int tok = i / groups, f = f0 + (i - tok * groups) * 8, a = p.adapter[t0 + tok];
        float v[8] = {};
        if (a >= p.n_adapters && p.status) atomicExch(p.status, XEMA_DEVICE_STATUS_ADAPTER);
        if (a >= 0 && a < p.n_adapters) {
          const uint4* w = reinterpret_cast<const uint4*>(p.lora_b + ((size_t)a * p.cols + f) * p.rank);
          const uint4* t = reinterpret_cast<const uint4*>(p.t + (size_t)(t0 + tok) * p.rank);
          const int steps = p.rank / 8;
#pragma unroll 2
          for (int g = 0; g < steps; ++g) {
            const uint4 tv = ld_u4(t + g);
            uint4 wv[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) wv[k] = ld_u4(w + k * steps + g);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = dot8(tv, wv[k], v[k]);
          }
        }
        if (p.bias) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] += __bfloat162float(p.bias[f + k]);
        }
        float4* d = reinterpret_cast<float4*>(delta + (i - first) * 8);
        d[0] = make_float4(v[0], v[1], v[2], v[3]);
        d[1] = make_float4(v[4], v[5], v[6], v[7]);
      }
    }
    if constexpr (PACKED) {
      if (et < p.slots && b0 + et < p.batch && p.adapter[b0 + et] >= p.n_adapters && p.status) atomicExch(p.status, XEMA_DEVICE_STATUS_ADAPTER);
    }
    __syncwarp();              // (the lanes' last groups differ; the loads from TMEM want whole warps)
    const bool ok = aligned && mbar_wait_warp(done, 0, abort_flag);
    if (!ok) report_timeout(p.status);
    tc_fence_after();
    if (ok) {
      // all MMAs are done, so the ring is free: sums as [token][row] (fp32), row = gate features, then up
      const int row = quad * 32 + lane;
      const uint32_t t_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
      const int rows_in = p.split ? p.R : w_rows;          // rows of one product
#pragma unroll 1
      for (int h = 0; h < (GATED && p.split ? 2 : 1); ++h) {
#pragma unroll 1
        for (int c = 0; c < n_tok; c += 16) {
          uint32_t r[16];
          tmem_ld16(t_addr + h * NT + c, r);
          tmem_ld_wait_on(r);
          if (row < rows_in) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
              if (c + k < n_tok) sums[(c + k) * w_rows + h * p.R + row] = __uint_as_float(r[k]);
          }
        }
      }
      tc_fence_before();
    }
  }

  tc_fence_before();
  __syncthreads();
  // TMEM goes back before the cluster meets: a CTA that waits for its peers holds nothing that one of them may still wait for
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, TMEM_COLS);
  }
  __syncwarp();
  if (p.S > 1) {
    cluster_arrive();
    cluster_wait();
  }
  if (!*abort_flag) {
    for (int i = first + threadIdx.x; i < last; i += kThreads) {
      const int tok = i / groups, f = (i - tok * groups) * 8;
      long long row = t0 + tok;
      if constexpr (PACKED) {
        const int j = tok / p.pad;
        const long long at = t0 + tok - j * p.pad;
        if (at >= p.rows || b0 + j >= p.batch) continue;
        row = (b0 + j) * p.out_batch_rows + at;
      }
      if constexpr (SHRINK) row += (long long)b0 * p.rows;
      if constexpr (LORA) row *= p.out_batch_rows;
      float v[8];
      add_partials(sums + tok * w_rows + f, p.S, v);
      if constexpr (LORA) {
        const float* d = delta + (i - first) * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += d[k];
      }
      if constexpr (PACKED) {
        if (p.bias) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] += __bfloat162float(p.bias[f0 + f + k]);
        }
      }
      if constexpr (SHRINK) {
        const float scale = p.adapter_scale[valid_adapter(p, b0)];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= scale;
      }
      if constexpr (GATED) {
        float w[8];
        add_partials(sums + tok * w_rows + p.R + f, p.S, w);
        if constexpr (F8) {
          const float rs = p.row_scale[row];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            v[k] *= rs * p.gate_scale[f0 + f + k];
            w[k] *= rs * p.up_scale[f0 + f + k];
          }
        }
        if (!F8 && p.z) {
          store_bf16x8(p.z + row * p.cols + f0 + f, v);
          store_bf16x8(p.z + ((long long)p.rows + row) * p.cols + f0 + f, w);
          uint32_t low[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) low[k] = tiles::low_bytes(v[2 * k], w[2 * k]) | tiles::low_bytes(v[2 * k + 1], w[2 * k + 1]) << 16;
          *reinterpret_cast<uint4*>(p.z + (2LL * p.rows + row) * p.cols + f0 + f) = make_uint4(low[0], low[1], low[2], low[3]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] * tiles::sigmoid_f(tiles::act_q(v[k], p.act)) * w[k];
      }
      store_bf16x8(p.out + row * p.ldo + f0 + f, v);
    }
  }
  if (p.S > 1) {
    __syncwarp();              // (the lanes' last groups differ; the barrier wants whole warps)
    cluster_arrive();          // nobody leaves while its sums may still be read
    cluster_wait();
  }
}

// The instance for a tile of `nt` columns.
template <Kind KIND, bool F8, int NT>
int launch_clusters(const Maps& maps, const Params& p, cudaStream_t stream, int* max_clusters) {
  static PerDeviceInt attr_done, clusters[kMaxSplit + 1];
  auto kern = skinny_kernel<KIND, F8, NT>;
  if (int rc = ensure_smem_attr(kern, kSmem, attr_done)) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = p.S;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  if (max_clusters) {       // only asked how many clusters of S CTAs the device holds
    const int dev = current_device(), i = p.S;
    *max_clusters = clusters[i].get(dev);
    if (*max_clusters) return XEMA_OK;
    cfg.gridDim = dim3(sm_count() / p.S * p.S, 1, 1);
    cfg.numAttrs = 1;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(max_clusters, kern, &cfg);
    if (e != cudaSuccess || *max_clusters <= 0) {
      set_last_cuda_error((int)e);
      return XEMA_ECUDA;
    }
    clusters[i].set(dev, *max_clusters);
    return XEMA_OK;
  }
  const long long ctas = (long long)p.f_tiles * p.S * p.tiles;
  if (ctas > 0x7fffffffLL) return XEMA_EINVAL;
  cfg.gridDim = dim3((unsigned)ctas, 1, 1);
  cfg.numAttrs = KIND == Kind::kGradX ? 1 : 2;       // (tile_gemm.cuh: the gradients' products are not chained)
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, maps, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    set_last_cuda_error((int)e);
    return XEMA_ECUDA;
  }
  return XEMA_OK;
}
template <Kind KIND, bool F8>
int launch(const Maps& maps, const Params& p, cudaStream_t stream, int* max_clusters = nullptr) {
  if constexpr (KIND == Kind::kPacked) {
    return launch_clusters<KIND, F8, 128>(maps, p, stream, max_clusters);
  } else {
    switch (p.nt) {
      case 16: return launch_clusters<KIND, F8, 16>(maps, p, stream, max_clusters);
      case 32: return launch_clusters<KIND, F8, 32>(maps, p, stream, max_clusters);
      case 64: return launch_clusters<KIND, F8, 64>(maps, p, stream, max_clusters);
      default: return launch_clusters<KIND, F8, 128>(maps, p, stream, max_clusters);
    }
  }
}

// Token tiles: fills nt, tiles, and slots and pad of kPacked, from rows and batch.
template <Kind KIND>
inline int tile_tokens(Params* p) {
  long long tiles;
  if constexpr (KIND == Kind::kPacked) {
    p->pad = p->rows > 128 ? 128 : (p->rows + 15) / 16 * 16;
    p->slots = p->rows > 128 ? 1 : std::min(128 / p->pad, p->batch);
    p->nt = p->slots * p->pad;
    tiles = (long long)((p->batch + p->slots - 1) / p->slots) * ((p->rows + p->pad - 1) / p->pad);
  } else {
    p->nt = p->rows <= 16 ? 16 : p->rows <= 32 ? 32 : p->rows <= 64 ? 64 : 128;
    tiles = (long long)((p->rows + p->nt - 1) / p->nt) * (KIND == Kind::kShrink ? p->batch : 1);
  }
  if (tiles > 0x7fffffffLL) return XEMA_EINVAL;
  p->tiles = (int)tiles;
  return XEMA_OK;
}

// Fills S, R, split and what follows from them: the pair with the shortest estimate, in clocks, of what bounds a CTA -- its MMAs (26
// clocks + operand bytes / 170 each, and the round of a stage's barriers), its fill (57 bytes a clock) or its share of the memory's
// rate (3400 bytes a clock for all).  *ns: the estimate.  only_s, only_r: this S or R and no other.
template <Kind KIND, bool F8>
int plan(Params* p, long long* ns, int only_s = 0, int only_r = 0) {
  constexpr bool GATED = KIND == Kind::kGated, PACKED = KIND == Kind::kPacked;
  if (only_r < 0 || only_r > 128 || only_r % (KIND == Kind::kGradX ? 64 : 8)) return XEMA_EINVAL;
  if (int rc = tile_tokens<KIND>(p)) return rc;
  const int nt = p->nt, groups = p->cols / 8, token_tiles = p->tiles;
  const long long mma = 26 + (4096 + nt * 32) / 170;
  long long best = 0;
  Params q = *p;
  for (int s = 1; s <= kMaxSplit; s *= 2) {
    q.S = s;
    q.per_cta = (p->k_blocks + s - 1) / s;
    if ((s - 1) * q.per_cta >= p->k_blocks) continue;          // a CTA without a block
    if (only_s && s != only_s) continue;
    int clusters = 0;
    q.smem = kSmem;
    if (int rc = launch<KIND, F8>(Maps{}, q, nullptr, &clusters)) return rc;
    const long long units = (long long)groups * token_tiles;
    const int waves0 = (int)std::min<long long>((units + 16LL * clusters - 1) / (16LL * clusters), 1 << 20);
    // features of a CTA: as few waves as 128 allow, one more, or 128; one CTA an SM, or two that hide each other's ends
    for (int choice = 0; choice < 6; ++choice) {
      const int waves = waves0 + choice / 2, per_sm = 1 + choice % 2;
      const long long fit = (units + (long long)clusters * waves - 1) / ((long long)clusters * waves);
      q.R = choice >= 4 ? 128 : (int)std::min<long long>(128, 8 * fit);
      if (only_r) q.R = only_r;
      if (KIND == Kind::kGradX) q.R = q.R > 64 ? 128 : 64;
      if (KIND == Kind::kShrink) q.R = p->cols;
      q.split = GATED && q.R > 64;
      const int w_rows = (GATED ? 2 : 1) * q.R, block = (w_rows + nt) * 128, sums = nt * w_rows * 4;
      q.tail = std::max(kTail, KIND == Kind::kLora ? (nt * q.R * 4 / s + 2047) / 1024 * 1024 : 0);
      const int room = (per_sm == 2 ? kHalfSmem : kSmem) - 512 - q.tail;
      q.ks = std::max(1, std::min(std::min(4, q.per_cta), room / (4 * block)));
      const int more = PACKED ? (q.slots + s - 1) / s * ((p->rank + 63) / 64) : 0;
      q.stages = std::min(std::min(kMaxStages, room / (q.ks * block)), (q.per_cta + q.ks - 1) / q.ks + more);
      if (q.stages < 1 || room < sums) continue;
      q.smem = 512 + q.tail + (std::max(q.stages * q.ks * block, sums) + 1023) / 1024 * 1024;
      q.f_tiles = (p->cols + q.R - 1) / q.R;
      const long long ctas = (long long)q.f_tiles * token_tiles * s, slots = (long long)clusters * s * per_sm, rounds = (ctas + slots - 1) / slots;
      const long long issue = PACKED ? std::max(4 * mma + 300 / q.ks, 60LL * (q.slots + 1)) * 3 / 2 : 4 * (q.split ? 2 : 1) * mma + 300 / q.ks;   // (kPacked: several loads a block)
      auto work = [&](int n) {      // of a CTA with n on its SM
        return (q.per_cta + more) * std::max({n * issue, n * block / 57LL, std::min(ctas, (long long)clusters * s * n) * w_rows * 128 / 3400 / token_tiles});
      };
      const long long ends = 3300 + nt * q.R / 6 + (s > 1 ? 1500 + nt * w_rows / 3 : 0);
      const long long clocks = per_sm == 2 && ctas > (long long)clusters * s ? rounds * std::max(work(2), work(1) + ends) + ends : rounds * (work(1) + ends);
      if (best == 0 || clocks < best) {
        best = clocks;
        *p = q;
      }
    }
  }
  *ns = best * 10 / 19;
  return best ? XEMA_OK : XEMA_EINVAL;
}

}  // namespace skinny
}  // namespace xema
