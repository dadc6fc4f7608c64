// Persistent tcgen05 products of the gated feed-forward, its gradients and the projections with adapters.
//
//   kGated   h = act(x Wg^T) * (x Wu^T): half of a tile's columns are gate, half up, for the same features, so that the product
//            happens in the epilogue and neither projection goes to memory (unless the gradient asks for them)
//   kLinear  y = x W^T + bias + t B^T: the adapter's second product is further steps along K of the same accumulator
//   kGradX   dx = dg Wg + du Wu: one accumulator over both; the weights are read as they lie (N-major operand)
//   kGradW   dWg = dg^T x, dWu = du^T x: both operands are read as they lie (M- and N-major), the reduction is over tokens
//
// Shapes: two neighbouring SMs on a tile of 256 rows and 128 to 256 columns (PAIR, cta_group::2: each CTA has its 128 rows of A and one
// half of B), and one CTA on a 128 x 128 tile.  A step along the reduction is 128 bytes of an operand's row: 64 bf16 or 128 e4m3 values;
// whatever lies past an end reads as zero and is not written.
//
//   warp 0    TMA producer into a ring of stages (128-byte swizzle)
//   warp 1    owns TMEM; one elected lane issues the MMAs into one of two accumulators
//   warps 2-9 epilogue of the finished accumulator (thread = row, two warps a row take 32 columns in turn) while the next tile's products
//             fill the other one
// Barriers and ends of the pair form are those of the block's GEMM: all loads of a pair complete on the even CTA's full[], releases
// are multicast commits, every wait on an mbarrier is bounded and reported where it gives up, and no CTA leaves while its peer may still
// touch it.  griddepcontrol.wait, the TMEM allocation, __syncthreads and the cluster barriers have no limit, and a launch that stood in one of them
// would leave no status: they wait for earlier launches, which hold nothing of this one, and for warps whose own waits end.
//
// Bound by the tensor pipe and, in long runs, by the board's power: launches by themselves of 8192 x 4096 x 11264 gated 926 to 937 us (1614 to
// 1633 TFLOP/s; 963 with z), its dx 948 (1595) and dW 974 (1552; 19.03 waves of tiles), 8192 x 4096 x 12288 gated in e4m3 525 us (3.1 PFLOP/s),
// 4 x 4608 x 4096 x 4096 with adapters of rank 64 386 us (1630).  Eight epilogue warps against four: 5 to 12 % faster where the reduction is short, no difference where it is long.
#pragma once
#include <algorithm>

#include "kernels.h"
#include "sm100.cuh"

namespace xema {
namespace tiles {
using namespace sm100;

enum class Form { kGated, kLinear, kGradX, kGradW };

constexpr int kThreads = 320, kEpilogue = 256;  // epilogue: eight warps
constexpr int kRows = 128;                    // of A, and of B, that a CTA holds per step
constexpr int kStepBytes = 128;               // of a row of either operand
constexpr int kOperandBytes = kRows * kStepBytes;
constexpr int kHalfOperand = kOperandBytes / 2;
constexpr int kChunk = 32;                    // columns per epilogue step
constexpr int kBufBytes = 2048;               // 32 rows x 32 columns of bf16
constexpr int kRing = 2;                      // staging buffers per epilogue warp
constexpr int kGroupM = 8;
constexpr int kMaxSize = 0x7fffff00;          // of a dimension: a tile's last row and column, and one request more, stay within 32 bits

constexpr int kStageArea = 196608;            // for the ring of stages
constexpr int kMaxStages = 8;
constexpr int kOffRing = kStageArea;
constexpr int kOffCols = kOffRing + kEpilogue / 32 * kRing * kBufBytes;   // float [256]: bias, or the factors of the columns
constexpr int kOffBar = kOffCols + 1024;
constexpr int kSmemBytes = kOffBar + 256;
static_assert((2 * kMaxStages + 4) * 8 + 8 <= 256, "barrier area");
static_assert(kSmemBytes <= 232448, "shared memory of one SM");

// Operands and results by form:        a           a2   b    b2   out   out2
//   kGated                             x                Wg   Wu   h     z (batch 3: gate, up, low bytes)
//   kLinear                            x           t    W    B    y
//   kGradX                             d (batch 2)      Wg   Wu   dx
//   kGradW                             d (batch 2)      x         dWg   dWu
struct Maps {
  CUtensorMap a, a2, b, b2, out, out2;
};
struct Params {
  int batch, rows, cols;           // of the result; kGradW: batch 2, rows = features
  int bn;                          // columns of the product per tile (kGated: gate and up)
  int b_bytes, stages;             // of B that a CTA loads per step; stages
  int off_line;                    // rows of an operand do not begin on 128-byte lines
  int k_main, k_more;              // steps; kGradX: k_main of each half; kLinear: k_more beside a2 and b2 where there is an adapter
  int act, keep;                   // kGated; keep: write z
  const float *row_scale, *gate_scale, *up_scale;   // kGated, e4m3
  const __nv_bfloat16* bias;       // kLinear, or null
  const int* adapter;              // kLinear [batch], or null
  int n_adapters;
  int behind;                      // kLinear: launched right behind the kernel that makes t, which waited for everything before it
  unsigned int* status;
};

struct Coord {
  int b, mt, nt;
};
__device__ __forceinline__ Coord coord_of(int tile, int m_tiles, int n_tiles) {
  const int per_batch = m_tiles * n_tiles;
  Coord c;
  c.b = tile / per_batch;
  const int t = tile - c.b * per_batch;
  const int group = kGroupM * n_tiles;
  const int g = t / group;
  const int first_m = g * kGroupM;
  const int gm = min(kGroupM, m_tiles - first_m);
  const int in_group = t - g * group;
  c.mt = first_m + in_group % gm;
  c.nt = in_group / gm;
  return c;
}

// Index of the batch element's adapter, or -1.
__device__ __forceinline__ int adapter_of(const Params& p, int b) {
  if (!p.adapter) return -1;
  const int a = p.adapter[b];
  return a >= 0 && a < p.n_adapters ? a : -1;
}
template <Form FORM>
__device__ __forceinline__ int steps_of(const Params& p, int b) {
  if constexpr (FORM == Form::kLinear) return p.k_main + (adapter_of(p, b) >= 0 ? p.k_more : 0);
  else return FORM == Form::kGradX ? 2 * p.k_main : p.k_main;
}

// z / (1 + exp(-q)): silu with q = z, gelu's tanh form with q = 2 sqrt(2/pi) (z + 0.044715 z^3).  From the exponential and not from
// tanh.approx, whose absolute error of 2^-11 is as large as the result for z below -6.
__device__ __forceinline__ float act_q(float z, int act) {
  return act == XEMA_ACT_SILU ? z : 1.5957691216057308f * fmaf(0.044715f * z * z, z, z);
}
__device__ __forceinline__ float sigmoid_f(float q) { return __fdividef(1.f, 1.f + __expf(-q)); }

// What the gradient is given of zg and zu: both in bf16, and in a third plane what that leaves out, a signed byte each in steps of 2^-15 of
// the value's power of two (zg in the low one).  zg and zu in bf16 alone would nearly double the square of the gradients' error: relative
// to the norm 3.1e-3 against 2.35e-3, which is what the roundings of dg and du and of the results leave.
__device__ __forceinline__ int low_byte(float z) {
  const float h = __bfloat162float(__float2bfloat16_rn(z));
  const uint32_t e = __float_as_uint(h) & 0x7f800000u;
  return min(__float2int_rn((z - h) * (__uint_as_float(0x7f000000u - e) * 32768.f)), 127);      // (a NaN gives 0)
}
__device__ __forceinline__ uint32_t low_bytes(float zg, float zu) { return (low_byte(zg) & 0xff) | (low_byte(zu) & 0xff) << 8; }
__device__ __forceinline__ float with_low(float h, int low) {
  const uint32_t e = __float_as_uint(h) & 0x7f800000u;
  return e == 0x7f800000u ? h : fmaf((float)low, __uint_as_float(e) * (1.f / 32768.f), h);
}

__device__ __forceinline__ uint8_t* piece(uint8_t* buf, int lane, int q) { return buf + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4); }

// KSUB steps make a stage: those of a small tile are shorter than a barrier round.
template <Form FORM, bool F8, bool PAIR, int KSUB>
__device__ __forceinline__ void body(const Maps& maps, const Params& p) {
  constexpr int TM = PAIR ? 256 : 128, ACC_COLS = PAIR ? 256 : 128;       // rows of a tile; TMEM columns of an accumulator
  constexpr int STEP = F8 ? kStepBytes : kStepBytes / 2;                  // values per step
  const int out_cols = FORM == Form::kGated ? p.bn / 2 : p.bn;            // result columns per tile
  const int stage_bytes = KSUB * (kOperandBytes + p.b_bytes);
  constexpr bool A_MN = FORM == Form::kGradW, B_MN = FORM == Form::kGradW || FORM == Form::kGradX;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + kOffBar);
  uint64_t* empty = full + kMaxStages;
  uint64_t* tmem_full = empty + kMaxStages;
  uint64_t* tmem_empty = tmem_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tmem_empty + 2);
  volatile uint32_t* abort_flag = tmem_slot + 1;

  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)cluster_ctarank() : 0;
  const int worker = PAIR ? blockIdx.x >> 1 : blockIdx.x, n_workers = PAIR ? gridDim.x >> 1 : gridDim.x;
  const int m_tiles = (p.rows + TM - 1) / TM, n_tiles = (p.cols + out_cols - 1) / out_cols;
  const bool aligned = (smem_u32(smem) & 1023u) == 0;
  const int total_tiles = aligned ? p.batch * m_tiles * n_tiles : 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&tmem_full[s], 1);
      mbar_init(&tmem_empty[s], (PAIR ? 2 : 1) * kEpilogue / 32);
    }
    *abort_flag = aligned ? 0u : 1u;
    fence_mbar_init();
    prefetch_tmap(&maps.a);
    prefetch_tmap(&maps.b);
    prefetch_tmap(&maps.out);
    if (FORM == Form::kGradW || (FORM == Form::kGated && p.keep)) prefetch_tmap(&maps.out2);
    if (FORM == Form::kGradX) prefetch_tmap(&maps.b2);
  }
  if (warp == 1) {
    if (PAIR) {
      tmem_alloc_pair(tmem_slot, 2 * ACC_COLS);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(tmem_slot, 2 * ACC_COLS);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) {
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  // The launch may start while the one before it still runs, and waits for it before anything else -- or, behind the launch that makes
  // t (which lets this one start only after its own wait), before t is read and before the results are written.  The next launch may start
  // after that wait: CTAs of two launches share the SMs, never of three.
  const bool late = FORM == Form::kLinear && p.behind;
  if (!late) {
    grid_dep_wait();
    if (threadIdx.x == 0) grid_dep_launch();
    __syncwarp();
  }

  if (warp == 0) {
    // ---------------- TMA producer ----------------
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    auto load = [&](uint8_t* dst, const CUtensorMap& m, int st, int x, int y, int z) {
      if constexpr (PAIR) tma_load_3d_pair(dst, &m, mapa_shared(smem_u32(&full[st]), 0), x, y, z);
      else tma_load_3d(dst, &m, &full[st], x, y, z);
    };
    for (int tile = worker; ok && tile < total_tiles; tile += n_workers) {
      const Coord c = coord_of(tile, m_tiles, n_tiles);
      const int row = c.mt * TM + rank * kRows, col = c.nt * p.bn + rank * (p.bn / 2);
      const int adapter = FORM == Form::kLinear ? adapter_of(p, c.b) : -1;
      const int steps = steps_of<FORM>(p, c.b);
      for (int s0 = 0; s0 < steps; s0 += KSUB) {
        if (late && s0 + KSUB > p.k_main) grid_dep_wait();      // (returns at once after the first time)
        if (!(ok = mbar_wait_warp(&empty[stage], phase ^ 1, abort_flag))) break;
        if (elect_one()) {
          uint8_t* st = smem + stage * stage_bytes;
          const int bytes = min(KSUB, steps - s0) * (kOperandBytes + p.b_bytes);
          if (!PAIR) mbar_expect_tx(&full[stage], bytes);
          else if (rank == 0) mbar_expect_tx(&full[stage], 2 * bytes);
#pragma unroll
          for (int u = 0; u < KSUB; ++u) {
            const int s = s0 + u;
            if (KSUB > 1 && s >= steps) break;
            uint8_t *sa = st + u * kOperandBytes, *sb = st + KSUB * kOperandBytes + u * p.b_bytes;
            if constexpr (FORM == Form::kGated) {
              load(sa, maps.a, stage, s * STEP, row, 0);
              if constexpr (PAIR) {
                load(sb, rank ? maps.b2 : maps.b, stage, s * STEP, c.nt * out_cols, 0);
              } else {
                load(sb, maps.b, stage, s * STEP, c.nt * out_cols, 0);
                load(sb + p.b_bytes / 2, maps.b2, stage, s * STEP, c.nt * out_cols, 0);
              }
            } else if constexpr (FORM == Form::kLinear) {
              if (s < p.k_main) {
                load(sa, maps.a, stage, s * STEP, row, c.b);
                load(sb, maps.b, stage, s * STEP, col, 0);
              } else {
                load(sa, maps.a2, stage, (s - p.k_main) * STEP, row, c.b);
                load(sb, maps.b2, stage, (s - p.k_main) * STEP, col, adapter);
              }
            } else if constexpr (FORM == Form::kGradX) {
              const int half = s >= p.k_main, k = (s - half * p.k_main) * STEP;
              const CUtensorMap& w = half ? maps.b2 : maps.b;
              load(sa, maps.a, stage, k, row, half);
              load(sb, w, stage, col, k, 0);
              if (p.b_bytes > kHalfOperand) load(sb + kHalfOperand, w, stage, col + 64, k, 0);
            } else {
              load(sa, maps.a, stage, row, s * STEP, c.b);
              load(sa + kHalfOperand, maps.a, stage, row + 64, s * STEP, c.b);
              load(sb, maps.b, stage, col, s * STEP, 0);
              if (p.b_bytes > kHalfOperand) load(sb + kHalfOperand, maps.b, stage, col + 64, s * STEP, 0);
            }
          }
        }
        __syncwarp();
        if (++stage == p.stages) { stage = 0; phase ^= 1; }
      }
    }
    // The waits of as many further fills: the multicast commits that release this CTA's last ones have then landed here.
    if constexpr (PAIR) {
      for (int s = 0; ok && s < p.stages; ++s) {
        ok = mbar_wait_warp(&empty[stage], phase ^ 1, abort_flag);
        if (++stage == p.stages) { stage = 0; phase ^= 1; }
      }
    }
    if (!ok) {
      report_timeout(p.status);
      // Gave up: copies under way must land before a CTA leaves.  All of a pair complete on the even CTA's barriers; the closing
      // cluster barrier keeps the peer until then, a short settling time covers a stage that only one of them still asked for.
      if (rank == 0 && lane == 0) {
        for (int s = 0; s < p.stages; ++s) {
          const int st = (stage + s) % p.stages;
          volatile uint32_t dummy = 0;
          mbar_wait_slow(&full[st], st < stage ? phase : phase ^ 1, &dummy, 100000000ll);
        }
      }
      for (int i = 0; i < 64; ++i) __nanosleep(1000);
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer (pair: even CTA only) ----------------
    if (rank == 0) {
      const uint32_t idesc = F8 ? idesc_e4m3_f32(TM, p.bn) : idesc_bf16_f32(TM, p.bn, A_MN, B_MN);
      // An MMA covers 32 bytes along K of a K-major row, or 16 rows of 128 bytes of an operand that is stored by K.
      constexpr uint64_t A_ADV = A_MN ? 2048 >> 4 : 2, B_ADV = B_MN ? 2048 >> 4 : 2;
      const uint64_t a_desc0 = smem_desc_sw128(smem_u32(smem), A_MN ? kHalfOperand : 16, 1024);
      const uint64_t b_desc0 = smem_desc_sw128(smem_u32(smem + KSUB * kOperandBytes), B_MN ? kHalfOperand : 16, 1024);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int tile = worker; ok && tile < total_tiles; tile += n_workers) {
        const int steps = steps_of<FORM>(p, coord_of(tile, m_tiles, n_tiles).b);
        if (!(ok = __all_sync(0xffffffffu, mbar_wait_cluster(&tmem_empty[acc], acc_phase ^ 1, abort_flag)))) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * ACC_COLS;
#pragma unroll 1
        for (int s0 = 0; s0 < steps; s0 += KSUB) {
          if (!(ok = mbar_wait_warp(&full[stage], phase, abort_flag))) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t soff = (uint64_t)(stage * (stage_bytes >> 4));
#pragma unroll
            for (int u = 0; u < KSUB; ++u) {
              if (KSUB > 1 && s0 + u >= steps) break;
              const uint64_t da = a_desc0 + soff + (uint64_t)(u * (kOperandBytes >> 4));
              const uint64_t db = b_desc0 + soff + (uint64_t)(u * (p.b_bytes >> 4));
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t accumulate = k > 0 || u > 0 || s0 > 0;
                if constexpr (F8 && PAIR) mma_ss_f8_pair(d_tmem, da + k * A_ADV, db + k * B_ADV, idesc, accumulate);
                else if constexpr (F8) mma_ss_f8(d_tmem, da + k * A_ADV, db + k * B_ADV, idesc, accumulate);
                else if constexpr (PAIR) mma_ss_pair(d_tmem, da + k * A_ADV, db + k * B_ADV, idesc, accumulate);
                else mma_ss(d_tmem, da + k * A_ADV, db + k * B_ADV, idesc, accumulate);
              }
            }
            if constexpr (PAIR) mma_commit_pair(&empty[stage]);
            else mma_commit(&empty[stage]);
          }
          __syncwarp();
          if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        if (elect_one()) {
          if (PAIR) mma_commit_pair(&tmem_full[acc]);
          else mma_commit(&tmem_full[acc]);
        }
        __syncwarp();
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      }
      if (!ok) report_timeout(p.status);
    }
  } else {
    // ---------------- epilogue (pair: each CTA its own 128 rows) ----------------
    const int quad = warp & 3, side = (warp - 2) >> 2;   // TMEM lanes [32*quad, 32*quad + 32); of 64 columns this warp has the first 32 or the others
    const int et = threadIdx.x - 64;     // 0..255
    float* s_cols = reinterpret_cast<float*>(smem + kOffCols);
    uint8_t* ring = smem + kOffRing + (warp - 2) * kRing * kBufBytes;
    uint32_t used = 0;
    if (late) {
      grid_dep_wait();
      if (et == 0) grid_dep_launch();
      __syncwarp();
    }
    // 32 columns of the warp's rows, 16 bits each, on their way to the map's (x, y, z)
    auto send_raw = [&](const uint32_t (&w)[kChunk / 2], const CUtensorMap& m, int x, int y, int z) {
      uint8_t* buf = ring + (used % kRing) * kBufBytes;
      if (lane == 0) bulk_wait_read<kRing - 1>();
      __syncwarp();
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<uint4*>(piece(buf, lane, q)) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        tma_store_3d(&m, buf, x, y, z);
        bulk_commit();
      }
      __syncwarp();          // (the next load from TMEM, or vote, wants whole warps)
      ++used;
    };
    auto send = [&](const float (&v)[kChunk], const CUtensorMap& m, int x, int y, int z) {
      uint32_t w[kChunk / 2];
#pragma unroll
      for (int t = 0; t < kChunk / 2; ++t) w[t] = pack_bf16x2(v[2 * t], v[2 * t + 1]);
      send_raw(w, m, x, y, z);
    };
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int tile = worker; tile < total_tiles; tile += n_workers) {
      // the warps meet (the previous tile's factors are no longer read) and agree on going on
      if (!(ok = named_barrier_and(1, kEpilogue, ok))) break;
      const Coord c = coord_of(tile, m_tiles, n_tiles);
      const int row0 = c.mt * TM + rank * kRows + quad * 32, n_base = c.nt * out_cols;
      float row_scale = 1.f;
      if constexpr (FORM == Form::kGated && F8) {
        row_scale = p.row_scale[min(row0 + lane, p.rows - 1)];
        for (int i = et; i < p.bn; i += kEpilogue) {
          const bool up = i >= out_cols;
          const int f = n_base + (up ? i - out_cols : i);
          s_cols[i] = f < p.cols ? (up ? p.up_scale[f] : p.gate_scale[f]) : 0.f;
        }
      }
      if constexpr (FORM == Form::kLinear) {
        for (int i = et; i < p.bn; i += kEpilogue)
          s_cols[i] = p.bias && n_base + i < p.cols ? __bfloat162float(p.bias[n_base + i]) : 0.f;
      }
      named_barrier(1, kEpilogue);
      ok = mbar_wait_warp(&tmem_full[acc], acc_phase, abort_flag);
      tc_fence_after();
      const uint32_t t_addr = tmem_base + ((uint32_t)(quad * 32) << 16) + acc * ACC_COLS;
      if (ok && row0 < p.rows) {
#pragma unroll 1
        for (int col = side * kChunk; col < out_cols && n_base + col < p.cols; col += 2 * kChunk) {
          float v[kChunk];
          tmem_ld32(t_addr + col, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
          if constexpr (FORM == Form::kGated) {
            float w[kChunk];
            tmem_ld32(t_addr + out_cols + col, *reinterpret_cast<uint32_t(*)[32]>(&w[0]));
            tmem_ld_wait_on(*reinterpret_cast<uint32_t(*)[32]>(&v[0]));
            tmem_ld_wait_on(*reinterpret_cast<uint32_t(*)[32]>(&w[0]));
            if constexpr (F8) {
#pragma unroll
              for (int t = 0; t < kChunk; ++t) {
                v[t] *= row_scale * s_cols[col + t];
                w[t] *= row_scale * s_cols[out_cols + col + t];
              }
            }
            if (!F8 && p.keep) {
              send(v, maps.out2, n_base + col, row0, 0);
              send(w, maps.out2, n_base + col, row0, 1);
              uint32_t low[kChunk / 2];
#pragma unroll
              for (int t = 0; t < kChunk / 2; ++t) low[t] = low_bytes(v[2 * t], w[2 * t]) | low_bytes(v[2 * t + 1], w[2 * t + 1]) << 16;
              send_raw(low, maps.out2, n_base + col, row0, 2);
            }
#pragma unroll
            for (int t = 0; t < kChunk; ++t) v[t] = v[t] * sigmoid_f(act_q(v[t], p.act)) * w[t];
            send(v, maps.out, n_base + col, row0, 0);
          } else {
            tmem_ld_wait_on(*reinterpret_cast<uint32_t(*)[32]>(&v[0]));
            if constexpr (FORM == Form::kLinear) {
#pragma unroll
              for (int t = 0; t < kChunk; ++t) v[t] += s_cols[col + t];
            }
            if constexpr (FORM == Form::kGradW) send(v, c.b ? maps.out2 : maps.out, n_base + col, row0, 0);
            else send(v, maps.out, n_base + col, row0, c.b);
          }
        }
      }
      // only the tile after the next asks for this accumulator
      if (tile + 2 * n_workers < total_tiles) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) mbar_arrive_cluster(mapa_shared(smem_u32(&tmem_empty[acc]), 0));
          else mbar_arrive(&tmem_empty[acc]);
        }
        __syncwarp();
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
    if (!ok) report_timeout(p.status);
    if (lane == 0) bulk_wait<0>();       // this warp's stores are complete
    __syncwarp();
    if (FORM == Form::kLinear && blockIdx.x == 0 && p.adapter && p.status) {
      for (int b = et; b < p.batch; b += kEpilogue)
        if (p.adapter[b] >= p.n_adapters) atomicExch(p.status, XEMA_DEVICE_STATUS_ADAPTER);
    }
  }

  // Neither CTA of a pair leaves (or frees TMEM) while the other may still touch its memory or barriers.
  tc_fence_before();
  __syncthreads();
  if (PAIR) {
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem_base, 2 * ACC_COLS);
    else tmem_dealloc(tmem_base, 2 * ACC_COLS);
  }
  if (threadIdx.x == 0 && !aligned) report_timeout(p.status);
}

template <Form FORM, bool F8>
__global__ void __launch_bounds__(kThreads, 1) tile_kernel(const __grid_constant__ Maps maps, const Params p) {
  body<FORM, F8, false, 2>(maps, p);
}
template <Form FORM, bool F8, int KSUB>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
tile_pair_kernel(const __grid_constant__ Maps maps, const Params p) {
  body<FORM, F8, true, KSUB>(maps, p);
}

// A shape: CTA pairs on 256 x bn tiles, or single CTAs on 128 x 128 ones.
struct Shape {
  int pair, bn;
};
inline long long tile_count(const Params& p, const Shape& s, bool gated) {
  const int tm = s.pair ? 256 : 128, out_cols = gated ? s.bn / 2 : s.bn;
  return (long long)p.batch * ((p.rows + tm - 1) / tm) * ((p.cols + out_cols - 1) / out_cols);
}
// Estimated time of a shape.  A step takes 300 ns of a pair with 256 columns, 243 with 192, 189 with 128, and 225 of a single CTA (729 x
// 4096 x 4104 gated, 128 to 192 steps), or longer where weights that nobody shares come from memory at 6.2 TB/s (128 x 4096 x 8192: 340) and
// where the rows of an operand do not lie on 128-byte lines, so that each 128 bytes of a step meet two (729 x 1544 x 4104: 400, 356, 304
// and 400, 12.5 ns a KB).  The first waves and the last tile's epilogue add up to 1 us a wave + 10 ns a column.
inline long long shape_ns(const Params& p, const Shape& s, long long steps, bool gated) {
  const int workers = std::max(1, s.pair ? sm_count() / 2 : sm_count()), tm = s.pair ? 256 : 128;
  const long long tiles = tile_count(p, s, gated), full = tiles / workers, rest = tiles % workers, waves = full + (rest > 0);
  const long long sharing = std::min(kGroupM, (p.rows + tm - 1) / tm) * (long long)p.batch;
  auto from_memory = [&](long long n) { return n * s.bn * kStepBytes / std::max(1LL, sharing) / 6200; };
  const long long over_lines = p.off_line ? (kOperandBytes + (s.pair ? s.bn / 2 : s.bn) * kStepBytes) * 125LL / 10240 : 0;
  const long long step = std::max<long long>(s.pair ? 66 + s.bn * 92 / 100 : 225, over_lines);
  return steps * (full * std::max(step, from_memory(workers)) + (rest ? std::max(step, from_memory(rest)) : 0)) + std::min(waves, 3LL) * 1000 +
         (s.pair ? s.bn * 10 : 900);
}
inline Shape pick_shape(const Params& p, long long steps, bool gated) {
  Shape best = {0, 128};
  for (int bn = 256; bn >= 128; bn -= gated ? 64 : 32)
    if (shape_ns(p, {1, bn}, steps, gated) < shape_ns(p, best, steps, gated)) best = {1, bn};
  return best;
}
// That one, or the one that a caller asks for, and whether there is such a one.
inline Shape take_shape(const Params& p, long long steps, bool gated, const xema_ff_shape* in) {
  return in && in->kernel == XEMA_FF_TILES ? Shape{in->pair != 0, in->columns} : pick_shape(p, steps, gated);
}
inline bool is_tile(const xema_ff_shape& in, bool gated) {
  const int bn = in.columns;
  return in.kernel == XEMA_FF_TILES && (in.pair ? bn >= 128 && bn <= 256 && bn % (gated ? 64 : 32) == 0 : bn == 128);
}
// Rows of B that one load brings: of one of two halves where a tile has two (gated), or a CTA's share.
inline int b_box(const Shape& s, bool gated) { return s.pair || gated ? s.bn / 2 : s.bn; }

template <Form FORM, bool F8>
int launch(const Maps& maps, Params p, const Shape& shape, cudaStream_t stream) {
  const long long tiles = tile_count(p, shape, FORM == Form::kGated);
  if (tiles > (1LL << 30)) return XEMA_EINVAL;
  // an operand that is stored by K comes in blocks of 64 columns
  const int b_rows = shape.pair ? shape.bn / 2 : shape.bn, ksub = shape.pair && shape.bn >= 192 ? 1 : 2;
  p.bn = shape.bn;
  p.b_bytes = (FORM == Form::kGradX || FORM == Form::kGradW ? (b_rows + 63) / 64 * 64 : b_rows) * kStepBytes;
  p.stages = std::min(kMaxStages, kStageArea / (ksub * (kOperandBytes + p.b_bytes)));
  // The gradients' products start when everything before them has ended: chained to each other and to the kernel that makes dg and du,
  // a backward pass in a graph stopped for good in some ten thousands of passes, for a reason that was not found.  (Instructions that
  // want whole warps followed single lanes' work then, named barriers without a limit among them; the chain has not run since that is mended.)
  constexpr bool CHAINED = FORM != Form::kGradX && FORM != Form::kGradW;
  if (!shape.pair) {
    static PerDeviceInt attr_done;
    auto kern = tile_kernel<FORM, F8>;
    if (int rc = ensure_smem_attr(kern, kSmemBytes, attr_done)) return rc;
    return launch_kernel(kern, dim3((unsigned)std::min<long long>(tiles, sm_count())), kThreads, kSmemBytes, stream, CHAINED, maps, p);
  }
  static PerDeviceInt attr_done[2], pairs_cache[2];
  auto kern = ksub == 1 ? tile_pair_kernel<FORM, F8, 1> : tile_pair_kernel<FORM, F8, 2>;
  if (int rc = ensure_smem_attr(kern, kSmemBytes, attr_done[ksub - 1])) return rc;
  // all pairs of a persistent grid have to be resident at once
  const int dev = current_device();
  int max_pairs = pairs_cache[ksub - 1].get(dev);
  if (max_pairs == 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (sm_count() / 2), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = kSmemBytes;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, kern, &cfg);
    if (e != cudaSuccess || n <= 0) {
      set_last_cuda_error((int)e);
      return XEMA_ECUDA;
    }
    max_pairs = std::min(n, sm_count() / 2);
    pairs_cache[ksub - 1].set(dev, max_pairs);
  }
  return launch_kernel(kern, dim3((unsigned)(2 * std::min<long long>(tiles, max_pairs))), kThreads, kSmemBytes, stream, CHAINED, maps, p);
}

}  // namespace tiles
}  // namespace xema
