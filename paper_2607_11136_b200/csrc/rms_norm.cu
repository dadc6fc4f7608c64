// RMSNorm with the residual's addition in front of it and, where asked for, a result in e4m3 with a factor per row.
#include <cuda_fp8.h>
#include <float.h>

#include <algorithm>

#include "kernels.h"
#include "sm100.cuh"

namespace xema {
using namespace sm100;

namespace {
constexpr float kE4m3Max = 448.f;

// E neighbouring values of a row as they lie in memory: one load or store of up to 16 bytes (two for eight fp32 values).
template <typename T, int E>
struct Raw {
  static constexpr int BYTES = E * (int)sizeof(T), WORDS = BYTES < 4 ? 1 : BYTES / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (BYTES == 32) {
      asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
      asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p + 4));
    } else if constexpr (BYTES == 16) {
      asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    } else if constexpr (BYTES == 8) {
      asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    } else if constexpr (BYTES == 4) {
      asm volatile("ld.global.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    } else {
      unsigned short h;
      asm volatile("ld.global.u16 %0, [%1];" : "=h"(h) : "l"(p));
      w[0] = h;
    }
  }
  __device__ __forceinline__ float value(int k) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
    else return k & 1 ? bf16_hi(w[k / 2]) : bf16_lo(w[k / 2]);
  }
  __device__ __forceinline__ void put(const float (&v)[E]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < E; ++k) w[k] = __float_as_uint(v[k]);
    } else if constexpr (sizeof(T) == 2) {
      if constexpr (E == 1) w[0] = pack_bf16x2(v[0], 0.f);
      else
#pragma unroll
        for (int k = 0; k < E; k += 2) w[k / 2] = pack_bf16x2(v[k], v[k + 1]);
    } else {
#pragma unroll
      for (int k = 0; k < WORDS; ++k) w[k] = 0u;
#pragma unroll
      for (int k = 0; k < E; k += 2)
        w[k / 4] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[k], E == 1 ? 0.f : v[E == 1 ? 0 : k + 1]), __NV_SATFINITE, __NV_E4M3) << (8 * (k % 4));
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (BYTES == 32) {
      asm volatile("st.global.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
      asm volatile("st.global.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p + 4), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else if constexpr (BYTES == 16) {
      asm volatile("st.global.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    } else if constexpr (BYTES == 8) {
      asm volatile("st.global.v2.u32 [%0], {%1, %2};" ::"l"(p), "r"(w[0]), "r"(w[1]) : "memory");
    } else if constexpr (BYTES == 4) {
      asm volatile("st.global.u32 [%0], %1;" ::"l"(p), "r"(w[0]) : "memory");
    } else if constexpr (BYTES == 2) {
      asm volatile("st.global.u16 [%0], %1;" ::"l"(p), "h"((unsigned short)w[0]) : "memory");
    } else {
      *reinterpret_cast<uint8_t*>(p) = (uint8_t)w[0];
    }
  }
};

// Sum, or largest (a NaN stays one), over the block; every thread gets the same value.
template <bool MAX>
__device__ __forceinline__ float block_reduce(float v, float* s, int warps) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = MAX ? max3_nan(v, u, u) : v + u;
  }
  if (warps == 1) return v;
  if (lane == 0) s[warp] = v;
  __syncthreads();
  v = lane < warps ? s[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = MAX ? max3_nan(v, u, u) : v + u;
  }
  return v;
}

// The sum of a row's squares, and the same of its values times 2^-80 for rows whose squares leave fp32: beside those eps is nothing.
// (Adding the second sum up from the registers where it is asked for costs registers that hold a block more an SM: 1015 x 2298,
// residual in fp32, 6.0 us -> 7.2.)
struct Squares {
  float sum = 0.f, small = 0.f;
  __device__ __forceinline__ void add(float v) {
    sum = fmaf(v, v, sum);
    const float t = v * 0x1p-80f;
    small = fmaf(t, t, small);
  }
  // 1 / sqrt(mean + eps), the same on every thread; an infinity among the values gives NaN.
  __device__ __forceinline__ float rstd(float* s, int warps, int D, float eps) {
    sum = block_reduce<false>(sum, s, warps);
    if (sum > FLT_MAX) {                         // (on all threads of the row, or on none)
      if (warps > 1) __syncthreads();            // (the first partials have been read)
      small = block_reduce<false>(small, s, warps);
      return small > FLT_MAX ? __int_as_float(0x7fffffff) : rsqrtf(small / (float)D) * 0x1p-80f;
    }
    return rsqrtf(sum / (float)D + eps);
  }
};

// v / scale, rounded to nearest, from inv = 1 / scale: the remainder of a first quotient corrects it (Markstein's step).
__device__ __forceinline__ float quotient(float v, float scale, float inv) {
  const float q = v * inv;
  return fmaf(fmaf(-q, scale, v), inv, q);
}

// A block per row, or (WARP) a warp of eight, the row in registers: every byte is read and written once.  Thread t holds the groups of E
// values t, t + T, ...  (T threads, V groups); E is what the strides and addresses allow to be moved at once.
// Bound by HBM: 16384 x 4096, residual in bf16, result in e4m3, 70 us (6.7 TB/s; 73 with 16 values a thread, 85 with 8), 8192 x 8192 in
// bf16 79 us (6.8), one row 2.2 us.  Streaming stores change nothing, loads past the L1 lose 9 %.
template <typename R, typename Out, int E, int V, bool WARP>
__global__ void __launch_bounds__(WARP || E * V <= 8 ? 256 : E * V <= 32 ? 512 : 1024) rms_norm_kernel(const xema_rms_norm_args p) {
  __shared__ float s_sum[32], s_max[32];
  grid_dep_wait();
  grid_dep_launch();     // (after the wait: CTAs of two launches share the SMs, never of three)
  const int T = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x & 31 : threadIdx.x, warps = WARP ? 1 : blockDim.x >> 5;
  const size_t row = WARP ? (size_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
  if (WARP && row >= p.rows) return;
  const int groups = p.D / E;
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(p.x) + row * p.ldx;
  const R* res = static_cast<const R*>(p.resid) + row * p.ldr;
  float v[V][E];
  Squares squares;
  {
    Raw<__nv_bfloat16, E> xr[V];
    Raw<R, E> rr[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int g = tid + j * T;
      if (p.x && g < groups) xr[j].load(x + g * E);
      if (p.resid && g < groups) rr[j].load(res + g * E);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const bool in = tid + j * T < groups;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        v[j][k] = in && p.x ? xr[j].value(k) : 0.f;
        if (in && p.resid) v[j][k] += rr[j].value(k);
        squares.add(v[j][k]);
      }
    }
  }
  if (p.resid_out) {
    R* out = static_cast<R*>(p.resid_out) + row * p.ldro;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int g = tid + j * T;
      Raw<R, E> r;
      r.put(v[j]);
      if (g < groups) r.store(out + g * E);
    }
  }
  constexpr bool kAhead = E > 1 || V < 32;       // values one by one: no registers left for the gain's on the way
  Raw<__nv_bfloat16, E> w[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int g = tid + j * T;
    if (kAhead && g < groups) w[j].load(static_cast<const __nv_bfloat16*>(p.gain) + g * E);
  }
  const float rstd = squares.rstd(s_sum, warps, p.D, p.eps);
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const bool in = tid + j * T < groups;
    if (!kAhead && in) w[j].load(static_cast<const __nv_bfloat16*>(p.gain) + (tid + j * T) * E);
#pragma unroll
    for (int k = 0; k < E; ++k) {
      v[j][k] = in ? v[j][k] * rstd * w[j].value(k) : 0.f;
      if constexpr (sizeof(Out) == 1) {
        const float size = fabsf(v[j][k]);
        top = max3_nan(top, size, size);
      }
    }
  }
  float scale = 1.f, inv = 1.f;
  if constexpr (sizeof(Out) == 1) {
    top = block_reduce<true>(top, s_max, warps);
    scale = top / kE4m3Max;
    if (scale < FLT_MIN) scale = FLT_MIN;      // (false for a NaN)
    if (tid == 0) p.out_scale[row] = scale;
    inv = 1.f / scale;
  }
  Out* out = static_cast<Out*>(p.out) + row * p.ldo;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int g = tid + j * T;
    if constexpr (sizeof(Out) == 1) {
#pragma unroll
      for (int k = 0; k < E; ++k) v[j][k] = quotient(v[j][k], scale, inv);
    }
    Raw<Out, E> r;
    r.put(v[j]);
    if (g < groups) r.store(out + g * E);
  }
}

template <typename R, typename Out, int E>
int launch(const xema_rms_norm_args& a, cudaStream_t st) {
  // A warp per row up to 1024 columns.  Beyond, values of a thread: 8 up to 256 threads, 16 and 32 up to 512, 64; 32 from 2048 rows on up
  // to 4096 columns, where fewer threads a row leave room for more rows at once.
  auto threads = [&](int values) { return ((a.D + values - 1) / values + 31) / 32 * 32; };
  const dim3 eight((unsigned)((a.rows + 7LL) / 8));
  if (a.D <= 256) return launch_kernel(rms_norm_kernel<R, Out, E, 8 / E, true>, eight, 256, 0, st, true, a);
  if (a.D <= 512) return launch_kernel(rms_norm_kernel<R, Out, E, 16 / E, true>, eight, 256, 0, st, true, a);
  if (a.D <= 1024 && a.rows >= 1024) return launch_kernel(rms_norm_kernel<R, Out, E, 32 / E, true>, eight, 256, 0, st, true, a);
  const dim3 one(a.rows);
  if (threads(8) <= 256) return launch_kernel(rms_norm_kernel<R, Out, E, 8 / E, false>, one, threads(8), 0, st, true, a);
  if (threads(16) <= 512 && (E < 8 || a.D > 4096 || a.rows < 2048))
    return launch_kernel(rms_norm_kernel<R, Out, E, 16 / E, false>, one, threads(16), 0, st, true, a);
  if (threads(32) <= 512) return launch_kernel(rms_norm_kernel<R, Out, E, 32 / E, false>, one, threads(32), 0, st, true, a);
  return launch_kernel(rms_norm_kernel<R, Out, E, 64 / E, false>, one, threads(64), 0, st, true, a);
}

// Rows whose values lie on no common boundary (an odd width or stride): the row goes through shared memory, so that all but its ends
// moves 16 bytes at a time, with all of a row's loads under way together.  9000 x 2299, result in e4m3: 54 us (2.7 TB/s; 168 one value after the other).  Bound by the accesses
// to shared memory, two or three a value and two bytes each, and by the gain, which comes value by value for each row.
constexpr int kOddValues = 16, kOddMaxD = 8192;       // values of a thread
template <typename T>
struct RowLoad {
  uint4 body[sizeof(T)];
  T head, tail;
  int n_head, n_body, n_tail;
  __device__ __forceinline__ void load(const T* g, int n) {
    constexpr int E = 16 / (int)sizeof(T);
    n_head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(g) & 15)) & 15) / (int)sizeof(T));
    n_body = (n - n_head) / E;
    n_tail = n - n_head - n_body * E;
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i)
      if (t + i * blockDim.x < n_body) body[i] = ld_u4(reinterpret_cast<const uint4*>(g + n_head) + t + i * blockDim.x);
    if (t < n_head) head = g[t];
    if (t < n_tail) tail = g[n_head + n_body * E + t];
  }
  __device__ __forceinline__ void put(T* s) const {        // s: at the same place in 16 bytes as g
    constexpr int E = 16 / (int)sizeof(T);
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i)
      if (t + i * blockDim.x < n_body) reinterpret_cast<uint4*>(s + n_head)[t + i * blockDim.x] = body[i];
    if (t < n_head) s[t] = head;
    if (t < n_tail) s[n_head + n_body * E + t] = tail;
  }
};
template <typename T>
__device__ __forceinline__ void row_out(T* g, const T* s, int n) {
  const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(g) & 15)) & 15) / (int)sizeof(T)), body = (n - head) * (int)sizeof(T) / 16;
  for (int i = threadIdx.x; i < head; i += blockDim.x) g[i] = s[i];
  for (int i = threadIdx.x; i < body; i += blockDim.x) reinterpret_cast<uint4*>(g + head)[i] = reinterpret_cast<const uint4*>(s + head)[i];
  for (int i = head + body * (16 / (int)sizeof(T)) + threadIdx.x; i < n; i += blockDim.x) g[i] = s[i];
}
template <typename T>
__device__ __forceinline__ T* like(uint8_t* s, const T* g) { return reinterpret_cast<T*>(s + (reinterpret_cast<uintptr_t>(g) & 15)); }

template <typename R, typename Out>
__global__ void __launch_bounds__(512) rms_norm_odd_kernel(const xema_rms_norm_args p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_sum[32], s_max[32];
  grid_dep_wait();
  grid_dep_launch();
  const size_t row = blockIdx.x;
  const int T = blockDim.x, tid = threadIdx.x;
  uint8_t* second = smem + (p.D * (int)sizeof(R) + 47) / 16 * 16;
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(p.x) + row * p.ldx;
  const R* res = static_cast<const R*>(p.resid) + row * p.ldr;
  __nv_bfloat16* sx = like(second, x);
  R* sr = like(smem, res);
  {
    RowLoad<__nv_bfloat16> lx;
    RowLoad<R> lr;
    if (p.x) lx.load(x, p.D);
    if (p.resid) lr.load(res, p.D);
    if (p.x) lx.put(sx);
    if (p.resid) lr.put(sr);
  }
  __syncthreads();
  float v[kOddValues];
  Squares squares;
#pragma unroll
  for (int j = 0; j < kOddValues; ++j) {
    const int k = tid + j * T;
    v[j] = 0.f;
    if (k < p.D && p.x) v[j] = __bfloat162float(sx[k]);
    if (k < p.D && p.resid) v[j] += (float)sr[k];
    squares.add(v[j]);
  }
  const float rstd = squares.rstd(s_sum, T >> 5, p.D, p.eps);
  __syncthreads();                       // the rows have been read (one warp does not meet in the sum)
  R* so = nullptr;
  if (p.resid_out) {
    R* out = static_cast<R*>(p.resid_out) + row * p.ldro;
    so = like(smem, out);
#pragma unroll
    for (int j = 0; j < kOddValues; ++j)
      if (tid + j * T < p.D) so[tid + j * T] = (R)v[j];
  }
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < kOddValues; ++j) {
    const int k = tid + j * T;
    v[j] = k < p.D ? v[j] * rstd * __bfloat162float(static_cast<const __nv_bfloat16*>(p.gain)[k]) : 0.f;
    top = max3_nan(top, fabsf(v[j]), fabsf(v[j]));
  }
  float scale = 1.f, inv = 1.f;
  if constexpr (sizeof(Out) == 1) {
    top = block_reduce<true>(top, s_max, T >> 5);
    scale = top / kE4m3Max;
    if (scale < FLT_MIN) scale = FLT_MIN;
    if (tid == 0) p.out_scale[row] = scale;
    inv = 1.f / scale;
  }
  Out* out = static_cast<Out*>(p.out) + row * p.ldo;
  Out* sy = like(second, out);
#pragma unroll
  for (int j = 0; j < kOddValues; ++j) {
    if (tid + j * T >= p.D) continue;
    if constexpr (sizeof(Out) == 1) reinterpret_cast<uint8_t*>(sy)[tid + j * T] = __nv_cvt_float_to_fp8(quotient(v[j], scale, inv), __NV_SATFINITE, __NV_E4M3);
    else sy[tid + j * T] = __float2bfloat16_rn(v[j]);
  }
  __syncthreads();
  if (p.resid_out) row_out(static_cast<R*>(p.resid_out) + row * p.ldro, so, p.D);
  row_out(reinterpret_cast<uint8_t*>(out), reinterpret_cast<const uint8_t*>(sy), p.D * (int)sizeof(Out));
}

template <typename R, typename Out>
int launch_odd(const xema_rms_norm_args& a, cudaStream_t st) {
  const int threads = ((a.D + kOddValues - 1) / kOddValues + 31) / 32 * 32;
  const int smem = (a.D * (int)sizeof(R) + 47) / 16 * 16 + (a.D * 2 + 47) / 16 * 16;
  static PerDeviceInt attr_done;
  if (int rc = ensure_smem_attr(rms_norm_odd_kernel<R, Out>, kOddMaxD * 6 + 96, attr_done)) return rc;
  return launch_kernel(rms_norm_odd_kernel<R, Out>, dim3(a.rows), threads, smem, st, true, a);
}
template <typename R, typename Out>
int launch(const xema_rms_norm_args& a, int at_once, cudaStream_t st) {
  if (at_once == 1 && a.D >= 512 && a.D <= kOddMaxD) return launch_odd<R, Out>(a, st);
  return at_once == 8 ? launch<R, Out, 8>(a, st) : at_once == 2 ? launch<R, Out, 2>(a, st) : launch<R, Out, 1>(a, st);
}
}  // namespace

int launch_rms_norm(const xema_rms_norm_args& a, cudaStream_t stream) {
  if (a.rows < 0 || a.D < 1 || a.D > XEMA_RMS_NORM_MAX_D || !(a.eps >= 0.f)) return XEMA_EINVAL;
  if (a.rows == 0) return XEMA_OK;
  if ((!a.x && !a.resid) || !a.gain || !a.out || (a.resid_out && !a.resid)) return XEMA_EINVAL;
  if (a.out_is_e4m3 ? !a.out_scale : a.out_scale != nullptr) return XEMA_EINVAL;
  // rows of a result lie behind one another
  if (a.rows > 1 && (a.ldo < a.D || (a.resid_out && a.ldro < a.D))) return XEMA_EINVAL;
  const uintptr_t rsize = a.resid_is_f32 ? 4 : 2, osize = a.out_is_e4m3 ? 1 : 2;
  auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if ((at(a.x) | at(a.gain)) & 1 || (at(a.resid) | at(a.resid_out)) % rsize || at(a.out) % osize || at(a.out_scale) & 3) return XEMA_EALIGN;
  // A thread writes resid_out where it has read, and others may not have: over an operand only value for value.
  auto rows_of = [&](const void* p, long long cols, long long ld, long long size) {
    const long long pitch = ld * size;
    return pitch < 0 ? Rows{static_cast<const char*>(p) + (p ? (a.rows - 1) * pitch : 0), a.rows, cols * size, -pitch} : Rows{p, a.rows, cols * size, pitch};
  };
  const Rows x = rows_of(a.x, a.D, a.ldx, 2), resid = rows_of(a.resid, a.D, a.ldr, rsize), gain = {a.gain, 1, 2LL * a.D, 0};
  const Rows out = rows_of(a.out, a.D, a.ldo, osize), resid_out = rows_of(a.resid_out, a.D, a.ldro, rsize), factors = {a.out_scale, 1, 4LL * a.rows, 0};
  auto in_place = [&](const Rows& in) { return in.p == resid_out.p && in.bytes == resid_out.bytes && (a.rows == 1 || in.pitch == resid_out.pitch); };
  for (const Rows& in : {x, resid, gain})
    if (rows_meet(out, in) || rows_meet(factors, in)) return XEMA_EINVAL;
  if (rows_meet(resid_out, gain) || (!in_place(x) && rows_meet(resid_out, x)) || (!in_place(resid) && rows_meet(resid_out, resid))) return XEMA_EINVAL;
  if (rows_meet(out, resid_out) || rows_meet(out, factors) || rows_meet(resid_out, factors)) return XEMA_EINVAL;
  // values that every row allows to be moved at once
  auto allows = [&](int e) {
    auto row = [&](const void* p, long long ld, uintptr_t size) {
      return !p || (at(p) % std::min<uintptr_t>(16, e * size) == 0 && (a.rows == 1 || ld % e == 0));
    };
    return a.D % e == 0 && row(a.gain, 0, 2) && row(a.x, a.ldx, 2) && row(a.resid, a.ldr, rsize) && row(a.resid_out, a.ldro, rsize) &&
           row(a.out, a.ldo, osize);
  };
  const int at_once = allows(8) ? 8 : allows(2) ? 2 : 1;
  if (a.resid_is_f32)
    return a.out_is_e4m3 ? launch<float, __nv_fp8_e4m3>(a, at_once, stream) : launch<float, __nv_bfloat16>(a, at_once, stream);
  return a.out_is_e4m3 ? launch<__nv_bfloat16, __nv_fp8_e4m3>(a, at_once, stream) : launch<__nv_bfloat16, __nv_bfloat16>(a, at_once, stream);
}

}  // namespace xema
