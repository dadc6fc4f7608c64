// A projection that all requests of a batch share, beside each request's own low-rank adapter:
//   y[b] = x[b] W^T + bias + t[b] B_a^T,  t[b] = scale_a (x[b] A_a^T),  a = adapter[b].
// Two launches: t, and the projection.  With many tokens the projection's accumulator takes t B^T as further steps along K; with
// few it streams W, and t B^T is worked out beside it.  us, back to back in a graph: 4 x 4608 tokens of 4096 x 4096, rank 64, 426 (t alone 30);
// 60 x 30 tokens of 1024 x 2048 18 (30 with a tile of 128 rows a request); 256 single tokens of 4096 x 4096 26 (204 with 16 columns each).
#include "skinny_gemm.cuh"

namespace xema {
using namespace tiles;

namespace {
constexpr int kShrinkWarps = 4;
constexpr int kFewTokens = 1024;      // single tokens: up to which t B^T on the CUDA cores is considered
constexpr int kFewRows = 512;         // of a request: up to which the kernel with requests side by side in a tile is considered
constexpr int kShrinkRows = 8;        // of a request: up to which t is made by the CUDA cores

// t for few tokens: a block takes up to TOK tokens of one request and RANKS columns of its adapter; its warps share K.
template <int TOK, int RANKS>
__global__ void __launch_bounds__(kShrinkWarps * 32) shrink_kernel(const __nv_bfloat16* x, long long ldx, long long x_batch_rows,
                                                                   const __nv_bfloat16* lora_a, const float* scale, const int* adapter,
                                                                   __nv_bfloat16* t, int rows, int K, int rank, int n_adapters) {
  __shared__ float s_part[kShrinkWarps][TOK * RANKS];
  grid_dep_wait();       // before the next launch may start: it reads x and W ahead of its own wait
  grid_dep_launch();
  const int b = blockIdx.x, i0 = blockIdx.z * TOK, j0 = blockIdx.y * RANKS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int a = adapter[b];
  if (a < 0 || a >= n_adapters) return;
  const __nv_bfloat16* xr[TOK];
  const __nv_bfloat16* ar[RANKS];
#pragma unroll
  for (int i = 0; i < TOK; ++i) xr[i] = x + ((long long)b * x_batch_rows + min(i0 + i, rows - 1)) * ldx;
#pragma unroll
  for (int j = 0; j < RANKS; ++j) ar[j] = lora_a + ((long long)a * rank + j0 + j) * K;
  float sum[TOK][RANKS] = {};
#pragma unroll 2
  for (int g = warp * 32 + lane; g < K / 8; g += kShrinkWarps * 32) {
    uint4 av[RANKS], xv[TOK];
#pragma unroll
    for (int j = 0; j < RANKS; ++j) av[j] = ld_u4(reinterpret_cast<const uint4*>(ar[j]) + g);
#pragma unroll
    for (int i = 0; i < TOK; ++i) xv[i] = ld_u4(reinterpret_cast<const uint4*>(xr[i]) + g);
#pragma unroll
    for (int i = 0; i < TOK; ++i)
#pragma unroll
      for (int j = 0; j < RANKS; ++j) sum[i][j] = skinny::dot8(xv[i], av[j], sum[i][j]);
  }
#pragma unroll
  for (int i = 0; i < TOK; ++i)
#pragma unroll
    for (int j = 0; j < RANKS; ++j) {
      float v = sum[i][j];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane == 0) s_part[warp][i * RANKS + j] = v;
    }
  __syncthreads();
  if (threadIdx.x < TOK * RANKS) {
    const int i = threadIdx.x / RANKS, j = threadIdx.x % RANKS;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kShrinkWarps; ++w) v += s_part[w][threadIdx.x];
    if (i0 + i < rows) t[((long long)b * rows + i0 + i) * rank + j0 + j] = __float2bfloat16_rn(v * scale[a]);
  }
}

// The rows of `batch` requests, `step` rows from one to the next.
struct Batches {
  Rows one;
  int batch;
  long long step;
  // all rows from the first to the last, those between the requests too
  Rows all() const { return {one.p, (batch - 1) * (batch > 1 ? step : 0) + one.rows, one.bytes, one.pitch}; }
};
// Whether two of them share a byte.  With the same steps that is so for all pairs of requests if it is for one pair so far apart, and only
// those count whose ranges meet: two or three where requests do not overlap.  Otherwise the rows between the requests count too.
bool batches_meet(const Batches& a, const Batches& b) {
  if (!rows_meet(a.all(), b.all())) return false;
  if (a.batch == 1 || a.one.pitch != b.one.pitch || a.step != b.step || a.step < a.one.rows) return true;
  const long long pitch = a.one.pitch * a.step, off = (long long)reinterpret_cast<uintptr_t>(b.one.p) - (long long)reinterpret_cast<uintptr_t>(a.one.p);
  for (long long d = -off / pitch - 2; d <= -off / pitch + 2; ++d) {
    if (d <= -a.batch || d >= a.batch) continue;
    Rows shifted = b.one;
    shifted.p = static_cast<const char*>(b.one.p) + d * pitch;
    if (rows_meet(a.one, shifted)) return true;
  }
  return false;
}

// CTAs that share K of t, for a projection of `tiles` CTAs or (pair) pairs.  The projection starts on the SMs that t leaves free (a pair needs
// both SMs of two neighbours) and has its first waves to go before it needs t: one CTA a tile where the projection fills the device for longer
// than a wave, else as many as there is room for beside it, and (with enough of K to share) four where there is none and everything waits for
// t.  us with 1 / 2 / 4, rank 16: pairs of 192 columns 5 x 397 tokens 1544 x 2312 26.5 / 27.8 / 31.8, 3 x 1000 4096 x 2048 39.0 / 45.1 / 43.7; 128 x
// 128 2 x 100 4096 x 4096 20.4 / 20.3 / 20.1, 1 x 333 2048 x 2048 13.9 / 11.5 / 10.9, 1 x 2000 1024 x 1024 11.2 / 13.6 / 13.4.  Where it picks worse:
// 7 x 300 3000 x 1024, pairs of 256, 25.1 / 31.7 / 31.6.
// *beside: whether t runs beside the projection's first tiles and takes no time of its own.
int shrink_split(const skinny::Params& s, long long tiles, bool pair, bool* beside) {
  const long long slots = pair ? sm_count() / 2 : sm_count(), left = slots - tiles;
  auto takes = [&](int n) { return (long long)s.tiles * (pair ? (n + 1) / 2 : n); };
  // (of several waves the workers that start late are those without a tile of the last one, where that is not full)
  *beside = (left >= 0 ? left : (slots - tiles % slots) % slots) >= takes(1);
  int split = 1;
  if (left >= 0) split = left >= takes(4) || (left < takes(1) && s.k_blocks >= 32) ? 4 : left >= takes(2) ? 2 : 1;
  while (split > 1 && (split - 1) * ((s.k_blocks + split - 1) / split) >= s.k_blocks) split /= 2;
  return split;
}

template <int TOK, int RANKS>
int launch_shrink(const xema_lora_args& a, cudaStream_t stream) {
  return launch_kernel(shrink_kernel<TOK, RANKS>, dim3(a.batch, a.rank / RANKS, (a.rows + TOK - 1) / TOK), kShrinkWarps * 32, 0, stream, true,
                       static_cast<const __nv_bfloat16*>(a.x), (long long)a.ldx, (long long)a.x_batch_rows, static_cast<const __nv_bfloat16*>(a.lora_a),
                       a.scale, a.adapter, static_cast<__nv_bfloat16*>(a.work), a.rows, a.K, a.rank, a.n_adapters);
}
}  // namespace

unsigned long long lora_work_bytes(int batch, int rows, int rank) {
  if (batch < 0 || rows < 0 || rank < 0) return 0;
  return 2ull * batch * rows * rank;
}

int launch_lora(const xema_lora_args& a, unsigned int* status, cudaStream_t stream, const xema_ff_shape* in, int share_t) {
  if (a.batch < 0 || a.rows < 0 || a.K < 8 || a.K % 8 || a.N < 8 || a.N % 8 || a.n_adapters < 0) return XEMA_EINVAL;
  if (a.batch > kMaxSize || a.rows > kMaxSize || a.K > kMaxSize || a.N > kMaxSize) return XEMA_EINVAL;
  if (a.rank < 8 || a.rank % 8 || a.rank > XEMA_LORA_MAX_RANK) return XEMA_EINVAL;
  if (a.batch == 0 || a.rows == 0) return XEMA_OK;
  if (!a.x || !a.w || !a.out || !a.adapter) return XEMA_EINVAL;
  if (a.n_adapters > 0 && (!a.lora_a || !a.lora_b || !a.scale || !a.work)) return XEMA_EINVAL;
  const long long total = (long long)a.batch * a.rows;
  if (a.ldw < a.K || (total > 1 && (a.ldx < a.K || a.ldo < a.N))) return XEMA_EINVAL;
  if (a.batch > 1 && (a.x_batch_rows < 1 || a.out_batch_rows < a.rows)) return XEMA_EINVAL;
  auto mis = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; };
  if (mis(a.x) || mis(a.w) || mis(a.out) || mis(a.lora_a) || mis(a.lora_b) || mis(a.work)) return XEMA_EALIGN;
  if (a.ldw % 8 || (total > 1 && (a.ldx % 8 || a.ldo % 8))) return XEMA_EALIGN;
  if ((reinterpret_cast<uintptr_t>(a.adapter) | reinterpret_cast<uintptr_t>(a.scale)) & 3) return XEMA_EALIGN;
  if (reinterpret_cast<uintptr_t>(a.bias) & 1) return XEMA_EALIGN;
  const Batches x = {{a.x, a.rows, a.K * 2LL, a.ldx * 2}, a.batch, a.x_batch_rows}, out = {{a.out, a.rows, a.N * 2LL, a.ldo * 2}, a.batch, a.out_batch_rows};
  const Rows work = {a.n_adapters > 0 ? a.work : nullptr, 1, (long long)lora_work_bytes(a.batch, a.rows, a.rank), 0};
  const Rows operands[] = {{a.w, a.N, a.K * 2LL, a.ldw * 2}, {a.lora_a, 1, 2LL * a.n_adapters * a.rank * a.K, 0},
                     {a.lora_b, 1, 2LL * a.n_adapters * a.rank * a.N, 0}, {a.bias, 1, 2LL * a.N, 0}, {a.adapter, 1, 4LL * a.batch, 0},
                     {a.n_adapters > 0 ? a.scale : nullptr, 1, 4LL * a.n_adapters, 0}};
  for (const Rows& i : operands)
    if (rows_meet(out.all(), i) || rows_meet(work, i)) return XEMA_EINVAL;
  if (rows_meet(out.all(), work) || rows_meet(x.all(), work) || batches_meet(x, out)) return XEMA_EINVAL;
  Params p = {};
  p.batch = a.batch;
  p.rows = a.rows;
  p.cols = a.N;
  p.k_main = (a.K + 63) / 64;
  p.k_more = (a.rank + 63) / 64;
  p.bias = static_cast<const __nv_bfloat16*>(a.bias);
  p.adapter = a.adapter;
  p.n_adapters = a.n_adapters;
  p.behind = a.n_adapters > 0;
  p.status = status;
  p.off_line = ((total > 1 ? a.ldx : 0) | a.ldw) * 2 % 128 != 0;
  if (in && !is_tile(*in, false) && !(in->kernel == XEMA_FF_FEW && a.rows <= kFewRows) &&
      !(in->kernel == XEMA_FF_SINGLE && a.rows == 1 && total <= kFewTokens))
    return XEMA_EINVAL;
  const Shape shape = take_shape(p, p.k_main + p.k_more, false, in);
  const long long shared_ns = shape_ns(p, shape, p.k_main + p.k_more, false);

  // The kernels for few tokens: single tokens, or a few rows a request.  (Strides count in the choice where they take rows off the 128-byte lines,
  // through the estimate for tiles; results then differ in their last bits.)
  using skinny::Kind;
  skinny::Params q = {};
  long long ns = 0, ns1 = 0;
  q.cols = a.N;
  q.k_blocks = p.k_main;
  q.out = static_cast<__nv_bfloat16*>(a.out);
  q.ldo = total > 1 ? a.ldo : a.N;
  q.out_batch_rows = a.batch > 1 ? a.out_batch_rows : 0;
  q.bias = p.bias;
  q.t = static_cast<const __nv_bfloat16*>(a.work);
  q.lora_b = static_cast<const __nv_bfloat16*>(a.lora_b);
  q.adapter = a.adapter;
  q.n_adapters = a.n_adapters;
  q.rank = a.rank;
  q.behind = p.behind;
  q.status = status;
  skinny::Params q1 = q;
  int rc = XEMA_OK;
  const int only_s = in ? in->share : 0, only_r = in ? in->features : 0;
  if (a.rows <= kFewRows && (!in || in->kernel == XEMA_FF_FEW)) {
    q.rows = a.rows;
    q.batch = a.batch;
    if ((rc = skinny::plan<Kind::kPacked, false>(&q, &ns, only_s, only_r))) return rc;
  }
  if (a.rows == 1 && total <= kFewTokens && (!in || in->kernel == XEMA_FF_SINGLE)) {
    q1.rows = (int)total;
    if ((rc = skinny::plan<Kind::kLora, false>(&q1, &ns1, only_s, only_r))) return rc;
    ns1 += total * a.N * a.rank / 3000;        // t B^T beside the products
  }
  // t: by the CUDA cores beside a projection of either kind, or by a launch that takes SMs of its own
  const bool tokens_alone = a.rows <= kShrinkRows || a.n_adapters == 0;
  skinny::Params s[2] = {};
  long long packed_ns = ns, tiled_ns = shared_ns;
  if (!tokens_alone) {
    for (int i = 0; i < 2; ++i) {
      if (i == 1 && !ns) continue;
      s[i].rows = a.rows;
      s[i].batch = a.batch;
      s[i].cols = a.rank;
      s[i].k_blocks = p.k_main;
      s[i].out = static_cast<__nv_bfloat16*>(a.work);
      s[i].ldo = a.rank;
      s[i].adapter = a.adapter;
      s[i].adapter_scale = a.scale;
      s[i].n_adapters = a.n_adapters;
      s[i].status = status;
      bool beside = false;
      long long t_ns = 0;
      if ((rc = skinny::tile_tokens<Kind::kShrink>(&s[i]))) return rc;
      const int split = share_t ? share_t : shrink_split(s[i], i ? (long long)q.f_tiles * q.tiles * q.S : tile_count(p, shape, false), i ? false : shape.pair, &beside);
      if ((rc = skinny::plan<Kind::kShrink, false>(&s[i], &t_ns, split))) return rc;
      if (!beside) (i ? packed_ns : tiled_ns) += t_ns;
    }
  }
  const bool packed = ns && (in || (packed_ns < tiled_ns && (!ns1 || packed_ns < ns1))), flat = !packed && ns1 && (in || ns1 < tiled_ns);

  if (a.n_adapters > 0) {
    if (flat || tokens_alone) {
      rc = a.rows == 1 ? launch_shrink<1, 4>(a, stream) : launch_shrink<8, 2>(a, stream);
    } else {
      const skinny::Params& t = s[packed];
      skinny::Maps m = {};
      rc = encode_tmap_tile(&m.a, a.lora_a, 2, a.K, a.rank, a.n_adapters, a.K, (long long)a.rank * a.K, 64, t.R);
      if (!rc) rc = encode_tmap_tile(&m.x, a.x, 2, a.K, a.rows, a.batch, a.ldx, a.x_batch_rows * a.ldx, 64, t.nt);
      if (!rc) rc = skinny::launch<Kind::kShrink, false>(m, t, stream);
    }
    if (rc) return rc;
  }

  if (packed || flat) {
    skinny::Maps m = {};
    const skinny::Params& f = packed ? q : q1;
    rc = encode_tmap_tile(&m.a, a.w, 2, a.K, a.N, 1, a.ldw, 0, 64, f.R);
    if (flat) {
      if (!rc) rc = encode_tmap_tile(&m.x, a.x, 2, a.K, total, 1, a.x_batch_rows * a.ldx, 0, 64, f.nt);
      return rc ? rc : skinny::launch<Kind::kLora, false>(m, f, stream);
    }
    if (!rc) rc = encode_tmap_tile(&m.x, a.x, 2, a.K, a.rows, a.batch, a.ldx, a.x_batch_rows * a.ldx, 64, f.pad);
    if (!rc && a.n_adapters > 0) rc = encode_tmap_tile(&m.a2, a.lora_b, 2, a.rank, a.N, a.n_adapters, a.rank, (long long)a.N * a.rank, 64, f.R);
    if (!rc && a.n_adapters > 0) rc = encode_tmap_tile(&m.t, a.work, 2, a.rank, a.rows, a.batch, a.rank, (long long)a.rows * a.rank, 64, f.pad);
    if (a.n_adapters == 0) m.a2 = m.t = m.a;
    return rc ? rc : skinny::launch<Kind::kPacked, false>(m, f, stream);
  }
  const int box = b_box(shape, false);
  Maps m = {};
  rc = encode_tmap_tile(&m.a, a.x, 2, a.K, a.rows, a.batch, a.ldx, a.x_batch_rows * a.ldx, 64, 128);
  if (!rc) rc = encode_tmap_tile(&m.b, a.w, 2, a.K, a.N, 1, a.ldw, 0, 64, box);
  if (!rc) rc = encode_tmap_tile(&m.out, a.out, 2, a.N, a.rows, a.batch, a.ldo, a.out_batch_rows * a.ldo, 32, 32);
  if (!rc && a.n_adapters > 0) rc = encode_tmap_tile(&m.a2, a.work, 2, a.rank, a.rows, a.batch, a.rank, (long long)a.rows * a.rank, 64, 128);
  if (!rc && a.n_adapters > 0) rc = encode_tmap_tile(&m.b2, a.lora_b, 2, a.rank, a.N, a.n_adapters, a.rank, (long long)a.N * a.rank, 64, box);
  if (rc) return rc;
  return launch<Form::kLinear, false>(m, p, shape, stream);
}

}  // namespace xema
