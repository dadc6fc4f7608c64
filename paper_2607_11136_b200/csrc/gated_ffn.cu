// Gated feed-forward h = act(x Wg^T) * (x Wu^T) and its gradients.
#include "skinny_gemm.cuh"

namespace xema {
using namespace tiles;

namespace {
// Rows up to which the kernels for few tokens are considered.
constexpr int kFewRows = 1024;

// Whether a product of so many rows can run in the kernel that is asked for.
bool can_run(const xema_ff_shape* in, int rows, bool gated) { return !in || is_tile(*in, gated) || (in->kernel == XEMA_FF_FEW && rows <= kFewRows); }

bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// dg = dh * zu * act'(zg), du = dh * act(zg), eight neighbouring features a thread.  `d` may be `z`: a thread reads what it overwrites.
// With a = z s(q), s the logistic function: a' = s + z s (1 - s) q'.  Bound by HBM: 8192 x 11264 (1.1 GB) 190 us, 5.8 TB/s.
__global__ void __launch_bounds__(256) gated_grad_kernel(const __nv_bfloat16* dh, long long lddh, const __nv_bfloat16* z,
                                                         __nv_bfloat16* d, int rows, int ffn, int act) {
  grid_dep_wait();
  grid_dep_launch();     // (after the wait: CTAs of two launches share the SMs, never of three; no call is slower for it)
  const int groups = ffn / 8;
  const long long total = (long long)rows * groups, plane = (long long)rows * ffn;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
    const long long row = i / groups;
    const int g = (int)(i - row * groups);
    const uint4 a = ld_u4(dh + row * lddh + g * 8), zg = ld_u4(z + i * 8), zu = ld_u4(z + plane + i * 8), low = ld_u4(z + 2 * plane + i * 8);
    const uint32_t *pa = &a.x, *pg = &zg.x, *pu = &zu.x, *pl = &low.x;
    uint32_t og[4], ou[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float dg[2], du[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float in = e ? bf16_hi(pa[k]) : bf16_lo(pa[k]);
        const float v = with_low(e ? bf16_hi(pg[k]) : bf16_lo(pg[k]), (int8_t)(pl[k] >> (16 * e)));
        const float u = with_low(e ? bf16_hi(pu[k]) : bf16_lo(pu[k]), (int8_t)(pl[k] >> (16 * e + 8)));
        const float s = sigmoid_f(act_q(v, act));
        const float dq = act == XEMA_ACT_SILU ? 1.f : 1.5957691216057308f * fmaf(3.f * 0.044715f * v, v, 1.f);
        const float slope = s > 0.f && s < 1.f ? fmaf(v * s * (1.f - s), dq, s) : s;   // (dq may overflow at the ends)
        dg[e] = in * u * slope;
        du[e] = in * v * s;
      }
      og[k] = pack_bf16x2(dg[0], dg[1]);
      ou[k] = pack_bf16x2(du[0], du[1]);
    }
    *reinterpret_cast<uint4*>(d + i * 8) = make_uint4(og[0], og[1], og[2], og[3]);
    *reinterpret_cast<uint4*>(d + plane + i * 8) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
  }
}
}  // namespace

int launch_gated_ffn(const xema_gated_ffn_args& a, unsigned int* status, cudaStream_t stream, const xema_ff_shape* in) {
  const int unit = a.is_e4m3 ? 16 : 8, elem = a.is_e4m3 ? 1 : 2;
  if (a.rows < 0 || a.width < unit || a.width % unit || a.ffn < 8 || a.ffn % 8) return XEMA_EINVAL;
  if (a.rows > kMaxSize || a.width > kMaxSize || a.ffn > kMaxSize) return XEMA_EINVAL;
  if (a.activation != XEMA_ACT_SILU && a.activation != XEMA_ACT_GELU_TANH) return XEMA_EINVAL;
  if (a.rows == 0) return XEMA_OK;
  if (!a.x || !a.w_gate || !a.w_up || !a.h) return XEMA_EINVAL;
  if (a.is_e4m3 ? (!a.x_scale || !a.gate_scale || !a.up_scale || a.z) : (a.x_scale || a.gate_scale || a.up_scale)) return XEMA_EINVAL;
  if ((a.rows > 1 && (a.ldx < a.width || a.ldh < a.ffn)) || a.ldw < a.width) return XEMA_EINVAL;
  if (!on16(a.x) || !on16(a.w_gate) || !on16(a.w_up) || !on16(a.h) || !on16(a.z)) return XEMA_EALIGN;
  if ((a.rows > 1 && (a.ldx % unit || a.ldh % 8)) || a.ldw % unit) return XEMA_EALIGN;
  for (const float* f : {a.x_scale, a.gate_scale, a.up_scale})
    if (reinterpret_cast<uintptr_t>(f) & 3) return XEMA_EALIGN;
  const Rows x = {a.x, a.rows, (long long)a.width * elem, a.ldx * elem}, h = {a.h, a.rows, a.ffn * 2LL, a.ldh * 2};
  const Rows wg = {a.w_gate, a.ffn, (long long)a.width * elem, a.ldw * elem}, wu = {a.w_up, a.ffn, (long long)a.width * elem, a.ldw * elem};
  const Rows z = {a.z, 1, 6LL * a.rows * a.ffn, 0};
  for (const Rows& in : {x, wg, wu})
    if (rows_meet(h, in) || rows_meet(z, in)) return XEMA_EINVAL;
  const Rows sx = {a.x_scale, 1, 4LL * a.rows, 0}, sg = {a.gate_scale, 1, 4LL * a.ffn, 0}, su = {a.up_scale, 1, 4LL * a.ffn, 0};
  if (rows_meet(h, z) || rows_meet(h, sx) || rows_meet(h, sg) || rows_meet(h, su)) return XEMA_EINVAL;      // (no z with factors)
  const int step = 128 / elem;
  Params p = {};
  p.batch = 1;
  p.rows = a.rows;
  p.cols = a.ffn;
  p.k_main = (a.width + step - 1) / step;
  p.act = a.activation;
  p.keep = a.z != nullptr;
  p.row_scale = a.x_scale;
  p.gate_scale = a.gate_scale;
  p.up_scale = a.up_scale;
  p.status = status;
  p.off_line = ((a.rows > 1 ? a.ldx : 0) | a.ldw) * elem % 128 != 0;
  if (!can_run(in, a.rows, true)) return XEMA_EINVAL;
  const Shape shape = take_shape(p, p.k_main, true, in);
  if (a.rows <= kFewRows && (!in || in->kernel == XEMA_FF_FEW)) {
    skinny::Params q = {};
    q.rows = a.rows;
    q.cols = a.ffn;
    q.k_blocks = p.k_main;
    q.act = a.activation;
    q.row_scale = a.x_scale;
    q.gate_scale = a.gate_scale;
    q.up_scale = a.up_scale;
    q.out = static_cast<__nv_bfloat16*>(a.h);
    q.ldo = a.rows > 1 ? a.ldh : a.ffn;
    q.z = static_cast<__nv_bfloat16*>(a.z);
    q.status = status;
    long long ns = 0;
    const int s = in ? in->share : 0, r = in ? in->features : 0;
    int rc = a.is_e4m3 ? skinny::plan<skinny::Kind::kGated, true>(&q, &ns, s, r) : skinny::plan<skinny::Kind::kGated, false>(&q, &ns, s, r);
    if (rc) return rc;
    if (in || ns < shape_ns(p, shape, p.k_main, true)) {
      skinny::Maps m = {};
      rc = encode_tmap_tile(&m.a, a.w_gate, elem, a.width, a.ffn, 1, a.ldw, 0, step, q.R);
      if (!rc) rc = encode_tmap_tile(&m.a2, a.w_up, elem, a.width, a.ffn, 1, a.ldw, 0, step, q.R);
      if (!rc) rc = encode_tmap_tile(&m.x, a.x, elem, a.width, a.rows, 1, a.ldx, 0, step, q.nt);
      if (rc) return rc;
      return a.is_e4m3 ? skinny::launch<skinny::Kind::kGated, true>(m, q, stream) : skinny::launch<skinny::Kind::kGated, false>(m, q, stream);
    }
  }
  Maps m = {};
  int rc = encode_tmap_tile(&m.a, a.x, elem, a.width, a.rows, 1, a.ldx, 0, step, 128);
  if (!rc) rc = encode_tmap_tile(&m.b, a.w_gate, elem, a.width, a.ffn, 1, a.ldw, 0, step, b_box(shape, true));
  if (!rc) rc = encode_tmap_tile(&m.b2, a.w_up, elem, a.width, a.ffn, 1, a.ldw, 0, step, b_box(shape, true));
  if (!rc) rc = encode_tmap_tile(&m.out, a.h, 2, a.ffn, a.rows, 1, a.ldh, 0, 32, 32);
  if (!rc && a.z) rc = encode_tmap_tile(&m.out2, a.z, 2, a.ffn, a.rows, 3, a.ffn, (long long)a.rows * a.ffn, 32, 32);
  if (rc) return rc;
  return a.is_e4m3 ? launch<Form::kGated, true>(m, p, shape, stream) : launch<Form::kGated, false>(m, p, shape, stream);
}

int launch_gated_ffn_grad(const xema_gated_ffn_grad_args& a, unsigned int* status, cudaStream_t stream, const xema_ff_shape* dx_in,
                          const xema_ff_shape* dw_in) {
  if (a.rows < 0 || a.width < 8 || a.width % 8 || a.ffn < 8 || a.ffn % 8) return XEMA_EINVAL;
  if (a.rows > kMaxSize || a.width > kMaxSize || a.ffn > kMaxSize) return XEMA_EINVAL;
  if (a.activation != XEMA_ACT_SILU && a.activation != XEMA_ACT_GELU_TANH) return XEMA_EINVAL;
  if ((a.dw_gate == nullptr) != (a.dw_up == nullptr)) return XEMA_EINVAL;
  const bool want_w = a.dw_gate != nullptr, want_x = a.dx != nullptr;
  if (want_w && a.lddw < a.width) return XEMA_EINVAL;
  if (want_w && (!on16(a.dw_gate) || !on16(a.dw_up) || a.lddw % 8)) return XEMA_EALIGN;
  if (a.rows == 0) {
    for (void* w : {a.dw_gate, a.dw_up}) {
      const cudaError_t e = want_w ? cudaMemset2DAsync(w, (size_t)a.lddw * 2, 0, (size_t)a.width * 2, a.ffn, stream) : cudaSuccess;
      if (e != cudaSuccess) {
        set_last_cuda_error((int)e);
        return XEMA_ECUDA;
      }
    }
    return XEMA_OK;
  }
  if (!want_w && !want_x) return XEMA_OK;
  if (!a.dh || !a.z || !a.work || (want_w && !a.x) || (want_x && (!a.w_gate || !a.w_up))) return XEMA_EINVAL;
  if (a.rows > 1 && (a.lddh < a.ffn || (want_w && a.ldx < a.width) || (want_x && a.lddx < a.width))) return XEMA_EINVAL;
  if (want_x && a.ldw < a.width) return XEMA_EINVAL;
  if (!on16(a.dh) || !on16(a.z) || !on16(a.work)) return XEMA_EALIGN;
  if (want_w && !on16(a.x)) return XEMA_EALIGN;
  if (want_x && (!on16(a.w_gate) || !on16(a.w_up) || !on16(a.dx) || a.ldw % 8)) return XEMA_EALIGN;
  if (a.rows > 1 && (a.lddh % 8 || (want_w && a.ldx % 8) || (want_x && a.lddx % 8))) return XEMA_EALIGN;

  if (!can_run(dx_in, a.rows, false) || (dw_in && !is_tile(*dw_in, false))) return XEMA_EINVAL;

  const long long row = 2LL * a.width, z_bytes = 2LL * a.rows * a.ffn;
  const Rows in[] = {{a.dh, a.rows, 2LL * a.ffn, a.lddh * 2}, {want_w ? a.x : nullptr, a.rows, row, a.ldx * 2},
                     {want_x ? a.w_gate : nullptr, a.ffn, row, a.ldw * 2}, {want_x ? a.w_up : nullptr, a.ffn, row, a.ldw * 2}};
  const Rows z = {a.z, 1, 3 * z_bytes, 0}, work = {a.work, 1, 2 * z_bytes, 0}, dx = {a.dx, a.rows, row, a.lddx * 2};
  const Rows dwg = {a.dw_gate, a.ffn, row, a.lddw * 2}, dwu = {a.dw_up, a.ffn, row, a.lddw * 2};
  for (const Rows& out : {work, dx, dwg, dwu})
    for (const Rows& i : in)
      if (rows_meet(out, i)) return XEMA_EINVAL;
  if (a.work != a.z && rows_meet(work, z)) return XEMA_EINVAL;
  for (const Rows& out : {dx, dwg, dwu})
    if (rows_meet(out, z) || rows_meet(out, work)) return XEMA_EINVAL;
  if (rows_meet(dx, dwg) || rows_meet(dx, dwu) || rows_meet(dwg, dwu)) return XEMA_EINVAL;

  const long long groups = (long long)a.rows * (a.ffn / 8);
  const int grid = (int)std::min<long long>((groups + 255) / 256, 16LL * sm_count());
  int rc = launch_kernel(gated_grad_kernel, dim3(grid), 256, 0, stream, true, static_cast<const __nv_bfloat16*>(a.dh), (long long)a.lddh,
                         static_cast<const __nv_bfloat16*>(a.z), static_cast<__nv_bfloat16*>(a.work), a.rows, a.ffn, a.activation);
  const long long plane = (long long)a.rows * a.ffn;
  if (!rc && want_x) {
    Params p = {};
    p.batch = 1;
    p.rows = a.rows;
    p.cols = a.width;
    p.k_main = (a.ffn + 63) / 64;
    p.status = status;
    p.off_line = (a.ffn | a.ldw) * 2 % 128 != 0;
    const Shape shape = take_shape(p, 2 * p.k_main, false, dx_in);
    skinny::Params q = {};
    long long ns = 0;
    if (a.rows <= kFewRows && (!dx_in || dx_in->kernel == XEMA_FF_FEW)) {
      q.rows = a.rows;
      q.cols = a.width;
      q.k_blocks = 2 * p.k_main;
      q.k_half = p.k_main;
      q.out = static_cast<__nv_bfloat16*>(a.dx);
      q.ldo = a.rows > 1 ? a.lddx : a.width;
      q.status = status;
      rc = skinny::plan<skinny::Kind::kGradX, false>(&q, &ns, dx_in ? dx_in->share : 0, dx_in ? dx_in->features : 0);
    }
    if (!rc && ns && (dx_in || ns < shape_ns(p, shape, 2 * p.k_main, false))) {
      skinny::Maps m = {};
      rc = encode_tmap_tile(&m.a, a.w_gate, 2, a.width, a.ffn, 1, a.ldw, 0, 64, 64);
      if (!rc) rc = encode_tmap_tile(&m.a2, a.w_up, 2, a.width, a.ffn, 1, a.ldw, 0, 64, 64);
      if (!rc) rc = encode_tmap_tile(&m.x, a.work, 2, a.ffn, a.rows, 2, a.ffn, plane, 64, q.nt);
      if (!rc) rc = skinny::launch<skinny::Kind::kGradX, false>(m, q, stream);
    } else if (!rc) {
      Maps m = {};
      rc = encode_tmap_tile(&m.a, a.work, 2, a.ffn, a.rows, 2, a.ffn, plane, 64, 128);
      if (!rc) rc = encode_tmap_tile(&m.b, a.w_gate, 2, a.width, a.ffn, 1, a.ldw, 0, 64, 64);
      if (!rc) rc = encode_tmap_tile(&m.b2, a.w_up, 2, a.width, a.ffn, 1, a.ldw, 0, 64, 64);
      if (!rc) rc = encode_tmap_tile(&m.out, a.dx, 2, a.width, a.rows, 1, a.lddx, 0, 32, 32);
      if (!rc) rc = launch<Form::kGradX, false>(m, p, shape, stream);
    }
  }
  if (!rc && want_w) {
    Params p = {};
    p.batch = 2;
    p.rows = a.ffn;
    p.cols = a.width;
    p.k_main = (a.rows + 63) / 64;
    p.off_line = (a.ffn | (a.rows > 1 ? a.ldx : 0)) * 2 % 128 != 0;
    p.status = status;
    Maps m = {};
    rc = encode_tmap_tile(&m.a, a.work, 2, a.ffn, a.rows, 2, a.ffn, plane, 64, 64);
    if (!rc) rc = encode_tmap_tile(&m.b, a.x, 2, a.width, a.rows, 1, a.ldx, 0, 64, 64);
    if (!rc) rc = encode_tmap_tile(&m.out, a.dw_gate, 2, a.width, a.ffn, 1, a.lddw, 0, 32, 32);
    if (!rc) rc = encode_tmap_tile(&m.out2, a.dw_up, 2, a.width, a.ffn, 1, a.lddw, 0, 32, 32);
    if (!rc) rc = launch<Form::kGradW, false>(m, p, take_shape(p, p.k_main, false, dw_in), stream);
  }
  return rc;
}

}  // namespace xema
