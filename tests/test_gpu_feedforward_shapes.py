"""The feed-forward products in every kernel and shape that the estimates choose from, against plain implementations in 64 bits: each
tile's operand layouts, ragged ends and second rounds, and each share of K among CTAs, whatever sizes would take them.  Tolerances as derived in
test_gpu_feedforward."""
import math

import pytest
import torch

from paper_2607_11136_b200 import binding as xb
from test_gpu_feedforward import BF, DEV, _act_ref, _close, _close_grad, _gen, _grads_ref, _lora_case, _lora_ref, _quant, _randn

pytestmark = pytest.mark.gpu
T_ROUND = 6 * 2.0 ** -8 / math.sqrt(3)      # of t to bf16
TILES = [(0, 128)] + [(1, n) for n in (128, 160, 192, 224, 256)]
SHARES = (1, 2, 4)


def _tile(pair, columns):
    return xb.xema_ff_shape(kernel=xb.FF_TILES, pair=pair, columns=columns)


def _few(share, features, kernel=xb.FF_FEW):
    return xb.xema_ff_shape(kernel=kernel, share=share, features=features)


class _Status:
    def __init__(self):
        self.word = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.stream = torch.cuda.current_stream().cuda_stream

    def ok(self):
        torch.cuda.synchronize()
        assert self.word.item() == 0


def _nan(*shape):
    return torch.full(shape, math.nan, dtype=BF, device=DEV)


def _gated(status, shape, x, wg, wu, act, scales=None, keep=False):
    rows, width, ffn = x.shape[0], x.shape[1], wg.shape[0]
    h, z = _nan(rows, ffn), torch.zeros(3, rows, ffn, dtype=torch.int16, device=DEV) if keep else None
    a = xb.xema_gated_ffn_args(x=x.data_ptr(), ldx=width, w_gate=wg.data_ptr(), w_up=wu.data_ptr(), ldw=width, h=h.data_ptr(), ldh=ffn,
                               z=z.data_ptr() if keep else None, rows=rows, width=width, ffn=ffn, activation=act)
    if scales:
        a.is_e4m3 = 1
        a.x_scale, a.gate_scale, a.up_scale = (s.data_ptr() for s in scales)
    xb.xema_op_gated_ffn_in(a, shape, status.word.data_ptr(), status.stream)
    return h, z


def _check_gated(rows, width, ffn, shapes, e4m3):
    """Every shape with both activations, bf16 with and without what the gradient needs."""
    gen = _gen(rows, width, ffn, e4m3, 40)
    x, wg, wu = _randn(gen, (rows, width)), _randn(gen, (ffn, width), width ** -0.5), _randn(gen, (ffn, width), width ** -0.5)
    scales = None
    if e4m3:
        (x, sx), (wg, sg), (wu, su) = map(_quant, (x, wg, wu))
        scales = (sx, sg, su)
        xd, gd, ud = (t.double() * s.double()[:, None] for t, s in ((x, sx), (wg, sg), (wu, su)))
    else:
        xd, gd, ud = x.double(), wg.double(), wu.double()
    zg, zu = xd @ gd.t(), xd @ ud.t()
    status = _Status()
    for act, name in ((xb.ACT_SILU, "silu"), (xb.ACT_GELU_TANH, "gelu_tanh")):
        want = _act_ref(zg, name)[0] * zu
        for what, shape in shapes:
            h, _ = _gated(status, shape, x, wg, wu, act, scales)
            status.ok()
            _close(h, want, (what, name))
            if not e4m3:
                h2, z = _gated(status, shape, x, wg, wu, act, keep=True)
                status.ok()
                assert torch.equal(h, h2), what
                _close(z[0].view(BF), zg, (what, "zg"))
                _close(z[1].view(BF), zu, (what, "zu"))


GATED_TILES = [(p, n) for p, n in TILES if n % 64 == 0]


# two tiles of rows and several of columns with ragged ends; more than two rounds of tiles of every shape
@pytest.mark.parametrize("rows,width,ffn", [(300, 264, 520), (5200, 72, 1032), (20, 456, 136)])
@pytest.mark.parametrize("pair,columns", GATED_TILES)
def test_gated_tiles(rows, width, ffn, pair, columns):
    _check_gated(rows, width, ffn, [((pair, columns), _tile(pair, columns))], False)


@pytest.mark.parametrize("rows,width,ffn", [(300, 272, 520), (5200, 80, 1032), (20, 912, 136)])
@pytest.mark.parametrize("pair,columns", GATED_TILES)
def test_gated_tiles_e4m3(rows, width, ffn, pair, columns):
    _check_gated(rows, width, ffn, [((pair, columns), _tile(pair, columns))], True)


# each width of the MMA; features of a CTA with one and with two products, not all of them multiples of 16
@pytest.mark.parametrize("rows", [1, 16, 17, 32, 40, 64, 100, 128, 129, 300, 1024])
@pytest.mark.parametrize("e4m3", [False, True])
def test_gated_few_tokens(rows, e4m3):
    shapes = [((s, r), _few(s, r)) for s in SHARES for r in (8, 24, 64, 72, 128)]
    _check_gated(rows, 912 if e4m3 else 456, 328, shapes, e4m3)


def _grad(status, dx_in, dw_in, dh, x, wg, wu, z, act):
    rows, width, ffn = x.shape[0], x.shape[1], wg.shape[0]
    work, dx, dg, du = _nan(2, rows, ffn), _nan(rows, width), _nan(ffn, width), _nan(ffn, width)
    a = xb.xema_gated_ffn_grad_args(dh=dh.data_ptr(), lddh=ffn, x=x.data_ptr(), ldx=width, w_gate=wg.data_ptr(), w_up=wu.data_ptr(), ldw=width,
                                    z=z.data_ptr(), work=work.data_ptr(), dx=dx.data_ptr(), lddx=width, dw_gate=dg.data_ptr(),
                                    dw_up=du.data_ptr(), lddw=width, rows=rows, width=width, ffn=ffn, activation=act)
    xb.xema_op_gated_ffn_grad_in(a, dx_in, dw_in, status.word.data_ptr(), status.stream)
    return dx, dg, du


def _grad_case(rows, width, ffn):
    gen = _gen(rows, width, ffn, 41)
    x, dh = _randn(gen, (rows, width)), _randn(gen, (rows, ffn))
    wg, wu = _randn(gen, (ffn, width), width ** -0.5), _randn(gen, (ffn, width), width ** -0.5)
    return dh, x, wg, wu


# ragged tiles of both products; more than two rounds of dx's tiles, and of dW's
@pytest.mark.parametrize("rows,width,ffn", [(300, 840, 200), (5200, 2056, 72), (70, 2056, 2600)])
@pytest.mark.parametrize("pair,columns", TILES)
def test_gradients_in_tiles(rows, width, ffn, pair, columns):
    dh, x, wg, wu = _grad_case(rows, width, ffn)
    status = _Status()
    _, z = _gated(status, _tile(0, 128), x, wg, wu, xb.ACT_SILU, keep=True)
    got = _grad(status, _tile(pair, columns), _tile(pair, columns), dh, x, wg, wu, z, xb.ACT_SILU)
    status.ok()
    for name, g, r, off in zip(("dx", "dw_gate", "dw_up"), got, *_grads_ref(dh, x, wg, wu, "silu")):
        _close_grad(g, r, off, (name, pair, columns))


@pytest.mark.parametrize("rows", [1, 16, 31, 64, 100, 129, 300, 1000])
def test_input_gradient_for_few_tokens(rows):
    dh, x, wg, wu = _grad_case(rows, 328, 392)
    status = _Status()
    _, z = _gated(status, _tile(0, 128), x, wg, wu, xb.ACT_GELU_TANH, keep=True)
    refs, offs = _grads_ref(dh, x, wg, wu, "gelu_tanh")
    for share in SHARES:
        for features in (64, 128):
            got = _grad(status, _few(share, features), _tile(0, 128), dh, x, wg, wu, z, xb.ACT_GELU_TANH)
            status.ok()
            _close_grad(got[0], refs[0], offs[0], (share, features))


def _lora(status, shape, x, w, la, lb, scale, adapter, bias, share_t=0):
    batch, rows, K = x.shape
    N, (n, rank) = w.shape[0], la.shape[:2]
    out = _nan(batch, rows, N)
    work = torch.zeros(xb.xema_lora_work_bytes(batch, rows, rank), dtype=torch.uint8, device=DEV)
    a = xb.xema_lora_args(x=x.data_ptr(), ldx=K, x_batch_rows=rows, w=w.data_ptr(), ldw=K, bias=bias.data_ptr(), lora_a=la.data_ptr(),
                          lora_b=lb.data_ptr(), scale=scale.data_ptr(), adapter=adapter.data_ptr(), work=work.data_ptr(), out=out.data_ptr(),
                          ldo=N, out_batch_rows=rows, batch=batch, rows=rows, N=N, K=K, rank=rank, n_adapters=n)
    xb.xema_op_lora_in(a, shape, share_t, status.word.data_ptr(), status.stream)
    return out


def _check_lora(batch, rows, K, N, rank, shapes):
    gen = _gen(batch, rows, K, N, rank, 42)
    case = _lora_case(gen, batch, rows, K, N, rank, 3)
    case[5][0] = 1
    want, status = _lora_ref(*case), _Status()
    for what, shape, share_t in shapes:
        got = _lora(status, shape, *case, share_t=share_t)
        status.ok()
        _close(got, want, (what, share_t), rms=T_ROUND)


# (K in eight blocks, so that two and four CTAs can share it)
@pytest.mark.parametrize("batch,rows,K,N,rank", [(3, 300, 456, 840, 24), (2, 2600, 456, 2056, 64), (5, 7, 456, 200, 128)])
@pytest.mark.parametrize("pair,columns", TILES)
def test_adapters_in_tiles(batch, rows, K, N, rank, pair, columns):
    _check_lora(batch, rows, K, N, rank, [((pair, columns), _tile(pair, columns), t) for t in (0,) + SHARES])


@pytest.mark.parametrize("batch,rows,rank", [(9, 1, 16), (5, 3, 64), (11, 16, 24), (7, 17, 8), (10, 30, 128), (4, 60, 40), (3, 127, 16), (2, 128, 72), (3, 129, 24), (2, 300, 16)])
def test_adapters_of_requests_side_by_side(batch, rows, rank):
    _check_lora(batch, rows, 456, 328, rank, [((s, r), _few(s, r), t) for s, t in zip(SHARES, (4, 1, 2)) for r in (8, 24, 64, 72, 128)])


@pytest.mark.parametrize("batch,rank", [(1, 8), (5, 16), (48, 24), (65, 64), (130, 128), (300, 16)])
def test_adapters_of_single_tokens(batch, rank):
    _check_lora(batch, 1, 456, 328, rank, [((s, r), _few(s, r, xb.FF_SINGLE), 0) for s in SHARES for r in (8, 24, 64, 72, 128)])


def test_shapes_that_are_refused():
    gen = _gen(43)
    x, wg, wu = _randn(gen, (40, 72)), _randn(gen, (136, 72)), _randn(gen, (136, 72))
    status = _Status()
    case = _lora_case(gen, 3, 5, 72, 136, 16, 2)
    many = _lora_case(gen, 1, 600, 72, 136, 16, 2)
    z = torch.zeros(3, 40, 136, dtype=torch.int16, device=DEV)
    # (four CTAs find no share of the two blocks along K, or of dx's six)
    for call in (lambda s: _gated(status, s, x, wg, wu, 0), lambda s: _lora(status, s, *case), lambda s: _grad(status, s, _tile(0, 128), x.new_zeros(40, 136), x, wg, wu, z, 0)):
        for shape in (_tile(0, 64), _tile(0, 256), _tile(1, 64), _tile(1, 288), _tile(1, 144), _few(3, 0), _few(4, 0), _few(8, 0), _few(0, 7), _few(0, 136), _few(0, -8),
                      xb.xema_ff_shape(), xb.xema_ff_shape(kernel=9)):
            with pytest.raises(xb.XemaError):
                call(shape)
    with pytest.raises(xb.XemaError):
        _gated(status, _tile(1, 160), x, wg, wu, 0)                                   # half of a gated tile is no whole step of the epilogue
    with pytest.raises(xb.XemaError):
        _gated(status, _few(1, 0), _randn(gen, (1025, 72)), wg, wu, 0)
    with pytest.raises(xb.XemaError):
        _lora(status, _few(1, 0, xb.FF_SINGLE), *case)                                # more than a row a request
    with pytest.raises(xb.XemaError):
        _lora(status, _few(1, 0), *many)
    with pytest.raises(xb.XemaError):
        _lora(status, _tile(0, 128), *many, share_t=3)
    status.ok()
