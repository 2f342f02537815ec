"""Add + RMS norm and its backward against the 64-bit formulas, through the C ABI."""
import math

import pytest
import torch

import layer_ref as ref
from paper_2604_07853_amd import synth

pytestmark = pytest.mark.gpu

EPS = 1e-6
# fp32: a lane adds up to 64 squares, the row's lanes meet in 8 more steps, then a division, a root, a reciprocal and two
# products: fewer than 100 roundings of 2^-24 each
SLACK = 100 * ref.F32
ROWS_K = [(1, 8), (3, 64), (5, 120), (7, 128), (33, 136), (4, 504), (1, 512), (9, 520), (2, 768), (1, 2048), (130, 2048), (17, 2056), (3, 4096),
          (5, 4104), (2, 8192), (3, 8200), (2, 16384), (1031, 1024), (1100, 4096), (600, 8192)]


@pytest.fixture(scope="module")
def q():
    from paper_2604_07853_amd import binding
    binding.lib()
    return binding


def _padded(t, pad, lead=0):
    wide = torch.full((t.shape[0], t.shape[1] + pad + lead), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, lead: lead + t.shape[1]] = t
    return wide[:, lead: lead + t.shape[1]]


def _case(rows, K, stream, seed):
    x = synth.normal_bf16((rows, K), 0.7, seed)
    g = torch.Generator().manual_seed(seed + 1)
    r = torch.randn((rows, K), generator=g) * torch.exp(torch.randn((rows, 1), generator=g))
    w = synth.normal_bf16((K,), 0.2, seed + 2, mean=1.0)
    return x, None if stream is None else r.to(stream), w


def _check_y(y, want):
    assert ((y.double().cpu() - want).abs() <= want.abs() * (ref.HALF_BF16 + SLACK)).all()


@pytest.mark.parametrize("stream", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,K", ROWS_K)
def test_forward(q, rows, K, stream):
    x, r, w = _case(rows, K, stream, rows * 31 + K)
    want, h = ref.rmsnorm(x, r, w, EPS)
    rd = None if r is None else r.cuda()
    got = q.qarl_add_rmsnorm(x.cuda(), w.cuda(), EPS, residual=rd, quantize=True, y=torch.empty((rows, K), dtype=torch.bfloat16, device="cuda"))
    _check_y(got["y"], want)
    if r is not None:
        half = ref.HALF_BF16 if stream == torch.bfloat16 else ref.F32
        assert got["residual"].dtype == stream
        assert ((got["residual"].double().cpu() - h).abs() <= h.abs() * (half + 2 * ref.F32)).all()
    scale = got["scales"].double().cpu()
    top = want.abs().amax(1) / 448
    assert ((scale - top).abs() <= top * SLACK).all()
    deq = ref.e4m3_values(got["codes"].cpu()) * scale[:, None]
    assert ((deq - want).abs() <= want.abs() * (ref.HALF_E4M3 + 2 * SLACK) + scale[:, None] * ref.SUB_E4M3).all()
    # by way of bf16: the bytes that the row quantizer makes of y, and that the routed GEMM makes of it inside
    via = q.qarl_add_rmsnorm(x.cuda(), w.cuda(), EPS, residual=rd, quantize=True, via_bf16=True)
    codes, scales = q.qarl_quantize_rows_fp8(got["y"])
    assert torch.equal(via["codes"], codes) and torch.equal(via["scales"], scales)


@pytest.mark.parametrize("K", [128, 520, 2048, 4104])
def test_strided_rows_and_in_place(q, K):
    rows = 6
    x, r, w = _case(rows, K, torch.bfloat16, K)
    want, h = ref.rmsnorm(x, r, w, EPS)
    plain = q.qarl_add_rmsnorm(x.cuda(), w.cuda(), EPS, residual=r.cuda())
    xs, rs = _padded(x, 24, 8), _padded(r, 40)
    ys, os_ = _padded(torch.zeros_like(x), 16), _padded(torch.zeros_like(x), 72, 16)
    got = q.qarl_add_rmsnorm(xs, w.cuda(), EPS, residual=rs, residual_out=os_, y=ys)
    assert torch.equal(got["y"], plain["y"]) and torch.equal(got["residual"], plain["residual"])
    for t, lead in ((ys, 0), (os_, 16)):      # nothing outside the rows is written
        base = t._base
        keep = torch.ones(base.shape, dtype=torch.bool, device="cuda")
        keep[:, lead: lead + K] = False
        assert base[keep].isnan().all()
    got = q.qarl_add_rmsnorm(xs, w.cuda(), EPS, residual=rs, residual_out=rs, y=xs)
    assert torch.equal(xs, plain["y"]) and torch.equal(rs, plain["residual"])


@pytest.mark.parametrize("K", [128, 2048, 4104])
def test_zero_infinite_and_nan_rows(q, K):
    x, _, w = _case(5, K, None, 3)
    x[1] = 0
    x[2, K // 2] = float("inf")
    x[3, 5] = float("nan")
    got = q.qarl_add_rmsnorm(x.cuda(), w.cuda(), EPS, quantize=True, y=torch.empty_like(x, device="cuda"))
    y, s, c = got["y"].cpu(), got["scales"].cpu(), got["codes"].cpu()
    assert (y[1] == 0).all() and s[1] == 0 and ((c[1] & 127) == 0).all()
    assert y[2, K // 2].isnan() and y[3].isnan().all()
    assert s[2].isnan() and s[3].isnan() and ((c[2:4] & 127) == 127).all()
    for row in (0, 4):
        want, _ = ref.rmsnorm(x[row: row + 1], None, w, EPS)
        _check_y(y[row: row + 1], want)


@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,K", ROWS_K)
@pytest.mark.parametrize("with_dh", [True, False])
def test_backward(q, rows, K, stream, with_dh):
    dy = synth.normal_bf16((rows, K), 1e-2, 5)
    _, h, w = _case(rows, K, stream, 7)
    dh = torch.randn((rows, K), generator=torch.Generator().manual_seed(8)).mul(1e-2).to(stream) if with_dh else None
    dx, dw, size, dwsize = ref.rmsnorm_backward(dy, h, w, EPS, dh)
    half = ref.HALF_BF16 if stream == torch.bfloat16 else ref.F32
    got = q.qarl_add_rmsnorm_backward(_padded(dy, 8), _padded(h, 16), w.cuda(), EPS, dh=None if dh is None else _padded(dh, 24))
    assert ((got["dx"].double().cpu() - dx).abs() <= dx.abs() * half + size * 2 * SLACK).all()
    # dw: a lane adds at most rows / 4 rows, the partial sums meet in at most 16 + 9 steps
    chain = (rows + 100) * ref.F32
    assert ((got["dw"].double().cpu() - dw).abs() <= dwsize * (chain + SLACK)).all()
    short = q.qarl_add_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), EPS, dh=None if dh is None else dh.cuda(), dw_dtype=q.QARL_OUT_BF16)
    assert torch.equal(short["dx"], got["dx"])
    assert torch.equal(short["dw"], got["dw"].to(torch.bfloat16))
    again = q.qarl_add_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), EPS, dh=None if dh is None else dh.cuda())
    assert torch.equal(again["dw"], got["dw"])                           # the order of the sums is fixed


def test_backward_many_rows_and_no_rows(q):
    rows, K = 5003, 256
    dy, (_, h, w) = synth.normal_bf16((rows, K), 1e-2, 5), _case(rows, K, torch.bfloat16, 7)
    dx, dw, size, dwsize = ref.rmsnorm_backward(dy, h, w, EPS, None)
    hd = h.cuda()
    got = q.qarl_add_rmsnorm_backward(dy.cuda(), hd, w.cuda(), EPS, dx=hd)     # in place
    assert ((got["dx"].double().cpu() - dx).abs() <= dx.abs() * ref.HALF_BF16 + size * 2 * SLACK).all()
    assert ((got["dw"].double().cpu() - dw).abs() <= dwsize * ((rows + 100) * ref.F32 + SLACK)).all()
    none = torch.zeros((0, K), dtype=torch.bfloat16, device="cuda")
    dw0 = torch.ones((K,), dtype=torch.float32, device="cuda")
    assert (q.qarl_add_rmsnorm_backward(none, none, w.cuda(), EPS, dw=dw0)["dw"] == 0).all()
    assert q.qarl_add_rmsnorm(none, w.cuda(), EPS)["y"].shape == (0, K)
    assert q.qarl_add_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), EPS, want_dw=False)["dw"] is None


def test_gradient_against_differences(q):
    """d/de of sum(dy * y(h + e u)) + sum(dh * (h + e u)), by central differences in 64 bits, against the kernel's <dx, u>."""
    rows, K, e = 9, 768, 1e-5
    dy, (_, h, w) = synth.normal_bf16((rows, K), 1.0, 5), _case(rows, K, torch.float32, 7)
    dh = torch.randn((rows, K), generator=torch.Generator().manual_seed(8))
    got = q.qarl_add_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), EPS, dh=dh.cuda())

    def loss(hh, ww):
        y = hh / torch.sqrt((hh * hh).mean(1, keepdim=True) + EPS) * ww
        return float((dy.double() * y).sum() + (dh.double() * hh).sum())

    for seed in range(4):
        u = torch.randn((rows, K), generator=torch.Generator().manual_seed(20 + seed), dtype=torch.float64)
        d = (loss(h.double() + e * u, w.double()) - loss(h.double() - e * u, w.double())) / (2 * e)
        dx = got["dx"].double().cpu()
        assert abs(float((dx * u).sum()) - d) <= 1e-6 * float((dx * u).abs().sum())      # differences: e^2 and 1e-16 / e
        z = torch.randn((K,), generator=torch.Generator().manual_seed(30 + seed), dtype=torch.float64)
        d = (loss(h.double(), w.double() + e * z) - loss(h.double(), w.double() - e * z)) / (2 * e)
        dw = got["dw"].double().cpu()
        assert abs(float((dw * z).sum()) - d) <= 1e-5 * float((dw * z).abs().sum())
    assert math.isfinite(d)


def test_graph_replays(q):
    rows, K = 300, 2048
    x, r, w = _case(rows, K, torch.bfloat16, 11)
    x, r, w = x.cuda(), r.cuda(), w.cuda()
    ro, y = torch.empty_like(r), torch.empty_like(x)
    codes, scales = torch.empty((rows, K), dtype=torch.uint8, device="cuda"), torch.empty((rows,), dtype=torch.float32, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty((K,), dtype=torch.float32, device="cuda")
    ws = torch.empty((q.qarl_add_rmsnorm_backward_workspace_bytes(rows, K),), dtype=torch.uint8, device="cuda")

    def step():
        q.qarl_add_rmsnorm(x, w, EPS, residual=r, residual_out=ro, y=y, codes=codes, scales=scales)
        q.qarl_add_rmsnorm_backward(y, ro, w, EPS, dx=dx, dw=dw, ws=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        x.copy_(synth.normal_bf16((rows, K), 1.0, 40 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (ro, y, codes, scales, dx, dw)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (ro, y, codes, scales, dx, dw)))
