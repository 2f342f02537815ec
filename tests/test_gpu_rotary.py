"""Rotary positions and the append to the paged cache with the rotation on the way, against the formulas in 64 bits, through the C ABI."""
import math
from fractions import Fraction

import pytest
import torch

import layer_ref as ref
from rollout_ref import e2m1_values
from paper_2604_07853_amd import synth

pytestmark = pytest.mark.gpu

TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
# cosines and sines: the angle's conversion and product with 2 pi (1.5 roundings of at most pi / 4), the series' sums (1.5), the amplitude (1); the two products
# and their sum (2): at most 6.2 roundings of (|a| + |b|) times the amplitude, 2e-9 of the series beside them
TURN = 8 * ref.F32


@pytest.fixture(scope="module")
def q():
    from paper_2604_07853_amd import binding
    binding.lib()
    return binding


def angles(rope, positions):
    """Angles modulo a turn, from exact fractions."""
    f = [Fraction(x) / TWO_PI for x in rope.frequencies]
    return torch.tensor([[float((int(p) * x) % 1) * 2 * math.pi for x in f] for p in positions], dtype=torch.float64)


def turned(q, rope, positions, x, inverse=False):
    """(turned x, |a| + |b| times the amplitude) in float64; x [T, heads, D] on the CPU."""
    x, rot = x.double(), rope.rotary_dim
    angle = angles(rope, positions)[:, None]
    c, s = torch.cos(angle) * rope.amplitude, torch.sin(angle) * rope.amplitude * (-1 if inverse else 1)
    ia = torch.arange(rot // 2) * (2 if rope.layout == q.QARL_ROPE_PAIRS else 1)
    ib = ia + (1 if rope.layout == q.QARL_ROPE_PAIRS else rot // 2)
    a, b = x[..., ia], x[..., ib]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = size[..., ib] = (a.abs() + b.abs()) * rope.amplitude
    far = max([1] + [abs(int(p)) for p in positions])
    return y, size * (TURN + 2.5 * far * 2.0 ** -64 * 2 * math.pi)        # (the frequencies' 64 bits)


def close(got, want, err, dtype):
    got = got.double().cpu()
    return ((got - want).abs() <= err + (want.abs() + err) * (ref.F32 if dtype == torch.float32 else ref.HALF_BF16)).all()


def heads_of(T, heads, dim, dtype, seed, extra=0):
    return synth.normal_bf16((T, heads + extra, dim), 1.0, seed).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("T,heads,kv_heads,dim,rot", [(1, 1, 1, 16, 16), (1, 32, 4, 128, 128), (3, 5, 1, 80, 80), (37, 8, 8, 64, 32), (5, 3, 0, 192, 64), (130, 4, 2, 256, 256),
                                                      (9, 7, 1, 96, 48), (2, 1, 300, 64, 64), (4, 2, 1, 1024, 256)])
def test_rotary(q, dtype, layout, T, heads, kv_heads, dim, rot):
    rope = q.Rope(rot, base=10000.0, layout=layout)
    pos = torch.randint(0, 20000, (T,), generator=torch.Generator().manual_seed(T))
    pos[0] = 0
    x = heads_of(T, heads + kv_heads, dim, dtype, T + dim, 2)
    dev = x.cuda()
    k = dev[:, heads: heads + kv_heads] if kv_heads else None
    for inverse in (False, True):
        got = q.qarl_rotary(rope, pos.cuda(), dev[:, :heads], k, inverse=inverse)
        for name, lo, hi in (("q", 0, heads), ("k", heads, heads + kv_heads)):
            if hi == lo:
                assert got["k"] is None
                continue
            want, err = turned(q, rope, pos, x[:, lo:hi], inverse)
            assert close(got[name], want, err, dtype), (name, inverse)
            assert torch.equal(got[name][..., rot:].cpu(), x[:, lo:hi, rot:])       # what is not turned is passed on
    assert torch.equal(dev.cpu(), x)


@pytest.mark.parametrize("scaling,kw", [("LINEAR", dict(factor=4.0)), ("YARN", dict(factor=8.0, original_len=4096)), ("BANDS", dict(factor=8.0, original_len=8192, high=4.0))])
def test_scaled_frequencies_and_many_tokens(q, scaling, kw):
    rope = q.Rope(128, base=1e6, scaling=getattr(q, "QARL_ROPE_" + scaling), **kw)
    T = 9000                    # several tokens a workgroup, the last one not full
    x = heads_of(T, 3, 128, torch.bfloat16, 5)
    pos = torch.arange(T) * 29
    got = q.qarl_rotary(rope, pos.cuda(), x.cuda()[:, :2], x.cuda()[:, 2:])
    rows = torch.tensor([0, 1, 7, 8, 4095, 8999])
    for name, lo, hi in (("q", 0, 2), ("k", 2, 3)):
        want, err = turned(q, rope, pos[rows], x[rows, lo:hi])
        assert close(got[name][rows.cuda()], want, err, torch.bfloat16)


def test_far_and_negative_positions(q):
    """Positions at which a product in 32 (from about 2^40 on in 64) bits says nothing about the angle."""
    rope = q.Rope(64, base=500000.0)
    pos = torch.tensor([131071, 1 << 20, (1 << 31) + 7, -5, -(1 << 33) - 1, (1 << 40) + 3, 1 << 45])
    x = heads_of(7, 2, 64, torch.float32, 3)
    got = q.qarl_rotary(rope, pos.cuda(), x.cuda())["q"]
    for i in range(7):
        want, err = turned(q, rope, pos[i: i + 1], x[i: i + 1])
        assert close(got[i: i + 1], want, err, torch.float32), int(pos[i])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place_and_strides(q, dtype):
    rope = q.Rope(32, layout=q.QARL_ROPE_PAIRS)
    pos = torch.tensor([3, 1, 4, 1, 5], device="cuda")
    x = heads_of(5, 6, 64, dtype, 9).cuda()
    want = q.qarl_rotary(rope, pos, x[:, :4].contiguous(), x[:, 4:].contiguous())
    y = x.clone()
    got = q.qarl_rotary(rope, pos, y[:, :4], y[:, 4:], q_out=y[:, :4], k_out=y[:, 4:])
    assert got["q"].data_ptr() == y.data_ptr() and torch.equal(y[:, :4], want["q"]) and torch.equal(y[:, 4:], want["k"])
    # heads outermost, as attention by batched products keeps them
    t = x.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty((6, 5, 64), dtype=dtype, device="cuda").transpose(0, 1)
    assert torch.equal(q.qarl_rotary(rope, pos, t, q_out=out)["q"], q.qarl_rotary(rope, pos, x)["q"])
    # a single token or head at any stride
    odd = torch.zeros((3, 64 * 4 + 1), dtype=dtype, device="cuda")
    odd[0, :256] = x[0, :4].reshape(-1)
    assert torch.equal(q.qarl_rotary(rope, pos[:1], odd.as_strided((1, 4, 64), (257, 64, 1)))["q"], want["q"][:1])


def test_no_tokens(q):
    rope = q.Rope(64)
    x = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    none = torch.zeros((0,), dtype=torch.int64, device="cuda")
    assert q.qarl_rotary(rope, none, x, x)["k"].shape == (0, 4, 64)
    c = q.KVCache.empty(q.QARL_KV_E2M1, 2, 16, 4, 64)
    assert q.qarl_rotary_kv_write(c, rope, none, x, x, x, none).shape == (0, 4, 64)


@pytest.mark.parametrize("layout", [0, 1])
def test_the_inverse_is_the_gradient(q, layout):
    """Of sum(w y): against differences (y is linear: steps of 1 and the two evaluations' roundings), and as the transpose, <y(x), w> = <x, g(w)>."""
    rope = q.Rope(32, layout=layout, scaling=q.QARL_ROPE_YARN, factor=8.0, original_len=64)
    pos = torch.tensor([0, 100, 70000], device="cuda")
    x, w = (heads_of(3, 2, 48, torch.float32, s).cuda() for s in (1, 2))
    g = q.qarl_rotary(rope, pos, w, inverse=True)["q"].double()
    y0 = q.qarl_rotary(rope, pos, x)["q"].double()
    left, right = (y0 * w.double()), (x.double() * g)
    size = rope.amplitude * 2 * (x.double().abs().amax() * w.double().abs().amax())
    assert abs(left.sum() - right.sum()) <= x.numel() * size * 2 * TURN
    for d in range(0, 48, 5):
        step = x.clone()
        step[..., d] += 1.0
        y1 = q.qarl_rotary(rope, pos, step)["q"].double()
        slope = ((y1 - y0) * w.double()).sum(-1)
        # w meets two elements of y that changed; each evaluation is off by TURN (|a| + |b|), steps by a rounding of x
        bound = 2 * w.double().abs().amax(-1) * 2 * TURN * (2 * step.double().abs().amax(-1) * rope.amplitude + 1)
        assert ((slope - g[..., d]).abs() <= 3 * bound).all(), d


# ---- the append ----

FMT = {"bf16": "QARL_KV_BF16", "fp8": "QARL_KV_E4M3", "fp4": "QARL_KV_E2M1"}


def read_back(q, c, slots):
    """(k, v, their errors' scale) of the tokens at `slots`, in float64 [T, heads, dim]"""
    got = []
    for store, scales in ((c.k, c.k_scales), (c.v, c.v_scales)):
        rows, s = [], []
        for sl in slots.tolist():
            page, off = sl // c.page_size, sl % c.page_size
            row = store[page, :, off].cpu()
            if c.fmt == q.QARL_KV_E4M3:
                sc = scales[page, :, off].cpu().double()[:, None]
                row = ref.e4m3_values(row) * sc
            elif c.fmt == q.QARL_KV_E2M1:
                row, sc = e2m1_values(row, scales[page, :, off].cpu())
            else:
                row, sc = row.double(), torch.zeros((1, 1))
            rows.append(row)
            s.append(sc.expand(row.shape))
        got += [torch.stack(rows), torch.stack(s)]
    return got


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("T,heads,kv_heads,dim,rot,layout,page", [(1, 32, 4, 128, 128, 0, 16), (7, 3, 1, 64, 64, 0, 8), (40, 6, 2, 128, 80, 0, 32), (33, 5, 5, 64, 48, 1, 16),
                                                                  (300, 8, 2, 128, 128, 1, 64), (2, 0, 17, 64, 16, 0, 8), (9000, 1, 1, 64, 64, 0, 128)])
def test_append(q, fmt, T, heads, kv_heads, dim, rot, layout, page):
    rope = q.Rope(rot, layout=layout, scaling=q.QARL_ROPE_YARN, factor=4.0, original_len=2048)
    g = torch.Generator().manual_seed(T + dim)
    pages = -(-T // page) + 3
    slots = torch.randperm(pages * page, generator=g)[:T]
    gone = torch.zeros(T, dtype=torch.bool)
    if T > 3:
        gone[torch.tensor([1, 2, 3])] = True
        slots[1], slots[2], slots[3] = -1, pages * page, -(1 << 40)
    pos = torch.randint(0, 100000, (T,), generator=g)
    x = heads_of(T, heads + 2 * kv_heads, dim, torch.bfloat16, T + 1, 1)
    x[0, heads] = 0
    c = q.KVCache.empty(getattr(q, FMT[fmt]), pages, page, kv_heads, dim)
    for t in (c.k, c.v, c.k_scales, c.v_scales):
        if t is not None:
            t.view(torch.uint8).fill_(0x5a)
    dev = x.cuda()
    query = dev[:, :heads] if heads else None
    out = q.qarl_rotary_kv_write(c, rope, pos.cuda(), query, dev[:, heads: heads + kv_heads], dev[:, heads + kv_heads: heads + 2 * kv_heads], slots.cuda())
    pick = torch.arange(T) if T < 500 else torch.tensor([0, 5, 8, 1000, T - 2, T - 1])
    if heads:       # the queries: what qarl_rotary makes of them, bit for bit
        assert torch.equal(out, q.qarl_rotary(rope, pos.cuda(), query)["q"])
    live = pick[~gone[pick]]
    k, ks, v, vs = read_back(q, c, slots[live])
    want, err = turned(q, rope, pos[live], x[live, heads: heads + kv_heads])
    half = {"bf16": ref.HALF_BF16, "fp8": ref.HALF_E4M3 * (1 + 4 * ref.F32), "fp4": 0.0}[fmt]
    for got, scale, src, e in ((k, ks, want, err), (v, vs, x[live, heads + kv_heads: heads + 2 * kv_heads].double(), torch.zeros_like(want))):
        # e4m3: half a step, subnormals half of theirs; e2m1: half a step is 1/4 of the scale up to 2, 1/2 up to 4, 1 up to 6
        a = src.abs() + e
        low = {"bf16": 0.0 * a, "fp8": scale * ref.SUB_E4M3, "fp4": torch.where(a < 2 * scale, 0.25 * scale, torch.where(a < 4 * scale, 0.5 * scale, scale))}[fmt]
        assert ((got - src).abs() <= a * half + low * (1 + 1e-6) + e).all()
        if fmt == "fp4":    # the scale: the smallest power of two whose sixfold reaches the quarter's largest
            top = a.view(*a.shape[:-1], 4, -1).amax(-1)
            sc = scale.view(*a.shape[:-1], 4, -1)[..., 0]
            assert (top <= 6 * sc * (1 + 1e-6)).all() and ((top >= 3 * sc * (1 - 1e-6)) | (sc == 2.0 ** -100)).all()
        if fmt == "fp8":
            assert ((scale[..., 0] * 448 - src.abs().amax(-1)).abs() <= err.amax(-1) + src.abs().amax(-1) * 4 * ref.F32).all()
    # bf16: the same bytes as the two calls; every format: values as the plain write leaves them, and nothing beside the slots
    other = q.KVCache.empty(getattr(q, FMT[fmt]), pages, page, kv_heads, dim)
    for t in (other.k, other.v, other.k_scales, other.v_scales):
        if t is not None:
            t.view(torch.uint8).fill_(0x5a)
    rk = q.qarl_rotary(rope, pos.cuda(), dev[:, heads: heads + kv_heads])["q"]
    q.qarl_kv_cache_write(other, rk, dev[:, heads + kv_heads: heads + 2 * kv_heads], slots.cuda())
    assert torch.equal(c.v.view(torch.uint8), other.v.view(torch.uint8))
    if fmt == "bf16":
        assert torch.equal(c.k.view(torch.uint8), other.k.view(torch.uint8))
    else:
        assert torch.equal(c.v_scales.view(torch.uint8), other.v_scales.view(torch.uint8))
    untouched = torch.ones((pages, page), dtype=torch.bool)
    untouched.view(-1)[slots[~gone]] = False
    for t in (c.k, c.k_scales):
        if t is not None:
            b = t.view(torch.uint8).cpu().view(pages, kv_heads, page, -1).permute(0, 2, 1, 3)
            assert (b[untouched] == 0x5a).all()


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_append_of_infinities_and_nan(q, fmt):
    """A quarter (e4m3: a row) with one reads as NaN, its neighbours as they are.  Through the rotation an infinity reaches its partner too."""
    rope = q.Rope(64, layout=q.QARL_ROPE_PAIRS)
    k = heads_of(4, 2, 64, torch.bfloat16, 1)
    v = heads_of(4, 2, 64, torch.bfloat16, 2)
    k[1, 0, 5] = math.inf
    v[2, 1, 40] = math.nan
    c = q.KVCache.empty(getattr(q, FMT[fmt]), 1, 16, 2, 64)
    slots = torch.arange(4, device="cuda")
    q.qarl_rotary_kv_write(c, rope, slots + 10, None, k.cuda(), v.cuda(), slots)
    rk, rv = q.qarl_kv_cache_read(c, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda"), 4)
    for got, t, h, d in ((rk, 1, 0, 5), (rv, 2, 1, 40)):
        bad = torch.zeros((4, 2, 64), dtype=torch.bool)
        bad[t, h, (slice(None) if fmt == "fp8" else slice(d // 16 * 16, d // 16 * 16 + 16))] = True
        assert torch.equal(got.isnan().cpu(), bad)


def test_on_another_stream_and_in_a_graph(q):
    rope = q.Rope(128)
    pos, slots = torch.tensor([7, 9000], device="cuda"), torch.tensor([3, 17], device="cuda")
    x = heads_of(2, 8, 128, torch.bfloat16, 4).cuda()
    caches = [q.KVCache.empty(q.QARL_KV_E2M1, 2, 16, 2, 128) for _ in range(2)]
    for c in caches:
        for t in (c.k, c.v, c.k_scales, c.v_scales):
            t.zero_()
    out, grad = torch.empty((2, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda")

    def step(c, out, grad):
        q.qarl_rotary_kv_write(c, rope, pos, x[:, :4], x[:, 4:6], x[:, 6:], slots, q_out=out)
        q.qarl_rotary(rope, pos, x, inverse=True, q_out=grad)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(caches[0], out, grad)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], out, grad)
    for seed in range(3):
        x.copy_(heads_of(2, 8, 128, torch.bfloat16, 40 + seed))
        pos.add_(11)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(out), torch.empty_like(grad)
        step(caches[1], *want)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(grad, want[1])
        for n in ("k", "v", "k_scales", "v_scales"):
            assert torch.equal(getattr(caches[0], n), getattr(caches[1], n))


def test_offsets_past_32_bits(q):
    """The last page of a 4-bit cache of more than 2^32 bytes per half."""
    page, heads, dim = 1024, 8, 128
    pages = (1 << 32) // (page * heads * dim // 2) + 9
    c = q.KVCache(q.QARL_KV_E2M1, *[torch.zeros((pages, heads, page, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2)],
                  *[torch.zeros((pages, heads, page, 4), dtype=torch.uint8, device="cuda") for _ in range(2)])
    small = q.KVCache.empty(q.QARL_KV_E2M1, 1, page, heads, dim)
    for t in (small.k, small.v, small.k_scales, small.v_scales):
        t.zero_()
    rope, x = q.Rope(128), heads_of(3, 16, dim, torch.bfloat16, 6).cuda()
    slots = torch.tensor([pages * page - 3, pages * page - 2, pages * page - 1], device="cuda")
    for cache, at in ((c, slots), (small, slots - (pages - 1) * page)):
        q.qarl_rotary_kv_write(cache, rope, torch.arange(3, device="cuda"), None, x[:, :heads], x[:, heads:], at)
    assert not c.k[:4].any() and torch.equal(c.k[-1], small.k[0]) and torch.equal(c.v_scales[-1], small.v_scales[0]) and c.k[-1].any()


def random_heads(T, heads, dim, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((T, heads, dim), generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout,inverse", [(0, False), (1, True)])
def test_large_calls_equal_small_ones(q, dtype, layout, inverse):
    """Calls that move more than 64 MB pass the caches: the bits of the same tokens in smaller calls."""
    T, step, heads, dim = (9001, 1500, 24, 128) if dtype == torch.bfloat16 else (5001, 1000, 24, 128)
    rope = q.Rope(96, base=1e6, layout=layout)
    x, pos = random_heads(T, heads + 1, dim, dtype, 3), torch.arange(T, device="cuda") * 7 + 100
    whole = q.qarl_rotary(rope, pos, x[:, :20], x[:, 20:24], inverse=inverse)
    for lo in range(0, T, step):
        part = q.qarl_rotary(rope, pos[lo: lo + step], x[lo: lo + step, :20], x[lo: lo + step, 20:24], inverse=inverse)
        assert all(torch.equal(whole[n][lo: lo + step], part[n]) for n in whole), lo
    y = x.clone()
    q.qarl_rotary(rope, pos, y[:, :20], y[:, 20:24], inverse=inverse, q_out=y[:, :20], k_out=y[:, 20:24])
    assert torch.equal(y[:, :20], whole["q"]) and torch.equal(y[:, 20:24], whole["k"]) and torch.equal(y[:, 24], x[:, 24])


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("T,step,dim,layout", [(9001, 3000, 128, 0), (18001, 6000, 64, 1)])
def test_large_appends_equal_small_ones(q, fmt, T, step, dim, layout):
    heads, kv_heads, page = 16, 4, 16
    rope = q.Rope(dim, base=1e6, layout=layout)
    x, pos = random_heads(T, heads + 2 * kv_heads, dim, torch.bfloat16, 4), torch.arange(T, device="cuda") * 3
    pages = T // page + 5
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(T))[:T].cuda()
    slots[::1000] = -1
    caches, outs = [], []
    for size in (T, step):
        c = q.KVCache.empty(getattr(q, FMT[fmt]), pages, page, kv_heads, dim)
        for t in (c.k, c.v, c.k_scales, c.v_scales):
            if t is not None:
                t.view(torch.uint8).fill_(0x5a)
        outs.append(torch.cat([q.qarl_rotary_kv_write(c, rope, pos[lo: lo + size], x[lo: lo + size, :heads], x[lo: lo + size, heads: heads + kv_heads],
                                                      x[lo: lo + size, heads + kv_heads:], slots[lo: lo + size]) for lo in range(0, T, size)]))
        caches.append(c)
    assert torch.equal(*outs)
    for n in ("k", "v", "k_scales", "v_scales"):
        a, b = (getattr(c, n) for c in caches)
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)), n
