"""What the norm, the cache and attention refuse, on the host before any launch (no GPU needed), and the 64-bit references of their tests."""
import ctypes

import pytest
import torch

import layer_ref as ref

P = 4096            # an aligned address that no refused call looks at


@pytest.fixture(scope="module")
def q():
    import os
    from paper_2604_07853_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


def _refused(q, status, word, fn, args):
    got = fn(*args.values())
    assert got == status, (got, q.lib().qarl_last_error())
    assert word in q.lib().qarl_last_error().decode()


def _norm(**kw):
    a = dict(x=P, xs=256, r=P, rs=256, w=P, rows=3, K=256, eps=1e-6, sd=0, ro=P, ros=256, y=P, ys=256, codes=P, scales=P, via=0, stream=None)
    a.update(kw)
    return a


def test_norm(q):
    fn = q.lib().qarl_add_rmsnorm
    inv, uns, ali = q.QARL_ERR_INVALID_ARG, q.QARL_ERR_UNSUPPORTED, q.QARL_ERR_ALIGNMENT
    for status, word, kw in [(inv, "rows", dict(rows=-1)), (inv, "K > 0", dict(K=0)), (inv, "eps", dict(eps=-1.0)), (inv, "eps", dict(eps=float("nan"))),
                             (inv, "eps", dict(eps=float("inf"))), (uns, "K % 8", dict(K=252)), (uns, "16384", dict(K=16392)), (inv, "stream_dtype", dict(sd=2)),
                             (inv, "null", dict(x=None)), (inv, "null", dict(w=None)), (inv, "no output", dict(y=None, codes=None, scales=None, ro=None)),
                             (inv, "together", dict(scales=None)), (inv, "together", dict(codes=None)), (inv, "overlap", dict(xs=248)), (inv, "overlap", dict(ys=0)),
                             (ali, "residual ", dict(rs=260)), (ali, "residual_out", dict(ro=P + 8)), (ali, "x must", dict(x=P + 2)), (ali, "codes", dict(codes=P + 4)),
                             (ali, "weight", dict(w=P + 8))]:
        _refused(q, status, word, fn, _norm(**kw))
    assert fn(*_norm(rows=0, x=None).values()) == q.QARL_OK


def test_norm_backward(q):
    fn = q.lib().qarl_add_rmsnorm_backward

    def args(**kw):
        a = dict(dy=P, dys=256, h=P, hs=256, dh=None, dhs=0, w=P, rows=3, K=256, eps=1e-6, sd=0, dx=P, dxs=256, dw=P, dwd=1, ws=P, wsb=1 << 30, stream=None)
        a.update(kw)
        return a

    inv, uns, ali = q.QARL_ERR_INVALID_ARG, q.QARL_ERR_UNSUPPORTED, q.QARL_ERR_ALIGNMENT
    for status, word, kw in [(inv, "rows", dict(rows=-1)), (uns, "K % 8", dict(K=12)), (inv, "dw_dtype", dict(dwd=5)), (inv, "null", dict(dy=None)),
                             (inv, "null", dict(dx=None)), (ali, "dw", dict(dw=P + 2)), (inv, "overlap", dict(dh=P, dhs=8)), (ali, "dh", dict(dh=P, dhs=257)),
                             (q.QARL_ERR_WORKSPACE, "workspace", dict(ws=None)), (q.QARL_ERR_WORKSPACE, "workspace", dict(wsb=8)),
                             (q.QARL_ERR_WORKSPACE, "workspace", dict(ws=P + 8))]:
        _refused(q, status, word, fn, args(**kw))
    assert q.qarl_add_rmsnorm_backward_workspace_bytes(0, 256) == 0 and q.qarl_add_rmsnorm_backward_workspace_bytes(3, 256) >= 1024


def _cache(q, **kw):
    a = dict(fmt=q.QARL_KV_E4M3, num_pages=10, page_size=16, kv_heads=2, head_dim=64, k=P, v=P, k_scales=P, v_scales=P)
    a.update(kw)
    return ctypes.byref(q.qarl_kv_cache(**a))


def test_cache_descriptor(q):
    inv, uns, ali = q.QARL_ERR_INVALID_ARG, q.QARL_ERR_UNSUPPORTED, q.QARL_ERR_ALIGNMENT
    bad = [(uns, "format", dict(fmt=7)), (inv, "positive", dict(num_pages=0)), (inv, "positive", dict(page_size=-16)), (uns, "page_size", dict(page_size=24)),
           (uns, "page_size", dict(page_size=4)), (uns, "page_size", dict(page_size=2048)), (uns, "head_dim", dict(head_dim=96)), (uns, "kv_heads", dict(kv_heads=2000)),
           (inv, "null cache", dict(k=None)), (inv, "null cache", dict(v_scales=None)), (ali, "16-byte", dict(v=P + 8)), (ali, "16-byte", dict(k_scales=P + 4))]
    for status, word, kw in bad:
        c = _cache(q, **kw)
        _refused(q, status, word, q.lib().qarl_kv_cache_write, dict(c=c, k=P, kt=128, kh=64, v=P, vt=128, vh=64, T=1, slots=P, s=None))
        _refused(q, status, word, q.lib().qarl_kv_cache_read, dict(c=c, t=P, ts=4, tw=4, o=P, S=1, total=5, ko=P, vo=P, s=None))
        _refused(q, status, word, q.lib().qarl_paged_attention, _attention(q, c=c))
    _refused(q, inv, "descriptor", q.lib().qarl_kv_cache_write, dict(c=None, k=P, kt=128, kh=64, v=P, vt=128, vh=64, T=1, slots=P, s=None))
    sizes = (10, 16, 2, 64)
    assert q.lib().qarl_kv_cache_bytes(q.QARL_KV_E4M3, *sizes) == 20480 and q.lib().qarl_kv_cache_bytes(q.QARL_KV_BF16, *sizes) == 40960
    assert q.lib().qarl_kv_scales_bytes(q.QARL_KV_E4M3, *sizes) == 1280 and q.lib().qarl_kv_scales_bytes(q.QARL_KV_BF16, *sizes) == 0
    assert q.lib().qarl_kv_cache_bytes(9, *sizes) == 0 and q.lib().qarl_kv_cache_bytes(q.QARL_KV_BF16, -1, 16, 2, 64) == 0


def test_cache_write_and_read(q):
    inv, ali = q.QARL_ERR_INVALID_ARG, q.QARL_ERR_ALIGNMENT
    w = dict(c=_cache(q), k=P, kt=128, kh=64, v=P, vt=128, vh=64, T=1, slots=P, s=None)
    for status, word, kw in [(inv, "T >= 0", dict(T=-1)), (inv, "null", dict(k=None)), (inv, "null", dict(slots=None)), (ali, "strides", dict(kt=132)),
                             (ali, "strides", dict(vh=4)), (ali, "aligned", dict(v=P + 8)), (ali, "aligned", dict(slots=P + 4))]:
        _refused(q, status, word, q.lib().qarl_kv_cache_write, dict(w, **kw))
    assert q.lib().qarl_kv_cache_write(*dict(w, T=0, k=None).values()) == q.QARL_OK
    r = dict(c=_cache(q), t=P, ts=4, tw=4, o=P, S=2, total=5, ko=P, vo=P, s=None)
    for status, word, kw in [(inv, "negative", dict(S=-1)), (inv, "negative", dict(total=-1)), (inv, "null", dict(o=None)), (inv, "null", dict(t=None)),
                             (inv, "overlap", dict(ts=3)), (inv, "null output", dict(vo=None)), (ali, "aligned", dict(ko=P + 8)), (ali, "aligned", dict(t=P + 1))]:
        _refused(q, status, word, q.lib().qarl_kv_cache_read, dict(r, **kw))
    assert q.lib().qarl_kv_cache_read(*dict(r, total=0, ko=None).values()) == q.QARL_OK


def _attention(lib_q, **kw):
    a = dict(q=P, qt=256, qh=64, T=5, heads=4, c=_cache(lib_q), t=P, ts=4, tw=4, kv=P, qo=P, S=2, mq=4, mkv=60, scale=0.1, window=0, out=P, od=0, lse=P, ws=P,
             wsb=1 << 30, stream=None)
    a.update(kw)
    return a


def test_attention(q):
    fn = q.lib().qarl_paged_attention
    inv, uns, ali = q.QARL_ERR_INVALID_ARG, q.QARL_ERR_UNSUPPORTED, q.QARL_ERR_ALIGNMENT
    for status, word, kw in [(inv, "out_dtype", dict(od=3)), (inv, "negative", dict(T=-1)), (inv, "negative", dict(S=-2)), (inv, "negative", dict(window=-1)),
                             (inv, "negative", dict(mkv=-1)), (inv, "positive", dict(heads=0)), (inv, "finite", dict(scale=float("nan"))),
                             (inv, "finite", dict(scale=float("inf"))), (uns, "multiple", dict(heads=5)), (uns, "1024", dict(heads=2048)), (inv, "null", dict(q=None)),
                             (inv, "null", dict(out=None)), (inv, "null", dict(kv=None)), (inv, "null", dict(t=None)), (inv, "max_q_len", dict(mq=0)),
                             (inv, "overlap", dict(ts=2)), (ali, "aligned", dict(q=P + 8)), (ali, "strides", dict(qt=260)), (ali, "aligned", dict(lse=P + 2)),
                             (ali, "aligned", dict(out=P + 4))]:
        _refused(q, status, word, fn, _attention(q, **kw))
    need = q.lib().qarl_paged_attention_workspace_bytes(_cache(q), 3, 4, 3, 1, 20000)
    if need:
        _refused(q, q.QARL_ERR_WORKSPACE, "workspace", fn, _attention(q, T=3, S=3, mq=1, mkv=20000, wsb=need - 1))
        _refused(q, q.QARL_ERR_WORKSPACE, "workspace", fn, _attention(q, T=3, S=3, mq=1, mkv=20000, ws=None))
    assert fn(*_attention(q, T=0, q=None).values()) == q.QARL_OK and fn(*_attention(q, S=0, q=None).values()) == q.QARL_OK


def test_attention_refuses_scales_and_lengths_that_overflow_inside(q):
    """scale * log2 e has to stay finite; a row's number of pieces has to fit the join's lists."""
    fn = q.lib().qarl_paged_attention
    for scale in (3e38, -3e38, 2.5e38):
        _refused(q, q.QARL_ERR_INVALID_ARG, "finite", fn, _attention(q, scale=scale))
    _refused(q, q.QARL_ERR_UNSUPPORTED, "2^28", fn, _attention(q, mkv=(1 << 28) + 1))
    assert fn(*_attention(q, T=0, q=None, mkv=1 << 28, scale=1e38).values()) == q.QARL_OK


def test_binding_refuses_tensors_of_other_shapes_and_types(q):
    """On the host, before a pointer is taken: CPU tensors, other types, other sizes."""
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="x must be"):
        q.qarl_add_rmsnorm(x, w, 1e-6)
    c = q.KVCache.empty(q.QARL_KV_BF16, 4, 16, 2, 64, "cpu")
    with pytest.raises(ValueError, match="k must be"):
        q.qarl_kv_cache_write(c, x.view(2, 2, 64), x.view(2, 2, 64), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="query must be"):
        q.qarl_paged_attention(torch.zeros((2, 4, 64), dtype=torch.bfloat16), c, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                               torch.zeros(2, dtype=torch.int32), 2, 20)
    with pytest.raises(ValueError, match="contiguous"):
        q.KVCache(q.QARL_KV_BF16, c.k, c.v[:2])
    with pytest.raises(ValueError, match="k_scales"):
        q.KVCache(q.QARL_KV_E4M3, c.k.view(torch.uint8)[..., :64].contiguous(), c.v.view(torch.uint8)[..., :64].contiguous())
    with pytest.raises(ValueError, match="format"):
        q.KVCache(5, c.k, c.v)


def test_reference_gradient_against_differences():
    """The formula that the GPU tests compare with, by central differences."""
    g = torch.Generator().manual_seed(1)
    dy, h, dh = (torch.randn((3, 40), generator=g, dtype=torch.float64) for _ in range(3))
    w = torch.randn(40, generator=g, dtype=torch.float64)
    dx, dw, _, _ = ref.rmsnorm_backward(dy, h, w, 1e-6, dh)

    def loss(hh, ww):
        return float((dy * (hh / torch.sqrt((hh * hh).mean(1, keepdim=True) + 1e-6) * ww)).sum() + (dh * hh).sum())

    e = 1e-6
    for i in (0, 7, 39):
        u = torch.zeros_like(h)
        u[1, i] = e
        assert abs((loss(h + u, w) - loss(h - u, w)) / (2 * e) - float(dx[1, i])) < 1e-7
        z = torch.zeros_like(w)
        z[i] = e
        assert abs((loss(h, w + z) - loss(h, w - z)) / (2 * e) - float(dw[i])) < 1e-7


def test_reference_attention_on_closed_forms():
    q = torch.zeros((3, 2, 4))
    k, v = torch.randn((5, 1, 4), dtype=torch.float64), torch.arange(20, dtype=torch.float64).view(5, 1, 4)
    out, lse, _, _ = ref.attention(q, k, v, torch.ones(5, dtype=torch.bool), 5, 1.0, 0)       # equal scores: means
    for i in range(3):
        assert torch.allclose(out[i, 0], v[: 3 + i, 0].mean(0)) and torch.allclose(lse[i], torch.full((2,), float(torch.log(torch.tensor(3.0 + i))), dtype=torch.float64))
    out, lse, _, _ = ref.attention(q, k, v, torch.ones(5, dtype=torch.bool), 5, 1.0, 1)       # a window of one: the token itself
    assert torch.equal(out[:, 0], v[2:, 0]) and (lse == 0).all()
    out, lse, _, _ = ref.attention(q, k, v, torch.ones(5, dtype=torch.bool), 1, 1.0, 0)       # two queries in front of the first position
    assert (out[:2] == 0).all() and (lse[:2] == -float("inf")).all() and torch.equal(out[2, 0], v[0, 0])


def test_binding_refuses_buffers_that_a_kernel_cannot_reach(q):
    """Host memory, another GPU, strided workspaces: every pointer of a call is looked at, the cache's and the workspace's too."""
    c = q.KVCache.empty(q.QARL_KV_E4M3, 4, 16, 2, 64, "cpu")
    for gpu in (0, 3, -1):
        with pytest.raises(ValueError, match="cache must be on"):
            q._cache(c, gpu)
        with pytest.raises(ValueError, match="ws must be"):
            q._ws(torch.empty(64, dtype=torch.uint8), gpu)
        with pytest.raises(ValueError, match="y must be"):
            q._rows(torch.zeros((4, 64), dtype=torch.bfloat16), "y", torch.bfloat16, (4, 64), gpu)
        with pytest.raises(ValueError, match="lse must be"):
            q._flat(torch.zeros((4, 8)), "lse", torch.float32, (4, 8), gpu)
        with pytest.raises(ValueError, match="v must be"):
            q._heads(torch.zeros((4, 2, 64), dtype=torch.bfloat16), "v", (4, 2, 64), gpu)
        with pytest.raises(ValueError, match="block_table must be"):
            q._table(torch.zeros((4, 2), dtype=torch.int32), 4, gpu)
    assert q._ws(None, 0) == (None, 0)
    for bad in (dict(v=c.v.to("meta")), dict(k_scales=c.k_scales.to("meta")), dict(v_scales=c.v_scales.to("meta"))):
        with pytest.raises(ValueError, match="one device"):
            q.KVCache(q.QARL_KV_E4M3, **dict(dict(k=c.k, v=c.v, k_scales=c.k_scales, v_scales=c.v_scales), **bad))


def test_decoder_layer_refuses_what_it_cannot_run(q):
    """In the constructor, and not in the middle of the first step: e4m3 projections, head counts that do not divide, experts whose down does not fit."""
    from paper_2604_07853_amd.decoder import DecoderLayer
    H, heads, kv, D, E, I = 256, 4, 2, 64, 64, 128
    weight = lambda fmt, e, n, k: q.QWeight.empty(fmt, e, n, k, "cpu")
    norm = torch.ones(H, dtype=torch.bfloat16)
    good = dict(norm1=norm, norm2=norm, qkv=weight(q.QARL_W4A16_G128, 1, (heads + 2 * kv) * D, H), o=weight(q.QARL_W4A16_G128, 1, H, heads * D),
                router=torch.zeros((E, H), dtype=torch.bfloat16), gate_up=weight(q.QARL_FP8_E4M3_CH, E, 2 * I, H), down=weight(q.QARL_FP8_E4M3_CH, E, H, I),
                cache=q.KVCache.empty(q.QARL_KV_BF16, 4, 16, kv, D, "cpu"), topk=8)
    DecoderLayer(**good)
    DecoderLayer(**dict(good, gate_up=weight(q.QARL_W4A8_G128, E, 2 * I, H)))          # both on e4m3 rows
    for fmt in q.E4M3_ACT_FORMATS:
        with pytest.raises(ValueError, match="bf16 rows"):
            DecoderLayer(**dict(good, qkv=weight(fmt, 1, (heads + 2 * kv) * D, H)))
        with pytest.raises(ValueError, match="bf16 rows"):
            DecoderLayer(**dict(good, o=weight(fmt, 1, H, heads * D)))
    with pytest.raises(ValueError, match="query heads"):
        DecoderLayer(**dict(good, cache=q.KVCache.empty(q.QARL_KV_BF16, 4, 16, 3, D, "cpu"), qkv=weight(q.QARL_W4A16_G128, 1, (heads + 6) * D, H)))
    for down in (weight(q.QARL_FP8_E4M3_CH, E, H, 2 * I), weight(q.QARL_FP8_E4M3_CH, E, 2 * H, I), weight(q.QARL_FP8_E4M3_CH, 2 * E, H, I),
                 weight(q.QARL_W4A16_G128, E, H, I)):
        with pytest.raises(ValueError, match="down must be"):
            DecoderLayer(**dict(good, down=down))
    for topk in (0, 33):
        with pytest.raises(ValueError, match="picks 1 to 32"):
            DecoderLayer(**dict(good, topk=topk))
