"""The paged KV cache: writing (plain and quantized) and reading back, through the C ABI."""
import math

import pytest
import torch

import layer_ref as ref
from paper_2604_07853_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    from paper_2604_07853_amd import binding
    binding.lib()
    return binding


def _fmt(q, name):
    return q.QARL_KV_E4M3 if name == "fp8" else q.QARL_KV_BF16


def _filled(q, fmt, pages, page, heads, dim):
    """A cache of 0x5a bytes and 1.5 scales, to see what is written."""
    c = q.KVCache.empty(_fmt(q, fmt), pages, page, heads, dim)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0x5a)
    for t in (c.k_scales, c.v_scales):
        if t is not None:
            t.fill_(1.5)
    return c


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("T,heads,dim,page", [(1, 1, 64, 8), (1, 4, 128, 16), (5, 3, 64, 16), (37, 2, 128, 32), (300, 4, 128, 16), (9, 8, 128, 1024)])
def test_write(q, oracle, fmt, T, heads, dim, page):
    pages = -(-T // page) + 3
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(T))[:T].to(torch.int64)
    if T > 3:
        slots[1], slots[2], slots[3] = -1, pages * page, -(1 << 40)        # outside: skipped
    qkv = synth.normal_bf16((T, 2 * heads + 5, dim), 1.0, T + dim)
    qkv[0, 5] = 0
    if T > 5:
        qkv[4, 5, 3] = float("inf")
        qkv[5, 5 + heads, 1] = float("nan")
    k, v = qkv[:, 5: 5 + heads], qkv[:, 5 + heads:]
    c = _filled(q, fmt, pages, page, heads, dim)
    dev = qkv.cuda()
    q.qarl_kv_cache_write(c, dev[:, 5: 5 + heads], dev[:, 5 + heads:], slots.cuda())
    for src, store, scales in ((k, c.k, c.k_scales), (v, c.v, c.v_scales)):
        want = torch.full((pages, heads, page, dim * (1 if fmt == "fp8" else 2)), 0x5a, dtype=torch.uint8)
        wscale = torch.full((pages, heads, page), 1.5)
        if fmt == "fp8":
            codes, s = (torch.from_numpy(a) for a in oracle.quantize_fp8_rows(synth.bits(src.contiguous())))
            for t in range(T):
                for h in range(heads):
                    if not src[t, h].isfinite().all():
                        codes[t, h], s[t, h] = 0x7f, math.nan
        else:
            codes = src.contiguous().view(torch.uint8).reshape(T, heads, dim * 2)
        for t in range(T):
            sl = int(slots[t])
            if 0 <= sl < pages * page:
                want[sl // page, :, sl % page] = codes[t]
                if fmt == "fp8":
                    wscale[sl // page, :, sl % page] = s[t]
        assert torch.equal(store.view(torch.uint8).cpu().reshape(want.shape), want)
        if fmt == "fp8":
            assert torch.equal(scales.cpu().nan_to_num(-1.0), wscale.nan_to_num(-1.0))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("heads,dim,page", [(1, 64, 8), (4, 128, 16), (3, 128, 64), (2, 64, 128)])
@pytest.mark.parametrize("lens", [[1], [0, 5, 0, 131], [40, 1, 7, 300, 16, 0], [0]])
def test_read(q, fmt, heads, dim, page, lens):
    g = torch.Generator().manual_seed(sum(lens) + dim)
    need = [-(-n // page) for n in lens]
    pages, width = sum(need) + 2, max(need + [1]) + 1
    perm = torch.randperm(pages, generator=g)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at: at + n]
        at += n
    if lens[-1] > 2 * page:
        table[len(lens) - 1, 1] = pages             # a bad page reads as zeros
        if lens[-1] > 3 * page:
            table[len(lens) - 1, 2] = -7
    c = q.KVCache.empty(_fmt(q, fmt), pages, page, heads, dim)
    if fmt == "fp8":
        for t in (c.k, c.v):
            t.copy_(torch.randint(0, 256, t.shape, generator=g).masked_fill_(torch.rand(t.shape, generator=g) < 0.1, 0))
            t[(t & 127) == 127] = 1
        for t in (c.k_scales, c.v_scales):
            t.copy_(torch.rand(t.shape, generator=g) + 0.01)
    else:
        for t in (c.k, c.v):
            t.copy_(torch.randn(t.shape, generator=g))
    offsets = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    total = sum(lens) + 3                            # three rows behind the last sequence
    out = tuple(torch.full((total, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wide = torch.full((len(lens), width + 5), 0, dtype=torch.int32, device="cuda")
    wide[:, :width] = table.cuda()
    q.qarl_kv_cache_read(c, wide[:, :width], offsets.cuda(), total, out=out)
    for got, store, scales in ((out[0], c.k, c.k_scales), (out[1], c.v, c.v_scales)):
        want = torch.zeros((total, heads, dim), dtype=torch.float64)
        for s, n in enumerate(lens):
            rows, _ = ref.cached(store.cpu(), None if scales is None else scales.cpu(), table[s], n, page)
            want[int(offsets[s]): int(offsets[s]) + n] = rows
        assert ((got.double().cpu() - want).abs() <= want.abs() * (ref.HALF_BF16 + 2 * ref.F32 if fmt == "fp8" else 0)).all()


def test_round_trip_of_a_finished_sequence(q):
    """Written token by token and in chunks, read back whole: bf16 bit for bit, e4m3 to half a step."""
    T, heads, dim, page = 203, 4, 128, 16
    k, v = (synth.normal_bf16((T, heads, dim), 1.0, s).cuda() for s in (1, 2))
    pages = -(-T // page)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(4)).to(torch.int32).cuda()[None]
    pos = torch.arange(T, device="cuda")
    slots = table[0, pos // page].to(torch.int64) * page + pos % page
    for fmt in ("bf16", "fp8"):
        c = q.KVCache.empty(_fmt(q, fmt), pages, page, heads, dim)
        for lo, hi in ((0, 100), (100, 101), (101, 102), (102, 203)):
            q.qarl_kv_cache_write(c, k[lo:hi], v[lo:hi], slots[lo:hi])
        rk, rv = q.qarl_kv_cache_read(c, table, torch.tensor([0, T], dtype=torch.int32, device="cuda"), T)
        for got, src in ((rk, k), (rv, v)):
            if fmt == "bf16":
                assert torch.equal(got, src)
            else:
                s = src.double().abs().amax(-1, keepdim=True) / 448
                bound = src.double().abs() * (ref.HALF_E4M3 + 1.07 * ref.HALF_BF16) + s * ref.SUB_E4M3     # code, then bf16(code * scale)
                assert ((got.double() - src.double()).abs() <= bound).all()


def test_offsets_past_32_bits(q):
    """A cache of more than 2^32 bytes per half: the last page is written and read, the first is left alone."""
    page, heads, dim = 1024, 8, 128
    pages = (1 << 32) // (page * heads * dim) + 9                    # e4m3: one byte per element, 4.3 GB each
    c = q.KVCache(q.QARL_KV_E4M3, *[torch.zeros((pages, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2)],
                  *[torch.zeros((pages, heads, page), dtype=torch.float32, device="cuda") for _ in range(2)])
    k, v = (synth.normal_bf16((3, heads, dim), 1.0, s).cuda() for s in (1, 2))
    slots = torch.tensor([pages * page - 3, pages * page - 2, pages * page - 1], device="cuda")
    q.qarl_kv_cache_write(c, k, v, slots)
    assert not c.k[:4].any() and not c.v[:4].any()
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda")
    rk, rv = q.qarl_kv_cache_read(c, table, torch.tensor([0, page], dtype=torch.int32, device="cuda"), page)
    small = q.KVCache.empty(q.QARL_KV_E4M3, 1, page, heads, dim)
    for t in (small.k, small.v, small.k_scales, small.v_scales):
        t.zero_()
    q.qarl_kv_cache_write(small, k, v, slots - (pages - 1) * page)
    wk, wv = q.qarl_kv_cache_read(small, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([0, page], dtype=torch.int32, device="cuda"), page)
    assert torch.equal(rk, wk) and torch.equal(rv, wv) and rk[-3:].abs().sum() > 0


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_buffers_in_host_memory_are_refused(q, fmt):
    """Beside operands on the GPU: a cache, a workspace or an index array in host memory reaches no kernel."""
    host, c = q.KVCache.empty(_fmt(q, fmt), 4, 16, 2, 64, "cpu"), q.KVCache.empty(_fmt(q, fmt), 4, 16, 2, 64)
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    query = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    slots, table = torch.arange(2, device="cuda"), torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    lens, offsets = torch.tensor([2], dtype=torch.int32, device="cuda"), torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    for call in (lambda a: q.qarl_kv_cache_write(a, k, k, slots), lambda a: q.qarl_kv_cache_read(a, table, offsets, 2),
                 lambda a: q.qarl_paged_attention(query, a, table, lens, offsets, 2, 2)):
        with pytest.raises(ValueError, match="cache must be on cuda"):
            call(host)
        call(c)
    for bad in (torch.empty(4096, dtype=torch.uint8), torch.empty(8192, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="ws must be"):
            q.qarl_paged_attention(query, c, table, lens, offsets, 2, 2, ws=bad)
        with pytest.raises(ValueError, match="ws must be"):
            q.qarl_add_rmsnorm_backward(k.view(2, 128), k.view(2, 128), k.view(-1)[:128], 1e-6, ws=bad)
    with pytest.raises(ValueError, match="slots must be"):
        q.qarl_kv_cache_write(c, k, k, slots.cpu())
    with pytest.raises(ValueError, match="block_table must be"):
        q.qarl_paged_attention(query, c, table.cpu(), lens, offsets, 2, 2)
