"""The 4-bit paged cache: writing, reading back and attention over it, against the 64-bit formulas, through the C ABI."""
import math

import pytest
import torch

import layer_ref as ref
from rollout_ref import e2m1_quantized, e2m1_values
from paper_2604_07853_amd import synth
from test_gpu_attention import SHAPES, call, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    from paper_2604_07853_amd import binding
    binding.lib()
    return binding


def dense(codes, scales):
    """The cache's values in bf16, which holds them exactly."""
    v = e2m1_values(codes.cpu(), scales.cpu())[0]
    b = v.to(torch.bfloat16)
    assert torch.equal(b.double().nan_to_num(-1.0), v.nan_to_num(-1.0))
    return b


def make(q, seqs, heads, kv_heads, dim, page, seed, lo=118, hi=128):
    """seqs: [(new tokens, cached tokens)].  Any codes, scales from 2^(lo - 127) on; slots that no sequence uses hold NaN, unused table entries a bad page."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for _, n in seqs]
    pages, width = sum(need) + 2, max(need + [1]) + 1
    perm = torch.randperm(pages, generator=g)
    table = torch.full((len(seqs), width), pages + 5, dtype=torch.int32)
    c = q.KVCache.empty(q.QARL_KV_E2M1, pages, page, kv_heads, dim)
    used = torch.zeros((pages, page), dtype=torch.bool)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at: at + n]
        for p in range(seqs[s][1]):
            used[int(perm[at + p // page]), p % page] = True
        at += n
    host = []
    for store, scales in ((c.k, c.k_scales), (c.v, c.v_scales)):
        codes = torch.randint(0, 256, store.shape, generator=g).to(torch.uint8)
        sc = torch.randint(lo, hi, scales.shape, generator=g).to(torch.uint8)
        sc[(~used)[:, None, :].expand(sc.shape[:3])] = 255
        store.copy_(codes)
        scales.copy_(sc)
        host.append((dense(codes, sc), None))
    T = sum(n for n, _ in seqs)
    return dict(c=c, host=host, table=table, query=synth.normal_bf16((T, heads + 3, dim), 1.0, seed + 1), heads=heads, T=T, seqs=seqs,
                kv_lens=torch.tensor([n for _, n in seqs], dtype=torch.int32), offsets=torch.tensor([0] + [n for n, _ in seqs]).cumsum(0).to(torch.int32))


# ---- writing and reading ----

@pytest.mark.parametrize("T,heads,dim,page", [(1, 1, 64, 8), (1, 4, 128, 16), (9, 3, 64, 16), (37, 2, 128, 32), (300, 4, 128, 16), (9, 8, 128, 1024)])
def test_write(q, T, heads, dim, page):
    pages = -(-T // page) + 3
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(T))[:T]
    x = synth.normal_bf16((T, 2 * heads + 1, dim), 1.0, T + dim)
    if T > 8:
        slots[1], slots[2], slots[3] = -1, pages * page, -(1 << 40)        # outside: skipped
        x[0, 1] = 0
        x[4, 1, 3], x[5, 1 + heads, dim - 1] = math.inf, math.nan
        x[6, 1] = (torch.arange(dim) % 25 * 0.25).to(torch.bfloat16)       # borders between codes, and every code
        x[7, 1:], x[8, 1:] = x[7, 1:] * 2.0 ** 125, x[8, 1:] * 2.0 ** -110          # the largest scale (saturating), the smallest
        x[7, 1, 0] = 3.3e38
    c = q.KVCache.empty(q.QARL_KV_E2M1, pages, page, heads, dim)
    for t in (c.k, c.v, c.k_scales, c.v_scales):
        t.fill_(0x5a)
    dev = x.cuda()
    q.qarl_kv_cache_write(c, dev[:, 1: 1 + heads], dev[:, 1 + heads:], slots.cuda())
    for src, store, scales in ((x[:, 1: 1 + heads], c.k, c.k_scales), (x[:, 1 + heads:], c.v, c.v_scales)):
        codes, sc = e2m1_quantized(src)
        want, wscale = torch.full(store.shape, 0x5a, dtype=torch.uint8), torch.full(scales.shape, 0x5a, dtype=torch.uint8)
        for t in range(T):
            sl = int(slots[t])
            if 0 <= sl < pages * page:
                want[sl // page, :, sl % page], wscale[sl // page, :, sl % page] = codes[t], sc[t]
        have = store.cpu()
        written = wscale != 0x5a
        for shift in (0, 4):        # (a negative zero is a zero)
            a = have >> shift & 15
            a = torch.where(written.any(-1)[..., None] & (a == 8), 0, a)
            assert torch.equal(a, want >> shift & 15)
        assert torch.equal(scales.cpu(), wscale)


@pytest.mark.parametrize("heads,dim,page", [(1, 64, 8), (4, 128, 16), (3, 128, 64), (2, 64, 128)])
@pytest.mark.parametrize("lens", [[1], [0, 5, 0, 131], [40, 1, 7, 300, 16, 0], [0]])
def test_read(q, heads, dim, page, lens):
    m = make(q, [(0, n) for n in lens], heads, heads, dim, page, sum(lens) + dim, 27, 253)
    if lens[-1] > 2 * page:
        m["table"][len(lens) - 1, 1] = -1           # a bad page reads as zeros
    offsets = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    total = sum(lens) + 3                            # three rows behind the last sequence
    out = tuple(torch.full((total, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q.qarl_kv_cache_read(m["c"], m["table"].cuda(), offsets.cuda(), total, out=out)
    for got, (store, _) in zip(out, m["host"]):
        want = torch.zeros((total, heads, dim), dtype=torch.float64)
        for s, n in enumerate(lens):
            want[int(offsets[s]): int(offsets[s]) + n] = ref.cached(store, None, m["table"][s], n, page)[0]
        assert torch.equal(got.double().cpu(), want)


@pytest.mark.parametrize("fmt", ["QARL_KV_BF16", "QARL_KV_E4M3", "QARL_KV_E2M1"])
@pytest.mark.parametrize("S,longest", [(64, 30), (65, 30), (256, 2), (257, 70), (600, 3), (1500, 40)])
def test_read_of_many_sequences(q, fmt, S, longest):
    """Each row is the one that a read of the pages in their own order has there; some sequences are empty, two rows stand behind the last."""
    page, heads, dim = 16, 2, 64
    g = torch.Generator().manual_seed(S)
    lens = torch.randint(0, longest + 1, (S,), generator=g)
    lens[::7] = 0
    width = -(-longest // page)
    table = torch.randperm(S * width, generator=g).to(torch.int32).view(S, width)
    c = q.KVCache.empty(getattr(q, fmt), S * width, page, heads, dim)
    if fmt == "QARL_KV_BF16":
        for t in (c.k, c.v):
            t.copy_(torch.randn(t.shape, generator=g))
    else:
        for t in (c.k, c.v):
            t.copy_(torch.randint(0, 120, t.shape, generator=g))
        for t in (c.k_scales, c.v_scales):
            t.copy_(torch.randint(100, 140, t.shape, generator=g))
    n = S * width * page
    whole = q.qarl_kv_cache_read(c, torch.arange(S * width, dtype=torch.int32, device="cuda")[None], torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
    total = int(offsets[-1]) + 2
    got = q.qarl_kv_cache_read(c, table.cuda(), offsets.to(torch.int32).cuda(), total)
    seq = torch.repeat_interleave(torch.arange(S), lens)
    at = torch.arange(total - 2) - offsets[seq]
    rows = (table[seq, at // page].to(torch.int64) * page + at % page).cuda()
    for have, all_rows in zip(got, whole):
        assert torch.equal(have[:-2], all_rows[rows]) and not have[-2:].any()


# ---- attention ----

@pytest.mark.parametrize("heads,kv_heads,dim,page", SHAPES)
def test_single_tokens(q, heads, kv_heads, dim, page):
    m = make(q, [(1, n) for n in (1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 130, 257, 0)], heads, kv_heads, dim, page, heads * dim + page)
    check(m, call(q, m))


@pytest.mark.parametrize("heads,kv_heads,dim,page", SHAPES)
def test_chunks(q, heads, kv_heads, dim, page):
    m = make(q, [(5, 5), (1, 40), (0, 12), (17, 90), (3, 2), (33, 33), (70, 150), (4, 0), (2, 67)], heads, kv_heads, dim, page, heads * dim + page + 1)
    check(m, call(q, m))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,context", [(2, 0), (2, 300), (5, 61), (16, 500), (130, 0), (257, 100), (300, 1000)])
def test_lengths_of_one_sequence(q, dim, n, context):
    m = make(q, [(n, context + n)], 8, 2, dim, 16, n + context)
    check(m, call(q, m), rows=sorted({0, 1, n // 3, n // 2, n - 2, n - 1} & set(range(n))))


@pytest.mark.parametrize("dim", [64, 128])
def test_pieces_of_every_number_in_one_call(q, dim):
    tokens = [(1, n) for n in (1, 300, 513, 1600, 2047, 4100, 6000)]
    for seqs in (tokens, tokens + [(600, 700), (1, 5900), (300, 1400), (2, 4800)]):
        m = make(q, seqs, 16, 2, dim, 16, 41)
        check(m, call(q, m), rows=[0, 1, 299, 599])


@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 1000])
def test_window(q, window):
    for dim in (64, 128):
        m = make(q, [(1, 257), (1, 3), (40, 200), (90, 90), (3, 130)], 8, 2, dim, 16, window)
        check(m, call(q, m, window=window), window=window)


def test_long_contexts_fp32_output_and_scale(q):
    m = make(q, [(1, 5000), (2, 3001), (1, 17), (20, 2500)], 16, 2, 128, 16, 77)
    check(m, call(q, m, out_dtype=q.QARL_OUT_F32, scale=0.03), scale=0.03, rows=[0, 1, 19], out_f32=True)
    check(m, call(q, m, scale=-0.05), scale=-0.05, rows=[0, 10])


def test_scales_far_apart(q):
    """Quarters of a row up to 2^40 apart: a small quarter keeps its digits beside a large one."""
    for dim, seqs in ((128, [(1, 300), (2, 40)]), (64, [(1, 300), (2, 40)]), (128, [(70, 200)]), (64, [(70, 200)])):
        m = make(q, seqs, 8, 2, dim, 16, 3, 80, 128)
        check(m, call(q, m), rows=[0, 1, 69])


def test_prompts_equal_those_over_a_16_bit_cache(q):
    """The many-row kernel widens codes times scales exactly: the same bits as over the same values in bf16."""
    for dim in (64, 128):
        m = make(q, [(200, 300), (130, 130)], 8, 2, dim, 16, 8)
        c16 = q.KVCache(q.QARL_KV_BF16, m["host"][0][0].cuda(), m["host"][1][0].cuda())
        a, b = call(q, m), call(q, dict(m, c=c16))
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("n", [1, 3, 40, 100])
@pytest.mark.parametrize("dim", [64, 128])
def test_unseen_values_never_reach_a_result(q, n, dim):
    """NaN at positions that some rows see and others do not: later tokens of the chunk, tokens in front of the window.  A quarter's NaN among the values stays
    in its quarter."""
    for window, bad in ((0, [130 + n - 1, 130 + n // 2 + 1]), (50, [3, 70, 131])):
        m = make(q, [(n, 130 + n)], 8, 2, dim, 16, 5)
        clean = call(q, m, window=window)
        for which in (0, 1):
            for p in bad:
                if p >= 130 + n:
                    continue
                page, off = int(m["table"][0, p // 16]), p % 16
                store, scales = (m["c"].k, m["c"].k_scales) if which == 0 else (m["c"].v, m["c"].v_scales)
                keep = store[page, :, off].clone(), scales[page, :, off].clone()
                for code in (0, 0x77, 0x12):
                    store[page, :, off], scales[page, :, off, 2] = code, 255
                    got = call(q, m, window=window)
                    for i in range(n):
                        at = 130 + i
                        if p > at or (window and p <= at - window):
                            assert torch.equal(got["out"][i], clean["out"][i]) and torch.equal(got["lse"][i], clean["lse"][i]), (which, p, i)
                        elif which == 1:
                            quarter = slice(dim // 2, dim // 4 * 3)
                            assert got["out"][i][:, quarter].isnan().all() and got["out"][i][:, : dim // 2].isfinite().all(), (p, i, code)
                            assert got["out"][i][:, dim // 4 * 3:].isfinite().all()
                        else:
                            assert got["out"][i].isnan().all()
                    store[page, :, off], scales[page, :, off] = keep


@pytest.mark.parametrize("n", [1, 4, 70])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_nan_that_all_rows_see(q, n, dim):
    """In a tile that nothing is masked in: NaN whatever the codes, keys' in all of the row, values' in their quarter."""
    m = make(q, [(n, 400 + n)], 8, 2, dim, 16, 5)
    for p in (64, 100):
        page, off = int(m["table"][0, p // 16]), p % 16
        for which, (store, scales) in enumerate(((m["c"].k, m["c"].k_scales), (m["c"].v, m["c"].v_scales))):
            keep = store[page, :, off].clone(), scales[page, :, off].clone()
            for code in (0, 0x77, 0x12):
                store[page, :, off], scales[page, :, off, 1] = code, 255
                got = call(q, m)["out"]
                if which == 0:
                    assert got.isnan().all()
                else:
                    quarter = slice(dim // 4, dim // 2)
                    assert got[..., quarter].isnan().all() and got[..., : dim // 4].isfinite().all() and got[..., dim // 2:].isfinite().all()
            store[page, :, off], scales[page, :, off] = keep


def test_bad_pages_hold_nothing(q):
    m = make(q, [(1, 100), (3, 90), (80, 200)], 8, 2, 64, 16, 13)
    m["table"][0, 0], m["table"][0, 4], m["table"][2, 3] = -1, 1 << 30, -1
    m["table"][1, :] = -5
    check(m, call(q, m))


def test_rows_of_no_sequence_are_left_alone(q):
    m = make(q, [(1, 30), (5, 40)], 4, 2, 64, 16, 15)
    out = torch.full((m["T"] + 4, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    m["query"] = torch.roll(torch.cat([m["query"], m["query"][:4]]), 2, 0)
    m["offsets"] = m["offsets"] + 2
    call(q, m, out=out)
    assert (out[:2] == 9).all() and (out[8:] == 9).all() and (out[2:8] != 9).any()


@pytest.mark.parametrize("heads,kv_heads,dim", [(65, 1, 64), (96, 1, 128), (160, 2, 64), (48, 1, 128), (32, 1, 64)])
def test_many_query_heads_per_cached_one(q, heads, kv_heads, dim):
    m = make(q, [(1, 1), (1, 700), (3, 65), (0, 9), (1, 0), (2, 1300)], heads, kv_heads, dim, 16, heads)
    check(m, call(q, m))


def test_a_step_and_its_attention_in_a_graph(q):
    """As a decode step runs them: append with the rotation, then attention over the cache; replayed with new tokens, against the eager calls."""
    rope = q.Rope(128)
    m = make(q, [(1, 3000), (1, 900), (1, 1)], 8, 2, 128, 16, 16)
    c, table, kv_lens, offsets = m["c"], m["table"].cuda(), m["kv_lens"].cuda(), m["offsets"].cuda()
    slots = torch.tensor([int(m["table"][s, (n - 1) // 16]) * 16 + (n - 1) % 16 for s, (_, n) in enumerate(m["seqs"])], device="cuda")
    pos = (kv_lens - 1).long()
    x = synth.normal_bf16((3, 12, 128), 1.0, 1).cuda()
    rotated, out, lse = torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 8), device="cuda")
    ws = torch.empty((max(1, q.qarl_paged_attention_workspace_bytes(c, 3, 8, 3, 1, 3000)),), dtype=torch.uint8, device="cuda")

    def step():
        q.qarl_rotary_kv_write(c, rope, pos, x[:, :8], x[:, 8:10], x[:, 10:], slots, q_out=rotated)
        q.qarl_paged_attention(rotated, c, table, kv_lens, offsets, 1, 3000, out=out, lse=lse, ws=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        x.copy_(synth.normal_bf16((3, 12, 128), 1.0, 30 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), c.k.clone(), c.v_scales.clone()
        ws.fill_(255)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse) and torch.equal(got[2], c.k) and torch.equal(got[3], c.v_scales)
    for store, scales, i in ((c.k, c.k_scales, 0), (c.v, c.v_scales, 1)):
        m["host"][i] = (dense(store, scales), None)
    full = torch.zeros((3, 11, 128), dtype=torch.bfloat16)
    full[:, 1:9] = rotated.cpu()
    check(dict(m, query=full), dict(out=out, lse=lse))


def test_offsets_past_32_bits(q):
    page, heads, dim = 1024, 8, 128
    pages = (1 << 32) // (page * heads * dim // 2) + 9
    big = q.KVCache(q.QARL_KV_E2M1, *[torch.zeros((pages, heads, page, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2)],
                    *[torch.zeros((pages, heads, page, 4), dtype=torch.uint8, device="cuda") for _ in range(2)])
    small = q.KVCache.empty(q.QARL_KV_E2M1, 2, page, heads, dim)
    for n in ("k", "v", "k_scales", "v_scales"):
        b = getattr(small, n)
        b.random_(0, 256) if "scales" not in n else b.random_(120, 128)
        getattr(big, n)[-2:].copy_(b)
    query = synth.normal_bf16((70, 16, dim), 1.0, 1).cuda()
    for n in (1, 70):
        args = [torch.tensor([1500], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, 1500]
        a = q.qarl_paged_attention(query[:n], big, torch.tensor([[pages - 2, pages - 1]], dtype=torch.int32, device="cuda"), *args)["out"]
        b = q.qarl_paged_attention(query[:n], small, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), *args)["out"]
        assert torch.equal(a, b) and a.isfinite().all() and a.abs().sum() > 0


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("S,kv_heads,lens", [(70, 8, "ragged"), (300, 2, "ragged"), (512, 2, "equal"), (513, 2, "ragged"), (129, 4, "bound"), (64, 9, "few")])
def test_sequences_taken_in_the_order_of_their_lengths(q, fmt, S, kv_heads, lens):
    """More (sequence, head)s than workgroups begin at once: each is worked on, once, whatever the lengths (idle slots, equal ones, a bound far above them)."""
    import test_gpu_attention as base
    g = torch.Generator().manual_seed(S)
    n = torch.randint(0, 90, (S,), generator=g).tolist()
    if lens == "equal":
        n = [33] * S
    if lens == "few":
        n = [0] * (S - 2) + [1, 70]
    seqs = [(1, v) for v in n]
    m = make(q, seqs, 2 * kv_heads, kv_heads, 64, 16, S) if fmt == "fp4" else base.make(q, fmt, seqs, 2 * kv_heads, kv_heads, 64, 16, S)
    out = torch.full((S, 2 * kv_heads, 64), math.nan, dtype=torch.bfloat16, device="cuda")
    got = call(q, m, max_kv=100000 if lens == "bound" else None, out=out)
    assert got["out"].isfinite().all()
    check(m, got)


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("S,kv_heads,dim", [(130, 4, 128), (66, 8, 64), (512, 2, 64), (512, 8, 128)])
def test_long_caches_first_or_in_their_own_order(q, fmt, S, kv_heads, dim):
    """A few long caches among short ones: workgroups take them first where one of the first 64 sequences is long, and in the order of the call where they stand
    behind.  Either way every sequence gets the same bits."""
    import test_gpu_attention as base
    n = torch.randint(0, 60, (S,), generator=torch.Generator().manual_seed(S)).tolist()
    n[3], n[7], n[40], n[S // 2], n[S - 1] = 0, 5000, 3700, 3600, 4100
    seqs = [(1, v) for v in n]
    m = make(q, seqs, 2 * kv_heads, kv_heads, dim, 16, S) if fmt == "fp4" else base.make(q, fmt, seqs, 2 * kv_heads, kv_heads, dim, 16, S)
    outs = [torch.full((S, 2 * kv_heads, dim), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    got = call(q, m, out=outs[0])
    assert got["out"].isfinite().all()
    check(m, got)
    order = torch.tensor(sorted(range(S), key=lambda s: n[s]))
    again = call(q, dict(m, query=m["query"][order], table=m["table"][order], kv_lens=m["kv_lens"][order]), out=outs[1])
    assert torch.equal(again["out"].cpu(), got["out"].cpu()[order]) and torch.equal(again["lse"].cpu(), got["lse"].cpu()[order])


@pytest.mark.parametrize("fmt", ["QARL_KV_BF16", "QARL_KV_E4M3", "QARL_KV_E2M1"])
@pytest.mark.parametrize("dim,page", [(128, 16), (64, 128)])
def test_large_reads_equal_small_ones(q, fmt, dim, page):
    """Reads that move more than 64 MB pass the caches, those of up to 6144 rows take fewer rows a workgroup: the same bits, sequence by sequence and whole."""
    heads, lens = 4, [9000, 0, 1, 14001, 5000] if dim == 128 else [20001, 0, 1, 30003, 6000]
    g = torch.Generator(device="cuda")
    g.manual_seed(dim)
    need = [-(-n // page) for n in lens]
    c = q.KVCache.empty(getattr(q, fmt), sum(need), page, heads, dim)
    for t in (c.k, c.v):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda") if fmt == "QARL_KV_BF16" else torch.randint(0, 127, t.shape, generator=g, device="cuda"))
    for t in (c.k_scales, c.v_scales):
        if t is not None:
            t.copy_(torch.randint(100, 140, t.shape, generator=g, device="cuda"))
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    perm = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = perm[sum(need[:s]): sum(need[:s]) + n]
    table = table.cuda()
    offsets = torch.tensor([0] + lens, dtype=torch.int64).cumsum(0).to(torch.int32)
    total = int(offsets[-1])
    whole = q.qarl_kv_cache_read(c, table, offsets.cuda(), total)
    for s, n in enumerate(lens):
        for lo in range(0, n, 96 * page):       # (at most 12288 rows, a few pages at a time)
            rows = min(96 * page, n - lo)
            part = q.qarl_kv_cache_read(c, table[s: s + 1, lo // page:].contiguous(), torch.tensor([0, rows], dtype=torch.int32, device="cuda"), rows)
            at = int(offsets[s]) + lo
            assert all(torch.equal(a[at: at + rows], b) for a, b in zip(whole, part)), (s, lo)


@pytest.mark.parametrize("fmt", ["QARL_KV_BF16", "QARL_KV_E4M3", "QARL_KV_E2M1"])
@pytest.mark.parametrize("S,longest", [(96, 60), (97, 30), (97, 70), (200, 5), (255, 30)])
def test_read_of_about_a_hundred_sequences(q, fmt, S, longest):
    """Where the search for a row's sequence begins among the offsets in LDS, and fewer sequences than there is room for."""
    test_read_of_many_sequences(q, fmt, S, longest)
