"""Attention of new tokens over the paged cache against the 64-bit formulas, through the C ABI."""
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


def make(q, fmt, seqs, heads, kv_heads, dim, page, seed, garbage=True):
    """seqs: [(new tokens, cached tokens)].  Slots that no sequence uses hold NaN (garbage) and unused table entries a bad page."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for _, n in seqs]
    pages, width = sum(need) + 2, max(need + [1]) + 1
    perm = torch.randperm(pages, generator=g)
    table = torch.full((len(seqs), width), pages + 5, dtype=torch.int32)
    c = q.KVCache.empty(q.QARL_KV_E4M3 if fmt == "fp8" else q.QARL_KV_BF16, pages, page, kv_heads, dim)
    host = []
    used = torch.zeros((pages, page), dtype=torch.bool)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at: at + n]
        for p in range(seqs[s][1]):
            used[int(perm[at + p // page]), p % page] = True
        at += n
    for store, scales, mean in ((c.k, c.k_scales, 0.2), (c.v, c.v_scales, 0.5)):
        if fmt == "fp8":
            codes = torch.randint(0, 256, store.shape, generator=g).to(torch.uint8)
            codes[(codes & 127) == 127] = 1
            sc = torch.rand(scales.shape, generator=g) * 0.01 + 1e-3
            if garbage:
                sc[(~used)[:, None, :].expand(sc.shape)] = math.nan
                codes[(~used)[:, None, :].expand(sc.shape)] = 0x7f
            store.copy_(codes)
            scales.copy_(sc)
            host.append((codes, sc))
        else:
            x = (torch.randn(store.shape, generator=g) + mean).to(torch.bfloat16)
            if garbage:
                x[(~used)[:, None, :].expand(x.shape[:3])] = math.nan
            store.copy_(x)
            host.append((x, None))
    T = sum(n for n, _ in seqs)
    query = synth.normal_bf16((T, heads + 3, dim), 1.0, seed + 1)       # a slice of wider rows
    return dict(c=c, host=host, table=table, query=query, heads=heads, T=T, seqs=seqs,
                kv_lens=torch.tensor([n for _, n in seqs], dtype=torch.int32),
                offsets=torch.tensor([0] + [n for n, _ in seqs]).cumsum(0).to(torch.int32))


def call(q, m, max_kv=None, **kw):
    return q.qarl_paged_attention(m["query"].cuda()[:, 1: 1 + m["heads"]], m["c"], m["table"].cuda(), m["kv_lens"].cuda(), m["offsets"].cuda(),
                                  max([1] + [n for n, _ in m["seqs"]]), max([1] + [n for _, n in m["seqs"]]) if max_kv is None else max_kv,
                                  want_lse=True, **kw)


def check(m, got, scale=None, window=0, rows=None, out_f32=False):
    """Error of an output: a rounding of every probability to bf16 (half a step of p |v| each), the scores' fp32 error (it changes p by as much,
    in the numerator and in the sum), 2^-19 for exp2, the sums and the rescaling, and the output's own rounding."""
    scale = m["query"].shape[2] ** -0.5 if scale is None else scale
    for s, (n, total) in enumerate(m["seqs"]):
        lo = int(m["offsets"][s])
        k, ok = ref.cached(*m["host"][0], m["table"][s], total, m["c"].page_size)
        v, _ = ref.cached(*m["host"][1], m["table"][s], total, m["c"].page_size)
        pick = range(n) if rows is None else [i for i in rows if i < n]
        for i in pick:
            o, e, mag, zerr = ref.attention(m["query"][lo + i: lo + i + 1, 1: 1 + m["heads"]], k, v, ok, total - n + i + 1, scale, window)
            have, lse = got["out"][lo + i].double().cpu(), got["lse"][lo + i].double().cpu()
            tol = mag[0] * (ref.HALF_BF16 + 2 * zerr[0][:, None] + 2.0 ** -19) + o[0].abs() * (ref.F32 if out_f32 else 1.01 * ref.HALF_BF16)
            assert ((have - o[0]).abs() <= tol).all(), (s, i, float(((have - o[0]).abs() - tol).max()))
            seen = torch.isfinite(e[0])
            assert torch.equal(lse == -math.inf, ~seen), (s, i)
            assert ((lse - e[0]).abs()[seen] <= (zerr[0] + 2.0 ** -19 * (1 + e[0].abs()))[seen]).all(), (s, i)


SHAPES = [(1, 1, 64, 8), (8, 1, 128, 16), (4, 4, 64, 16), (14, 2, 128, 32), (6, 2, 64, 128), (32, 4, 128, 16), (40, 2, 128, 8), (5, 1, 128, 64)]


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", SHAPES)
def test_single_tokens(q, fmt, heads, kv_heads, dim, page):
    seqs = [(1, n) for n in (1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 130, 257, 0)]
    m = make(q, fmt, seqs, heads, kv_heads, dim, page, heads * dim + page)
    check(m, call(q, m))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", SHAPES)
def test_chunks(q, fmt, heads, kv_heads, dim, page):
    """Whole prompts, chunks behind a context, single tokens, sequences without new tokens, more queries than cached positions."""
    seqs = [(5, 5), (1, 40), (0, 12), (17, 90), (3, 2), (33, 33), (70, 150), (4, 0), (2, 67)]
    m = make(q, fmt, seqs, heads, kv_heads, dim, page, heads * dim + page + 1)
    check(m, call(q, m))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("n,context", [(2, 0), (2, 300), (5, 61), (16, 500), (130, 0), (257, 100), (300, 1000)])
def test_lengths_of_one_sequence(q, fmt, n, context):
    m = make(q, fmt, [(n, context + n)], 8, 2, 128, 16, n + context)
    check(m, call(q, m), rows=sorted({0, 1, n // 3, n // 2, n - 2, n - 1} & set(range(n))))


@pytest.mark.parametrize("dim", [64, 128])
def test_pieces_of_every_number_in_one_call(q, dim):
    """Rows of one piece, of a few and of many (single tokens over caches of all lengths), alone and beside long chunks with thousands of rows."""
    tokens = [(1, n) for n in (1, 300, 512, 513, 1100, 1600, 2047, 3000, 4100, 4609, 5200, 6000)]
    for seqs in (tokens, tokens + [(600, 700), (1, 5900), (300, 1400), (2, 4800)]):
        m = make(q, "bf16", seqs, 16, 2, dim, 16, 41)
        check(m, call(q, m), rows=[0, 1, 299, 599])


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("dim", [64, 128])
def test_more_row_blocks_than_cus(q, fmt, dim):
    """Several rounds of workgroups, 70 sequences (more than a wavefront looks up at once), every row of every block written."""
    lens = [(1 + 37 * s % 130, 1 + 37 * s % 130 + 11 * s % 60) for s in range(66)] + [(700, 700), (3, 900), (520, 1000), (900, 901)]
    m = make(q, fmt, lens, 16, 2, dim, 16, 31)
    out = torch.full((m["T"], 16, dim), math.nan, dtype=torch.bfloat16, device="cuda")
    got = call(q, m, out=out)
    assert got["out"].isfinite().all() and got["lse"].isfinite().all()
    check(m, got, rows=[0, 40, 129, 350, 519, 699, 899])


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 1000])
def test_window(q, fmt, window):
    m = make(q, fmt, [(1, 257), (1, 3), (40, 200), (90, 90), (3, 130)], 8, 2, 64, 16, window)
    check(m, call(q, m, window=window), window=window)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_long_contexts_fp32_output_and_scale(q, fmt):
    m = make(q, fmt, [(1, 5000), (2, 3001), (1, 17), (20, 2500)], 16, 2, 128, 16, 77)
    check(m, call(q, m, out_dtype=q.QARL_OUT_F32, scale=0.3), scale=0.3, rows=[0, 1, 19], out_f32=True)
    check(m, call(q, m, scale=-0.05), scale=-0.05, rows=[0, 10])


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("n", [1, 3, 40, 100])
def test_unseen_values_never_reach_a_result(q, fmt, n):
    """NaN and infinities at positions that some rows see and others do not: later tokens of the chunk, tokens in front of the window."""
    for window, bad in ((0, [130 + n - 1, 130 + n // 2 + 1]), (50, [3, 70, 131])):
        m = make(q, fmt, [(n, 130 + n)], 8, 2, 128, 16, 5)
        clean = call(q, m, window=window)
        for which in (0, 1):
            for p in bad:
                if p >= 130 + n:
                    continue
                page, off = int(m["table"][0, p // 16]), p % 16
                for value in ((0x7f, math.nan), (0x10, math.inf)) if fmt == "fp8" else ((math.nan,), (math.inf,), (-math.inf,)):
                    store, scales = (m["c"].k, m["c"].k_scales) if which == 0 else (m["c"].v, m["c"].v_scales)
                    keep = store[page, :, off].clone(), None if scales is None else scales[page, :, off].clone()
                    store[page, :, off] = value[0]
                    if fmt == "fp8":
                        scales[page, :, off] = value[1]
                    got = call(q, m, window=window)
                    for i in range(n):
                        at = 130 + i
                        if p > at or (window and p <= at - window):
                            assert torch.equal(got["out"][i], clean["out"][i]) and torch.equal(got["lse"][i], clean["lse"][i]), (which, p, i)
                        elif which == 1:
                            assert not got["out"][i].isfinite().any() or value[0] == 0x10, (p, i)
                    store[page, :, off] = keep[0]
                    if fmt == "fp8":
                        scales[page, :, off] = keep[1]


@pytest.mark.parametrize("n", [1, 60])
def test_extreme_scores(q, n):
    """Scores far apart (the softmax is one token), equal scores, and a first token that outweighs all others."""
    for factor in (40.0, 0.0, -40.0):
        m = make(q, "bf16", [(n, 200 + n)], 8, 2, 128, 16, 9)
        m["query"] = (m["query"].float() * factor).to(torch.bfloat16)
        check(m, call(q, m), rows=[0, n - 1])


def test_bad_pages_hold_nothing(q):
    m = make(q, "bf16", [(1, 100), (3, 90)], 8, 2, 64, 16, 13)
    m["table"][0, 0], m["table"][0, 4] = -1, 1 << 30
    m["table"][1, :] = -5
    check(m, call(q, m))


def test_lengths_are_cut_at_the_bounds(q):
    m = make(q, "bf16", [(1, 400)], 8, 2, 64, 16, 14)
    whole = call(q, m)
    m["kv_lens"][0] = 400
    m["table"] = m["table"][:, : 400 // 16].contiguous()
    assert torch.equal(call(q, m)["out"], whole["out"])
    cut = call(q, m, max_kv=160)                       # positions 0 .. 159 of a query at 399
    k, ok = ref.cached(*m["host"][0], m["table"][0], 160, 16)
    v, _ = ref.cached(*m["host"][1], m["table"][0], 160, 16)
    o, e, mag, zerr = ref.attention(m["query"][:1, 1:9], k, v, ok, 400, 64 ** -0.5, 0)
    assert ((cut["out"][0].double().cpu() - o[0]).abs() <= mag[0] * (ref.HALF_BF16 + 1e-5) + o[0].abs() * 1.01 * ref.HALF_BF16).all()


def test_rows_of_no_sequence_are_left_alone(q):
    m = make(q, "fp8", [(1, 30), (5, 40)], 4, 2, 64, 16, 15)
    out = torch.full((m["T"] + 4, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    m["query"] = torch.cat([m["query"], m["query"][:4]])
    m["offsets"] = m["offsets"] + 2
    m["query"] = torch.roll(m["query"], 2, 0)
    call(q, m, out=out)
    assert (out[:2] == 9).all() and (out[8:] == 9).all() and (out[2:8] != 9).any()


def test_same_results_every_time_and_in_a_graph(q):
    m = make(q, "fp8", [(1, 3000), (1, 900), (40, 700), (1, 1)], 8, 2, 128, 16, 16)
    query, table, kv_lens, offsets = m["query"].cuda()[:, 1:9], m["table"].cuda(), m["kv_lens"].cuda(), m["offsets"].cuda()
    out, lse = torch.empty((m["T"], 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((m["T"], 8), device="cuda")
    ws = torch.empty((max(1, q.qarl_paged_attention_workspace_bytes(m["c"], m["T"], 8, 4, 40, 3000)),), dtype=torch.uint8, device="cuda")
    slots = torch.tensor([int(m["table"][0, 2999 // 16]) * 16 + 2999 % 16], device="cuda")
    new = synth.normal_bf16((1, 2, 128), 1.0, 3).cuda()

    def step():
        q.qarl_kv_cache_write(m["c"], new, new, slots)
        q.qarl_paged_attention(query, m["c"], table, kv_lens, offsets, 40, 3000, out=out, lse=lse, ws=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        new.copy_(synth.normal_bf16((1, 2, 128), 1.0, 30 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        ws.fill_(255)                                  # nothing of an earlier call is used
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)


@pytest.mark.parametrize("n,S", [(1, 1), (1, 3), (3, 2), (70, 1), (70, 3)])
def test_the_workspace_asked_for_is_enough(q, n, S):
    """Behind the bytes that the query names nothing is written, whatever the window (it changes how a cache is cut)."""
    m = make(q, "bf16", [(n, 4700 - 100 * s) for s in range(S)], 8, 2, 64, 16, 21)
    for max_kv in (4700, 4701, 5000, 6143, 9000):
        need = q.qarl_paged_attention_workspace_bytes(m["c"], m["T"], 8, S, n, max_kv)
        ws = torch.full((need + 65536,), 0x5a, dtype=torch.uint8, device="cuda")
        for window in (0, 1, 700, 1500, 2560, 4000, 4600):
            got = call(q, m, max_kv=max_kv, window=window, ws=ws)
            assert (ws[need:] == 0x5a).all(), (max_kv, window)
            if max_kv in (4701, 9000) and window in (0, 2560):
                check(m, got, window=window, rows=[0, n - 1])


def test_offsets_past_32_bits(q):
    """A cache of more than 2^32 bytes: the last pages hold the sequence."""
    page, heads, dim = 1024, 8, 128
    pages = (1 << 31) // (page * heads * dim) + 9
    big = q.KVCache(q.QARL_KV_BF16, *[torch.zeros((pages, heads, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    small = q.KVCache.empty(q.QARL_KV_BF16, 2, page, heads, dim)
    for a, b in ((big.k, small.k), (big.v, small.v)):
        b.normal_()
        a[-2:].copy_(b)
    query = synth.normal_bf16((40, 16, dim), 1.0, 1).cuda()
    for n in (1, 40):
        args = [torch.tensor([1500], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, 1500]
        a = q.qarl_paged_attention(query[:n], big, torch.tensor([[pages - 2, pages - 1]], dtype=torch.int32, device="cuda"), *args)["out"]
        b = q.qarl_paged_attention(query[:n], small, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), *args)["out"]
        assert torch.equal(a, b) and a.isfinite().all() and a.abs().sum() > 0


@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_visible_infinities_at_the_ends_reach_the_result(q, fmt, n):
    """An infinity at the last or the first position that a query sees gives infinities, however much of its tile lies outside (a product with the
    probability 0 of a position that is not there would give NaN)."""
    window = 50
    for total in (n, n + 17, n + 95):
        for first in (False, True):
            m = make(q, fmt, [(n, total)], 8, 2, 64, 16, total + 5)
            at = max(0, total - window) if first else total - 1             # the last query's ends
            page, off = int(m["table"][0, at // 16]), at % 16
            v, scales = m["host"][1]
            if fmt == "fp8":
                v[page, :, off] = 0x38 + (torch.arange(64) % 2 * 128).to(torch.uint8)        # 1 and -1 in turn
                scales[page, :, off] = math.inf
                m["c"].v_scales.copy_(scales)
            else:
                v[page, :, off] = torch.where(torch.arange(64) % 2 == 0, math.inf, -math.inf).to(torch.bfloat16)
            m["c"].v.copy_(v)
            got = call(q, m, window=window)["out"][n - 1].double().cpu()
            assert torch.equal(got, torch.where(torch.arange(64) % 2 == 0, math.inf, -math.inf).double().expand(8, 64)), (total, first)


@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("scale", [0.0, 1e-36, -1e-33])
def test_scales_of_small_size(q, n, scale):
    """Scores that are large before they are scaled (16 coordinates of up to 2^60 each): the scale counts as it is, however small."""
    m = make(q, "bf16", [(n, n + 30)], 4, 2, 64, 16, 3)
    m["query"] = (m["query"].float() * 2.0 ** 55).to(torch.bfloat16)
    k = (m["host"][0][0].float() * 2.0 ** 55).to(torch.bfloat16)
    m["host"][0] = (k, None)
    m["c"].k.copy_(k)
    check(m, call(q, m, scale=scale), scale=scale)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("n,total,window", [(9, 700, 0), (33, 33, 0), (300, 300, 0), (300, 700, 40), (290, 1000, 200), (257, 400, 1)])
def test_wavefronts_that_see_different_tiles(q, fmt, n, total, window):
    """One query head per cached one and eight: wavefronts without rows, behind the diagonal, in front of a window's start, in one piece and in several."""
    for heads, S in ((2, 1), (16, 1), (2, 40)):
        m = make(q, fmt, [(n, total)] * S if S == 1 else [(n - s % 3, total - s) if total - s >= n else (n, total) for s in range(S)], heads, 2, 64, 16, n)
        got = call(q, m, window=window)
        check(dict(m, seqs=m["seqs"][:2]), got, window=window, rows=sorted({r for r in (0, 1, 31, 32, 33, 63, 64, 127, 128, n - 34, n - 33, n - 2, n - 1) if r >= 0}))


def test_strides_of_single_tokens_and_heads_do_not_matter(q):
    """A batch of one token, or one head, cut out of rows whose length is no multiple of eight."""
    m = make(q, "bf16", [(1, 40)], 4, 1, 64, 16, 9)
    wide = torch.zeros((2, 4 * 64 + 3), dtype=torch.bfloat16, device="cuda")
    wide[0, :256] = m["query"][0, 1:5].reshape(-1).cuda()
    view = wide.as_strided((1, 4, 64), (259, 64, 1))
    args = (m["c"], m["table"].cuda(), m["kv_lens"].cuda(), m["offsets"].cuda(), 1, 40)
    assert view.stride()[0] % 8 and torch.equal(q.qarl_paged_attention(view, *args)["out"], q.qarl_paged_attention(view.contiguous(), *args)["out"])
    k = torch.randn((8, 64), device="cuda").to(torch.bfloat16).as_strided((8, 1, 64), (64, 3, 1))
    before = m["c"].k.clone()
    q.qarl_kv_cache_write(m["c"], k, k, torch.arange(8, device="cuda"))
    assert torch.equal(m["c"].k[0, 0, :8], k[:, 0]) and torch.equal(m["c"].k[0, 0, 8:].view(torch.int16), before[0, 0, 8:].view(torch.int16))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("heads,max_q,window,seqs", [
    (2, 65, 1, [(300, 300)]), (16, 4, 1, [(90, 700), (1, 40)]),                                 # a window's positions in more pieces than max_q_len lets expect
    (16, 1, 0, [(1, 3000), (5, 4000), (1, 2500)]), (2, 1, 0, [(40, 3000), (1, 3000)]),          # single tokens
    (2, 70, 0, [(70, 2000), (1, 3000), (200, 2500), (3, 50)]), (16, 70, 0, [(70, 2000), (1, 3000), (71, 2500), (2, 50)]),
    (2, 70, 40, [(70, 2000), (500, 800), (1, 3000)]), (2, 40, 0, [(33, 900), (41, 900), (64, 64), (65, 70)])])
def test_sequences_longer_than_the_bound_are_left_alone(q, fmt, heads, max_q, window, seqs):
    """max_q_len is the caller's bound: a longer sequence's rows stay as they are, whatever the workspace held, and the others are right."""
    m = make(q, fmt, seqs, heads, 2, 64, 16, 51)
    max_kv = max(n for _, n in seqs)
    ws = torch.full((q.qarl_paged_attention_workspace_bytes(m["c"], m["T"], heads, len(seqs), max_q, max_kv),), 1, dtype=torch.uint8, device="cuda")
    out = torch.full((m["T"], heads, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((m["T"], heads), 9.0, device="cuda")
    got = q.qarl_paged_attention(m["query"].cuda()[:, 1: 1 + heads], m["c"], m["table"].cuda(), m["kv_lens"].cuda(), m["offsets"].cuda(), max_q, max_kv,
                                 window=window, out=out, lse=lse, ws=ws)
    for s, (n, _) in enumerate(seqs):
        lo = int(m["offsets"][s])
        if n > max_q:
            assert (out[lo: lo + n] == 9).all() and (lse[lo: lo + n] == 9).all(), s
    check(dict(m, seqs=[(n if n <= max_q else 0, total) for n, total in seqs]), got, window=window)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("n", [1, 3, 70, 300])
def test_windows_that_start_behind_the_last_position_there_is(q, fmt, n):
    """kv_lens past what the table holds (80 positions) or max_kv_len allows, and a window that starts there: zeros and lse -inf; rows whose window reaches
    back before it see what is left."""
    for total, window, max_kv in ((1000 + n, 10, 1000 + n), (81 + n + 20, 20, 81 + n + 20), (80 + n, 40, 80 + n), (n + 400, 30, 72), (n + 75, 30, 72)):
        m = make(q, fmt, [(n, total), (2, 90)], 8, 2, 64, 16, n + 7)
        m["table"] = m["table"][:, :5].contiguous()
        got = call(q, m, max_kv=max_kv, window=window)
        if max_kv >= 80:
            check(m, got, window=window)
        for i in range(n):
            if total - n + i - window + 1 >= min(80, max_kv):
                assert (got["out"][i] == 0).all() and (got["lse"][i] == -math.inf).all(), (total, window, i)
            else:
                assert got["out"][i].isfinite().all() and got["lse"][i].isfinite().all() and (got["out"][i] != 0).any(), (total, window, i)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("scale", [2e-38, -3e-38, 1e-39, -5e-40])
def test_scales_below_the_smallest_normal_ones(q, fmt, n, scale):
    """Scores of up to 2^126 before they are scaled: in both kernels the scale counts as it is.  Its product with log2 e is then a subnormal number, and so is
    that with a key's scale (0.13 or more here): half a step of 2^-149 on each."""
    m = make(q, fmt, [(n, n + 30)], 4, 2, 64, 16, 3)
    if fmt == "bf16":
        m["query"] = (m["query"].float() * 2.0 ** 60).to(torch.bfloat16)
        k = (m["host"][0][0].float() * 2.0 ** 61).to(torch.bfloat16)
        m["host"][0] = (k, None)
        m["c"].k.copy_(k)
    else:                                                   # codes of up to 448 and scales of about 0.005
        m["query"] = (m["query"].float() * 2.0 ** 113).to(torch.bfloat16)
        sc = m["host"][0][1] * 2.0 ** 7
        m["host"][0] = (m["host"][0][0], sc)
        m["c"].k_scales.copy_(sc)
    got = call(q, m, scale=scale)
    low = 2.0 ** -149 / abs(scale) * (1 if fmt == "bf16" else 8)
    as_given = torch.tensor(scale, dtype=torch.float32).item()
    for i in range(n):
        k, ok = ref.cached(*m["host"][0], m["table"][0], n + 30, 16)
        v, _ = ref.cached(*m["host"][1], m["table"][0], n + 30, 16)
        o, e, mag, zerr = ref.attention(m["query"][i: i + 1, 1:5], k, v, ok, 31 + i, as_given, 0)
        top = zerr[0] / ((64 + 8) * ref.F32)                # the scores' own size
        err = zerr[0] + low * top
        tol = mag[0] * (ref.HALF_BF16 + 2 * err[:, None] + 2.0 ** -19) + o[0].abs() * 1.01 * ref.HALF_BF16
        assert ((got["out"][i].double().cpu() - o[0]).abs() <= tol).all(), (i, float(top.max()))
        assert ((got["lse"][i].double().cpu() - e[0]).abs() <= err + 2.0 ** -19 * (1 + e[0].abs())).all(), (i, float(top.max()))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(65, 1, 64), (96, 1, 128), (160, 2, 64), (256, 1, 64)])
def test_more_query_heads_per_cached_one_than_few_rows_hold(q, fmt, heads, kv_heads, dim):
    """Single tokens whose heads alone are more than the kernel for few rows takes, and up to a whole row block per token."""
    seqs = [(1, 1), (1, 700), (3, 65), (0, 9), (1, 0), (2, 1300)]
    m = make(q, fmt, seqs, heads, kv_heads, dim, 16, heads)
    check(m, call(q, m))
    m = make(q, fmt, [(1, 3000), (1, 40)], heads, kv_heads, dim, 16, heads + 1)
    check(m, call(q, m, window=700), window=700)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("max_q,max_kv", [(1, 20000), (2, 700), (64, 20000), (2048, 1 << 20), (1 << 30, 1 << 24)])
def test_bounds_that_no_sequence_reaches(q, fmt, max_q, max_kv):
    """max_q_len and max_kv_len as a server names them, once and for all: the results stay within the same bound."""
    seqs = [(1, 600), (1, 33), (1, 0), (1, 1)] if max_q == 1 else [(1, 600), (2, 33), (0, 4), (2, 130)]
    m = make(q, fmt, seqs, 16, 2, 64, 16, 61)
    got = q.qarl_paged_attention(m["query"].cuda()[:, 1:17], m["c"], m["table"].cuda(), m["kv_lens"].cuda(), m["offsets"].cuda(), max_q, max_kv, want_lse=True)
    check(m, got)
    many = make(q, fmt, [(70, 300), (1, 900), (5, 5)], 16, 2, 64, 16, 62)
    if max_q > 70:
        check(many, q.qarl_paged_attention(many["query"].cuda()[:, 1:17], many["c"], many["table"].cuda(), many["kv_lens"].cuda(), many["offsets"].cuda(), max_q,
                                           max_kv, window=100, want_lse=True), window=100)
