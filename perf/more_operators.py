"""What a rollout step needs beside its experts, norms and 16- or 8-bit caches, as measured calls: rotary positions (and their gradient), keys and
values appended to the paged cache with the rotation on the way, a cache held in 4 bits with the attention over it, and the choice of the next token.

listed() names the cases, draw() gives more of the same ranges, prepare() makes what a program holds before the call,
run() is one pass (the framework's kernels where `own` is true, elementary torch operations where it is false), work() the
bytes and operations a pass cannot do without, exact() the same outputs from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

HEADS = dict(heads=32, kv_heads=4, dim=128)     # the layer's attention: 32 query heads over 4 cached ones
PROMPT, RESPONSE = 2048, 16384                  # longest prompt and response of a rollout
VOCAB = 151936
E4M3_MAX = 448.0
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # the learner's forward over 8 sequences x 2048 tokens: queries and keys are slices of one projection
        dict(HEADS, name="rotary_16384tok", kind="rotary", rows=16384, rot=128, layout="half", scaling="none", type="bf16", inverse=False, far=PROMPT, sliced=True),
        # gradients in 32 bits of a ragged batch over far positions: part of the head rotated, pairs side by side, frequencies stretched for long contexts
        dict(name="rotary_backward_f32_1733tok", kind="rotary", heads=28, kv_heads=4, dim=128, rows=1733, rot=64, layout="pairs", scaling="yarn", type="f32",
             inverse=True, far=130000, sliced=False),
        # one decode step of an ordinary rollout batch: a token per sequence, each to a page of its own
        dict(HEADS, name="append_fp8_256tok", kind="append", fmt="fp8", rows=256, page=16, scattered=True, skipped=3, rot=128, layout="half", scaling="none",
             far=PROMPT + RESPONSE),
        # prompts being filled in, 16-bit cache
        dict(HEADS, name="append_bf16_16384tok", kind="append", fmt="bf16", rows=16384, page=16, scattered=False, skipped=0, rot=128, layout="half",
             scaling="linear", far=PROMPT),
        # short prompts of a ragged batch filled into a 4-bit cache, which another engine then gets in 16 bits
        dict(HEADS, name="store_read_fp4_37seq", kind="store", fmt="fp4", seqs=37, len_min=1, len_max=110, page=16, rot=128, layout="half", scaling="none", lens=1),
        # the last of a batch still being generated: a single token over the longest context, 4-bit cache
        dict(HEADS, name="attention_fp4_1tok_18432", kind="attention", fmt="fp4", seqs=1, q_min=1, q_max=1, ctx_min=PROMPT + RESPONSE - 1,
             ctx_max=PROMPT + RESPONSE - 1, window=0, idle=0, page=16, lens=2),
        # one decode step of a rollout batch at all stages of its responses
        dict(HEADS, name="attention_fp4_256tok", kind="attention", fmt="fp4", seqs=256, q_min=1, q_max=1, ctx_min=0, ctx_max=PROMPT + RESPONSE - 1,
             window=0, idle=5, page=16, lens=3),
        # chunks of prompts beside single tokens, over contexts of all lengths: continuous batching of a model with 28 heads over 4
        dict(name="attention_fp4_chunks", kind="attention", heads=28, kv_heads=4, dim=128, fmt="fp4", seqs=12, q_min=1, q_max=700, ctx_min=0,
             ctx_max=8192, window=0, idle=0, page=32, lens=5),
        # one sequence being generated: the usual truncation, latency alone
        dict(name="sample_1tok", kind="sample", rows=1, vocab=VOCAB, type="bf16", flat=False, pad=0, masked=0.0, ways="usual"),
        # a decode step of rollouts for training: the whole softmax at temperature 1
        dict(name="sample_256tok_whole", kind="sample", rows=256, vocab=VOCAB, type="bf16", flat=False, pad=0, masked=0.0, ways="whole"),
        # a served batch whose requests ask for different things, some of them greedy
        dict(name="sample_256tok_mixed", kind="sample", rows=256, vocab=VOCAB, type="bf16", flat=False, pad=0, masked=0.0, ways="mixed"),
        # logits in 32 bits of an odd vocabulary in padded rows, flat, most tokens excluded by a grammar
        dict(name="sample_f32_37tok_masked", kind="sample", rows=37, vocab=32003, type="f32", flat=True, pad=61, masked=0.6, ways="mixed"),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "store", "attention", "attention", "attention", "sample", "sample", "sample"])
    if kind == "sample":
        vocab = _log_uniform(rng, 100, 160000)
        return dict(kind=kind, rows=_log_uniform(rng, 1, min(1024, max(1, (VOCAB * 256) // vocab))), vocab=vocab, type=rng.choice(["bf16", "bf16", "f32"]),
                    flat=rng.random() < 0.3, pad=rng.choice([0, 0, rng.randint(1, 200)]), masked=rng.choice([0.0, 0.0, 0.5, 0.97]),
                    ways=rng.choice(["usual", "whole", "mixed", "mixed"]))
    kv_heads = rng.choice([1, 2, 4, 4, 8])
    group = rng.choice([1, 2, 4, 6, 7, 8, 8, 12, 16])
    c = dict(kind=kind, heads=kv_heads * group, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]))
    if kind != "attention":
        c.update(layout=rng.choice(["half", "half", "pairs"]), scaling=rng.choice(["none", "none", "linear", "yarn", "bands"]))
        if kind == "rotary":
            c["dim"] = rng.choice([64, 80, 96, 128, 128, 192, 256])
        c["rot"] = c["dim"] if rng.random() < 0.6 else 16 * rng.randint(1, c["dim"] // 16)
    row = kv_heads * c["dim"]
    if kind == "rotary":
        per = (c["heads"] + kv_heads) * c["dim"]
        c.update(rows=_log_uniform(rng, 1, min(30000, (72 << 20) // per)), type=rng.choice(["bf16", "bf16", "f32"]), inverse=rng.random() < 0.4,
                 far=_log_uniform(rng, 1, 1 << 20), sliced=rng.random() < 0.5)
        if c["type"] == "f32":
            c["rows"] = max(1, c["rows"] // 2)
        return c
    c["page"] = rng.choice([8, 16, 16, 32, 64, 128])
    if kind == "append":
        per = (c["heads"] + 2 * kv_heads) * c["dim"]
        c.update(fmt=rng.choice(["bf16", "fp8"]), rows=_log_uniform(rng, 1, min(30000, (72 << 20) // per)), scattered=rng.random() < 0.5, far=_log_uniform(rng, 1, 1 << 20))
        c["skipped"] = rng.choice([0, 0, min(c["rows"], rng.randint(1, 9))])
        return c
    c["lens"] = rng.randint(10, 1 << 30)
    c["fmt"] = "fp4"
    if kind == "store":
        total = (1 << 20) // row
        c["seqs"] = _log_uniform(rng, 1, min(60, max(1, total // 2)))
        c["len_max"] = _log_uniform(rng, 1, max(1, total // c["seqs"]))
        c["len_min"] = rng.randint(1, c["len_max"])
        return c
    # attention: single tokens, a few of them, or chunks; bounded by the padded scores and caches that the plain form makes
    step = rng.choice(["one", "one", "few", "chunk", "chunk"])
    c["seqs"] = _log_uniform(rng, 1, 256 if step != "chunk" else 24)
    c["q_max"] = {"one": 1, "few": rng.randint(2, 9), "chunk": _log_uniform(rng, 10, 2048)}[step]
    c["q_min"] = c["q_max"] if step == "one" or rng.random() < 0.4 else rng.randint(0, c["q_max"])
    most = min(PROMPT + RESPONSE, (500 << 20) // (c["seqs"] * row), (1 << 29) // (c["seqs"] * c["q_max"] * c["heads"]))
    if most <= c["q_max"]:
        c["seqs"] = max(1, c["seqs"] * most // (4 * c["q_max"]))
        most = min(PROMPT + RESPONSE, (500 << 20) // (c["seqs"] * row), (1 << 29) // (c["seqs"] * c["q_max"] * c["heads"]))
    most = max(most, c["q_max"])
    c["ctx_max"] = _log_uniform(rng, 1, most - c["q_max"] + 1) - 1 if rng.random() < 0.7 else most - c["q_max"]
    c["ctx_min"] = c["ctx_max"] if rng.random() < 0.3 else rng.randint(0, c["ctx_max"])
    c["window"] = 0 if rng.random() < 0.7 else _log_uniform(rng, 1, c["ctx_max"] + c["q_max"])
    c["idle"] = rng.choice([0, 0, 1, 2]) if c["seqs"] > 2 else 0
    return c


# ---- lengths of a case (the same for every seed: the work of a case is known from the case) ----

def _lens(case):
    """attention: [(new tokens, cached tokens with the new ones)] of each sequence; store: [tokens]."""
    rng = random.Random(case["lens"])
    if case["kind"] == "store":
        return [rng.randint(case["len_min"], case["len_max"]) for _ in range(case["seqs"])]
    got = []
    for i in range(case["seqs"]):
        n = rng.randint(case["q_min"], case["q_max"])
        got.append((n, rng.randint(case["ctx_min"], case["ctx_max"]) + n))
    got[0] = (case["q_max"], got[0][1] - got[0][0] + case["q_max"])
    for i in rng.sample(range(1, case["seqs"]), case["idle"]) if case["idle"] else []:
        got[i] = (got[i][0], 0)                 # a slot of the batch without a sequence: nothing to attend to
    return got


def _seen(case, n, total):
    """(visible (query, token) pairs of a sequence, tokens that at least one query sees)"""
    if total < n or n == 0:
        return 0, 0                             # an idle slot
    w = case["window"] or total
    first = total - n                           # position of the first new token
    full = max(0, min(n, w - 1 - first))        # queries that see everything in front of them
    pairs = full * first + full * (full + 1) // 2 + (n - full) * w
    return pairs, total - max(0, first - w + 1)


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std)


def _quantized_rows(x):
    """(e4m3 codes, one scale a row) of fp32 rows: scale = absmax / 448, code = e4m3(x / scale)"""
    scale = x.abs().amax(-1) / E4M3_MAX
    unit = torch.where(scale > 0, scale, torch.ones_like(scale))
    return (x / unit[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def _packed_rows(x):
    """(e2m1 codes, two a byte, and four scale bytes a row) of fp32 rows.  Scale: the smallest power of two whose sixfold reaches the quarter row's absmax;
    code: nearest, ties to even."""
    quarters = x.view(*x.shape[:-1], 4, x.shape[-1] // 4)
    absmax = quarters.abs().amax(-1)
    mantissa, exponent = torch.frexp(absmax)
    e = torch.where(mantissa <= 0.75, exponent - 3, exponent - 2).clamp(-100, 125)
    e = torch.where(absmax > 0, e, torch.full_like(e, -100))
    t = torch.ldexp(quarters, -e[..., None])
    a = t.abs()
    code = (a > 0.25).int()
    for border, included in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if included else (a > border)
    code = (code + 8 * (t < 0)).to(torch.uint8).view(*x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _cache(g, case, pages):
    """A cache whose pages have been in use: keys with a common direction, values with a mean per channel, as trained layers have."""
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    st = dict(fmt=case["fmt"], pages=pages, page=case["page"], kv_heads=case["kv_heads"], dim=case["dim"])
    for name in ("k", "v"):
        if case["fmt"] == "fp4":
            # pages of codes and scales as the quantizer leaves them: a normal row's codes, scales around the row's size
            if case["kind"] == "store":
                st[name] = torch.zeros(shape[:3] + (case["dim"] // 2,), dtype=torch.uint8, device="cuda")
                st[name + "_scales"] = torch.full(shape[:3] + (4,), 27, dtype=torch.uint8, device="cuda")
                continue
            st[name] = torch.empty(shape[:3] + (case["dim"] // 2,), dtype=torch.uint8, device="cuda")
            st[name + "_scales"] = torch.empty(shape[:3] + (4,), dtype=torch.uint8, device="cuda")
            mean = _normal(g, (1, case["kv_heads"], 1, case["dim"]), 0.5)
            step = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
            for at in range(0, pages, step):
                n = min(step, pages - at)
                st[name][at: at + n], st[name + "_scales"][at: at + n] = _packed_rows(_normal(g, (n,) + shape[1:]).add_(mean))
            continue
        x = _normal(g, shape).add_(_normal(g, (1, case["kv_heads"], 1, case["dim"]), 0.5))
        if case["fmt"] == "fp8":
            codes, st[name + "_scales"] = _quantized_rows(x)
            st[name] = codes.view(torch.uint8)
        else:
            st[name] = x.to(torch.bfloat16)
            st[name + "_scales"] = None
    return st


def _table(g, case, lens):
    """Pages of each sequence, drawn without order from a cache somewhat larger than they need; -1 where a sequence has none."""
    page = case["page"]
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 7
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    width = max(1, max(need))
    count = torch.tensor(need, device="cuda")
    first = torch.cumsum(count, 0) - count
    col = torch.arange(width, device="cuda")
    at = (first[:, None] + col).clamp(max=pages - 1)
    table = torch.where(col < count[:, None], perm[at], torch.full_like(perm[at], -1)).contiguous()
    return table, pages


def _offsets(lens):
    t = torch.tensor([0] + list(lens), dtype=torch.int64)
    return torch.cumsum(t, 0).to(torch.int32).cuda()


def _frequencies(case):
    """(radians a position of each pair, in 64 bits; what the rotated pairs are multiplied by)"""
    rot = case["rot"]
    base, factor, original = 1e6, 8.0, 4096.0
    i = torch.arange(rot // 2, dtype=torch.float64)
    f = base ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "yarn":       # pairs that turn often within the original length keep their frequency, slow ones are stretched
        def pair_of(turns):
            return rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rot - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0
    if case["scaling"] == "bands":      # the same between 1 and 4 turns, by the turns themselves
        s = ((original * f / (2 * math.pi) - 1.0) / 3.0).clamp(0, 1)
        return f * s + f / factor * (1 - s), 1.0
    return f, 1.0


def _rope(st, case):
    f, amplitude = _frequencies(case)
    st.update(frequencies=f.cuda(), amplitude=amplitude, rot=case["rot"], layout=case["layout"], scaling=case["scaling"])


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    if kind == "sample":
        return _prepare_sample(case, g)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if kind == "rotary":
        rows, dt = case["rows"], torch.float32 if case["type"] == "f32" else torch.bfloat16
        start = int(torch.randint(0, case["far"], (1,), generator=g, device="cuda")) if case["far"] > PROMPT else 0
        positions = (start + torch.arange(rows, device="cuda")) % case["far"]
        x = _normal(g, (rows, heads + 2 * kv_heads, dim), 1e-3 if case["inverse"] else 1.0).to(dt)
        q, k = x[:, :heads], x[:, heads: heads + kv_heads]
        if not case["sliced"]:
            q, k = q.contiguous(), k.contiguous()
        st = dict(kind=kind, q=q, k=k, positions=positions, inverse=case["inverse"], q_out=torch.empty((rows, heads, dim), dtype=dt, device="cuda"),
                  k_out=torch.empty((rows, kv_heads, dim), dtype=dt, device="cuda"))
        _rope(st, case)
        return st
    if kind == "append":
        rows, page = case["rows"], case["page"]
        if case["scattered"]:       # decode: every token in a page of its own
            pages = rows + 5
            slots = torch.randperm(pages, generator=g, device="cuda")[:rows] * page + torch.randint(0, page, (rows,), generator=g, device="cuda")
            positions = torch.randint(0, case["far"], (rows,), generator=g, device="cuda")
        else:                       # prefill: pages filled one behind the other, in no order
            pages = -(-rows // page) + 5
            at = torch.arange(rows, device="cuda")
            slots = torch.randperm(pages, generator=g, device="cuda")[at // page] * page + at % page
            positions = at % case["far"]
        if case["skipped"]:         # tokens that pad the batch
            slots[torch.randperm(rows, generator=g, device="cuda")[: case["skipped"]]] = -1
        st = _cache(g, case, pages)
    elif kind == "store":
        lens = _lens(case)
        table, pages = _table(g, case, lens)
        st = _cache(g, case, pages)
        rows = sum(lens)
        offsets = _offsets(lens)
        positions = torch.cat([torch.arange(n, device="cuda") for n in lens])
        seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
        slots = table[seq, positions // case["page"]].long() * case["page"] + positions % case["page"]
        st.update(table=table, offsets=offsets, total=rows)
        for name in ("k_out", "v_out"):
            st[name] = torch.empty((rows, kv_heads, dim), dtype=torch.bfloat16, device="cuda")
    else:
        lens = _lens(case)
        table, pages = _table(g, case, [total for _, total in lens])
        st = _cache(g, case, pages)
        rows = sum(n for n, _ in lens)
        qkv = _normal(g, (rows, heads + 2 * kv_heads, dim), 1.5).to(torch.bfloat16)   # the queries are a slice of one projection's rows
        st.update(kind=kind, q=qkv[:, :heads], table=table, q_offsets=_offsets([n for n, _ in lens]), rows=rows,
                  kv_lens=torch.tensor([total for _, total in lens], dtype=torch.int32, device="cuda"), max_q=max(n for n, _ in lens),
                  max_kv=max(1, max(total for _, total in lens)), scale=dim ** -0.5, window=case["window"],
                  out=torch.empty((rows, heads, dim), dtype=torch.bfloat16, device="cuda"),
                  lse=torch.empty((rows, heads), dtype=torch.float32, device="cuda"))
        return st
    # q, k and v are slices of one projection's rows
    qkv = _normal(g, (rows, heads + 2 * kv_heads, dim)).mul_(torch.exp(_normal(g, (rows, 1, 1), 0.7))).to(torch.bfloat16)
    st.update(kind=kind, q=qkv[:, :heads], new_k=qkv[:, heads: heads + kv_heads], new_v=qkv[:, heads + kv_heads:], slots=slots.to(torch.int64), positions=positions,
              q_out=torch.empty((rows, heads, dim), dtype=torch.bfloat16, device="cuda"))
    _rope(st, case)
    return st


def _prepare_sample(case, g):
    rows, vocab = case["rows"], case["vocab"]
    logits = _normal(g, (rows, vocab), 0.5 if case["flat"] else 2.2)
    if not case["flat"]:        # a few candidates stand out, in some rows one alone
        at = torch.randint(0, vocab, (rows, 48), generator=g, device="cuda")
        lift = 4.0 - 2.5 * torch.log(torch.rand((rows, 48), generator=g, device="cuda").clamp(min=1e-6))
        logits.scatter_add_(1, at, lift * torch.rand((rows, 1), generator=g, device="cuda"))
    if case["masked"]:
        out = torch.rand((rows, vocab), generator=g, device="cuda") < case["masked"]
        out[:, 0] = False
        logits.masked_fill_(out, float("-inf"))
    logits = logits.to(torch.float32 if case["type"] == "f32" else torch.bfloat16)
    if case["pad"]:
        wide = torch.zeros((rows, vocab + case["pad"]), dtype=logits.dtype, device="cuda")
        wide[:, :vocab] = logits
        logits = wide[:, :vocab]
    st = dict(kind="sample", logits=logits, u=torch.rand((rows,), generator=g, device="cuda"), temperature=None, top_k=None, top_p=None, min_p=None,
              token=torch.empty((rows,), dtype=torch.int32, device="cuda"), logprob=torch.empty((rows,), device="cuda"), kept_logprob=torch.empty((rows,), device="cuda"))
    if case["ways"] == "usual":
        st.update(temperature=torch.full((rows,), 0.6, device="cuda"), top_k=torch.full((rows,), 20, dtype=torch.int32, device="cuda"),
                  top_p=torch.full((rows,), 0.95, device="cuda"))
    elif case["ways"] == "mixed":
        def some(share, values, otherwise):
            return torch.where(torch.rand((rows,), generator=g, device="cuda") < share, values, torch.full_like(values, otherwise))
        unit = lambda: torch.rand((rows,), generator=g, device="cuda")      # noqa: E731
        st.update(temperature=some(0.95, 0.3 + 1.2 * unit(), 0.0), top_k=some(0.4, torch.exp(7.0 * unit()), 0.0).to(torch.int32), top_p=some(0.7, 0.5 + 0.5 * unit(), 1.0),
                  min_p=some(0.3, 0.2 * unit(), 0.0))
    return st


# ---- one pass ----

def run(state):
    if own:
        return _run_own(state)
    return {"rotary": _rotary, "append": _append, "store": _store, "attention": _attention, "sample": _sample}[state["kind"]](state)


def _run_own(st):
    from paper_2604_07853_amd import binding as q
    kind = st["kind"]
    if kind == "sample":
        r = q.qarl_sample(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"], token=st["token"],
                          logprob=st["logprob"], kept_logprob=st["kept_logprob"])
        return dict(token=r["token"], logprob=r["logprob"], kept_logprob=r["kept_logprob"])
    if kind != "attention" and "rope" not in st:      # the frequencies, which a program makes once
        layout = q.QARL_ROPE_PAIRS if st["layout"] == "pairs" else q.QARL_ROPE_HALF
        scaling = dict(none=q.QARL_ROPE_PLAIN, linear=q.QARL_ROPE_LINEAR, yarn=q.QARL_ROPE_YARN, bands=q.QARL_ROPE_BANDS)[st["scaling"]]
        low, high = (1.0, 4.0) if st["scaling"] == "bands" else (1.0, 32.0)
        st["rope"] = q.Rope(st["rot"], base=1e6, layout=layout, scaling=scaling, factor=8.0, original_len=4096, low=low, high=high)
    if kind == "rotary":
        r = q.qarl_rotary(st["rope"], st["positions"], st["q"], st["k"], inverse=st["inverse"], q_out=st["q_out"], k_out=st["k_out"])
        return dict(q=r["q"], k=r["k"])
    if "handle" not in st:      # the descriptor of the cache, which a program makes once
        fmt = dict(bf16=q.QARL_KV_BF16, fp8=q.QARL_KV_E4M3, fp4=q.QARL_KV_E2M1)[st["fmt"]]
        st["handle"] = q.KVCache(fmt, st["k"], st["v"], st["k_scales"], st["v_scales"])
    cache = st["handle"]
    if kind == "attention":
        r = q.qarl_paged_attention(st["q"], cache, st["table"], st["kv_lens"], st["q_offsets"], st["max_q"], st["max_kv"], scale=st["scale"],
                                   window=st["window"], out=st["out"], lse=st["lse"])
        return dict(out=r["out"], lse=r["lse"])
    query = q.qarl_rotary_kv_write(cache, st["rope"], st["positions"], st["q"], st["new_k"], st["new_v"], st["slots"], q_out=st["q_out"])
    if kind == "append":
        return dict(_cache_values(st), q=query)
    k, v = q.qarl_kv_cache_read(cache, st["table"], st["offsets"], st["total"], out=(st["k_out"], st["v_out"]))
    return dict(q=query, k=k, v=v)


def _cache_values(st):
    if st["fmt"] == "fp8":
        return dict(k=st["k"].view(torch.float8_e4m3fn), v=st["v"].view(torch.float8_e4m3fn), k_scales=st["k_scales"], v_scales=st["v_scales"])
    return dict(k=st["k"], v=st["v"])


def _rotated(st, x, inverse=False):
    """x [rows, heads, dim] rotated, in 32 bits; the angles of far positions in 64."""
    angle = st["positions"].double()[:, None] * st["frequencies"]
    cos, sin = (torch.cos(angle) * st["amplitude"]).float()[:, None], (torch.sin(angle) * st["amplitude"]).float()[:, None]
    if inverse:
        sin = -sin
    x = x.float()
    y = x.clone()
    rot = st["rot"]
    if st["layout"] == "pairs":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y[..., : rot // 2], y[..., rot // 2: rot] = a * cos - b * sin, b * cos + a * sin
    return y


def _rotary(st):
    dt = st["q"].dtype
    return dict(q=_rotated(st, st["q"], st["inverse"]).to(dt), k=_rotated(st, st["k"], st["inverse"]).to(dt))


def _write(st):
    """The new keys, rotated, and values into their slots."""
    keep = st["slots"] >= 0
    slots = st["slots"][keep]
    page, off = slots // st["page"], slots % st["page"]
    for name, x in (("k", _rotated(st, st["new_k"])[keep]), ("v", st["new_v"][keep].float())):
        if st["fmt"] == "fp8":
            codes, scales = _quantized_rows(x)
            st[name][page, :, off] = codes.view(torch.uint8)
            st[name + "_scales"][page, :, off] = scales
        elif st["fmt"] == "fp4":
            st[name][page, :, off], st[name + "_scales"][page, :, off] = _packed_rows(x)
        else:
            st[name][page, :, off] = x.to(torch.bfloat16)


def _append(st):
    _write(st)
    return dict(_cache_values(st), q=_rotated(st, st["q"]).to(torch.bfloat16))


def _wide(st, name, index):
    """Cached rows st[name][index] of the 4-bit cache in 32 bits."""
    code, scale = st[name][index], st[name + "_scales"][index]
    value = torch.tensor(E2M1 + [-x for x in E2M1], device="cuda")
    both = torch.stack([value[(code & 15).int()], value[(code >> 4).int()]], -1).view(*code.shape[:-1], 4, -1)
    return torch.ldexp(both, scale[..., None].int() - 127).view(*code.shape[:-1], -1)


def _store(st):
    _write(st)
    at = torch.arange(st["total"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(st["offsets"], at, right=True) - 1
    pos = at - st["offsets"][seq]
    page, off = st["table"][seq, pos // st["page"]].long(), (pos % st["page"]).long()
    index = (page[:, None], torch.arange(st["kv_heads"], device="cuda")[None, :], off[:, None])
    return dict(q=_rotated(st, st["q"]).to(torch.bfloat16), k=_wide(st, "k", index).to(torch.bfloat16), v=_wide(st, "v", index).to(torch.bfloat16))


def _attention(st):
    """All sequences at once, padded to the longest chunk and the longest context."""
    seqs, heads, kv_heads, dim = st["table"].shape[0], st["q"].shape[1], st["kv_heads"], st["dim"]
    group, max_q, max_kv = heads // kv_heads, st["max_q"], st["table"].shape[1] * st["page"]
    begin = st["q_offsets"][:-1].long()
    n = st["q_offsets"][1:].long() - begin
    i = torch.arange(max_q, device="cuda")
    row = begin[:, None] + i
    real = i < n[:, None]
    q = st["q"].float()[row.clamp(max=max(0, st["rows"] - 1))]                                          # [seqs, max_q, heads, dim]
    q = q.view(seqs, max_q, kv_heads, group, dim).permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, max_q * group, dim)
    pages = st["table"].clamp(min=0).long()
    k = _wide(st, "k", pages).permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, max_kv, dim)
    z = torch.matmul(q, k.transpose(2, 3)).mul_(st["scale"])                                            # [seqs, kv_heads, max_q * group, max_kv]
    del k
    j = torch.arange(max_kv, device="cuda")
    pos = st["kv_lens"].long()[:, None] - n[:, None] + i                                                # position of each query
    sees = (j <= pos[:, :, None]) & (j < st["kv_lens"].long()[:, None, None])
    if st["window"]:
        sees &= j > pos[:, :, None] - st["window"]
    sees = sees[:, None, :, None, :].expand(seqs, 1, max_q, group, max_kv).reshape(seqs, 1, max_q * group, max_kv)
    z.masked_fill_(~sees, float("-inf"))
    m = z.amax(-1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    p = z.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    v = _wide(st, "v", pages).permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, max_kv, dim)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (m + torch.log(total))[..., 0]
    o = o.view(seqs, kv_heads, max_q, group, dim).permute(0, 2, 1, 3, 4).reshape(seqs, max_q, heads, dim)
    lse = lse.view(seqs, kv_heads, max_q, group).permute(0, 2, 1, 3).reshape(seqs, max_q, heads)
    st["out"][row[real]] = o[real].to(torch.bfloat16)
    st["lse"][row[real]] = lse[real]
    return dict(out=st["out"], lse=st["lse"])


def _sample(st):
    """Tokens in the order of their logits (equal ones by index); weights in 64 bits: a random number may fall next to a border of the sums."""
    rows, vocab = st["logits"].shape
    z, index = torch.sort(st["logits"].float(), dim=1, descending=True, stable=True)
    t = torch.ones((rows,), device="cuda") if st["temperature"] is None else st["temperature"]
    greedy = t == 0
    scaled = (z.double() - z[:, :1].double()) / torch.where(greedy, torch.ones_like(t), t).double()[:, None]
    w = torch.exp(scaled)
    whole = w.sum(1)
    rank = torch.arange(vocab, device="cuda")
    keep = w > 0
    if st["top_k"] is not None:
        k = torch.where(st["top_k"] > 0, st["top_k"], torch.full_like(st["top_k"], vocab))
        keep &= rank < k[:, None]
    total = torch.where(keep, w, 0.0).cumsum(1)
    if st["top_p"] is not None:
        keep &= (total - w < st["top_p"].double()[:, None] * total[:, -1:]) | (st["top_p"] >= 1)[:, None]
    if st["min_p"] is not None:
        keep &= w >= st["min_p"].double()[:, None]
    keep &= ~greedy[:, None] | (rank == 0)
    keep[:, 0] = True
    total = torch.where(keep, w, 0.0).cumsum(1)
    place = (total <= st["u"].double()[:, None] * total[:, -1:]).sum(1)
    place = torch.minimum(place, keep.sum(1) - 1)[:, None]
    at = scaled.gather(1, place)[:, 0]
    return dict(token=index.gather(1, place)[:, 0].int(), logprob=(at - torch.log(whole)).float(), kept_logprob=(at - torch.log(total[:, -1])).float())


# ---- bytes and operations a pass cannot do without ----

def work(case):
    kind = case["kind"]
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4 if case["type"] == "f32" else 2) + 32 * case["rows"], "flops": 4 * n}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if kind == "rotary":
        n = case["rows"] * (heads + kv_heads)
        return {"bytes": n * dim * (8 if case["type"] == "f32" else 4) + 8 * case["rows"], "flops": 3 * n * case["rot"]}
    row = kv_heads * dim
    stored = {"bf16": 2 * row, "fp8": row + 4 * kv_heads, "fp4": row // 2 + 4 * kv_heads}[case["fmt"]]      # bytes of a token's keys (or values) in the cache
    if kind in ("append", "store"):
        rows = case["rows"] if kind == "append" else sum(_lens(case))
        written = rows - case.get("skipped", 0)
        queries = rows * heads * dim
        return {"bytes": 4 * queries + 2 * written * (2 * row + stored) + 16 * rows + (2 * rows * (stored + 2 * row) if kind == "store" else 0),
                "flops": 3 * (rows * heads + written * kv_heads) * case["rot"] + 4 * written * row}
    pairs, tokens, rows = 0, 0, 0
    for n, total in _lens(case):
        p, t = _seen(case, n, total)
        pairs, tokens, rows = pairs + p, tokens + t, rows + n
    return {"bytes": 2 * tokens * stored + rows * heads * (4 * dim + 4), "flops": 4 * dim * heads * pairs}


# ---- the definitions in 64 bits ----

def _exact_turned(case, positions, x, inverse=False):
    """Each pair as a complex number, turned by its angle."""
    f, amplitude = _frequencies(case)
    angle = positions.double()[:, None] * f.cuda()
    turn = torch.polar(torch.full_like(angle, amplitude), -angle if inverse else angle)[:, None]
    x = x.double()
    part, rest = x[..., : case["rot"]], x[..., case["rot"]:]
    if case["layout"] == "half":
        pair = part.reshape(*part.shape[:-1], 2, -1).transpose(-1, -2)
    else:
        pair = part.reshape(*part.shape[:-1], -1, 2)
    got = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
    if case["layout"] == "half":
        got = got.transpose(-1, -2)
    return torch.cat([got.reshape(part.shape), rest], -1)


def _e4m3_table():
    """The finite e4m3 values by code: 4 exponent bits (bias 7), 3 mantissa bits, subnormals below 2^-6."""
    vals = []
    for c in range(127):
        e, f = c >> 3, c & 7
        vals.append(f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10))
    return torch.tensor(vals, dtype=torch.float64, device="cuda")


def _exact_quantized(y):
    """(values of the e4m3 codes, scales) of 64-bit rows"""
    scale = y.abs().amax(-1, keepdim=True) / E4M3_MAX
    t = torch.where(scale > 0, y / scale, torch.zeros_like(y))
    a = t.abs()
    exponent = torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))
    exponent = torch.where(torch.exp2(exponent + 1) <= a, exponent + 1, exponent)
    step = torch.exp2(exponent.clamp(min=-6.0) - 3)
    return torch.sign(t) * (torch.round(a / step) * step).clamp(max=E4M3_MAX), scale[..., 0]


def _exact_packed(y):
    """What 64-bit rows are in e2m1 with a power-of-two scale for each quarter."""
    part = y.view(*y.shape[:-1], 4, -1)
    size = part.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2((size / 6).clamp(min=2.0 ** -100))))
    scale = torch.where(size > 6 * scale, 2 * scale, torch.where(size <= 3 * scale, scale / 2, scale)).clamp(min=2.0 ** -100, max=2.0 ** 125)
    a = (part / scale).abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.sign(part) * (torch.round(a / step) * step).clamp(max=6.0) * scale).view(y.shape)


def _exact_cached(st, name, index):
    code = st[name][index].long()
    value = torch.tensor([s * x for s in (1.0, -1.0) for x in E2M1], dtype=torch.float64, device="cuda")
    wide = torch.empty(code.shape[:-1] + (2 * code.shape[-1],), dtype=torch.float64, device="cuda")
    wide[..., 0::2] = value[code % 16]
    wide[..., 1::2] = value[code // 16]
    return wide * torch.exp2(st[name + "_scales"][index].double() - 127).repeat_interleave(wide.shape[-1] // 4, -1)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return _exact_sample(st)
    if kind == "rotary":
        return {n: _exact_turned(case, st["positions"], st[n], case["inverse"]) for n in ("q", "k")}
    if kind in ("append", "store"):
        got = dict(q=_exact_turned(case, st["positions"], st["q"]))
        new = dict(k=_exact_turned(case, st["positions"], st["new_k"]), v=st["new_v"].double())
        if kind == "store":     # every slot is written once, and read back in the order of the tokens
            return dict(got, **{n: _exact_packed(x.contiguous()) for n, x in new.items()})
        at = torch.nonzero(st["slots"] >= 0)[:, 0]
        where = st["slots"][at]
        for n, x in new.items():
            codes, scales = _exact_quantized(x) if case["fmt"] == "fp8" else (x, None)
            whole = (_e4m3_table()[(st[n] & 127).long()] * torch.where(st[n] >= 128, -1.0, 1.0).double()) if case["fmt"] == "fp8" else st[n].double()
            flat = whole.permute(0, 2, 1, 3).reshape(-1, case["kv_heads"], case["dim"])
            flat[where] = codes[at]
            got[n] = flat.view(-1, case["page"], case["kv_heads"], case["dim"]).permute(0, 2, 1, 3).contiguous()
            if scales is not None:
                flat = st[n + "_scales"].double().permute(0, 2, 1).reshape(-1, case["kv_heads"])
                flat[where] = scales[at]
                got[n + "_scales"] = flat.view(-1, case["page"], case["kv_heads"]).permute(0, 2, 1).contiguous()
        return got
    group = case["heads"] // case["kv_heads"]
    outs, lses = [], []
    start = 0
    for s, (n, total) in enumerate(_lens(case)):
        q = st["q"][start: start + n].double()
        start += n
        o = torch.zeros((n, case["heads"], case["dim"]), dtype=torch.float64, device="cuda")
        e = torch.full((n, case["heads"]), float("-inf"), dtype=torch.float64, device="cuda")
        if n and total >= n:
            pages = st["table"][s, : -(-total // case["page"])].long()
            keys, values = (_exact_cached(st, name, pages).permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, case["dim"])[:, :total] for name in ("k", "v"))
            pos = torch.arange(total - n, total, device="cuda")
            j = torch.arange(total, device="cuda")
            hidden = j[None, :] > pos[:, None]
            if case["window"]:
                hidden |= j[None, :] <= pos[:, None] - case["window"]
            for h in range(case["heads"]):
                z = (q[:, h] @ keys[h // group].T) * (case["dim"] ** -0.5)
                z[hidden] = float("-inf")
                e[:, h] = torch.logsumexp(z, 1)
                o[:, h] = torch.exp(z - e[:, h: h + 1]) @ values[h // group]
        outs.append(o)
        lses.append(e)
    return dict(out=torch.cat(outs), lse=torch.cat(lses))


def _exact_sample(st):
    """Row by row over its distinct logits, the largest first, each as often as it occurs."""
    rows, vocab = st["logits"].shape
    tokens, lps, kept_lps = [], [], []
    got = {n: (st[n].tolist() if st[n] is not None else [d] * rows) for n, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0), ("u", 0.0))}
    for r in range(rows):
        row = st["logits"][r].double()
        value, count = torch.unique(row[row > float("-inf")], return_counts=True)
        value, count = value.flip(0), count.flip(0)
        t = got["temperature"][r]
        y = (value - value[0]) / (t or 1.0)
        w, n = torch.exp(y), count.clone()
        log_all = torch.log((w * n).sum())
        if t == 0:
            n = torch.zeros_like(n)
            n[0] = 1
        if got["top_k"][r] > 0:
            n = torch.minimum(n, (got["top_k"][r] - (count.cumsum(0) - count)).clamp(min=0))
        mass = (w * n).cumsum(0)
        if got["top_p"][r] < 1:     # of a value's tokens those whose forerunners hold less than the share
            room = (got["top_p"][r] * mass[-1] - (mass - w * n)) / w
            n = torch.minimum(n, torch.ceil(room).clamp(min=0).nan_to_num(posinf=0.0).long())
        n = torch.where(w >= got["min_p"][r], n, 0)
        if n[0] == 0:
            n[0] = 1
        mass = (w * n).cumsum(0)
        goal = got["u"][r] * mass[-1]
        at = min(int((mass <= goal).sum()), int((n > 0).sum()) - 1)
        nth = min(int(torch.floor((goal - (mass[at] - w[at] * n[at])) / w[at]).clamp(min=0)), int(n[at]) - 1)
        tokens.append(int(torch.nonzero(row == value[at])[nth, 0]))
        lps.append(y[at] - log_all)
        kept_lps.append(y[at] - torch.log(mass[-1]))
    return dict(token=torch.tensor(tokens, dtype=torch.int32, device="cuda"), logprob=torch.stack(lps), kept_logprob=torch.stack(kept_lps))
