"""What surrounds the quantized experts in a decoder layer, as measured calls: residual addition with RMS norm (and its
backward), the paged KV cache (written quantized or plain, and read back) and the attention of new tokens over it.

listed() names the cases, draw() gives more of the same ranges, prepare() makes what a program holds before the call,
run() is one pass (the framework's kernels where `own` is true, elementary torch operations where it is false), work() the
bytes and operations a pass cannot do without, exact() the same outputs from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

HIDDEN = 2048                                   # hidden size of the layer the library is written around
HEADS = dict(heads=32, kv_heads=4, dim=128)     # its attention: 32 query heads over 4 cached ones
PROMPT, RESPONSE = 2048, 16384                  # longest prompt and response of a rollout
EPS = 1e-6
E4M3_MAX = 448.0


def listed():
    return [
        # one sequence being generated: the norm in front of a projection, latency alone
        dict(name="norm_1tok", kind="norm", rows=1, hidden=HIDDEN, stream="bf16", quant=False, pad=0),
        # the learner's forward over 8 sequences x 2048 tokens: the norm in front of W8A8 experts
        dict(name="norm_fp8_16384tok", kind="norm", rows=16384, hidden=HIDDEN, stream="bf16", quant=True, pad=0),
        # the same tokens in the learner's backward
        dict(name="norm_backward_16384tok", kind="norm_backward", rows=16384, hidden=HIDDEN, stream="bf16", pad=0),
        # a ragged batch of a wider model whose residual stream is kept in 32 bits
        dict(name="norm_backward_f32_1733tok", kind="norm_backward", rows=1733, hidden=4096, stream="f32", pad=0),
        # one decode step of an ordinary rollout batch: a token per sequence, each to a page of its own, k and v slices of one projection
        dict(HEADS, name="write_fp8_256tok", kind="write", fmt="fp8", rows=256, page=16, scattered=True, skipped=3),
        # prompts being filled in, 16-bit cache
        dict(HEADS, name="write_bf16_16384tok", kind="write", fmt="bf16", rows=16384, page=16, scattered=False, skipped=0),
        # 8 finished rollouts of the longest length handed on in 16 bits
        dict(HEADS, name="read_fp8_8x18432", kind="read", fmt="fp8", seqs=8, len_min=PROMPT + RESPONSE, len_max=PROMPT + RESPONSE, page=16, lens=0),
        # short prefixes of a ragged batch
        dict(HEADS, name="read_bf16_37seq", kind="read", fmt="bf16", seqs=37, len_min=1, len_max=500, page=16, lens=1),
        # the last of a batch still being generated: a single token over the longest context
        dict(HEADS, name="attention_1tok_18432", kind="attention", fmt="bf16", seqs=1, q_min=1, q_max=1, ctx_min=PROMPT + RESPONSE - 1,
             ctx_max=PROMPT + RESPONSE - 1, window=0, idle=0, page=16, lens=2),
        # one decode step of a rollout batch at all stages of its responses, quantized cache, some slots of the batch idle
        dict(HEADS, name="attention_256tok_fp8", kind="attention", fmt="fp8", seqs=256, q_min=1, q_max=1, ctx_min=0, ctx_max=PROMPT + RESPONSE - 1,
             window=0, idle=5, page=16, lens=3),
        # eight prompts filled in at once
        dict(HEADS, name="attention_8x2048", kind="attention", fmt="bf16", seqs=8, q_min=PROMPT, q_max=PROMPT, ctx_min=0, ctx_max=0, window=0,
             idle=0, page=16, lens=4),
        # chunks of prompts beside single tokens, over contexts of all lengths: continuous batching of a model with 28 heads over 4
        dict(name="attention_chunks_fp8", kind="attention", heads=28, kv_heads=4, dim=128, fmt="fp8", seqs=12, q_min=1, q_max=700, ctx_min=0,
             ctx_max=8192, window=0, idle=0, page=32, lens=5),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "write", "read", "attention", "attention", "attention"])
    if kind in ("norm", "norm_backward"):
        hidden = 8 * _log_uniform(rng, 16, 1024)
        c = dict(kind=kind, rows=_log_uniform(rng, 1, min(20000, (36 << 20) // hidden)), hidden=hidden, stream=rng.choice(["bf16", "bf16", "f32"]),
                 pad=8 * rng.choice([0, 0, rng.randint(1, 40)]))
        if kind == "norm":
            c["quant"] = rng.random() < 0.5
        return c
    kv_heads = rng.choice([1, 2, 4, 4, 8])
    group = rng.choice([1, 2, 4, 6, 7, 8, 8, 12, 16])
    c = dict(kind=kind, fmt=rng.choice(["bf16", "fp8"]), heads=kv_heads * group, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]),
             page=rng.choice([8, 16, 16, 32, 64, 128]), lens=rng.randint(10, 1 << 30))
    row = kv_heads * c["dim"]
    if kind == "write":
        c.update(rows=_log_uniform(rng, 1, min(30000, (8 << 20) // row)), scattered=rng.random() < 0.5)
        c["skipped"] = rng.choice([0, 0, min(c["rows"], rng.randint(1, 9))])
        return c
    if kind == "read":
        total = min(200000, (64 << 20) // row)
        c["seqs"] = _log_uniform(rng, 1, 300)
        c["len_max"] = _log_uniform(rng, 1, min(20000, max(1, total // c["seqs"])))
        c["len_min"] = rng.randint(0, c["len_max"])
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
    """attention: [(new tokens, cached tokens with the new ones)] of each sequence; read: [cached tokens]."""
    rng = random.Random(case["lens"])
    if case["kind"] == "read":
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
    pairs = 0
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


def _padded(t, pad):
    """The same rows, each `pad` elements further apart."""
    if not pad:
        return t
    wide = torch.zeros((t.shape[0], t.shape[1] + pad), dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def _quantized_rows(x):
    """(e4m3 codes, one scale a row) of fp32 rows: scale = absmax / 448, code = e4m3(x / scale)"""
    scale = x.abs().amax(-1) / E4M3_MAX
    unit = torch.where(scale > 0, scale, torch.ones_like(scale))
    return (x / unit[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def _cache(g, case, pages):
    """A cache whose pages have been in use: keys with a common direction, values with a mean per channel, as trained layers have."""
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    st = dict(fmt=case["fmt"], pages=pages, page=case["page"], kv_heads=case["kv_heads"], dim=case["dim"])
    for name in ("k", "v"):
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


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    if kind in ("norm", "norm_backward"):
        rows, hidden = case["rows"], case["hidden"]
        sd = torch.float32 if case["stream"] == "f32" else torch.bfloat16
        # a residual stream some layers deep: rows of different size, a few channels much larger than the others
        big = torch.ones(hidden, device="cuda")
        big[torch.randint(0, hidden, (max(1, hidden // 512),), generator=g, device="cuda")] = 20.0
        size = torch.exp(_normal(g, (rows, 1), 0.5))
        stream = _normal(g, (rows, hidden), 2.0).mul_(big).mul_(size)
        weight = _normal(g, (hidden,), 0.2).add_(1.0).to(torch.bfloat16)
        if kind == "norm":
            st = dict(kind=kind, x=_padded(_normal(g, (rows, hidden), 0.7).to(torch.bfloat16), case["pad"]), residual=_padded(stream.to(sd), case["pad"]),
                      weight=weight, quant=case["quant"], residual_out=torch.empty((rows, hidden), dtype=sd, device="cuda"))
            if case["quant"]:
                st["codes"] = torch.empty((rows, hidden), dtype=torch.uint8, device="cuda")
                st["scales"] = torch.empty((rows,), dtype=torch.float32, device="cuda")
            else:
                st["y"] = torch.empty((rows, hidden), dtype=torch.bfloat16, device="cuda")
            return st
        return dict(kind=kind, dy=_padded(_normal(g, (rows, hidden), 1e-3).to(torch.bfloat16), case["pad"]), h=_padded(stream.to(sd), case["pad"]),
                    dh=_padded(_normal(g, (rows, hidden), 1e-3).to(sd), case["pad"]), weight=weight)
    if kind == "write":
        rows, page, dim = case["rows"], case["page"], case["dim"]
        if case["scattered"]:       # decode: every token in a page of its own
            pages = rows + 5
            slots = torch.randperm(pages, generator=g, device="cuda")[:rows] * page + torch.randint(0, page, (rows,), generator=g, device="cuda")
        else:                       # prefill: pages filled one behind the other, in no order
            pages = -(-rows // page) + 5
            at = torch.arange(rows, device="cuda")
            slots = torch.randperm(pages, generator=g, device="cuda")[at // page] * page + at % page
        if case["skipped"]:         # tokens that pad the batch
            slots[torch.randperm(rows, generator=g, device="cuda")[: case["skipped"]]] = -1
        st = _cache(g, case, pages)
        # k and v are slices of one projection's rows
        qkv = _normal(g, (rows, case["heads"] + 2 * case["kv_heads"], dim)).mul_(torch.exp(_normal(g, (rows, 1, 1), 0.7))).to(torch.bfloat16)
        st.update(kind=kind, new_k=qkv[:, case["heads"]: case["heads"] + case["kv_heads"]], new_v=qkv[:, case["heads"] + case["kv_heads"]:], slots=slots.to(torch.int64))
        return st
    if kind == "read":
        lens = _lens(case)
        table, pages = _table(g, case, lens)
        st = _cache(g, case, pages)
        total = sum(lens)
        st.update(kind=kind, table=table, offsets=_offsets(lens), total=total)
        for name in ("k_out", "v_out"):
            st[name] = torch.empty((total, case["kv_heads"], case["dim"]), dtype=torch.bfloat16, device="cuda")
        return st
    lens = _lens(case)
    table, pages = _table(g, case, [total for _, total in lens])
    st = _cache(g, case, pages)
    rows = sum(n for n, _ in lens)
    qkv = _normal(g, (rows, case["heads"] + 2 * case["kv_heads"], case["dim"]), 1.5).to(torch.bfloat16)   # the queries are a slice of one projection's rows
    st.update(kind=kind, q=qkv[:, : case["heads"]], table=table, q_offsets=_offsets([n for n, _ in lens]), rows=rows,
              kv_lens=torch.tensor([total for _, total in lens], dtype=torch.int32, device="cuda"), max_q=max(n for n, _ in lens),
              max_kv=max(1, max(total for _, total in lens)), scale=case["dim"] ** -0.5, window=case["window"],
              out=torch.empty((rows, case["heads"], case["dim"]), dtype=torch.bfloat16, device="cuda"),
              lse=torch.empty((rows, case["heads"]), dtype=torch.float32, device="cuda"))
    return st


# ---- one pass ----

def run(state):
    if own:
        return _run_own(state)
    return {"norm": _norm, "norm_backward": _norm_backward, "write": _write, "read": _read, "attention": _attention}[state["kind"]](state)


def _run_own(st):
    from paper_2604_07853_amd import binding as q
    kind = st["kind"]
    if kind == "norm":
        if st["quant"]:
            r = q.qarl_add_rmsnorm(st["x"], st["weight"], EPS, residual=st["residual"], residual_out=st["residual_out"], codes=st["codes"], scales=st["scales"])
            return dict(codes=r["codes"].view(torch.float8_e4m3fn), scales=r["scales"], residual=r["residual"])
        r = q.qarl_add_rmsnorm(st["x"], st["weight"], EPS, residual=st["residual"], residual_out=st["residual_out"], y=st["y"])
        return dict(y=r["y"], residual=r["residual"])
    if kind == "norm_backward":
        r = q.qarl_add_rmsnorm_backward(st["dy"], st["h"], st["weight"], EPS, dh=st["dh"])
        return dict(dx=r["dx"], dw=r["dw"])
    if "handle" not in st:      # the descriptor of the cache, which a program makes once
        st["handle"] = q.KVCache(q.QARL_KV_E4M3 if st["fmt"] == "fp8" else q.QARL_KV_BF16, st["k"], st["v"], st["k_scales"], st["v_scales"])
    cache = st["handle"]
    if kind == "write":
        q.qarl_kv_cache_write(cache, st["new_k"], st["new_v"], st["slots"])
        return _cache_values(st)
    if kind == "read":
        k, v = q.qarl_kv_cache_read(cache, st["table"], st["offsets"], st["total"], out=(st["k_out"], st["v_out"]))
        return dict(k=k, v=v)
    r = q.qarl_paged_attention(st["q"], cache, st["table"], st["kv_lens"], st["q_offsets"], st["max_q"], st["max_kv"], scale=st["scale"],
                               window=st["window"], out=st["out"], lse=st["lse"])
    return dict(out=r["out"], lse=r["lse"])


def _cache_values(st):
    if st["fmt"] == "fp8":
        return dict(k=st["k"].view(torch.float8_e4m3fn), v=st["v"].view(torch.float8_e4m3fn), k_scales=st["k_scales"], v_scales=st["v_scales"])
    return dict(k=st["k"], v=st["v"])


def _norm(st):
    h = st["x"].float() + st["residual"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * st["weight"].float()
    if st["quant"]:
        codes, scales = _quantized_rows(y)
        return dict(codes=codes, scales=scales, residual=h.to(st["residual"].dtype))
    return dict(y=y.to(torch.bfloat16), residual=h.to(st["residual"].dtype))


def _norm_backward(st):
    dy, h = st["dy"].float(), st["h"].float()
    rstd = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    g = dy * st["weight"].float()
    dx = st["dh"].float() + rstd * (g - h * (rstd * rstd * (g * h).mean(-1, keepdim=True)))
    return dict(dx=dx.to(st["h"].dtype), dw=(dy * h * rstd).sum(0, dtype=torch.float64).float())


def _write(st):
    keep = st["slots"] >= 0
    slots = st["slots"][keep]
    page, off = slots // st["page"], slots % st["page"]
    for name in ("k", "v"):
        x = st["new_" + name][keep]
        if st["fmt"] == "fp8":
            codes, scales = _quantized_rows(x.float())
            st[name][page, :, off] = codes.view(torch.uint8)
            st[name + "_scales"][page, :, off] = scales
        else:
            st[name][page, :, off] = x
    return _cache_values(st)


def _wide(st, name, index):
    """Cached rows st[name][index] in 32 bits."""
    if st["fmt"] == "fp8":
        return st[name][index].view(torch.float8_e4m3fn).float() * st[name + "_scales"][index][..., None]
    return st[name][index].float()


def _read(st):
    at = torch.arange(st["total"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(st["offsets"], at, right=True) - 1
    pos = at - st["offsets"][seq]
    page, off = st["table"][seq, pos // st["page"]].long(), (pos % st["page"]).long()
    heads = torch.arange(st["kv_heads"], device="cuda")
    index = (page[:, None], heads[None, :], off[:, None])
    return dict(k=_wide(st, "k", index).to(torch.bfloat16), v=_wide(st, "v", index).to(torch.bfloat16))


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


# ---- bytes and operations a pass cannot do without ----

def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_backward"):
        n, s = case["rows"] * case["hidden"], 4 if case["stream"] == "f32" else 2
        if kind == "norm":
            return {"bytes": n * (2 + 2 * s + (1 if case["quant"] else 2)) + case["hidden"] * 2, "flops": 8 * n}
        return {"bytes": n * (2 + 3 * s) + case["hidden"] * 6, "flops": 14 * n}
    row = case["kv_heads"] * case["dim"]
    stored = row + 4 * case["kv_heads"] if case["fmt"] == "fp8" else 2 * row      # bytes of a token's keys (or values) in the cache
    if kind == "write":
        rows = case["rows"] - case["skipped"]
        return {"bytes": 2 * rows * (2 * row + stored) + 8 * case["rows"], "flops": 4 * rows * row}
    if kind == "read":
        total = sum(_lens(case))
        return {"bytes": 2 * total * (2 * row + stored), "flops": 2 * total * row}
    pairs, tokens, rows = 0, 0, 0
    for n, total in _lens(case):
        p, t = _seen(case, n, total)
        pairs, tokens, rows = pairs + p, tokens + t, rows + n
    return {"bytes": 2 * tokens * stored + rows * case["heads"] * (4 * case["dim"] + 4), "flops": 4 * case["dim"] * case["heads"] * pairs}


# ---- the definitions in 64 bits ----

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


def _exact_cached(st, name, index):
    if st["fmt"] != "fp8":
        return st[name][index].double()
    code = st[name][index]
    value = _e4m3_table()[(code & 127).long()]
    return torch.where(code >= 128, -value, value) * st[name + "_scales"][index].double()[..., None]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = st["x"].double() + st["residual"].double()
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["hidden"] + EPS) * st["weight"].double()
        if case["quant"]:
            codes, scales = _exact_quantized(y)
            return dict(codes=codes, scales=scales, residual=h)
        return dict(y=y, residual=h)
    if kind == "norm_backward":
        dy, h, w, dh = (st[n].double() for n in ("dy", "h", "weight", "dh"))
        hidden = case["hidden"]
        r = 1.0 / torch.sqrt((h * h).sum(1) / hidden + EPS)
        xhat = h * r[:, None]
        c = (dy * w * xhat).sum(1) / hidden
        return dict(dx=dh + r[:, None] * (dy * w - xhat * c[:, None]), dw=(dy * xhat).sum(0))
    if kind == "write":
        page = case["page"]
        got = {}
        for name in ("k", "v"):
            whole = _exact_cached(dict(st, **{name + "_scales": torch.ones_like(st[name + "_scales"])}) if case["fmt"] == "fp8" else st, name, slice(None))
            scales = st[name + "_scales"].double() if case["fmt"] == "fp8" else None
            x = st["new_" + name].double()
            codes, s = _exact_quantized(x) if case["fmt"] == "fp8" else (x, None)
            at = torch.nonzero(st["slots"] >= 0)[:, 0]
            where = st["slots"][at]
            flat = whole.permute(0, 2, 1, 3).reshape(-1, case["kv_heads"], case["dim"])
            flat[where] = codes[at]
            got[name] = flat.view(-1, page, case["kv_heads"], case["dim"]).permute(0, 2, 1, 3).contiguous()
            if scales is not None:
                flat = scales.permute(0, 2, 1).reshape(-1, case["kv_heads"])
                flat[where] = s[at]
                got[name + "_scales"] = flat.view(-1, page, case["kv_heads"]).permute(0, 2, 1).contiguous()
        return got
    if kind == "read":
        k, v = [], []
        for s, n in enumerate(_lens(case)):
            pages = st["table"][s, : -(-n // case["page"])].long()
            for out, name in ((k, "k"), (v, "v")):
                out.append(_exact_cached(st, name, pages).permute(0, 2, 1, 3).reshape(-1, case["kv_heads"], case["dim"])[:n].clone())
        return dict(k=torch.cat(k), v=torch.cat(v))
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
