"""The decoder layer that runs norm, cache, attention and the quantized experts together: prompts and single tokens, against the parts."""
import pytest
import torch

import layer_ref as ref
from paper_2604_07853_amd import synth

pytestmark = pytest.mark.gpu

H, HEADS, KV, D, E, I, TOPK, PAGE = 512, 8, 2, 64, 64, 256, 4, 16


@pytest.fixture(scope="module")
def q():
    from paper_2604_07853_amd import binding
    binding.lib()
    return binding


def layer_of(q, fmt, kv_fmt, pages):
    from paper_2604_07853_amd.decoder import DecoderLayer
    w = lambda seed, n, k, std=0.05: q.qarl_quantize_weights(synth.normal_bf16((1, n, k), std, seed).cuda(), q.QARL_W4A16_G128)
    gu, dn = synth.expert_weights(E, H, I, seed=3, std=0.05)
    return DecoderLayer(synth.normal_bf16((H,), 0.1, 4, mean=1.0).cuda(), w(5, (HEADS + 2 * KV) * D, H), w(6, H, HEADS * D),
                        synth.normal_bf16((H,), 0.1, 7, mean=1.0).cuda(), synth.normal_bf16((E, H), 0.05, 8).cuda(),
                        q.qarl_quantize_weights(gu.cuda(), fmt), q.qarl_quantize_weights(dn.cuda(), fmt),
                        q.KVCache.empty(kv_fmt, pages, PAGE, KV, D), TOPK)


def plan(lens, contexts, pages, seed=0):
    """Everything a call needs for `lens` new tokens behind `contexts` cached ones; every sequence owns a fixed run of shuffled pages."""
    S = len(lens)
    per = pages // S
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)[: per * S].view(S, per).cuda()
    slots = torch.cat([table[s, (c + torch.arange(n)) // PAGE].to(torch.int64) * PAGE + ((c + torch.arange(n)) % PAGE).cuda() for s, (n, c) in enumerate(zip(lens, contexts))])
    i32 = dict(dtype=torch.int32, device="cuda")
    kv = [n + c for n, c in zip(lens, contexts)]
    return dict(slots=slots, block_table=table, kv_lens=torch.tensor(kv, **i32), q_offsets=torch.tensor([0] + lens, **i32).cumsum(0).to(torch.int32),
                max_q_len=max(lens), max_kv_len=max(kv))


@pytest.mark.parametrize("fmt,kv_fmt", [("QARL_W4A16_G128", "QARL_KV_BF16"), ("QARL_FP8_E4M3_CH", "QARL_KV_E4M3"), ("QARL_W4A8_G128", "QARL_KV_E4M3")])
def test_prompt_then_tokens_against_the_whole(q, fmt, kv_fmt):
    """A prompt in one call against the same prompt in a chunk and two single tokens: the same cache, the same rows up to the order of sums."""
    lens, pages = [150, 70, 400], 120
    layer = layer_of(q, getattr(q, fmt), getattr(q, kv_fmt), pages)
    x = [synth.normal_bf16((n, H), 1.0, 20 + s).cuda() for s, n in enumerate(lens)]
    whole, stream = layer.forward(torch.cat(x), None, **plan(lens, [0, 0, 0], pages))
    assert whole.shape == stream.shape == (sum(lens), H) and whole.isfinite().all() and stream.isfinite().all()
    cache = [t.clone() for t in (layer.cache.k, layer.cache.v)]
    for t in (layer.cache.k, layer.cache.v):
        t.zero_()
    head = [n - 2 for n in lens]
    layer.forward(torch.cat([a[:-2] for a in x]), None, **plan(head, [0, 0, 0], pages))
    ends = torch.tensor(lens).cumsum(0) - 1
    for step in (2, 1):
        got, res = layer.forward(torch.cat([a[len(a) - step: len(a) - step + 1] for a in x]), None, **plan([1, 1, 1], [n - step for n in lens], pages))
        rows = (ends - (step - 1)).cuda()
        # attention's probabilities and its output round once to bf16 each way, the o projection's and the stream's bf16 follow: a few of 2^-8
        scale = stream[rows].double().square().mean(1, keepdim=True).sqrt()
        assert ((res - stream[rows]).double().abs() <= 6 * ref.HALF_BF16 * (stream[rows].double().abs() + scale)).all()
        same = layer._moe[3].routing.ids
        assert same.shape == (3, TOPK) and got.isfinite().all()
    # the cached keys and values are those of the whole prompt but for a rounding of the projection (the GEMM's paths add in different orders)
    used = torch.cat([plan(lens, [0, 0, 0], pages)["slots"]])
    for a, b in zip(cache, (layer.cache.k, layer.cache.v)):
        a, b = (t.permute(0, 2, 1, 3).reshape(-1, KV, D)[used] for t in (a, b))
        assert (a != b).double().mean() < 0.02


@pytest.mark.parametrize("T", [3, 600])
def test_the_layer_is_its_parts(q, T):
    """forward() against the same calls made one by one, e4m3 experts: from 513 tokens on the second norm writes the experts' rows itself, and the
    result is that of quantizing its bf16 output by a call of its own."""
    pages = 60
    layer = layer_of(q, q.QARL_FP8_E4M3_CH, q.QARL_KV_E4M3, pages)
    x, r = synth.normal_bf16((T, H), 1.0, 30).cuda(), synth.normal_bf16((T, H), 1.0, 31).cuda()
    p = plan([T], [0], pages)
    turned = []

    def rotate(a, b):
        turned.append((a.shape, b.shape))
        return a.flip(2).contiguous(), b.flip(2).contiguous()

    out, stream = layer.forward(x, r, rotate=rotate, **p)
    assert turned == [((T, HEADS, D), (T, KV, D))]
    n1 = q.qarl_add_rmsnorm(x, layer.norm1, 1e-6, residual=r)
    off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    qkv = q.qarl_qgemm_grouped(layer.qkv, n1["y"], off, T).view(T, HEADS + 2 * KV, D)
    c = q.KVCache.empty(q.QARL_KV_E4M3, pages, PAGE, KV, D)
    q.qarl_kv_cache_write(c, qkv[:, HEADS: HEADS + KV].flip(2).contiguous(), qkv[:, HEADS + KV:], p["slots"])
    att = q.qarl_paged_attention(qkv[:, :HEADS].flip(2).contiguous(), c, p["block_table"], p["kv_lens"], p["q_offsets"], T, T)["out"]
    o = q.qarl_qgemm_grouped(layer.o, att.view(T, HEADS * D), off, T)
    n2 = q.qarl_add_rmsnorm(o, layer.norm2, 1e-6, residual=n1["residual"])
    assert torch.equal(n2["residual"], stream)
    moe = q.MoELayer(layer.gu, layer.dn, T, TOPK, q.QARL_PATH_DECODE if T <= 512 else q.QARL_PATH_PREFILL)
    assert torch.equal(moe.forward(n2["y"], torch.matmul(n2["y"], layer.router.t())), out)


def test_sizes_that_do_not_fit_are_refused(q):
    from paper_2604_07853_amd.decoder import DecoderLayer
    a = layer_of(q, q.QARL_W4A16_G128, q.QARL_KV_BF16, 8)
    good = dict(norm1=a.norm1, qkv=a.qkv, o=a.o, norm2=a.norm2, router=a.router, gate_up=a.gu, down=a.dn, cache=a.cache)
    for bad in (dict(qkv=a.o), dict(norm1=a.norm1[:-1]), dict(router=a.router[:-1]), dict(cache=q.KVCache.empty(q.QARL_KV_BF16, 8, PAGE, KV * 2, D))):
        with pytest.raises(ValueError):
            DecoderLayer(**dict(good, **bad))


@pytest.mark.parametrize("fmt", ["QARL_W4A16_G128", "QARL_FP8_E4M3_CH"])
def test_batches_of_every_size_share_one_set_of_buffers(q, fmt):
    """A layer that meets many batch sizes holds the intermediates of one, and its results are those of a layer that has met no other."""
    pages = 40
    layer = layer_of(q, getattr(q, fmt), q.QARL_KV_BF16, pages)
    for T in (5, 300, 1, 17, 512, 5):
        x, p = synth.normal_bf16((T, H), 1.0, 40 + T).cuda(), plan([T], [0], pages)
        out, stream = (t.clone() for t in layer.forward(x, None, **p))
        fresh = layer_of(q, getattr(q, fmt), q.QARL_KV_BF16, pages)
        want = fresh.forward(x, None, **p)
        assert torch.equal(out, want[0]) and torch.equal(stream, want[1]), T
    assert len(layer._moe) == 5
    for name in ("a", "out"):
        assert len({getattr(m, name).untyped_storage().data_ptr() for m in layer._moe.values()}) == 1


@pytest.mark.parametrize("fmt", ["QARL_W4A16_G128", "QARL_FP8_E4M3_CH"])
def test_batches_on_two_streams(q, fmt):
    """Chunks on one stream and decode steps on another, each result read late: it is that of the same call alone."""
    calls, per = [(300, 0), (7, 1), (512, 0), (1, 1), (300, 1), (7, 0)], 32
    inputs = []
    for i, (T, _) in enumerate(calls):      # sequences of their own, in pages of their own
        p = plan([T], [0], per)
        inputs.append((synth.normal_bf16((T, H), 1.0, 60 + i).cuda(), dict(p, slots=p["slots"] + i * per * PAGE, block_table=p["block_table"] + i * per)))
    make = lambda: layer_of(q, getattr(q, fmt), q.QARL_KV_BF16, per * len(calls))
    want = [make().forward(x, None, **p)[0].clone() for x, p in inputs]
    layer, streams, got = make(), [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for (x, p), (_, on) in zip(inputs, calls):
        with torch.cuda.stream(streams[on]):
            out = layer.forward(x, None, **p)[0]
            torch.cuda._sleep(5_000_000)
            got.append(out.clone())
    torch.cuda.synchronize()
    for (T, _), a, b in zip(calls, got, want):
        assert torch.equal(a, b), T


@pytest.mark.parametrize("fmt,kv_fmt", [("QARL_W4A16_G128", "QARL_KV_BF16"), ("QARL_FP8_E4M3_CH", "QARL_KV_E4M3"), ("QARL_W4A8_G128", "QARL_KV_BF16")])
@pytest.mark.parametrize("T", [7, 600])
@pytest.mark.parametrize("met", [True, False])
def test_captured_steps(q, fmt, kv_fmt, T, met):
    """A step in a graph, of a size met before and of a new one: every replay gives what the same call gives outside, before and after it."""
    pages = 64
    layer = layer_of(q, getattr(q, fmt), getattr(q, kv_fmt), pages)
    x, r = (synth.normal_bf16((T, H), 1.0, s).cuda() for s in (70, 71))
    p = plan([T], [20], pages)
    for t in (layer.cache.k, layer.cache.v, layer.cache.k_scales, layer.cache.v_scales):
        if t is not None:
            t.zero_()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for n in (5, 700) + ((T,) if met else ()):
            layer.forward(synth.normal_bf16((n, H), 1.0, n).cuda(), None, **plan([n], [0], pages))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, stream = layer.forward(x, r, **p)
    if not met:         # a call of that size outside, in front of the first replay
        first = [t.clone() for t in layer.forward(x, r, **p)]
    for seed in range(3):
        if seed:
            x.copy_(synth.normal_bf16((T, H), 1.0, 80 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), stream.clone()
        if seed == 0 and not met:
            assert all(torch.equal(a, b) for a, b in zip(first, got))
        want = layer.forward(x, r, **p)
        torch.cuda.synchronize()
        assert got[0].isfinite().all() and all(torch.equal(a, b) for a, b in zip(got, want)), seed


@pytest.mark.parametrize("fmt", ["QARL_W4A16_G128", "QARL_FP8_E4M3_CH"])
def test_no_tokens(q, fmt):
    """A step without tokens, alone and between others."""
    layer = layer_of(q, getattr(q, fmt), q.QARL_KV_BF16, 8)
    i32 = dict(dtype=torch.int32, device="cuda")
    none = dict(slots=torch.empty(0, dtype=torch.int64, device="cuda"), block_table=torch.zeros((3, 2), **i32), kv_lens=torch.zeros(3, **i32),
                q_offsets=torch.zeros(4, **i32), max_q_len=1, max_kv_len=1)
    x = synth.normal_bf16((3, H), 1.0, 5).cuda()
    for _ in range(2):
        for stream in (None, x[:0]):
            out, res = layer.forward(x[:0], stream, **none)
            assert out.shape == res.shape == (0, H)
        want = [t.clone() for t in layer.forward(x, None, **plan([3], [0], 8))]
        assert want[0].isfinite().all()
