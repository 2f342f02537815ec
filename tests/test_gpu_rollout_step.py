"""Rotary positions, the 4-bit cache, attention and sampling together, as a rollout's steps run them, through the decoder layer."""
import pytest
import torch

import layer_ref as ref
from paper_2604_07853_amd import synth
from test_gpu_decoder_layer import D, H, HEADS, KV, PAGE, TOPK, layer_of, plan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    from paper_2604_07853_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("T", [3, 600])
@pytest.mark.parametrize("kv_fmt", ["QARL_KV_BF16", "QARL_KV_E2M1"])
def test_the_layer_is_its_parts(q, T, kv_fmt):
    pages = 60
    layer = layer_of(q, q.QARL_W4A16_G128, getattr(q, kv_fmt), pages)
    rope = q.Rope(D, base=1e6)
    x, p = synth.normal_bf16((T, H), 1.0, 30).cuda(), plan([T], [0], pages)
    pos = torch.arange(T, device="cuda") + 5
    out, stream = (t.clone() for t in layer.forward(x, None, rope=rope, positions=pos, **p))
    n1 = q.qarl_add_rmsnorm(x, layer.norm1, 1e-6)
    off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    qkv = q.qarl_qgemm_grouped(layer.qkv, n1["y"], off, T).view(T, HEADS + 2 * KV, D)
    c = q.KVCache.empty(getattr(q, kv_fmt), pages, PAGE, KV, D)
    query = q.qarl_rotary_kv_write(c, rope, pos, qkv[:, :HEADS], qkv[:, HEADS: HEADS + KV], qkv[:, HEADS + KV:], p["slots"])
    att = q.qarl_paged_attention(query, c, p["block_table"], p["kv_lens"], p["q_offsets"], T, T)["out"]
    o = q.qarl_qgemm_grouped(layer.o, att.view(T, HEADS * D), off, T)
    n2 = q.qarl_add_rmsnorm(o, layer.norm2, 1e-6, residual=x)
    assert torch.equal(n2["residual"], stream)
    moe = q.MoELayer(layer.gu, layer.dn, T, TOPK, q.QARL_PATH_DECODE if T <= 512 else q.QARL_PATH_PREFILL)
    assert torch.equal(moe.forward(n2["y"], torch.matmul(n2["y"], layer.router.t())), out)
    # a rope of its own accord, before the cache: over a 16-bit cache the same bits
    if kv_fmt == "QARL_KV_BF16":
        turned = lambda a, b: tuple(q.qarl_rotary(rope, pos, a, b).values())      # noqa: E731
        again, _ = layer.forward(x, None, rotate=turned, **p)
        assert torch.equal(again, out)
    with pytest.raises(ValueError, match="go together"):
        layer.forward(x, None, rope=rope, **p)


def test_attention_goes_by_the_distance_of_positions(q):
    """All positions shifted by as many: the same scores, so the same layer but for the roundings of turned queries and keys."""
    T, pages = 200, 30
    layer = layer_of(q, q.QARL_W4A16_G128, q.QARL_KV_BF16, pages)
    rope = q.Rope(D, base=1e4, layout=q.QARL_ROPE_PAIRS)
    x, p = synth.normal_bf16((T, H), 1.0, 31).cuda(), plan([T], [0], pages)
    a = layer.forward(x, None, rope=rope, positions=torch.arange(T, device="cuda"), **p)[1].double()
    b = layer.forward(x, None, rope=rope, positions=torch.arange(T, device="cuda") + 100003, **p)[1].double()
    c = layer.forward(x, None, rope=rope, positions=torch.arange(T, device="cuda") * 3, **p)[1].double()
    # scores of size s change by two roundings of q and k (2^-8 of |q| |k| each at most), probabilities by as much; stream and o projection round as well
    scale = a.square().mean(1, keepdim=True).sqrt()
    assert ((a - b).abs() <= 8 * ref.HALF_BF16 * (a.abs() + scale)).all()
    assert ((a - c).abs() > 8 * ref.HALF_BF16 * (a.abs() + scale)).any()


@pytest.mark.parametrize("kv_fmt", ["QARL_KV_E4M3", "QARL_KV_E2M1"])
def test_prompts_and_sampled_tokens(q, kv_fmt):
    """Prompts filled in, then tokens sampled and fed back: every step's log-prob is what the learner's kernel makes of the same rows, and the sampled
    sequences, filled in at once into a cache of their own, leave the bytes that the steps have left."""
    lens, steps, V, pages = [40, 7, 65], 6, 1000, 30
    layer = layer_of(q, q.QARL_W4A16_G128, getattr(q, kv_fmt), pages)
    rope = q.Rope(D, base=1e6)
    embed, w_lm = synth.normal_bf16((V, H), 1.0, 50).cuda(), synth.normal_bf16((V, H), 0.05, 51).cuda()
    seqs = [torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(n)).cuda() for n in lens]
    contexts, new = [0, 0, 0], [len(s) for s in seqs]
    first = torch.cat(seqs)
    sampled, lps = [], []
    g = torch.Generator().manual_seed(9)
    for step in range(steps):
        tokens = first if step == 0 else sampled[-1].long()
        pos = torch.cat([c + torch.arange(n) for n, c in zip(new, contexts)]).cuda()
        p = plan(new, contexts, pages)
        out, stream = layer.forward(embed[tokens], None, rope=rope, positions=pos, **p)
        ends = (torch.tensor(new).cumsum(0) - 1).cuda()
        hidden = (out[ends] + stream[ends])
        logits = torch.matmul(hidden.float(), w_lm.float().t())
        r = q.qarl_sample(logits, torch.rand((3,), generator=g).cuda(), temperature=torch.ones(3, device="cuda"), top_k=torch.tensor([0, 50, 1], dtype=torch.int32, device="cuda"))
        assert (r["token"] >= 0).all() and (r["token"] < V).all()
        assert int(r["token"][2]) == int(logits[2].argmax())
        want = q.qarl_token_logprob(hidden, w_lm, r["token"])["logprob"]
        size = torch.matmul(hidden.double().abs(), w_lm.double().abs().t()).amax(1)
        assert ((r["logprob"] - want).double().abs() <= 4 * (H + 8) * ref.F32 * size + 1e-5).all()
        delta = q.qarl_logprob_mismatch(want, r["logprob"])["delta"]
        assert (delta.abs() <= 1e-3).all()
        sampled.append(r["token"])
        contexts, new = [c + n for c, n in zip(contexts, new)], [1, 1, 1]
        lps.append(r["logprob"])
    whole = [torch.cat([s, torch.stack(sampled)[: steps - 1, i].long()]) for i, s in enumerate(seqs)]
    total = [len(s) for s in whole]
    other = layer_of(q, q.QARL_W4A16_G128, getattr(q, kv_fmt), pages)
    p = plan(total, [0, 0, 0], pages)
    other.forward(embed[torch.cat(whole)], None, rope=rope, positions=torch.cat([torch.arange(n) for n in total]).cuda(), **p)
    # keys and values come from the first layer's input alone: equal but for the projection's order of sums (a decode step and a prompt take different paths)
    for a, b in ((layer.cache.k, other.cache.k), (layer.cache.v, other.cache.v)):
        rows = [t.permute(0, 2, 1, 3).reshape(pages * PAGE, -1)[p["slots"]] for t in (a, b)]
        assert (rows[0] != rows[1]).double().mean() < 0.02
