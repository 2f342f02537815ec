"""Sampling of the next token against sorted sums in 64 bits, through the C ABI."""
import math

import numpy as np
import pytest
import torch

import rollout_ref as ref

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24


@pytest.fixture(scope="module")
def q():
    from paper_2604_07853_amd import binding
    binding.lib()
    return binding


def rows_of(T, V, kind, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((T, V), generator=g) * {"wide": 2.2, "flat": 0.3, "peaked": 1.0, "tiny": 1e-4}[kind]
    if kind == "peaked":
        z[torch.arange(T), torch.randint(0, V, (T,), generator=g)] += 9.0
    return z.to(dtype)


def ask(q, z, u, **ways):
    T = z.shape[0]
    dt = dict(temperature=torch.float32, top_k=torch.int32, top_p=torch.float32, min_p=torch.float32)
    kw = {n: torch.as_tensor(v, dtype=dt[n]).expand(T).contiguous().cuda() for n, v in ways.items()}
    return q.qarl_sample(z.cuda() if not z.is_cuda else z, torch.as_tensor(u, dtype=torch.float32).expand(T).contiguous().cuda(), want_kept=True, **kw)


def check(z, got, u, **ways):
    """Log-probs: a rounding to fp32 of a value of that size, weights left out of the integer sums (below 2^-44 each: 1e-8 at most of 2^20 of them)."""
    T = z.shape[0]
    wide = {n: torch.as_tensor(v).expand(T).tolist() for n, v in ways.items()}
    us = torch.as_tensor(u, dtype=torch.float32).expand(T).tolist()
    rows = z.cpu().double().numpy()
    token, lp, kept = got["token"].tolist(), got["logprob"].tolist(), got["kept_logprob"].tolist()
    for r in range(T):
        want = ref.sample(rows[r], us[r], **{n: v[r] for n, v in wide.items()})
        assert token[r] == want[0], (r, token[r], want)
        for have, w in ((lp[r], want[1]), (kept[r], want[2])):
            assert (math.isnan(w) and math.isnan(have)) or abs(have - w) <= abs(w) * 1.01 * F32 + 2e-8, (r, have, w)


WAYS = [dict(), dict(temperature=0.6, top_k=20, top_p=0.95), dict(top_p=0.9), dict(temperature=1.3, min_p=0.05), dict(top_k=1), dict(temperature=0.0),
        dict(temperature=0.7, top_k=300, top_p=0.8, min_p=0.01), dict(top_p=0.0), dict(top_k=5000, top_p=0.999), dict(temperature=0.01, top_p=0.5), dict(min_p=2.0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ways", WAYS)
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 32003])
def test_all_ways(q, dtype, ways, V):
    for i, kind in enumerate(("wide", "flat", "peaked", "tiny")):
        T = 9
        z = rows_of(T, V, kind, dtype, V + i)
        u = torch.rand((T,), generator=torch.Generator().manual_seed(V))
        u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
        check(z, ask(q, z, u, **ways), u, **ways)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_vocabularies_and_mixed_rows(q, dtype):
    for T, V in ((37, 151936), (5, (1 << 20) - 3), (3, 1 << 20)):
        g = torch.Generator().manual_seed(V)
        z = rows_of(T, V, "wide", dtype, 3)
        z[T - 1] = rows_of(1, V, "flat", dtype, 4)[0]
        ways = dict(temperature=torch.rand((T,), generator=g) + 0.5, top_k=torch.randint(0, 3000, (T,), generator=g) * (torch.rand((T,), generator=g) < 0.5),
                    top_p=torch.rand((T,), generator=g) * 0.6 + 0.5, min_p=torch.rand((T,), generator=g) * 0.01 * (torch.rand((T,), generator=g) < 0.4))
        ways["temperature"][1] = 0.0
        u = torch.rand((T,), generator=g)
        check(z, ask(q, z, u, **ways), u, **ways)


@pytest.mark.parametrize("offset", [0.0, -0.02, -9.0, 20.0])
@pytest.mark.parametrize("top_k", [2, 100, 255, 256, 257, 400, 1500])
def test_places_found_one_in_front_of_the_other(q, top_k, offset):
    """Logits in 32 bits: the first k tokens, those of them that hold p, the token: each place lies in front of the one before, among the same tokens or not."""
    T, V = 12, 32003
    z = rows_of(T, V, "wide", torch.float32, top_k)
    z[T // 2:] *= 0.01                                  # a few bins hold all
    z = z + offset
    z[1::2] = (z[1::2] * 4096).round() / 4096           # some equal ones
    u = torch.linspace(0.0, 1.0, T)
    for ways in (dict(top_k=top_k), dict(top_k=top_k, top_p=0.5), dict(top_k=top_k, top_p=0.97, min_p=0.02), dict(top_p=0.01, min_p=0.9)):
        check(z, ask(q, z, u, **ways), u, **ways)


@pytest.mark.parametrize("V", [20011, 200003])
@pytest.mark.parametrize("offset,spread", [(20.0, 1.0), (-60.0, 0.05), (100.0, 1e-3)])
def test_many_tokens_of_nearly_one_value(q, V, offset, spread):
    """Logits in 32 bits whose upper halves hardly differ: thousands share one, with different weights; from the last of few values on, the same ones."""
    T = 10
    z = rows_of(T, V, "wide", torch.float32, V) * spread + offset
    z[::3] = (z[::3] * 64).round() / 64
    u = torch.linspace(0.0, 1.0, T)
    for ways in (dict(), dict(top_p=0.7), dict(top_k=9000, top_p=0.6), dict(top_k=V - 1, min_p=0.3, temperature=0.05)):
        check(z, ask(q, z, u, **ways), u, **ways)


@pytest.mark.parametrize("T", [1, 2, 63, 300, 1500])
def test_many_rows(q, T):
    z = rows_of(T, 501, "wide", torch.bfloat16, T)
    u = torch.rand((T,), generator=torch.Generator().manual_seed(T))
    check(z, ask(q, z, u, top_p=0.9), u, top_p=0.9)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [0.0, -0.0, 5.0, -1e30, 3.3e38, -3.3895313892515355e38, 1e-30, -300.0, 300.0])
@pytest.mark.parametrize("V", [8, 1000, 70001])
def test_equal_logits_stand_by_index(q, dtype, value, V):
    """All V tokens weigh the same: the borders of the sums are whole numbers of weights, met exactly."""
    z = torch.full((6, V), value).to(dtype)
    if V > 8 and value == 0.0:
        z[:, ::2] = -0.0                                # the same value
    for j in (0, 1, V // 2, V - 1):
        u = (j + 0.5) / V if V > 8 else j / V          # eighths are exact: the running sum does not yet exceed u at token j - 1
        got = ask(q, z, u)
        assert (got["token"] == j).all(), (j, got["token"])
        assert ((got["logprob"] + math.log(V)).abs() <= math.log(V) * 2 * F32).all()
    for kw, n in ((dict(top_k=5), 5), (dict(top_p=0.5), -(-V // 2)), (dict(min_p=1.0), V), (dict(min_p=1.5), 1), (dict(top_k=8, top_p=0.25), 2)):
        for u, want in ((0.0, 0), (1.0, n - 1), (math.nan, 0), (-3.0, 0), (7.0, n - 1)):
            got = ask(q, z, u, **kw)
            assert (got["token"] == want).all(), (kw, u, got["token"])
            assert ((got["kept_logprob"] + math.log(n)).abs() <= math.log(V) * 2 * F32).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_logits(q, dtype):
    """-inf and the type's lowest value: in front of, behind and between the others; nearly all of a row, all but one."""
    low = torch.finfo(dtype).min
    for V, fill in ((50, -math.inf), (50, low), (151936, -math.inf), (151936, low), (70001, -1e4)):
        z = rows_of(4, V, "wide", dtype, V)
        z[0, :-3] = fill
        z[1, 1:] = fill
        z[2, ::2] = fill
        z[3, : V // 2] = fill
        for kw in WAYS[:8]:
            for u in (0.0, 0.3, 0.999999):
                check(z, ask(q, z, u, **kw), u, **kw)


def test_values_of_every_size(q):
    """A few large logits over tiny and subnormal ones, values around zero, far from it, and temperatures that make the one like the other."""
    g = torch.Generator().manual_seed(1)
    V = 4001
    for dtype in (torch.bfloat16, torch.float32):
        z = torch.stack([torch.randn(V, generator=g) * 2.0 ** e for e in (-140, -60, -9, -3, 0, 5, 9, 60, 120)]).to(dtype)
        z = torch.cat([z, (z[4:5].float() + 600).to(dtype), (z[4:5].float() - 600).to(dtype), (z[4:5].float() * 2.0 ** torch.randint(-20, 8, (V,), generator=g)).to(dtype)])
        u = torch.rand((z.shape[0],), generator=g)
        for t in (1.0, 1e-3, 1e-38, 30.0, 1e30):
            for kw in (dict(), dict(top_p=0.7), dict(top_k=100, min_p=0.2)):
                check(z, ask(q, z, u, temperature=t, **kw), u, temperature=t, **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_without_a_distribution(q, dtype):
    for V in (9, 5000):
        z = rows_of(8, V, "wide", dtype, 2)
        z[0, 3], z[1, V - 1], z[2] = math.nan, math.inf, -math.inf
        z[3, 1] = -math.nan
        t = torch.tensor([1.0, 1.0, 1.0, 1.0, -0.5, math.nan, math.inf, 1.0])
        got = ask(q, z, 0.4, temperature=t)
        assert got["token"][:7].tolist() == [-1] * 7 and got["logprob"][:7].isnan().all() and got["kept_logprob"][:7].isnan().all()
        check(z[7:], {n: v[7:] for n, v in got.items()}, 0.4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("first,pad", [(0, 0), (1, 2), (3, 61), (7, 8)])
def test_rows_at_any_address(q, dtype, first, pad):
    V = 3001
    wide = torch.full((5, first + V + pad), math.nan, dtype=dtype, device="cuda")
    z = rows_of(5, V, "wide", dtype, 6)
    wide[:, first: first + V] = z.cuda()
    view = wide[:, first: first + V]
    for u in (0.1, 0.9):
        check(z, ask(q, view, u, top_p=0.95), u, top_p=0.95)
    check(z[2:3], ask(q, view[2:3], 0.5), 0.5)


def test_frequencies_follow_the_probabilities(q):
    """Evenly spread random numbers: each token comes as often as its share says, to one in either direction."""
    z = torch.tensor([0.3, 1.7, -0.4, 1.7, 0.0, 2.1, -3.0], dtype=torch.float32)
    n = 20000
    u = (torch.arange(n) + 0.5) / n
    for kw in (dict(), dict(top_k=4), dict(top_p=0.8, temperature=0.7)):
        got = ask(q, z.expand(n, 7).contiguous(), u, **kw)
        count = torch.bincount(got["token"].cpu().long(), minlength=7).double()
        t = kw.get("temperature", 1.0)
        order = sorted(range(7), key=lambda i: (-float(z[i]), i))
        w = np.exp([(float(z[i]) - 2.1) / t for i in order])
        keep = 4 if "top_k" in kw else 1 + int((np.cumsum(w)[:-1] < 0.8 * w.sum()).sum()) if "top_p" in kw else 7
        for i, j in enumerate(order):
            want = n * w[i] / w[:keep].sum() if i < keep else 0.0
            assert abs(count[j] - want) <= 1.01, (kw, j)


def test_no_rows_and_results_that_do_not_change(q):
    assert ask(q, torch.zeros((0, 10), dtype=torch.bfloat16, device="cuda"), 0.5)["token"].shape == (0,)
    z = rows_of(200, 40001, "flat", torch.float32, 1).cuda()
    u = torch.rand((200,), generator=torch.Generator().manual_seed(1))
    first = ask(q, z, u, top_p=0.9)
    for _ in range(5):
        again = ask(q, z, u, top_p=0.9)
        assert all(torch.equal(first[n], again[n]) for n in first)
    for lo, hi in ((0, 1), (7, 19), (100, 200)):        # by itself or in a batch
        part = ask(q, z[lo:hi], u[lo:hi], top_p=0.9)
        assert all(torch.equal(first[n][lo:hi], part[n]) for n in first)


def test_graph_and_other_stream(q):
    T, V = 6, 151936
    z, u = rows_of(T, V, "wide", torch.bfloat16, 1).cuda(), torch.rand((T,), device="cuda")
    k, p = torch.tensor([20, 0, 1, 500, 0, 3], dtype=torch.int32, device="cuda"), torch.full((T,), 0.9, device="cuda")
    out = dict(token=torch.empty((T,), dtype=torch.int32, device="cuda"), logprob=torch.empty((T,), device="cuda"), kept_logprob=torch.empty((T,), device="cuda"))
    ws = torch.full((max(16, q.qarl_sample_workspace_bytes(T, V)),), 0x5a, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q.qarl_sample(z, u, top_k=k, top_p=p, ws=ws, **out)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.qarl_sample(z, u, top_k=k, top_p=p, ws=ws, **out)
    for seed in range(3):
        z.copy_(rows_of(T, V, ("wide", "flat", "peaked")[seed], torch.bfloat16, 20 + seed))
        u.copy_(torch.rand((T,)))
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        want = q.qarl_sample(z, u, top_k=k, top_p=p, want_kept=True)
        assert all(torch.equal(out[n], want[n]) for n in out)
        check(z, out, u, top_k=k.cpu(), top_p=0.9)


def test_nothing_is_written_behind_the_workspace(q):
    for T, V, dtype in ((1, 151936, torch.bfloat16), (70, 5000, torch.bfloat16), (3, 20001, torch.float32)):
        need = q.qarl_sample_workspace_bytes(T, V)
        ws = torch.full((need + 65536,), 0x5a, dtype=torch.uint8, device="cuda")
        z = rows_of(T, V, "wide", dtype, 1)
        u = torch.rand((T,), generator=torch.Generator().manual_seed(1))
        got = q.qarl_sample(z.cuda(), u.cuda(), want_kept=True, ws=ws)
        assert (ws[need:] == 0x5a).all()
        check(z, got, u)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [2000, 32003, 200003])
def test_a_share_of_nothing_keeps_the_first_token(q, dtype, V):
    """top_p of zero and less, whatever the other truncations leave: also where more tokens than a list holds share the upper half of the largest logit."""
    T = 8
    z = rows_of(T, V, "wide", dtype, V)
    z[1], z[2], z[3] = 5.0, -0.75, 0.0                          # all equal
    z[4] = (rows_of(1, V, "wide", torch.float32, 1)[0] * 1e-3 + 100.0).to(dtype)
    z[5] = (rows_of(1, V, "wide", torch.float32, 2)[0] * 1e-3 + 300.0).to(dtype)
    z[6] = (rows_of(1, V, "wide", torch.float32, 3)[0] * 1e-3 - 2.0).to(dtype)
    z[7, : V // 2] = -math.inf
    u = torch.linspace(0.0, 1.0, T)
    for share in (0.0, -0.5, -math.inf):
        for ways in (dict(), dict(top_k=1500), dict(top_k=V - 1, temperature=0.7), dict(min_p=0.2), dict(top_k=1100, min_p=0.9, temperature=3.0)):
            check(z, ask(q, z, u, top_p=share, **ways), u, top_p=share, **ways)


@pytest.mark.parametrize("dtype,V", [(torch.bfloat16, 81920), (torch.bfloat16, 163000), (torch.float32, 65536), (torch.float32, 90001)])
def test_a_row_does_not_depend_on_how_many_there_are(q, dtype, V):
    """Up to 64 rows are cut into parts, more are not: the same tokens and log-probs, bit for bit.  Rows 0 to 7 of 16 bits: more values below 2^-9 in one part than
    others hold in all; temperatures at which the weight of a value three steps below the largest lies so near a border between two units that an exponential
    and a product of three factors fall on either side of it, and random numbers between the two sums that follow: any change of way shows in the token."""
    T = 65
    z = rows_of(T, V, "wide", dtype, V)
    z[8:12] = rows_of(4, V, "flat", dtype, 1)
    u, t = torch.rand((T,), generator=torch.Generator().manual_seed(V)), torch.ones(T)
    if V == 163000:
        z[:8, :300] = 2.0 ** -10
        z[:8, 300:80300] = 5.09375
        z[:8, 80300:] = 5.0
        t[:8] = torch.tensor([0x3f0091f6, 0x3f00ecca, 0x3f01342c, 0x3f0091f6, 0x3f00ecca, 0x3f01342c, 0x3f0091f6, 0x3f00ecca], dtype=torch.int32).view(torch.float32)
        u[:8] = torch.tensor([14032438, 11532833, 11334061, 14032438, 11532833, 11334061, 14032438, 11532833]) / 2.0 ** 24
    for kw in (dict(), dict(top_p=0.9), dict(top_k=700, min_p=0.001)):
        way = dict(temperature=t, **kw)
        whole = ask(q, z, u, **way)
        for lo, hi in ((0, 64), (0, 1), (2, 9)):
            part = ask(q, z[lo:hi], u[lo:hi], **dict(way, temperature=t[lo:hi]))
            assert all(torch.equal(whole[n][lo:hi], part[n]) for n in whole), (kw, lo, hi, whole["token"][lo:hi].tolist(), part["token"].tolist())
        check(z[8:], {n: v[8:] for n, v in whole.items()}, u[8:], **dict(way, temperature=t[8:]))


@pytest.mark.parametrize("dtype,V", [(torch.bfloat16, 32762), (torch.bfloat16, 50001), (torch.bfloat16, 65530), (torch.bfloat16, 151936), (torch.bfloat16, 163833), (torch.bfloat16, 163834),
                                     (torch.bfloat16, 201088), (torch.float32, 65536), (torch.float32, 151936), (torch.float32, 163840)])
def test_large_vocabularies_of_more_rows_than_are_cut(q, dtype, V):
    """Rows of every length that one workgroup takes whole, and the first that it does not: all rows are sampled, some are checked; tokens at the row's very ends."""
    T = 70
    z = rows_of(T, V, "wide", dtype, V)
    z[20:40] = rows_of(20, V, "flat", dtype, 1)
    z[5, : V - 3], z[6, 2:] = -math.inf, -math.inf
    z[7] = 3.0                                          # all equal: the token is the number's place
    g = torch.Generator().manual_seed(V)
    u = torch.rand((T,), generator=g)
    u[7], u[8], u[9] = 0.99999, 0.0, 1.0
    ways = dict(temperature=torch.rand((T,), generator=g) + 0.5, top_k=torch.randint(0, 3000, (T,), generator=g) * (torch.rand((T,), generator=g) < 0.5),
                top_p=torch.rand((T,), generator=g) * 0.7 + 0.4, min_p=torch.rand((T,), generator=g) * 0.01 * (torch.rand((T,), generator=g) < 0.4))
    ways["temperature"][1] = 0.0
    ways["top_k"][7] = 0
    ways["top_p"][7] = 1.0
    pick = torch.tensor([0, 1, 5, 6, 7, 8, 9, 21, 38, 69])
    for kw in (dict(), ways):
        got = ask(q, z, u, **kw)
        assert (got["token"] >= 0).all() and (got["token"] < V).all()
        check(z[pick], {n: v[pick.cuda()] for n, v in got.items()}, u[pick], **{n: v[pick] for n, v in kw.items()})


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(1, 151936), (64, 81920), (3, 1 << 20), (70, 163834)])
def test_workspaces_of_cut_rows(q, dtype, T, V):
    """What a workspace holds before a call, other rows' sums among it, does not matter, and nothing is written behind it."""
    need = q.qarl_sample_workspace_bytes(T, V)
    assert need > 0
    ws = torch.full((need + 65536,), 0x5a, dtype=torch.uint8, device="cuda")
    u = torch.rand((T,), generator=torch.Generator().manual_seed(1)).cuda()
    for i, kind in enumerate(("wide", "flat", "tiny", "wide")):
        z = rows_of(T, V, kind, dtype, i).cuda()
        if i == 3:
            z[0] = math.nan
            ws[:need] = 0xff
        got = q.qarl_sample(z, u, want_kept=True, ws=ws)
        clean = q.qarl_sample(z, u, want_kept=True, ws=torch.zeros((need,), dtype=torch.uint8, device="cuda"))
        assert all(torch.equal(got[n].nan_to_num(7.0), clean[n].nan_to_num(7.0)) for n in got)
        assert (ws[need:] == 0x5a).all()
        lo = 1 if i == 3 and T > 1 else 0
        check(z[lo: lo + 1].cpu(), {n: v[lo: lo + 1] for n, v in got.items()}, u[lo: lo + 1].cpu())


@pytest.mark.parametrize("T,V", [(6, 151936), (70, 100003)])
def test_graph_of_32_bit_logits(q, T, V):
    z, u = rows_of(T, V, "wide", torch.float32, 1).cuda(), torch.rand((T,), device="cuda")
    k, p = torch.randint(0, 400, (T,), dtype=torch.int32, device="cuda"), torch.full((T,), 0.9, device="cuda")
    out = dict(token=torch.empty((T,), dtype=torch.int32, device="cuda"), logprob=torch.empty((T,), device="cuda"), kept_logprob=torch.empty((T,), device="cuda"))
    ws = torch.full((max(16, q.qarl_sample_workspace_bytes(T, V)),), 0x5a, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q.qarl_sample(z, u, top_k=k, top_p=p, ws=ws, **out)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.qarl_sample(z, u, top_k=k, top_p=p, ws=ws, **out)
    for seed in range(4):
        z.copy_(rows_of(T, V, ("wide", "flat", "peaked", "tiny")[seed], torch.float32, 20 + seed))
        u.copy_(torch.rand((T,)))
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        want = q.qarl_sample(z, u, top_k=k, top_p=p, want_kept=True)
        assert all(torch.equal(out[n], want[n]) for n in out)
        check(z[:3], {n: v[:3] for n, v in out.items()}, u[:3], top_k=k[:3].cpu(), top_p=0.9)
