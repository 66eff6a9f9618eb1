"""hydra_token_logprobs against log_softmax in 64 bits: masked and equal logits, rows of nothing, odd vocabularies, tokens that are not there."""
import math

import pytest
import torch

from paper_2402_05109_amd import binding as hb
from span_util import DEV, context

pytestmark = pytest.mark.gpu


def call(x, tok, tau=1.0, k=0, want=("logprob", "rank", "entropy")):
    B, T, V = x.shape
    c = context(2, 64, B, [-1] + list(range(T - 1)), vocab=V, max_pos=T + 1)
    o = {"logprob": torch.full((B, T), 5.0, device=DEV), "rank": torch.full((B, T), -9, dtype=torch.int32, device=DEV), "entropy": torch.full((B, T), 5.0, device=DEV)}
    ids, lps = (torch.full((B, T, k), -9, dtype=torch.int32, device=DEV), torch.full((B, T, k), 5.0, device=DEV)) if k else (None, None)
    c.hydra_token_logprobs(B, c.ws, x.to(DEV), None if tok is None else tok.to(DEV, torch.int32), tau, k, **{n: o[n] for n in want}, top_ids=ids, top_logprobs=lps)
    return o | {"ids": ids, "lps": lps, "flags": c.read_flags()}


def check(x, tok, tau=1.0, k=0):
    """Tolerance.  A weight is off by 2^-20 of itself (the exponential, and a sum of V terms by lanes of up to 64 in a row) and by the error of its exponent, a
    difference rounded once and multiplied by 1 / tau rounded once: 2^-22 z, with z its distance from the largest.  So the weights beside the peak, and
    their sum over z, by sums that can be taken; log1p and the last operations by 2^-21 of what they return.  (A first version took the largest z among weights over
    1e-12 in place of the sums, which left out rows all of whose weights are smaller.)  The reference takes the tokens
    that share the largest logit apart, as a sum that begins at 1 loses what is small beside it (V additions of 2^-53 each: torch.log_softmax in 64 bits has 9.4e-11 wrong in the
    fourth digit), and is itself held to log_softmax."""
    o = call(x, tok, tau, k)
    y = x.double().to(DEV) / tau
    z = (y.amax(dim=-1, keepdim=True) - y)
    lp = -z - torch.log1p(torch.where(z > 0, torch.exp(-z), 0.0).sum(dim=-1, keepdim=True) + ((z == 0).sum(dim=-1, keepdim=True) - 1))
    soft = torch.log_softmax(y, dim=-1)
    assert torch.equal(torch.isfinite(lp), torch.isfinite(soft)) and ((lp - soft).abs() <= 1e-10 + 1e-12 * z)[torch.isfinite(lp)].all()
    p = lp.exp()
    c = 2.0 ** -20 + 64 * 2.0 ** -24
    zz = torch.where(p > 0, z, 0.0)
    off = (torch.where(z > 0, p, 0.0) * (c + 2.0 ** -22 * zz)).sum(dim=-1)              # of the weights beside the peak, and of ln Z
    off_z = (p * zz * (c + 2.0 ** -22 * zz)).sum(dim=-1)                                # of their sum over z
    assert o["flags"] == 0
    given = tok.to(DEV) >= 0
    mine = lp.gather(2, tok.to(DEV).long().clamp(min=0)[..., None])[..., 0]
    zt = z.gather(2, tok.to(DEV).long().clamp(min=0)[..., None])[..., 0]
    lnz = -lp.amax(dim=-1)
    tol = off + 2.0 ** -21 * (lnz + zt) + 1e-37
    assert ((o["logprob"].double() - mine).abs() <= tol)[given & torch.isfinite(mine)].all()
    assert torch.equal(o["logprob"][given & (mine == -math.inf)], torch.full_like(o["logprob"][given & (mine == -math.inf)], -math.inf))
    assert (o["logprob"][~given] == 0).all() and (o["rank"][~given] == -1).all()
    xd = x.to(DEV)
    at = xd.gather(2, tok.to(DEV).long().clamp(min=0)[..., None])
    assert torch.equal(o["rank"][given], (xd > at).sum(dim=-1).to(torch.int32)[given])
    h = -(torch.where(p > 0, p * lp, 0.0)).sum(dim=-1)
    assert ((o["entropy"].double() - h).abs() <= off_z + off * (1 + h) + 2.0 ** -21 * h + 1e-37).all()
    if k:
        order = torch.sort(xd.cpu(), dim=-1, descending=True, stable=True).indices[..., :k].to(DEV)
        assert torch.equal(o["ids"], order.to(torch.int32))
        want, zk = lp.gather(2, order), z.gather(2, order)
        fin = torch.isfinite(want)
        assert ((o["lps"].double() - want).abs() <= off[..., None] + 2.0 ** -21 * (lnz[..., None] + zk) + 1e-37)[fin].all()
        assert (o["lps"][~fin] == -math.inf).all()
    return o


@pytest.mark.parametrize("V", [2, 3, 5, 63, 64, 65, 1000, 1024, 4097, 31999, 32000, 32003, 32769, 50257, 65536, 100003, 131072, 262147])
@pytest.mark.parametrize("k", [0, 1, 2, 5, 32])
def test_vocabularies(V, k):
    g = torch.Generator().manual_seed(V + k)
    x = torch.randn(2, 3, V, generator=g) * 3
    x[..., :4] += 9 * torch.rand(2, 3, min(V, 4), generator=g)
    tok = torch.randint(-1, V, (2, 3), generator=g)
    check(x, tok, k=min(k, V))


@pytest.mark.parametrize("rows", [(1, 1), (1, 128), (7, 33), (16, 64)])
@pytest.mark.parametrize("V", [1024, 32000])
def test_rows(rows, V):
    g = torch.Generator().manual_seed(V)
    x = torch.randn(*rows, V, generator=g) * 4
    check(x, torch.randint(-1, V, rows, generator=g), tau=0.7, k=10)


@pytest.mark.parametrize("tau", [0.05, 0.7, 1.0, 3.0, 1e4])
def test_temperatures(tau):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2, 4, 5000, generator=g) * 3
    check(x, torch.randint(0, 5000, (2, 4), generator=g), tau=tau, k=7)


@pytest.mark.parametrize("V", [700, 32000, 40000])
def test_equal_and_masked_logits(V):
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(6, 1, V, generator=g) * 2).round()                       # many ties
    x[1] = 0.0                                                                # all equal
    x[2] = -math.inf
    x[2, 0, [5, 77, V - 1]] = torch.tensor([1.0, 3.0, 1.0])                   # three tokens are left, fewer than k
    x[3] = -0.0
    x[3, 0, ::2] = 0.0                                                        # -0 and +0 are equal
    x[4] = torch.finfo(torch.float32).min                                     # the lowest value, and one that is not
    x[4, 0, V // 2] = 1.0
    x[5, 0, V - 2] = 60.0                                                     # nothing beside one token
    tok = torch.tensor([[3], [V - 1], [6], [1], [V // 2], [V - 2]])
    for k in (0, 5, 32):
        check(x, tok, k=k)


def test_small_probabilities_keep_their_digits():
    """One token far ahead: its log probability and the entropy are tiny and right to many digits."""
    x = torch.full((1, 3, 1000), -30.0)
    x[0, :, 17] = torch.tensor([0.0, -10.0, 5.0])
    o = check(x, torch.full((1, 3), 17))
    y = x.double()
    lp = torch.log_softmax(y, dim=-1)
    small = torch.log1p(999 * torch.exp(torch.tensor([-30.0, -20.0, -35.0]).double()))
    assert ((o["logprob"][0].cpu().double() + small).abs() <= 1e-5 * small).all()
    h = small + 999 * torch.exp(torch.tensor([-30.0, -20.0, -35.0]).double()) * torch.tensor([30.0, 20.0, 35.0]).double() / small.exp()
    assert ((o["entropy"][0].cpu().double() - h).abs() <= 1e-5 * h).all() and float(lp[0, 0, 17]) < 0


@pytest.mark.parametrize("V", [900, 40000])
def test_rows_without_a_distribution(V):
    x = torch.randn(5, 1, V, generator=torch.Generator().manual_seed(1))
    x[0, 0, 7] = math.nan
    x[1, 0, V - 3] = math.inf
    x[2] = -math.inf
    x[3, 0, V - 1] = math.nan
    o = call(x, torch.full((5, 1), 11), k=4)
    for name in ("logprob", "entropy"):
        assert torch.isnan(o[name][:4]).all() and torch.isfinite(o[name][4]).all()
    assert torch.isnan(o["lps"][:4]).all() and o["ids"][1, 0, 0] == V - 3 and o["ids"][2, 0].tolist() == [0, 1, 2, 3]
    y = x.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    assert torch.equal(o["ids"][0, 0].cpu().long(), torch.sort(y[0, 0], descending=True, stable=True).indices[:4])
    assert torch.equal(o["rank"].cpu()[:, 0].long(), (y[:, 0] > y[:, 0, 11:12]).sum(dim=-1)) and o["flags"] == 0


def test_tokens_that_are_not_there():
    V = 100
    x = torch.randn(1, 4, V, generator=torch.Generator().manual_seed(1))
    o = call(x, torch.tensor([[-1, V, -2, 5]]))
    lp = torch.log_softmax(x.double(), dim=-1)
    want = torch.tensor([0.0, lp[0, 1, 0], lp[0, 2, 0], lp[0, 3, 5]]).double()
    assert o["flags"] == 2 and ((o["logprob"][0].cpu().double() - want).abs() <= 1e-5).all()
    assert o["rank"][0].tolist() == [-1, int((x[0, 1] > x[0, 1, 0]).sum()), int((x[0, 2] > x[0, 2, 0]).sum()), int((x[0, 3] > x[0, 3, 5]).sum())]


@pytest.mark.parametrize("want", [("logprob",), ("rank",), ("entropy",), ("logprob", "entropy"), ()])
def test_outputs_that_are_not_wanted(want):
    V = 33000
    x = torch.randn(2, 2, V, generator=torch.Generator().manual_seed(1))
    tok = torch.randint(0, V, (2, 2), generator=torch.Generator().manual_seed(2))
    full = call(x, tok, k=3)
    some = call(x, tok if set(want) & {"logprob", "rank"} else None, k=3 if not want else 0, want=want)
    for name in want:
        assert torch.equal(some[name], full[name])
    if not want:
        assert torch.equal(some["ids"], full["ids"]) and torch.equal(some["lps"], full["lps"])


def test_on_another_stream_and_in_a_graph():
    B, T, V, k = 2, 5, 33001, 6
    c = context(2, 64, B, [-1] + list(range(T - 1)), vocab=V, max_pos=T + 1)
    x = torch.randn(B, T, V, device=DEV)
    tok = torch.randint(0, V, (B, T), device=DEV).to(torch.int32)
    outs = [torch.zeros(B, T, device=DEV), torch.zeros(B, T, dtype=torch.int32, device=DEV), torch.zeros(B, T, device=DEV), torch.zeros(B, T, k, dtype=torch.int32, device=DEV),
            torch.zeros(B, T, k, device=DEV)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        c.hydra_token_logprobs(B, c.ws, x, tok, 1.0, k, *outs)
    st.synchronize()
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.hydra_token_logprobs(B, c.ws, x, tok, 1.0, k, *outs)
    for i in range(4):
        x2 = x.clone()
        if i % 2:
            x.add_(1.0)                                                       # log probabilities do not change, sums do
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[1], want[1]) and torch.equal(outs[3], want[3])
        assert all((a - b).abs().max() <= 1e-4 for a, b in zip((outs[0], outs[2], outs[4]), (want[0], want[2], want[4])))
        x.copy_(x2)
    assert c.read_flags() == 0


@pytest.mark.parametrize("V", [3, 900, 40000])
@pytest.mark.parametrize("k", [0, 3])
def test_a_given_token_whose_logit_is_no_number(V, k):
    """It ranks as one of -infinity does, whatever the sign of the NaN: behind every token over that."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn(4, 2, V, generator=g)
    tok = torch.randint(0, V, (4, 2), generator=g)
    tok[0], tok[1] = 0, V - 1
    x.scatter_(2, tok[..., None], math.nan)
    x[1] = torch.where(torch.isnan(x[1]), -x[1], x[1])
    x[2, :, ::2] = torch.where(torch.isnan(x[2, :, ::2]), x[2, :, ::2], -math.inf)
    x[3, 1] = math.nan                                                        # nothing over -infinity: all rank first
    o = call(x, tok, k=k)
    want = (x.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf) > -math.inf).sum(dim=-1)
    assert torch.equal(o["rank"].cpu().long(), want) and want[3, 1] == 0
    assert torch.isnan(o["logprob"]).all() and torch.isnan(o["entropy"]).all() and o["flags"] == 0
