"""Sampling from given uniform numbers, against the definition in 64 bits."""
import math
import os
import random
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2505_24544_b200 import binding as b

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def draw(row, t, k, p, mp, u):
    """Token and ln probability; row: float64 array without NaN."""
    order = np.argsort(-row, kind="stable")
    top = row[order[0]]
    if top == -math.inf:
        return -1, math.nan
    if not t > 0:
        return int(order[0]), 0.0
    if 0 < k < len(order):
        order = order[:k]
    if p <= 0 or mp > 1:
        order = order[:1]
    with np.errstate(invalid="ignore"):
        d = np.where(row[order] == top, 0.0, (row[order] - top) / t)
    d = np.where(np.isnan(d) | (row[order] == -math.inf), -math.inf, d)          # infinite temperature below an infinite logit; masked
    if p < 1:
        run = np.cumsum(np.exp(d))
        n = min(int(np.searchsorted(run, p * run[-1], side="left")) + 1, len(order))
        order, d = order[:n], d[:n]
    if mp > 0:
        keep = d >= math.log(mp)
        keep[0] = True
        order, d = order[keep], d[keep]
    at = np.argsort(order, kind="stable")
    ids, w = order[at], np.exp(d[at])
    run = np.cumsum(w)
    i = min(int(np.searchsorted(run, u * run[-1], side="right")), len(ids) - 1)
    return int(ids[i]), float(d[at][i] - math.log(run[-1]))


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """Weights are off by 2^-46 of the largest and 2^-45 of themselves at most: a sum of V of them, relative to the total, by less than
    (V + 2) 2^-45.  A border that a sum comes nearer to may fall to either side: tokens of either are right."""
    rows, v = logits.shape
    dev = lambda x, dt: None if x is None else torch.tensor(x, dtype=dt, device="cuda")
    tokens, logp = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    b.beagle_sample(logits, dev(u, torch.float32), tokens, dev(temperature, torch.float32), dev(top_k, torch.int32), dev(top_p, torch.float32),
                    dev(min_p, torch.float32), logp)
    z = logits.detach().cpu().double().numpy()
    z = np.where(np.isnan(z), -math.inf, z)
    f32 = lambda x: float(np.float32(x))
    eps = (v + 2) * 2.0 ** -45
    for i in range(rows):
        t = 1.0 if temperature is None else f32(temperature[i])
        k = 0 if top_k is None else top_k[i]
        p = 1.0 if top_p is None or not f32(top_p[i]) < 1 else f32(top_p[i])
        mp = 0.0 if min_p is None or not f32(min_p[i]) > 0 else f32(min_p[i])
        ui = min(max(f32(u[i]), 0.0), 1.0)
        want = {}
        for dp in ([0.0] if p >= 1 or p <= 0 else [0.0, -eps, eps]):
            for du in (0.0, -eps, eps):
                tok, lp = draw(z[i], t, k, min(p + dp, 1.0), mp, min(max(ui + du, 0.0), 1.0 - 2.0 ** -53))
                want.setdefault(tok, []).append(lp)
        got, lp = int(tokens[i]), float(logp[i])
        assert got in want, (i, got, want, t, k, p, mp, ui)
        if got == -1:
            assert math.isnan(lp)
        else:
            # the total's relative error, double arithmetic, one rounding to fp32
            assert min(abs(lp - x) for x in want[got]) <= 2 * eps + 2.0 ** -24 * abs(lp) + 2.0 ** -40, (lp, want[got])
    again = torch.empty_like(tokens)
    b.beagle_sample(logits, dev(u, torch.float32), again, dev(temperature, torch.float32), dev(top_k, torch.int32), dev(top_p, torch.float32),
                    dev(min_p, torch.float32))
    assert torch.equal(tokens, again)
    return tokens.tolist()


def noise(rows, v, std, dtype, seed=0):
    return (torch.randn(rows, v, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * std).to(DT[dtype])


def params(rows, seed, v):
    r = random.Random(seed)
    return dict(u=[r.random() for _ in range(rows)], temperature=[r.choice([0.0, 0.3, 0.8, 1.0, 1.7]) for _ in range(rows)],
                top_k=[r.choice([0, -1, 1, 2, 40, 700, v, v + 5]) for _ in range(rows)], top_p=[r.choice([1.0, 0.1, 0.5, 0.9, 0.999, 2.0]) for _ in range(rows)],
                min_p=[r.choice([0.0, 0.01, 0.3, 1.0]) for _ in range(rows)])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,v", [(1, 1), (3, 2), (40, 33), (20, 1000), (5, 4099), (9, 32000), (40, 8193), (1, 128256), (3, 262144), (150, 20001)])
@pytest.mark.parametrize("std", [0.05, 3.0, 20.0])
def test_mixed_requests(dtype, rows, v, std):
    """bf16 logits have many equal values, std 0.05 a nearly flat distribution (whole vocabularies inside a filter)."""
    check(noise(rows, v, std, dtype, rows + v), **params(rows, v, v))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("only", ["temperature", "top_k", "top_p", "min_p"])
def test_one_filter(dtype, only):
    rows, v = 33, 50257
    p = params(rows, 5, v)
    check(noise(rows, v, 2.0, dtype, 8), u=p["u"], **{only: p[only]})


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_equal_logits(dtype):
    """Borders inside long runs of equal logits: the lower ids are kept.  (More of them than are compared pairwise.)"""
    v = 30011
    z = torch.zeros(8, v, dtype=DT[dtype], device="cuda")
    z[:, ::3] = 1.0
    z[:, 1::3] = -2.0
    z[:, 7] = 2.0
    us = [0.0, 0.3, 0.999, 0.5, 0.25, 0.75, 0.9999, 0.1]
    check(z, us, top_k=[1, 2, 5000, 10001, 10005, 25000, 29999, 600])
    check(z, us, top_p=[0.001, 0.1, 0.5, 0.9, 0.95, 0.99, 0.9999, 0.6])
    check(z, us, top_k=[20000] * 8, top_p=[0.001, 0.1, 0.5, 0.9, 0.95, 0.99, 0.9999, 0.6], temperature=[0.5, 1, 2, 4, 1, 1, 9, 1])


def test_borders_that_are_exact():
    """Equal weights: sums are exact on both sides, so are the borders."""
    v = 4096
    z = torch.full((6, v), 3.5, device="cuda")
    tokens = check(z, [0.0, 0.25, 0.5, 0.75, 0.25, 0.5], top_p=[1.0, 1.0, 1.0, 1.0, 0.5, 0.25])
    assert tokens[:3] == [0, 1024, 2048] and tokens[4:] == [512, 512]
    tokens = check(z, [0.0, 0.25, 0.5, 0.75, 0.25, 0.5], top_k=[4, 4, 4, 4, 1000, 0])
    assert tokens == [0, 1, 2, 3, 250, 2048]


@pytest.mark.parametrize("low", [-1e4, -3.0e38, -math.inf, math.nan])
def test_masked_tokens(low):
    """Masks of every kind, NaN among them, in rows that keep a few tokens, one, and none."""
    v = 20000
    z = torch.full((6, v), low, device="cuda")
    z[0, [5, 700, 19999]] = torch.tensor([1.0, 2.0, 1.5], device="cuda")
    z[1, 12345] = -7.0
    z[3, :9000] = noise(1, 9000, 2.0, "fp32", 4)[0]
    z[4, 100] = -3.0e38
    p = dict(u=[0.5, 0.9, 0.9, 0.3, 0.7, 0.0])
    check(z, **p)
    check(z, **p, temperature=[1.0, 0.5, 0.0, 2.0, 0.1, 1.0], top_k=[2, 0, 0, 50, 3, 0], top_p=[0.9, 0.5, 1.0, 0.8, 0.9, 0.9])
    tokens = check(z, **p, top_k=[2, 2, 2, 2, 2, 2], min_p=[0.5] * 6)
    if low != low or low == -math.inf:
        assert tokens[2] == -1 and tokens[5] == -1
    check(torch.nan_to_num(z, nan=low, neginf=low).to(torch.bfloat16), **p, top_p=[0.9] * 6)


def test_infinite_logits_and_parameters_at_their_ends():
    z = noise(12, 5000, 2.0, "fp32", 3)
    z[0, [17, 40]] = math.inf
    z[1, 3] = math.inf
    z[2, 3] = math.inf
    inf, nan = math.inf, math.nan
    check(z, u=[0.9, 0.2, 0.5, 0.0, 1.0, 0.99999994, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5], temperature=[1.0, 0.0, inf, inf, 1e-30, 1e-3, 1e30, nan, -1.0, 1.0, 1.0, 1.0],
          top_p=[0.9, 0.9, 1.0, 1.0, 0.9, 1e-30, 0.5, 0.5, 0.5, 0.0, -1.0, nan], min_p=[0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 2.0])
    check(z, u=[0.5] * 12, min_p=[nan, 1.0, 1.5, 0.5, -1.0, 0.0, 1e-30, 1e-8, 0.1, 0.2, 0.3, 0.9])


def test_unaligned_and_strided_rows_another_stream():
    big = noise(7, 4099 + 13, 3.0, "bf16", 5)
    side = torch.cuda.Stream()
    for off in (0, 1, 3, 8, 13):
        part = big[:, off:off + 4099]
        check(part, **params(7, off, 4099))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            check(part.float()[:, 1:], **params(7, off, 4098))
    torch.cuda.synchronize()


def test_captured_and_replayed_with_new_numbers():
    z, u = noise(4, 32000, 3.0, "fp32", 6), torch.rand(4, device="cuda")
    tokens, temp = torch.empty(4, dtype=torch.int32, device="cuda"), torch.full((4,), 0.7, device="cuda")
    b.beagle_sample(z, u, tokens, temperature=temp)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.beagle_sample(z, u, tokens, temperature=temp)
    for i in range(5):
        u.copy_(torch.rand(4, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
        z.copy_(noise(4, 32000, 3.0, "fp32", 100 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert tokens.tolist() == check(z, u.tolist(), temperature=[0.7] * 4)


def test_frequencies_follow_the_weights():
    """Evenly spaced numbers through the inverse distribution: every token as often as its share, to within one."""
    n = 5000
    z = torch.tensor([[0.0, 1.0, -1.0, 2.0, 0.5]], device="cuda").repeat(n, 1)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tokens = torch.empty(n, dtype=torch.int32, device="cuda")
    b.beagle_sample(z, u, tokens)
    share = torch.softmax(z[0].double(), 0) * n
    assert bool(((torch.bincount(tokens.long(), minlength=5).double() - share).abs() <= 1.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["negative", "positive", "zero top", "tiny", "mostly zero", "wide", "one value", "subnormal", "few codes"])
def test_where_the_logits_lie(dtype, kind):
    """All of one sign, around 0, of any size: codes of either sign, the logits nearest to 0, and rows whose border lies among those."""
    v, g = 30000, torch.Generator(device="cuda").manual_seed(9)
    z = torch.randn(10, v, generator=g, device="cuda")
    small = torch.rand(10, v, generator=g, device="cuda")
    z = {"negative": z.abs() * -3 - 0.5, "positive": z.abs() * 3, "zero top": torch.where(small < 0.01, 0.0, z.abs() * -2), "tiny": z * 1e-25, "mostly zero": torch.where(small < 0.02, z * 4, z * 1e-6),
         "wide": z * torch.exp(small * 40 - 35), "one value": z * 0 - 1.5, "subnormal": z * 1e-39, "few codes": torch.randint(0, 5, (10, v), generator=g, device="cuda") * 1.0 - 2}[kind]
    z = z.to(DT[dtype])
    us = [0.0, 0.1, 0.2, 0.3, 0.4, 0.5, 0.6, 0.7, 0.9, 0.999]
    if kind == "subnormal":                              # they count as 0: all equal
        z = torch.where(z.float().abs() < 1.1754944e-38, torch.zeros_like(z), z)
    check(z, us)
    check(z, us, top_p=[0.001, 0.2, 0.4, 0.5, 0.6, 0.7, 0.8, 0.9, 0.99, 0.9999])
    check(z, us, temperature=[0.2, 0.5, 1, 2, 5, 0.2, 0.5, 1, 2, 5], top_p=[0.5] * 10, min_p=[0.0, 0.5, 0.01, 0.9, 0.99, 0.001, 0.2, 0.7, 1e-6, 0.3])
    check(z, us, temperature=[0.3] * 10, top_k=[1, 3, 10, 100, 1000, 5000, 20000, 29999, 0, 2], top_p=[0.7] * 10)
    masked = torch.where(small < 0.7, torch.full_like(z, -math.inf), z)
    check(masked, us, top_p=[0.9] * 5 + [1.0] * 5)


def test_subnormal_logits_count_as_zero():
    z = torch.zeros(1, 8, device="cuda")
    z[0, 3], z[0, 5] = 1e-39, -1e-40
    tokens = torch.empty(1, dtype=torch.int32, device="cuda")
    for u, want in ((0.0, 0), (0.3, 2), (0.99, 7)):
        b.beagle_sample(z, torch.tensor([u], device="cuda"), tokens)
        assert tokens.item() == want
    b.beagle_sample(z, torch.tensor([0.9], device="cuda"), tokens, top_k=torch.tensor([2], dtype=torch.int32, device="cuda"))
    assert tokens.item() == 1
    b.beagle_sample(z, torch.tensor([0.9], device="cuda"), tokens, temperature=torch.zeros(1, device="cuda"))
    assert tokens.item() == 0


def test_many_rows_past_32_bit_offsets():
    """17000 rows of 128256 (2.2e9 logits): the blocks walk over the rows; each row's token is its own peak, its neighbours' NaN do not reach it."""
    rows, v = 17000, 128256
    z = torch.zeros(rows, v, dtype=torch.bfloat16, device="cuda")
    peak = torch.randint(0, v, (rows,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    z.scatter_(1, peak[:, None], 40.0)
    z[::7] = float("nan")
    tokens, u = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.rand(rows, device="cuda")
    b.beagle_sample(z, u, tokens)
    want = peak.to(torch.int32)
    want[::7] = -1
    assert torch.equal(tokens, want)
    b.beagle_sample(z, u, tokens, top_k=torch.full((rows,), 5, dtype=torch.int32, device="cuda"), top_p=torch.full((rows,), 0.5, device="cuda"))
    assert torch.equal(tokens, want)


def test_two_streams_at_once():
    z = noise(100, 50000, 3.0, "fp32", 12)
    p = params(100, 3, 50000)
    want = check(z, **p)
    dev = lambda x, dt: torch.tensor(x, dtype=dt, device="cuda")
    args = dict(temperature=dev(p["temperature"], torch.float32), top_k=dev(p["top_k"], torch.int32), top_p=dev(p["top_p"], torch.float32), min_p=dev(p["min_p"], torch.float32))
    u = dev(p["u"], torch.float32)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                t = torch.empty(100, dtype=torch.int32, device="cuda")
                b.beagle_sample(z, u, t, **args)
                outs.append(t)
    torch.cuda.synchronize()
    assert all(t.tolist() == want for t in outs)


def test_refusals_of_the_binding():
    z, u, t = torch.zeros(3, 10, device="cuda"), torch.zeros(3, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (dict(logits=z.double()), dict(logits=z[0]), dict(logits=z.t()), dict(logits=z.cpu()), dict(u=u[:2]), dict(u=u.double()), dict(tokens=t.long()), dict(tokens=t.cpu()),
                dict(temperature=u.cpu()), dict(top_k=u), dict(top_p=t), dict(logp=t)):
        a = dict(logits=z, u=u, tokens=t)
        a.update(bad)
        with pytest.raises(ValueError):
            b.beagle_sample(**a)
    with pytest.raises(b.BeagleError):
        b.beagle_sample(torch.zeros(1, 2 ** 18 + 1, device="cuda"), u[:1], t[:1])
    b.beagle_sample(z[:0], u[:0], t[:0])                 # no rows: nothing to do


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_drafts_for_acceptance_under_sampling(dtype):
    """Tokens drawn with beagle_sample from the draft's own distribution, then beagle_verify_sample: with equal draft and target logits every
    draft is accepted, and the extra token is the one that beagle_sample draws from the same numbers."""
    from paper_2505_24544_b200 import workloads as WL
    from paper_2505_24544_b200.binding import BeagleHead
    w = WL.WORKLOADS["c1_tiny_fp32"]
    head = BeagleHead.from_workload(w, WL.make_weights(w), device="cuda:0")
    gamma, B, v = 3, 4, w.vocab
    z = noise(B * (gamma + 1), v, 2.0, dtype, 5).view(B, gamma + 1, v)
    u = torch.rand(B, gamma + 1, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    temp = torch.full((B * (gamma + 1),), 0.8, device="cuda")
    tokens, _ = head.sample(z.view(-1, v), u.view(-1), temperature=temp)
    drafts = tokens.view(B, gamma + 1)
    accept, out = head.verify_sample(drafts[:, :gamma].contiguous(), z[:, :gamma].float().transpose(0, 1).contiguous(), z, torch.rand(B, gamma, device="cuda"), u[:, gamma].contiguous(), 0.8)
    assert accept.tolist() == [gamma] * B and torch.equal(out, drafts)


@pytest.mark.parametrize("v", [300, 5000, 32000, 128256])
@pytest.mark.parametrize("kind", ["noise", "ties", "one high", "two sides", "masked"])
def test_large_top_k_by_code(v, kind):
    """bf16 with top-k beyond the candidates that are compared pairwise: the border on a code, on one of many equal logits, among the
    logits next to 0 that have no code of their own, behind the last logit that weighs anything."""
    rows = 24
    z = noise(rows, v, 3.0, "bf16", v)
    if kind == "ties":
        z = (z * 2).round() / 2
    elif kind == "one high":                             # nearly all lie below 2^-11 of the largest
        z = z * 2.0 ** -10
        z[:, 17] = 9.0
    elif kind == "two sides":                            # -0.0, 0, both signs, far below the largest
        z = torch.where(z > 0, z * 2.0 ** -14, z)
        z[:, ::5] = 0.0
        z[:, 1::5] = -0.0
    elif kind == "masked":
        z[:, torch.arange(v, device="cuda") % 7 != 3] = float("-inf")
        z[:, ::11] = float("nan")
    r = random.Random(v)
    check(z, u=[r.random() for _ in range(rows)], temperature=[r.choice([0.3, 1.0, 1.7]) for _ in range(rows)],
          top_k=[r.choice([257, 258, 299, 400, 1000, 3000, v // 2, v - 1]) for _ in range(rows)], top_p=[r.choice([1.0, 0.2, 0.9, 0.9999]) for _ in range(rows)],
          min_p=[r.choice([0.0, 0.0, 0.05]) for _ in range(rows)])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 2, 31, 32, 33, 64, 65, 128, 129, 255, 256, 257, 258, 3499, 3500, 3501])
def test_numbers_of_candidates(dtype, m):
    """As many tokens as min-p keeps, around the borders between the ways to finish a row."""
    rows, v = 4, 20000
    z = torch.full((rows, v), -5.0, dtype=DT[dtype], device="cuda")
    at = torch.randperm(v, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda")[:m]
    z[:, at] = torch.rand(rows, m, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda").to(DT[dtype])
    check(z, u=[0.0, 0.3, 0.77, 0.99999994], min_p=[0.1] * rows)
    check(z, u=[0.0, 0.3, 0.77, 0.99999994], top_k=[m] * rows, top_p=[1.0, 0.5, 0.9, 0.99])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_more_rows_than_fit_the_gpu(dtype):
    """Clusters take over rows of others; captured and replayed too, with other parameters in the same tensors."""
    rows, v = 700, 33000
    z = noise(rows, v, 3.0, dtype, 4)
    p = params(rows, 6, v)
    want = check(z, **p)
    dev = lambda x, dt: torch.tensor(x, dtype=dt, device="cuda")
    args = dict(temperature=dev(p["temperature"], torch.float32), top_k=dev(p["top_k"], torch.int32), top_p=dev(p["top_p"], torch.float32), min_p=dev(p["min_p"], torch.float32))
    u, tokens = dev(p["u"], torch.float32), torch.zeros(rows, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.beagle_sample(z, u, tokens, **args)
    for turn in range(5):
        tokens.zero_()
        graph.replay()
        assert tokens.tolist() == want
    for x in (u, *args.values()):
        x.copy_(x.flip(0))
    z.copy_(z.flip(0))
    graph.replay()
    assert tokens.tolist() == want[::-1]


SHORT_WAIT = """
import os
import torch
from paper_2505_24544_b200 import binding as b
g = torch.Generator(device="cuda").manual_seed(4)
for dtype, rows, v in ((torch.bfloat16, 700, 33000), (torch.float32, 1000, 5000), (torch.float32, 600, 33000)):
    z, u = (torch.randn(rows, v, generator=g, device="cuda") * 3).to(dtype), torch.rand(rows, generator=g, device="cuda")
    want, right = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    b.beagle_sample(z, u, want, logp=right)
    tokens, logp = torch.full_like(want, 1 << 20), torch.full_like(right, 7.0)
    os.environ["BEAGLE_SAMPLE_TRIES"] = "0"
    b.beagle_sample(z, u, tokens, logp=logp)
    alone = torch.full_like(want, 1 << 20)
    b.beagle_sample(z, u, alone)
    del os.environ["BEAGLE_SAMPLE_TRIES"]
    torch.cuda.synchronize()
    for t in (tokens, alone):
        assert bool(((t == want) | (t == -1)).all()) and bool((t == -1).any()), t.tolist()
    assert bool(((logp == right) | logp.isnan()).all()) and bool(logp.isnan().any())
    b.beagle_sample(z, u, tokens, logp=logp)
    assert torch.equal(tokens, want) and torch.equal(logp, right)
print("no row kept what it had")
"""


def test_a_wait_that_runs_out_leaves_no_old_tokens():
    """In the build for tests the wait for another row can be given no tries: clusters then end after their first row, and of the rows that
    nobody does none keeps what was there; the next call is whole again."""
    from paper_2505_24544_b200 import build
    env = dict(os.environ, BEAGLE_LIBRARY=build.build(checked=True))
    r = subprocess.run([sys.executable, "-c", SHORT_WAIT], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "no row kept what it had" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
