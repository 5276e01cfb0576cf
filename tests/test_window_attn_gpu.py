"""Windowed attention over whole sequences, forward and backward, against the definition in 64 bits."""
import random

import pytest
import torch

from paper_2505_24544_b200 import binding as b

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def visible(n, m, window, sinks, strict):
    last = torch.arange(n)[:, None] + (m - n - int(strict))
    j = torch.arange(m)[None, :]
    seen = j <= last
    return seen & ((j > last - window) | (j < sinks)) if window > 0 else seen


def reference(q, k, v, do, q_len, kv_len, window, sinks, strict, dtype):
    """Outputs and gradients in 64 bits with a bound on each one's error: {name: (value, bound)}."""
    q, k, v, do = (x.detach().cpu().double() for x in (q, k, v, do))
    hq, dh = q.shape[1:]
    G = hq // k.shape[1]
    half, weight = HALF[dtype], HALF["bf16"] if dtype == "bf16" else 0.0         # weight: P and dS enter their products in bf16
    res = {n: [torch.zeros_like(x), torch.zeros_like(x)] for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    lse_all, lse_tol = torch.full(q.shape[:2], -torch.inf, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    a = c = 0
    u = 2.0 ** -24
    for n, m in zip(q_len, kv_len):
        seen = visible(n, m, window, sinks, strict)
        some = seen.any(-1)
        for h in range(hq):
            x, y, z, g = q[a:a + n, h], k[c:c + m, h // G], v[c:c + m, h // G], do[a:a + n, h]
            s = (x @ y.T) / dh ** 0.5
            size = torch.where(seen, (x.abs() @ y.abs().T) / dh ** 0.5, 0.0).amax(-1, keepdim=True) if m else torch.zeros(n, 1).double()
            s = s.masked_fill(~seen, -torch.inf)
            lse = torch.logsumexp(s, -1)
            p = torch.exp(s - torch.where(some, lse, 0.0)[:, None])
            score = (dh + 8) * u * size + 2.0 ** -21 * (1 + size)                # a score, its exponential's argument and the exponential
            l_err = score[:, 0] + m * u + 2.0 ** -21 * (1 + torch.where(some, lse, 0.0).abs())
            lse_all[a:a + n, h], lse_tol[a:a + n, h] = lse, l_err
            o, mass = p @ z, p @ z.abs()
            o_err = (2 * score + 2 * m * u + weight) * mass
            o_err = o_err + half * (o.abs() + o_err) + 2.0 ** -40
            res["out"][0][a:a + n, h], res["out"][1][a:a + n, h] = o, o_err
            p_err = (2 * score + l_err[:, None]) * p                             # recomputed from the log-sum-exp
            dp, dp_size = g @ z.T, g.abs() @ z.abs().T
            delta = (g * o).sum(-1, keepdim=True)
            d_err = (g.abs() * o_err).sum(-1, keepdim=True) + (dh + 2) * u * (g.abs() * o.abs()).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            ds_err = p_err * (dp - delta).abs() + p * ((dh + 2) * u * dp_size + d_err)
            ds_err = ds_err + weight * (ds.abs() + ds_err)
            pw_err = p_err + weight * (p + p_err)
            dq, dk, dv = ds @ y / dh ** 0.5, ds.T @ x / dh ** 0.5, p.T @ g
            eq = (ds_err @ y.abs() + m * u * ds.abs() @ y.abs()) / dh ** 0.5
            ek = (ds_err.T @ x.abs() + n * G * u * ds.abs().T @ x.abs()) / dh ** 0.5
            ev = pw_err.T @ g.abs() + n * G * u * p.T @ g.abs()
            res["dq"][0][a:a + n, h], res["dq"][1][a:a + n, h] = dq, eq + half * (dq.abs() + eq) + 2.0 ** -40
            res["dk"][0][c:c + m, h // G] += dk
            res["dk"][1][c:c + m, h // G] += ek
            res["dv"][0][c:c + m, h // G] += dv
            res["dv"][1][c:c + m, h // G] += ev
        a, c = a + n, c + m
    for x in ("dk", "dv"):                                                       # rounded once, after the heads were added
        res[x][1] += half * (res[x][0].abs() + res[x][1]) + 2.0 ** -40
    res["lse"] = (lse_all, lse_tol)
    return res


def compare(got, ref):
    for name, x in got.items():
        value, tol = ref[name]
        x = x.cpu().double()
        if name == "lse":
            none = torch.isinf(value)
            assert torch.equal(none, torch.isinf(x) & (x < 0)), name
            x, value, tol = x[~none], value[~none], tol[~none]
        bad = ~((x - value).abs() <= tol)
        assert not bool(bad.any()), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float(((x - value).abs() / tol).nan_to_num(9e9).max()):.3g} of the bound, first at {bad.nonzero()[0].tolist()}"


def inputs(q_len, kv_len, hq, hkv, dh, dtype, seed, spread=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rows(n, h, std=1.0):
        return (torch.randn(n, h, dh, generator=g, device="cuda") * std).to(DT[dtype])
    return rows(sum(q_len), hq, spread), rows(sum(kv_len), hkv), rows(sum(kv_len), hkv), rows(sum(q_len), hq)


def run(q, k, v, do, q_len, kv_len, window, sinks, strict):
    out, lse = torch.full_like(q, 7.0).contiguous(), torch.full(q.shape[:2], 7.0, device="cuda")
    b.beagle_window_attn_forward(q, k, v, q_len, kv_len, out, lse, window, sinks, strict)
    grads = [torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda") for x in (q, k, v)]
    b.beagle_window_attn_backward(q, k, v, out, lse, do, q_len, kv_len, *grads, window, sinks, strict)
    return dict(zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *grads)))


HEADS = [("bf16", 4, 4, 128), ("bf16", 8, 2, 128), ("bf16", 4, 1, 64), ("bf16", 3, 1, 128), ("fp32", 4, 4, 64), ("fp32", 4, 2, 128), ("fp32", 3, 1, 16),
         ("fp32", 2, 2, 32)]
LENGTHS = [([1], [1]), ([2, 1, 3], [2, 1, 3]), ([127, 128, 129], [127, 128, 129]), ([300], [300]), ([0, 70, 0, 5], [3, 70, 0, 5]), ([1, 1, 1], [500, 64, 1]),
           ([40, 200], [333, 201]), ([130, 65], [20, 0]), ([257], [400])]


@pytest.mark.parametrize("dtype,hq,hkv,dh", HEADS)
@pytest.mark.parametrize("q_len,kv_len", LENGTHS)
@pytest.mark.parametrize("window,sinks,strict", [(0, 0, False), (0, 5, True), (1, 0, False), (1, 2, True), (64, 4, True), (100, 0, False), (33, 150, False),
                                                (128, 128, True), (1000, 3, False)])
def test_against_the_definition(dtype, hq, hkv, dh, q_len, kv_len, window, sinks, strict):
    x = inputs(q_len, kv_len, hq, hkv, dh, dtype, 3)
    compare(run(*x, q_len, kv_len, window, sinks, strict), reference(*x, q_len, kv_len, window, sinks, strict, dtype))


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 2, 1, 128), ("bf16", 8, 1, 64), ("fp32", 2, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(200, 4), (0, 0), (640, 300), (7, 1)])
def test_long_sequences(dtype, hq, hkv, dh, window, sinks):
    """Many tiles, several segments of the sinks' gradients, rows that see tens of tiles."""
    q_len, kv_len = [1501, 700], [1501, 2100]
    x = inputs(q_len, kv_len, hq, hkv, dh, dtype, 5)
    compare(run(*x, q_len, kv_len, window, sinks, False), reference(*x, q_len, kv_len, window, sinks, False, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_sequences(dtype):
    """Sixty-four sequences of zero to a few hundred rows in one call."""
    r = random.Random(1)
    q_len = [r.choice([0, 1, 2, 17, 64, 130, 200]) for _ in range(64)]
    kv_len = [n + r.choice([0, 0, 1, 90]) for n in q_len]
    x = inputs(q_len, kv_len, 2, 1, 64, dtype, 6)
    compare(run(*x, q_len, kv_len, 48, 3, True), reference(*x, q_len, kv_len, 48, 3, True, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_steep_scores(dtype):
    """Scores that rise by tens of bits along the keys (the reference point moves in every tile) and rows with one dominant key."""
    q_len = kv_len = [400]
    q, k, v, do = inputs(q_len, kv_len, 2, 2, 64, dtype, 8)
    ramp = torch.linspace(0.1, 6, 400, device="cuda")[:, None, None]
    k = (torch.ones_like(k).float() * ramp + 0.1 * k.float()).to(k.dtype)
    q = (q.float().abs() * 0.5).to(q.dtype)
    for window, sinks in ((0, 0), (100, 4)):
        compare(run(q, k, v, do, q_len, kv_len, window, sinks, False), reference(q, k, v, do, q_len, kv_len, window, sinks, False, dtype))


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_slices_of_a_fused_projection(dtype, dh):
    """q, k, v and their gradients as column blocks of one matrix; what lies between and behind is left alone; the same bits as
    from dense tensors."""
    q_len, kv_len, hq, hkv = [100, 37], [100, 37], 4, 2
    rows, width = 137, (hq + 2 * hkv + 1) * dh
    fused = torch.randn(rows + 5, width, device="cuda").to(DT[dtype])
    grad = torch.full_like(fused, 3.0)

    def views(t):
        t = t[:rows]
        return (t[:, :hq * dh].unflatten(1, (hq, dh)), t[:, hq * dh:(hq + hkv) * dh].unflatten(1, (hkv, dh)),
                t[:, (hq + hkv) * dh:(hq + 2 * hkv) * dh].unflatten(1, (hkv, dh)))
    q, k, v = views(fused)
    do = torch.randn(rows, hq, dh, device="cuda").to(DT[dtype])
    dense = run(q.contiguous(), k.contiguous(), v.contiguous(), do, q_len, kv_len, 30, 2, False)
    out = torch.full((rows + 3, hq, dh), 7.0, dtype=DT[dtype], device="cuda")
    lse = torch.full((rows + 3, hq), 7.0, device="cuda")
    b.beagle_window_attn_forward(q, k, v, q_len, kv_len, out[:rows], lse[:rows], 30, 2)
    b.beagle_window_attn_backward(q, k, v, out[:rows], lse[:rows], do, q_len, kv_len, *views(grad), 30, 2)
    assert torch.equal(out[:rows], dense["out"]) and torch.equal(lse[:rows], dense["lse"])
    for x, n in zip(views(grad), ("dq", "dk", "dv")):
        assert torch.equal(x, dense[n])
    assert bool((out[rows:] == 7).all()) and bool((lse[rows:] == 7).all())
    assert bool((grad[rows:] == 3).all()) and bool((grad[:, (hq + 2 * hkv) * dh:] == 3).all())


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_sequences_do_not_mix(dtype, dh):
    """A sequence of NaN between two others changes no bit of theirs, forward or backward."""
    q_len, kv_len = [70, 90, 33], [130, 90, 40]
    x = inputs(q_len, kv_len, 4, 2, dh, dtype, 9)
    for window, sinks in ((0, 0), (20, 3)):
        clean = run(*x, q_len, kv_len, window, sinks, False)
        q, k, v, do = (t.clone() for t in x)
        q[70:160], do[70:160], k[130:220], v[130:220] = (float("nan"),) * 4
        got = run(q, k, v, do, q_len, kv_len, window, sinks, False)
        for name, t in got.items():
            keep = torch.ones(t.shape[0], dtype=torch.bool)
            keep[130:220] = False
            if name in ("out", "lse", "dq"):
                keep[:] = True
                keep[70:160] = False
            assert torch.equal(t[keep.cuda()], clean[name][keep.cuda()]), name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_repeats_streams_and_graphs(dtype):
    """The same bits run after run, on another stream, and from a captured forward and backward pass replayed on new inputs."""
    q_len, kv_len = [150, 260], [150, 300]
    x, y = inputs(q_len, kv_len, 4, 2, 64, dtype, 10), inputs(q_len, kv_len, 4, 2, 64, dtype, 11)
    first, other = run(*x, q_len, kv_len, 50, 4, True), run(*y, q_len, kv_len, 50, 4, True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = run(*x, q_len, kv_len, 50, 4, True)
    side.synchronize()
    assert all(torch.equal(first[n], again[n]) for n in first)
    z = [t.clone() for t in x]
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            res = run(*z, q_len, kv_len, 50, 4, True)
    for src, want in ((y, other), (x, first)):
        for t, s in zip(z, src):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[n], res[n]) for n in res)


def test_gradients_against_differences():
    """Directional derivatives of the definition in 64 bits (central differences) against the kernels' gradients."""
    q_len, kv_len, window, sinks = [40], [60], 16, 3
    x = inputs(q_len, kv_len, 2, 1, 64, "fp32", 12)
    got = run(*x, q_len, kv_len, window, sinks, True)
    ref = reference(*x, q_len, kv_len, window, sinks, True, "fp32")
    q, k, v, do = (t.cpu().double() for t in x)
    seen = visible(40, 60, window, sinks, True)

    def loss(q, k, v):
        s = (torch.einsum("ihd,jgd->hij", q, k) / 8).masked_fill(~seen, -torch.inf)
        return (torch.einsum("hij,jgd->ihd", torch.softmax(s, -1), v) * do).sum()
    for i, name in enumerate(("dq", "dk", "dv")):
        g = torch.Generator().manual_seed(i)
        d = torch.randn(x[i].shape, generator=g, dtype=torch.float64)
        h = 1e-4
        plus, minus = ([t + sign * h * d if j == i else t for j, t in enumerate((q, k, v))] for sign in (1, -1))
        slope = float((loss(*plus) - loss(*minus)) / (2 * h))
        mine = float((got[name].cpu().double() * d).sum())
        # the gradient's own bound along d; the differences are off by h^2 times a third derivative and 2^-52 |loss| / h
        tol = float((ref[name][1] * d.abs()).sum()) + 1e-4
        assert abs(slope - mine) <= tol


def test_refusals():
    x = inputs([5], [5], 2, 1, 64, "bf16", 1)
    q, k, v, do = x
    out, lse = torch.empty_like(q), torch.empty(5, 2, device="cuda")
    with pytest.raises(ValueError):
        b.beagle_window_attn_forward(q, k, v, [4], [5], out, lse)                    # rows and lengths disagree
    with pytest.raises(ValueError):
        b.beagle_window_attn_forward(q, k, v.float(), [5], [5], out, lse)
    with pytest.raises(ValueError):
        b.beagle_window_attn_forward(q.cpu(), k, v, [5], [5], out, lse)
    with pytest.raises(ValueError):
        b.beagle_window_attn_forward(q, k, v, [5], [5], out.transpose(0, 1).contiguous().transpose(0, 1), lse)
    with pytest.raises(b.BeagleError):
        b.beagle_window_attn_forward(q, k, v, [5], [5], out, lse, window=3, sinks=2000)
    with pytest.raises(b.BeagleError):
        b.beagle_window_attn_forward(q, k[:1].expand(5, 1, 64), v, [5], [5], out, lse)      # one key row for all
    b.beagle_window_attn_forward(q, k, v, [5], [5], out, lse)
    with pytest.raises(b.BeagleError):
        b.beagle_window_attn_backward(q, k, v, out, lse, do, [5], [5], torch.empty_like(q), torch.empty_like(k), torch.empty_like(v),
                                      ws=torch.empty(64, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("fp32", 16), ("fp32", 64)])
def test_a_nan_query_stays_in_its_row(dtype, dh):
    """A NaN in one query makes that row's outputs and lse NaN, in that head, and nothing else."""
    q_len, kv_len = [150, 40], [200, 40]
    q, k, v, do = inputs(q_len, kv_len, 4, 2, dh, dtype, 5)
    out, lse = torch.empty_like(q), torch.empty(190, 4, device="cuda")
    b.beagle_window_attn_forward(q, k, v, q_len, kv_len, out, lse, 70, 3)
    bad = q.clone()
    bad[131, 1, 3] = float("nan")
    out2, lse2 = torch.empty_like(q), torch.empty_like(lse)
    b.beagle_window_attn_forward(bad, k, v, q_len, kv_len, out2, lse2, 70, 3)
    assert bool(out2[131, 1].isnan().all()) and bool(lse2[131, 1].isnan())
    out2[131, 1], lse2[131, 1] = out[131, 1], lse[131, 1]
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_row_at_any_distance(dtype):
    """A single query and key taken out of a larger matrix whose rows are an odd number of elements apart."""
    g = torch.Generator(device="cuda").manual_seed(2)
    wide = [torch.randn(2 * (4 * 64 + 1), generator=g, device="cuda").to(DT[dtype]) for _ in range(4)]
    q, k, v, do = (torch.as_strided(x, (1, 4, 64), (257, 64, 1)) for x in wide)
    dense = [x.contiguous().clone() for x in (q, k, v, do)]
    got, want = run(q, k, v, do, [1], [1], 0, 0, False), run(*dense, [1], [1], 0, 0, False)
    for name in want:
        assert torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("hq,hkv,dh", [(2, 2, 64), (4, 1, 32), (2, 1, 128), (3, 3, 16)])
@pytest.mark.parametrize("window,sinks", [(64, 4), (30, 70), (5, 1), (200, 130)])
def test_sinks_past_the_band_fp32(hq, hkv, dh, window, sinks):
    """Long ragged fp32 sequences: the sinks' gradients come from several segments of queries, of several heads."""
    q_len, kv_len = [700, 0, 90, 1], [760, 20, 90, 0]
    q, k, v, do = inputs(q_len, kv_len, hq, hkv, dh, "fp32", 23)
    compare(run(q, k, v, do, q_len, kv_len, window, sinks, True), reference(q, k, v, do, q_len, kv_len, window, sinks, True, "fp32"))


@pytest.mark.parametrize("hq,hkv,dh", [(8, 1, 128), (8, 1, 64), (16, 2, 64), (6, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 0), (200, 4), (30, 140)])
def test_shared_key_tiles(hq, hkv, dh, window, sinks):
    """Few key tiles, many heads on each: several CTAs share a tile's jobs, with and without segments of the sinks."""
    q_len, kv_len = [600, 0, 130, 1], [650, 5, 130, 1]
    x = inputs(q_len, kv_len, hq, hkv, dh, "bf16", 29)
    first = run(*x, q_len, kv_len, window, sinks, False)
    compare(first, reference(*x, q_len, kv_len, window, sinks, False, "bf16"))
    again = run(*x, q_len, kv_len, window, sinks, False)
    for name in first:
        assert torch.equal(first[name], again[name]), name


# Ragged, with empty sequences, queries that see nothing and keys that nobody sees between the others.
MANY_Q = [400, 0, 130, 700, 1, 257, 520, 90, 300, 64, 129, 200]
MANY_KV = [400, 70, 130, 640, 1, 300, 720, 0, 200, 64, 40, 200]


def tiles(lengths, rows):
    return sum(-(-n // rows) for n in lengths)


@pytest.mark.parametrize("hq,hkv,dh", [(16, 16, 128), (16, 16, 64), (32, 16, 64), (32, 4, 128)])
@pytest.mark.parametrize("window,sinks,strict", [(0, 0, False), (64, 4, True), (300, 0, True), (300, 140, False)])
def test_more_items_than_sms(hq, hkv, dh, window, sinks, strict):
    """Every CTA of the backward's query side walks three items or more, its pipeline running on across them, and so does the key side
    where its items are short (a window, at most two query heads a K/V head); elsewhere that is a CTA an item, several waves of them."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert tiles(MANY_Q, 128) * hq >= 3 * sms and (hkv < 16 or tiles(MANY_KV, 128) * hkv >= 3 * sms)
    x = inputs(MANY_Q, MANY_KV, hq, hkv, dh, "bf16", 31)
    first = run(*x, MANY_Q, MANY_KV, window, sinks, strict)
    compare(first, reference(*x, MANY_Q, MANY_KV, window, sinks, strict, "bf16"))
    again = run(*x, MANY_Q, MANY_KV, window, sinks, strict)
    for name in first:
        assert torch.equal(first[name], again[name]), name


@pytest.mark.parametrize("hq,hkv", [(8, 8), (8, 2)])
@pytest.mark.parametrize("dh", [16, 32, 64, 128])
@pytest.mark.parametrize("window,sinks,strict", [(0, 0, False), (100, 70, True)])
def test_large_calls_fp32(hq, hkv, dh, window, sinks, strict):
    """Enough rows for the fp32 kernels' tiles of 64 (the calls of the other tests take 32), at every width."""
    q_len, kv_len = [520, 0, 700, 65], [600, 30, 640, 100]
    assert min(tiles(q_len, 64), tiles(kv_len, 64)) * hq >= 148
    x = inputs(q_len, kv_len, hq, hkv, dh, "fp32", 37)
    first = run(*x, q_len, kv_len, window, sinks, strict)
    compare(first, reference(*x, q_len, kv_len, window, sinks, strict, "fp32"))
    again = run(*x, q_len, kv_len, window, sinks, strict)
    for name in first:
        assert torch.equal(first[name], again[name]), name


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 4, 4, 128), ("bf16", 16, 16, 64), ("bf16", 8, 1, 64), ("fp32", 4, 2, 64), ("fp32", 12, 12, 32)])
@pytest.mark.parametrize("window,sinks", [(30, 140), (64, 4), (100, 600)])
def test_sinks_of_ragged_sequences(dtype, hq, hkv, dh, window, sinks):
    """Sequences with many segments of queries past the sinks' band, with one and with none side by side, some with fewer keys than
    there are sinks: each keeps its own partials."""
    q_len, kv_len = [40, 1400, 0, 131, 500, 1, 90, 300], [40, 1400, 200, 131, 90, 700, 90, 460]
    x = inputs(q_len, kv_len, hq, hkv, dh, dtype, 41)
    first = run(*x, q_len, kv_len, window, sinks, False)
    compare(first, reference(*x, q_len, kv_len, window, sinks, False, dtype))
    again = run(*x, q_len, kv_len, window, sinks, False)
    for name in first:
        assert torch.equal(first[name], again[name]), name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_past_32_bit_offsets(dtype):
    """Queries, outputs and gradients of more than 2^31 elements: a sequence behind them has the results that it has alone."""
    long, n, hq, hkv, dh, window = 530000, 900, 32, 16, 128, 100
    assert long * hq * dh > 2 ** 31
    q_len, kv_len = [long, n], [700, 1000]                   # (the long sequence's queries see its few keys at its end)
    x = inputs([n], [1000], hq, hkv, dh, dtype, 43)
    alone = run(*x, [n], [1000], window, 0, False)
    q, do, out = (torch.zeros(long + n, hq, dh, dtype=DT[dtype], device="cuda") for _ in range(3))
    k, v = (torch.ones(1700, hkv, dh, dtype=DT[dtype], device="cuda") for _ in range(2))
    q[long:], do[long:], k[700:], v[700:] = x[0], x[3], x[1], x[2]
    lse = torch.zeros(long + n, hq, device="cuda")
    b.beagle_window_attn_forward(q, k, v, q_len, kv_len, out, lse, window, 0)
    assert torch.equal(out[long:], alone["out"]) and torch.equal(lse[long:], alone["lse"])
    # scores 0: the mean of ones (a sum that is exact, times the sum's inverse: two roundings of half a step, 2 * 2^-24), and ln of how
    # many keys a query sees
    assert bool(((out[long - 700:long].double() - 1).abs() <= 2.0 ** -23 * (1 + 2.0 ** -20)).all()) and bool((out[:long - 700] == 0).all()) and bool(torch.isneginf(lse[:long - 700]).all())
    seen = torch.arange(1, 701, device="cuda").clamp(max=window).double().log()[:, None]
    assert bool(((lse[long - 700:long].double() - seen).abs() <= 2.0 ** -21 * (1 + seen)).all())
    dq, dk, dv = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    b.beagle_window_attn_backward(q, k, v, out, lse, do, q_len, kv_len, dq, dk, dv, window, 0)
    for got, name in ((dq[long:], "dq"), (dk[700:], "dk"), (dv[700:], "dv")):
        assert torch.equal(got, alone[name]), name
    assert not bool(dq[:long].any()) and not bool(dk[:700].any()) and not bool(dv[:700].any())
