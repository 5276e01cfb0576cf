"""Rotary positions on the GPU, alone and on the way into the paged cache, against the definition in 64 bits."""
import random

import pytest
import torch

from paper_2505_24544_b200 import binding as b
from test_pages_gpu import Model, new_cache, i32

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
U = 2.0 ** -24


def reference(rot, x, pos, inverse=False):
    """Value and bound.  x [rows, heads, dh], pos [rows]; 64 bits on the CPU."""
    s = rot.struct
    r, h = s.rot_dim, s.rot_dim // 2
    x, pos = x.detach().cpu().double(), pos.cpu().double()
    angle = pos[:, None] * torch.tensor(rot.frequencies, dtype=torch.float64)
    c, sn = torch.cos(angle)[:, None] * s.mscale, torch.sin(angle)[:, None] * s.mscale * (-1 if inverse else 1)
    ia = torch.arange(0, r, 2) if s.interleaved else torch.arange(h)
    ib = ia + 1 if s.interleaved else ia + h
    y, bound = x.clone(), torch.zeros_like(x)
    p, q = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = p * c - q * sn, q * c + p * sn
    # cosine and sine: the reduced turn rounded to fp32 (2 pi 2^-26 = 1.6 u), two units in the last place of the function (2 u), the
    # factor (u); the angle in double on both sides (its size * 2^-51); two products and their sum (3 u): 8 u
    size = (p.abs() + q.abs()) * s.mscale
    err = size * (8 * U + angle.abs()[:, None] * 2.0 ** -51)
    bound[..., ia], bound[..., ib] = err, err
    return y, bound


def close(got, want, bound, dtype):
    err = (got.detach().cpu().double() - want).abs()
    assert bool((err <= bound + HALF[dtype] * (want.abs() + bound) + 2.0 ** -126).all()), float(err.max())


def randn(*shape, dtype, seed=0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(DT[dtype])


# every unit size (16 bytes, 8, 4, one element), parts of the head, one pair, whole heads; widths that are no power of two
SHAPES = [("bf16", 128, 128), ("bf16", 128, 64), ("bf16", 128, 8), ("bf16", 64, 20), ("bf16", 64, 6), ("bf16", 64, 2), ("bf16", 80, 80), ("bf16", 256, 254), ("bf16", 8, 8),
          ("fp32", 64, 64), ("fp32", 128, 24), ("fp32", 64, 12), ("fp32", 20, 10), ("fp32", 256, 256), ("fp32", 4, 2)]


@pytest.mark.parametrize("dtype,dh,rot_dim", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk", [(1, 1, 0), (7, 5, 3), (33, 32, 8), (1201, 4, 4)])
def test_rotation_and_transpose(dtype, dh, rot_dim, interleaved, rows, hq, hk):
    rot = b.Rotary(dh, rot_dim, theta=10000.0, interleaved=interleaved)
    pos = torch.randint(-5, 200000, (rows,), generator=torch.Generator().manual_seed(rows), dtype=torch.int32)
    q, k = randn(rows, hq, dh, dtype=dtype, seed=1), randn(rows, max(hk, 1), dh, dtype=dtype, seed=2)
    for inverse in (False, True):
        qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
        if hk:
            b.beagle_rotary_apply(rot, q, qo, k, ko, pos.cuda(), inverse=inverse)
            close(ko, *reference(rot, k, pos, inverse), dtype)
        else:
            b.beagle_rotary_apply(rot, q, qo, pos=pos.cuda(), inverse=inverse)
        close(qo, *reference(rot, q, pos, inverse), dtype)
        assert torch.equal(qo[..., rot_dim:], q[..., rot_dim:])
        again = q.clone()
        b.beagle_rotary_apply(rot, again, again, pos=pos.cuda(), inverse=inverse)            # in place: the same bits
        assert torch.equal(again, qo)


@pytest.mark.parametrize("scaling,kw", [("linear", {}), ("base", {}), ("bands", {}), ("bands", dict(low=2.0, high=9.0)), ("ramp", {}), ("ramp", dict(mscale=0.7))])
def test_scaled_frequencies(scaling, kw):
    rot = b.Rotary(128, 96, theta=500000.0, scaling=scaling, factor=8.0, original=4096, **kw)
    pos = torch.randint(0, 32768, (50,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    x = randn(50, 3, 128, dtype="fp32")
    out = torch.empty_like(x)
    b.beagle_rotary_apply(rot, x, out, pos=pos.cuda())
    close(out, *reference(rot, x, pos), "fp32")


def test_far_positions():
    """Angles of more turns than fp32 counts, up to the last int32, and given frequencies."""
    rot = b.Rotary(64)
    rot.struct.freq[3] = -2.5
    rot.struct.freq[4] = 0.0
    pos = torch.tensor([0, 1, 16777217, 123456789, 2147483647, -2147483648], dtype=torch.int32)
    x = randn(6, 2, 64, dtype="fp32")
    out = torch.empty_like(x)
    b.beagle_rotary_apply(rot, x, out, pos=pos.cuda())
    close(out, *reference(rot, x, pos), "fp32")


def test_positions_without_a_tensor():
    rot = b.Rotary(64, 32)
    x = randn(30, 2, 64, dtype="bf16")
    out = torch.empty_like(x)
    b.beagle_rotary_apply(rot, x, out, pos0=5)
    close(out, *reference(rot, x, torch.arange(5, 35)), "bf16")
    b.beagle_rotary_apply(rot, x, out, pos0=2, period=10)                     # three sequences of ten
    close(out, *reference(rot, x, 2 + torch.arange(30) % 10), "bf16")


def test_strided_rows_another_stream_and_neighbours():
    """Queries and keys as slices of a fused projection, rotated in place there: what lies between stays as it was."""
    rot = b.Rotary(64, interleaved=True)
    fused = randn(300, 12 * 64, dtype="bf16")
    before = fused.clone()
    q, k = fused[:, :8 * 64].unflatten(1, (8, 64)), fused[:, 8 * 64:10 * 64].unflatten(1, (2, 64))
    pos = torch.arange(300, dtype=torch.int32, device="cuda")
    want_q, want_k = reference(rot, q, pos), reference(rot, k, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.beagle_rotary_apply(rot, q, q, k, k, pos)
    side.synchronize()
    close(q, *want_q, "bf16")
    close(k, *want_k, "bf16")
    assert torch.equal(fused[:, 10 * 64:], before[:, 10 * 64:])


def test_a_nan_stays_in_its_pair():
    rot = b.Rotary(64, 48)
    x = randn(4, 2, 64, dtype="fp32")
    clean = torch.empty_like(x)
    b.beagle_rotary_apply(rot, x, clean, pos0=3)
    x[1, 1, 5] = float("nan")
    out = torch.empty_like(x)
    b.beagle_rotary_apply(rot, x, out, pos0=3)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, 1, 5] = bad[1, 1, 5 + 24] = True
    assert torch.equal(torch.isnan(out), bad) and torch.equal(out[~bad], clean[~bad])


def test_gradient_against_differences():
    """sum(w * rotate(x)) has the gradient transpose(w): compared with differences, which are exact for a linear map but for rounding."""
    rot = b.Rotary(16, 12, theta=100.0, scaling="ramp", factor=4.0, original=64)
    x, w = randn(5, 2, 16, dtype="fp32", seed=3), randn(5, 2, 16, dtype="fp32", seed=4)
    pos = torch.tensor([0, 1, 7, 100, 3000], dtype=torch.int32, device="cuda")
    grad = torch.empty_like(w)
    b.beagle_rotary_apply(rot, w, grad, pos=pos, inverse=True)
    for at in [(0, 0, 0), (1, 1, 5), (2, 0, 11), (3, 1, 13), (4, 0, 3), (4, 1, 9)]:
        side = []
        for step in (1.0, -1.0):
            y = x.clone()
            y[at] += step
            out = torch.empty_like(y)
            b.beagle_rotary_apply(rot, y, out, pos=pos)
            side.append((out.double() * w.double()).sum())
        # each output is off by 9 u of the sizes in its pair, 16 outputs of at most |x| + 1 < 6 with |w| < 5 differ between the two sides
        assert abs(float((side[0] - side[1]) / 2 - grad[at])) < 16 * 5 * 9 * U * 12 * rot.struct.mscale


# ------------------------------------------------------------------------------------------------ into the cache

@pytest.mark.parametrize("dtype,hkv,hq,dh,rot_dim,interleaved,ps", [
    ("bf16", 8, 32, 128, 128, False, 64), ("bf16", 2, 4, 64, 20, False, 16), ("bf16", 1, 8, 32, 32, True, 8), ("bf16", 3, 6, 256, 64, True, 32), ("bf16", 2, 0, 64, 6, False, 16),
    ("fp32", 4, 4, 64, 64, False, 16), ("fp32", 2, 2, 16, 8, True, 8), ("fp32", 1, 5, 128, 10, False, 256)])
@pytest.mark.parametrize("offset", [0, 1, 1000])
def test_append(dtype, hkv, hq, dh, rot_dim, interleaved, ps, offset):
    """Ragged appends onto ragged slots, forks that copy their last page, rows that find no room: the cache as after the plain append of
    keys rotated beforehand (same pages, lengths, counts, values), the queries at their positions, everything else as it was."""
    rot = b.Rotary(dh, rot_dim, interleaved=interleaved, scaling="linear", factor=2.0)
    r = random.Random(dh + ps + offset)
    cache = new_cache(14, ps, hkv, dh, 6, 5, dtype)
    model = Model(cache)
    slots = [4, 0, 2, 1]

    def step(slots, T, n_new):
        B = len(slots)
        k, v = randn(B, T, hkv, dh, dtype=dtype, seed=T), randn(B, T, hkv, dh, dtype=dtype, seed=T + 1)
        n = [T] * B if n_new is None else [max(0, min(T, x)) for x in n_new]
        at = [model.length[s] for s in slots]
        # the model stores the keys as they are: hand it what the operator writes, checked below
        q = randn(B, T, max(hq, 1), dh, dtype=dtype, seed=T + 2)
        q_out = torch.full_like(q, 7.0)
        ok = torch.full((B,), 5, dtype=torch.int32, device="cuda")
        args = (q, q_out) if hq else (None, None)
        b.beagle_pages_append_rotary(cache, slots, rot, k, v, None if n_new is None else i32(n_new), ok, *args, q_offset=offset)
        pos = torch.tensor(at, dtype=torch.int32)[:, None] + torch.arange(T, dtype=torch.int32)
        turned = torch.empty_like(k)
        b.beagle_rotary_apply(rot, k.flatten(0, 1), turned.flatten(0, 1), pos=pos.reshape(-1).cuda())
        close(turned.flatten(0, 1), *reference(rot, k.flatten(0, 1), pos.reshape(-1)), dtype)
        assert ok.tolist() == model.append(slots, turned, v, n)
        assert cache.length.tolist() == model.length and cache.refs.tolist() == model.refs
        assert [[x for x in row if x >= 0] for row in cache.table.tolist()] == model.pages
        for s in range(6):
            for i in range(model.length[s]):
                p, row = model.pages[s][i // ps], i % ps
                assert torch.equal(cache.k[p, :, row].cpu(), model.k[p, :, row]) and torch.equal(cache.v[p, :, row].cpu(), model.v[p, :, row])
        if hq:
            want = reference(rot, q.flatten(0, 1), pos.reshape(-1) + offset)
            some = torch.arange(T)[None, :] < torch.tensor(n)[:, None]
            f = some.reshape(-1)
            close(q_out.flatten(0, 1)[f.cuda()], want[0][f], want[1][f], dtype)
            assert bool((q_out[~some.cuda()] == 7.0).all())

    step(slots, 3, [r.randint(0, 3) for _ in slots])
    step(slots, ps + 1, [ps, 1, ps + 1, -2])
    b.beagle_pages_fork(cache, [4, 2], [3, 5])
    model.fork([4, 2], [3, 5])
    step([3, 5, 4], 1, None)                               # copies of shared last pages
    step([0, 1, 2, 3, 4], 2 * ps, [1, 2 * ps, 2 * ps, 1, 1])         # some find no room
    step([1], 0, None)


def test_append_is_captured_and_replayed():
    rot = b.Rotary(64)
    cache = new_cache(20, 16, 2, 64, 2, 10, "bf16")
    k, v, q = randn(2, 1, 2, 64, dtype="bf16", seed=1), randn(2, 1, 2, 64, dtype="bf16", seed=2), randn(2, 1, 4, 64, dtype="bf16", seed=3)
    q_out, ok = torch.empty_like(q), torch.empty(2, dtype=torch.int32, device="cuda")
    b.beagle_pages_append_rotary(cache, [0, 1], rot, k, v, None, ok, q, q_out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.beagle_pages_append_rotary(cache, [0, 1], rot, k, v, None, ok, q, q_out)
    for i in range(1, 40):
        graph.replay()
        pos = torch.tensor([i, i], dtype=torch.int32)
        close(q_out[:, 0], *reference(rot, q[:, 0], pos), "bf16")
        got = torch.stack([cache.k[int(cache.table[s, i // 16]), :, i % 16] for s in (0, 1)])
        close(got, *reference(rot, k[:, 0], pos), "bf16")
    assert cache.length.tolist() == [40, 40]


def test_queries_rotated_in_place_and_from_a_fused_projection():
    rot = b.Rotary(64)
    cache = new_cache(20, 16, 2, 64, 2, 10, "bf16")
    fused = randn(2, 5, 8 * 64, dtype="bf16")
    q, k, v = fused[..., :4 * 64].unflatten(2, (4, 64)), fused[..., 4 * 64:6 * 64].unflatten(2, (2, 64)), fused[..., 6 * 64:].unflatten(2, (2, 64))
    out = torch.empty(2, 5, 4, 64, dtype=torch.bfloat16, device="cuda")
    b.beagle_pages_append_rotary(cache, [1, 0], rot, k, v, None, None, q, out)
    dense = q.contiguous()
    b.beagle_pages_truncate(cache, [0, 1])
    b.beagle_pages_append_rotary(cache, [1, 0], rot, k, v, None, None, dense, dense)
    assert torch.equal(out, dense)
    close(out.flatten(0, 1), *reference(rot, q.reshape(10, 4, 64), torch.arange(5).repeat(2)), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_past_32_bit_offsets(dtype):
    """Rows whose offsets pass 2^31 elements, in the input, the output, and both."""
    far = 2 ** 30 + 64
    big = torch.zeros(2 * far + 4096, dtype=DT[dtype], device="cuda")
    rot = b.Rotary(64)
    rows = torch.as_strided(big, (3, 2, 64), (far, 64, 1))
    x = randn(3, 2, 64, dtype=dtype, seed=1)
    rows.copy_(x)
    out = torch.empty_like(x)
    b.beagle_rotary_apply(rot, rows, out, pos0=5)
    close(out, *reference(rot, x, torch.arange(5, 8)), dtype)
    b.beagle_rotary_apply(rot, rows, rows, pos0=5)
    assert torch.equal(rows, out) and int((big != 0).sum()) <= 3 * 128
    del big


def test_append_past_32_bit_offsets():
    """Pools of more than 2^31 elements: keys and values land in the last pages, copies of shared pages come from there."""
    rot = b.Rotary(128)
    ps, hkv = 256, 8
    n_pages = 2 ** 31 // (ps * hkv * 128) + 40
    cache = new_cache(n_pages, ps, hkv, 128, 3, 6, "bf16")
    cache.refs[: n_pages - 12] = 1                       # only the last pages are free
    k, v = randn(1, 300, hkv, 128, dtype="bf16", seed=1), randn(1, 300, hkv, 128, dtype="bf16", seed=2)
    ok = torch.zeros(1, dtype=torch.int32, device="cuda")
    b.beagle_pages_append_rotary(cache, [0], rot, k, v, None, ok)
    b.beagle_pages_fork(cache, [0], [1])
    b.beagle_pages_append_rotary(cache, [1], rot, k[:, :5], v[:, :5], None, ok)
    assert ok.item() == 1 and cache.length.tolist()[:2] == [300, 305]
    for slot, n in ((0, 300), (1, 305)):
        pages = [int(x) for x in cache.table[slot, :2]]
        assert min(pages) >= n_pages - 12
        got = torch.cat([cache.k[p] for p in pages], 1)[:, :n].transpose(0, 1)
        src = torch.cat([k[0], k[0, :5]])[:n]
        close(got, *reference(rot, src, torch.arange(n)), "bf16")
        assert torch.equal(torch.cat([cache.v[p] for p in pages], 1)[:, :n].transpose(0, 1), torch.cat([v[0], v[0, :5]])[:n])
    assert int(cache.table[0, 1]) != int(cache.table[1, 1])


def test_a_damaged_table_stays_inside_the_pools():
    """Page ids and lengths out of range: nothing outside the cache is touched, the other slot gets its rows."""
    rot = b.Rotary(64)
    cache = new_cache(12, 16, 2, 64, 3, 4, "bf16")
    k, v = randn(2, 20, 2, 64, dtype="bf16", seed=1), randn(2, 20, 2, 64, dtype="bf16", seed=2)
    b.beagle_pages_append_rotary(cache, [0, 1], rot, k, v)
    cache.table[0, 1] = 2 ** 31 - 1
    cache.length[2] = 2 ** 31 - 1
    cache.table[2, 3] = -9
    ok = torch.zeros(3, dtype=torch.int32, device="cuda")
    q = randn(3, 4, 4, 64, dtype="bf16", seed=3)
    out = torch.zeros_like(q)
    k, v = randn(3, 4, 2, 64, dtype="bf16", seed=4), randn(3, 4, 2, 64, dtype="bf16", seed=5)
    b.beagle_pages_append_rotary(cache, [0, 2, 1], rot, k, v, None, ok, q, out)
    torch.cuda.synchronize()
    assert ok.tolist()[1:] == [0, 1]
    page = int(cache.table[1, 1])
    close(cache.k[page, :, 4:8].transpose(0, 1), *reference(rot, k[2], torch.arange(20, 24)), "bf16")
    close(out[2], *reference(rot, q[2], torch.arange(20, 24)), "bf16")
