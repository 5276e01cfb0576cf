"""Refusals of the rotary, shared-prefix and sampling entry points, all found on the host, and the rotary frequencies (no GPU needed)."""
import ctypes as C
import math

import pytest

from test_pages_cpu import CAPACITY, INVALID, OK, SHAPE, arr, lib, pages          # noqa: F401 (lib is a fixture)

P = 1 << 21


def rotary(lib, head_dim=64, rot_dim=64, interleaved=0, theta=10000.0, scaling=0, factor=1.0, original=0.0, low=1.0, high=4.0, mscale=0.0):
    from paper_2505_24544_b200.binding import BeagleRotary
    r = BeagleRotary()
    return lib.beagle_rotary_make(head_dim, rot_dim, interleaved, theta, scaling, factor, original, low, high, mscale, C.byref(r)), r


def test_structure_matches_header():
    from paper_2505_24544_b200.binding import BeagleRotary
    assert C.sizeof(BeagleRotary) == 4 * 4 + 8 + 128 * 8


@pytest.mark.parametrize("kw,want", [
    (dict(head_dim=0), INVALID), (dict(rot_dim=0), INVALID), (dict(rot_dim=-2), INVALID), (dict(interleaved=2), INVALID), (dict(head_dim=258, rot_dim=2), SHAPE),
    (dict(rot_dim=66), SHAPE), (dict(rot_dim=33), SHAPE), (dict(theta=1.0), INVALID), (dict(theta=0.0), INVALID), (dict(theta=math.nan), INVALID), (dict(theta=math.inf), INVALID),
    (dict(scaling=5), INVALID), (dict(scaling=-1), INVALID), (dict(scaling=1, factor=0.5), INVALID), (dict(scaling=1, factor=math.nan), INVALID),
    (dict(scaling=3, factor=2.0), INVALID), (dict(scaling=3, factor=2.0, original=100.0, low=4.0), INVALID), (dict(scaling=4, factor=2.0, original=100.0, low=0.0), INVALID),
    (dict(scaling=4, factor=2.0, original=math.inf), INVALID), (dict(scaling=2, factor=2.0, rot_dim=2), SHAPE), (dict(mscale=-1.0), INVALID), (dict(mscale=math.nan), INVALID),
    (dict(), OK), (dict(head_dim=256, rot_dim=2), OK), (dict(scaling=3, factor=2.0, original=100.0), OK)])
def test_make(lib, kw, want):
    assert rotary(lib, **kw)[0] == want


def test_make_without_output(lib):
    assert lib.beagle_rotary_make(64, 64, 0, 10000.0, 0, 1.0, 0.0, 1.0, 4.0, 0.0, None) == INVALID


def test_frequencies():
    """The properties that define each scaling."""
    from paper_2505_24544_b200.binding import Rotary
    plain = Rotary(128, 96, theta=500000.0).frequencies
    assert len(plain) == 48 and plain[0] == 1.0 and all(abs(y / x - 500000.0 ** (-1 / 48)) < 1e-12 for x, y in zip(plain, plain[1:]))
    kw = dict(theta=500000.0, factor=8.0, original=4096)
    linear = Rotary(128, 96, scaling="linear", **kw).frequencies
    assert all(abs(y * 8 / x - 1) < 1e-15 for x, y in zip(plain, linear))
    base = Rotary(128, 96, scaling="base", **kw).frequencies
    assert base[0] == 1.0 and abs(base[-1] * 8 / plain[-1] - 1) < 1e-12 and all(x / 8 < y <= x for x, y in zip(plain, base))
    turns = [4096 * f / (2 * math.pi) for f in plain]
    bands = Rotary(128, 96, scaling="bands", **kw)
    assert bands.struct.mscale == 1.0
    for f, n, y in zip(plain, turns, bands.frequencies):
        if n >= 4 or n <= 1:
            assert abs(y - (f if n >= 4 else f / 8)) <= 1e-15 * f
        else:
            assert f / 8 < y < f
    ramp = Rotary(128, 96, scaling="ramp", **kw)
    assert abs(ramp.struct.mscale - (1 + 0.1 * math.log(8))) < 1e-15
    ratio = [y / x for x, y in zip(plain, ramp.frequencies)]
    assert ratio[0] == 1.0 and abs(ratio[-1] - 1 / 8) < 1e-15 and all(x >= y - 1e-15 for x, y in zip(ratio, ratio[1:]))
    assert all(r == 1.0 for r, n in zip(ratio, turns) if n > 40) and all(abs(r - 1 / 8) < 1e-12 for r, n in zip(ratio, turns) if n < 0.7)
    with pytest.raises(ValueError):
        Rotary(64, scaling="other")
    with pytest.raises(ValueError):
        Rotary(64, mscale=0.0)


def test_apply_refusals(lib):
    _, r = rotary(lib)
    R = C.byref(r)

    def call(rot=R, dtype=1, rows=4, pos=None, pos0=0, period=0, hq=2, q=P, qs=128, qo=P, qos=128, hk=1, k=P, ks=64, ko=P, kos=64):
        return lib.beagle_rotary_apply(rot, dtype, rows, pos, pos0, period, hq, q, qs, qo, qos, hk, k, ks, ko, kos, 0, None)

    assert call(rows=0) == OK and call(rows=0, q=None) == OK
    assert call(rot=None) == INVALID
    for kw in (dict(dtype=2), dict(rows=-1), dict(hq=-1), dict(hk=-1), dict(hq=0, hk=0), dict(period=-1), dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(qs=127),
               dict(qos=120), dict(ks=56), dict(q=P + 2), dict(qo=P + 8), dict(qs=132, qos=132), dict(qs=136), dict(kos=72), dict(pos=P + 2)):
        assert call(**kw) == INVALID, kw
    assert call(hq=65536) == SHAPE
    assert call(pos0=2 ** 31 - 2, rows=4) == CAPACITY
    _, odd = rotary(lib, head_dim=20, rot_dim=20)
    assert call(rot=C.byref(odd), hq=0) == SHAPE                # 40 bytes a head: not in 16-byte pieces
    for bad in (dict(rot_dim=3), dict(rot_dim=66), dict(head_dim=300)):
        _, x = rotary(lib)
        for n, v in bad.items():
            setattr(x, n, v)
        assert call(rot=C.byref(x)) == SHAPE
    _, x = rotary(lib)
    x.freq[5] = math.nan
    assert call(rot=C.byref(x)) == INVALID
    _, x = rotary(lib)
    x.mscale = math.inf
    assert call(rot=C.byref(x)) == INVALID


def test_append_refusals(lib):
    _, r = rotary(lib)
    cache = pages(lib)

    def call(p=cache, rot=r, batch=1, slots=arr(0), T=1, k=P, ks=128, v=P, vs=128, hq=2, q=P, qs=128, qo=P, off=0):
        return lib.beagle_pages_append_rotary(C.byref(p), C.byref(rot), batch, slots, T, None, k, ks, v, vs, hq, q, qs, qo, off, None, None)

    assert call(batch=0) == OK
    assert call(p=pages(lib, k=0)) == INVALID and call(p=pages(lib, page_size=24)) == SHAPE and call(p=pages(lib, ws_bytes=16)) == CAPACITY
    assert lib.beagle_pages_append_rotary(C.byref(cache), None, 1, arr(0), 1, None, P, 128, P, 128, 0, None, 0, None, 0, None, None) == INVALID
    _, narrow = rotary(lib, head_dim=32, rot_dim=32)
    assert call(rot=narrow) == SHAPE
    for kw in (dict(slots=arr(4)), dict(slots=arr(-1)), dict(slots=None), dict(batch=2, slots=arr(1, 1)), dict(T=-1), dict(k=None), dict(v=None), dict(ks=120), dict(vs=120), dict(k=P + 2),
               dict(ks=132), dict(hq=-1), dict(q=None), dict(qo=None), dict(qs=120), dict(q=P + 4), dict(qo=P + 8), dict(qs=132), dict(qs=256), dict(off=-1)):
        assert call(**kw) == INVALID, kw
    assert call(batch=65, slots=arr(*range(65))) == CAPACITY
    assert call(T=2 ** 29 + 1) == CAPACITY and call(off=2 ** 29) == CAPACITY and call(hq=65536) == SHAPE


def test_shared_refusals(lib):
    cache = pages(lib)
    n = C.c_size_t()

    def size(p=cache, batch=3, hq=4, groups=arr(2, 1), n_groups=2, out=C.byref(n)):
        return lib.beagle_paged_attn_shared_workspace_bytes(C.byref(p) if p is not None else None, batch, hq, n_groups, groups, out)

    assert size() == OK and n.value % 256 == 0 and n.value > 0
    need = n.value
    assert size(p=None) == INVALID and size(out=None) == INVALID and size(p=pages(lib, page_size=24)) == SHAPE and size(hq=3) == SHAPE and size(hq=18) == SHAPE
    assert size(hq=0) == INVALID and size(batch=-1) == INVALID and size(batch=65, groups=arr(65), n_groups=1) == CAPACITY
    bad_groups = [(arr(2, 2), 2), (arr(3, 0), 2), (arr(4, -1), 2), (None, 2), (arr(3), -1), (arr(3), 0), (arr(1, 1), 2)]
    for g, m in bad_groups:
        assert size(groups=g, n_groups=m) == INVALID
    assert size(batch=0, groups=None, n_groups=0) == OK

    def call(p=cache, batch=3, slots=arr(0, 1, 2), groups=arr(2, 1), n_groups=2, shared=P, hq=4, q=P, qs=256, out=P, lse=None, ws=P, nb=need):
        return lib.beagle_paged_attn_shared(C.byref(p), batch, slots, n_groups, groups, shared, hq, q, qs, out, lse, ws, nb, None)

    assert call(batch=0, n_groups=0) == OK
    for g, m in bad_groups:
        assert call(groups=g, n_groups=m) == INVALID
        assert lib.beagle_pages_shared(C.byref(cache), 3, arr(0, 1, 2), m, g, P, None) == INVALID
    for kw in (dict(slots=arr(0, 1, 4)), dict(slots=arr(0, -1, 2)), dict(slots=None), dict(shared=None), dict(shared=P + 2), dict(q=None), dict(out=None), dict(ws=None), dict(q=P + 8),
               dict(out=P + 2), dict(ws=P + 8), dict(qs=255), dict(qs=260), dict(lse=P + 2), dict(hq=0)):
        assert call(**kw) == INVALID, kw
    assert call(nb=need - 1) == CAPACITY and call(hq=3) == SHAPE and call(p=pages(lib, v=0)) == INVALID
    for kw, want in ((dict(p=pages(lib, v=0)), INVALID), (dict(slots=arr(0, 1, 4)), INVALID), (dict(shared=None), INVALID), (dict(shared=P + 1), INVALID)):
        a = dict(p=cache, slots=arr(0, 1, 2), shared=P)
        a.update(kw)
        assert lib.beagle_pages_shared(C.byref(a["p"]), 3, a["slots"], 2, arr(2, 1), a["shared"], None) == want


def test_sample_refusals(lib):
    def call(logits=P, dtype=0, rows=2, vocab=100, stride=100, t=None, k=None, p=None, m=None, u=P, tokens=P, logp=None):
        return lib.beagle_sample(logits, dtype, rows, vocab, stride, t, k, p, m, u, tokens, logp, None)

    assert call(rows=0) == OK and call(rows=0, logits=None) == OK
    for kw in (dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(stride=99), dict(logits=None), dict(u=None), dict(tokens=None), dict(logits=P + 2), dict(dtype=1, logits=P + 1),
               dict(t=P + 1), dict(k=P + 2), dict(p=P + 3), dict(m=P + 2), dict(u=P + 2), dict(tokens=P + 2), dict(logp=P + 2)):
        assert call(**kw) == INVALID, kw
    assert call(vocab=2 ** 18 + 1, stride=2 ** 19) == SHAPE
    assert call(rows=2 ** 31 - 1) == CAPACITY


@pytest.mark.parametrize("dtype,dh,hq,hkv", [(1, 128, 32, 8), (1, 64, 8, 8), (1, 64, 7, 1), (1, 256, 4, 1), (0, 64, 4, 4)])
@pytest.mark.parametrize("groups", [[1, 1], [2], [9, 1], [64], [33, 2, 3]])
def test_shared_workspace_has_room_at_any_16_byte_border(lib, dtype, dh, hq, hkv, groups):
    """The partials are stored 32 bytes at once and lie on multiples of 256, the caller's memory on 16: the size has room for all of them
    behind the border that follows any such address."""
    G, sms = hq // hkv, 148
    mma = dtype == 1 and dh in (64, 128)
    many = [n * G for n in groups if mma and n > 1 and n * G > 8]               # query rows of the groups on 128-row tiles
    block, few = 128 // G * G, 4 if dh == 256 else 8
    entries = sum(groups) + sum(-(-n * G // few) for n in groups if n > 1 and not (mma and n * G > 8))
    tiles = sum(-(-n // block) for n in many)
    up = lambda x: -(-x // 256) * 256
    row, rows = (dh + 2) * 4, max([min(n, block) for n in many], default=0)
    parts = up(entries * hkv * 8) + up(tiles * hkv * 8) + up((entries * hkv + 2 * sms) * (4 if mma else 1) * 8 * row)
    if tiles:
        parts += up((tiles * hkv + 2 * sms) * -(-rows // 4) * 4 * row)
    n = C.c_size_t()
    p = pages(lib, dtype=dtype, head_dim=dh, n_kv_heads=hkv)
    assert lib.beagle_paged_attn_shared_workspace_bytes(C.byref(p), sum(groups), hq, len(groups), arr(*groups), C.byref(n)) == OK
    for at in range(P, P + 256, 16):
        assert up(at) + parts <= at + n.value


def test_whole_numbers_that_the_interface_cannot_hold_are_refused():
    """Their low bits would be a position, an offset or a width of their own."""
    import torch
    from paper_2505_24544_b200 import binding as b
    rot, q = b.Rotary(64), torch.zeros(3, 2, 64)
    for kw in (dict(pos0=2 ** 31), dict(pos0=2 ** 32 + 5), dict(pos0=-2 ** 31 - 1), dict(period=2 ** 63), dict(period=2 ** 64 + 1)):
        with pytest.raises(ValueError, match=next(iter(kw))):
            b.beagle_rotary_apply(rot, q, q, **kw)
    for off in (2 ** 32, 2 ** 32 + 1, -2 ** 32):
        with pytest.raises(ValueError, match="q_offset"):
            b.beagle_pages_append_rotary(None, [0], rot, q[None], q[None], q_offset=off)
    for kw in (dict(head_dim=2 ** 32 + 64), dict(head_dim=64, rot_dim=2 ** 32 + 32)):
        with pytest.raises(ValueError):
            b.Rotary(**kw)


@pytest.mark.parametrize("mscale", [1e39, -1e39, 1.7e308])
def test_a_factor_beyond_fp32_is_refused(lib, mscale):
    """The kernels multiply by it in fp32: it would be infinite, and NaN times 0."""
    assert mscale < 0 or rotary(lib, mscale=mscale)[0] == INVALID
    _, r = rotary(lib)
    r.mscale = mscale
    assert lib.beagle_rotary_apply(C.byref(r), 1, 0, None, 0, 0, 0, None, 0, None, 0, 1, None, 64, None, 64, 0, None) == INVALID
    p = pages(lib)
    assert lib.beagle_pages_append_rotary(C.byref(p), C.byref(r), 0, None, 0, None, None, 0, None, 0, 0, None, 0, None, 0, None, None) == INVALID
    r.mscale = 3e38
    assert lib.beagle_pages_append_rotary(C.byref(p), C.byref(r), 0, None, 0, None, None, 0, None, 0, 0, None, 0, None, 0, None, None) == OK
