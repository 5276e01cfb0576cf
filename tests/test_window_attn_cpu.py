"""Refusals of the windowed attention's entry points (host checks, no GPU needed)."""
import ctypes as C

import pytest

OK, INVALID, SHAPE, CAPACITY = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2505_24544_b200 import build
    from paper_2505_24544_b200.binding import load_library
    build.build()
    return load_library()


def attn(**kw):
    from paper_2505_24544_b200.binding import BeagleWindowAttn
    w = BeagleWindowAttn()
    base = dict(q_dev=1 << 20, k_dev=2 << 20, v_dev=3 << 20, q_stride=512, k_stride=256, v_stride=256, q_len_host=(5, 7), kv_len_host=(5, 9), dtype=1,
                n_q_heads=4, n_kv_heads=2, head_dim=128, window=4, sinks=1, strict=0)
    base.update(kw)
    base.setdefault("batch", len(base["q_len_host"] or ()))
    w.arrays = [(C.c_int32 * max(1, len(x)))(*x) for x in base.values() if isinstance(x, tuple)]         # kept alive by the structure
    arrays = iter(w.arrays)
    for n, x in base.items():
        setattr(w, n, C.addressof(next(arrays)) if isinstance(x, tuple) else x)
    return w


def forward(lib, w, out=4 << 20, lse=5 << 20):
    return lib.beagle_window_attn_forward(None if w is None else C.byref(w), out, lse, None)


def backward(lib, w, out=4 << 20, lse=5 << 20, do=6 << 20, ds=512, dq=7 << 20, dqs=512, dk=8 << 20, dks=256, dv=9 << 20, dvs=256, ws=10 << 20, n=1 << 30):
    return lib.beagle_window_attn_backward(None if w is None else C.byref(w), out, lse, do, ds, dq, dqs, dk, dks, dv, dvs, ws, n, None)


@pytest.mark.parametrize("kw, want", [
    (dict(dtype=2), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_kv_heads=-1), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(strict=2), INVALID), (dict(batch=-1), INVALID), (dict(q_len_host=None, batch=2), INVALID), (dict(kv_len_host=None), INVALID),
    (dict(q_len_host=(5, -1)), INVALID), (dict(kv_len_host=(-2, 3)), INVALID),
    (dict(n_q_heads=5), SHAPE), (dict(head_dim=96), SHAPE), (dict(head_dim=32), SHAPE), (dict(head_dim=256), SHAPE), (dict(n_q_heads=1 << 17), SHAPE),
    (dict(batch=65), CAPACITY), (dict(sinks=1025), CAPACITY), (dict(q_len_host=(1 << 27, 1)), CAPACITY), (dict(kv_len_host=(1, 1 << 27)), CAPACITY),
])
def test_bad_shapes(lib, kw, want):
    w = attn(**kw)
    n = C.c_size_t()
    assert forward(lib, w) == want
    assert backward(lib, w) == want
    assert lib.beagle_window_attn_workspace_bytes(C.byref(w), C.byref(n)) == want


def test_bad_pointers(lib):
    assert forward(lib, None) == INVALID and backward(lib, None) == INVALID
    for kw in (dict(q_dev=0), dict(k_dev=0), dict(v_dev=0), dict(q_dev=8 + (1 << 20)), dict(q_stride=511), dict(q_stride=516), dict(k_stride=255), dict(v_stride=0),
               dict(q_stride=-512)):
        assert forward(lib, attn(**kw)) == INVALID
        assert backward(lib, attn(**kw)) == INVALID
    w = attn()
    assert forward(lib, w, out=None) == INVALID and forward(lib, w, out=8) == INVALID and forward(lib, w, lse=2) == INVALID
    for kw in (dict(out=None), dict(lse=None), dict(do=None), dict(ds=500), dict(dq=None), dict(dqs=4), dict(dk=None), dict(dks=257), dict(dv=None), dict(dvs=0),
               dict(ws=None), dict(ws=16)):
        assert backward(lib, w, **kw) == INVALID
    assert backward(lib, w, n=64) == CAPACITY


def test_nothing_to_do(lib):
    empty = attn(q_len_host=(0, 0), kv_len_host=(0, 0), q_dev=0, k_dev=0, v_dev=0)
    assert forward(lib, empty, None, None) == OK
    assert backward(lib, empty, None, None, None, 0, None, 0, None, 0, None, 0, None, 0) == OK
    assert forward(lib, attn(batch=0, q_len_host=None, kv_len_host=None), None, None) == OK
    n = C.c_size_t()
    assert lib.beagle_window_attn_workspace_bytes(C.byref(empty), C.byref(n)) == OK
    assert lib.beagle_window_attn_workspace_bytes(C.byref(empty), None) == INVALID


def test_workspace_bytes(lib):
    """(log-sum-exp, delta) of every query in padded rows; fp32 partials of the sinks where a query lies past their band."""
    def size(**kw):
        n = C.c_size_t()
        assert lib.beagle_window_attn_workspace_bytes(C.byref(attn(**kw)), C.byref(n)) == OK
        return n.value
    stats = 4 * (128 + 256 + 128) * 8                            # 4 heads, 5 and 130 rows padded, one tile of slack
    short = dict(q_len_host=(5, 130), kv_len_host=(5, 130))
    assert size(window=0, sinks=9, **short) == stats
    assert size(window=500, sinks=9, **short) == stats           # no query lies past the window of the first keys
    assert size(window=2, sinks=3, **short) == stats + 2 * 2 * (1 + 1) * 3 * 2 * 128 * 4
    assert size(window=2, sinks=1000, **short) == stats + 2 * 2 * (1 + 1) * 130 * 2 * 128 * 4
    assert size(dtype=0, head_dim=32, **short) == -(-stats // 256) * 256 + 135 * 4 * 2 * 32 * 4


def test_backward_checks_its_workspace(monkeypatch):
    """A workspace in host memory, or with gaps, is refused like any other tensor."""
    torch = pytest.importorskip("torch")
    from paper_2505_24544_b200 import binding as b

    class Library:
        def beagle_window_attn_backward(self, *_):
            raise AssertionError("the library was reached")
    q, lse = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2)
    monkeypatch.setattr(b, "_check", lambda name, t, *_: t.data_ptr())           # the other tensors stand for ones on the device
    monkeypatch.setattr(b, "_stream", lambda: 0)
    monkeypatch.setattr(b, "load_library", Library)

    def call(ws):
        b.beagle_window_attn_backward(q, q, q, q, lse, q, [3], [3], q, q, q, ws=ws)
    with pytest.raises(ValueError, match="ws.*device"):
        call(torch.zeros(64, dtype=torch.uint8))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    with pytest.raises(ValueError, match="ws.*contiguous"):
        call(torch.zeros(64, 2, dtype=torch.uint8)[:, 0])
    with pytest.raises(AssertionError, match="the library was reached"):
        call(torch.zeros(64, dtype=torch.uint8))


def test_workspace_of_a_long_sequence_among_short_ones(lib):
    """Partials of the sinks are kept for the sequences that have queries past the band, in their own number of segments and rows: one
    sequence of 32768 among 63 of 200 (window 512, 1024 sinks) takes what it takes alone."""
    def size(*lengths, **kw):
        n = C.c_size_t()
        shape = dict(window=512, sinks=1024, n_q_heads=8, n_kv_heads=8, head_dim=128, q_stride=1024, k_stride=1024, v_stride=1024)
        shape.update(kw)
        assert lib.beagle_window_attn_workspace_bytes(C.byref(attn(q_len_host=lengths, kv_len_host=lengths, **shape)), C.byref(n)) == OK
        return n.value

    def stats(*lengths):
        return 8 * (sum(-(-n // 128) * 128 for n in lengths) + 128) * 8
    long, short = (32768,), (200,) * 63
    parts = 8 * (1 + 32) * 1024 * 2 * 128 * 4                    # 252 jobs past the band, eight a segment
    assert size(*long) == stats(*long) + parts
    assert size(*short) == stats(*short)
    assert size(*long, *short) == size(*short, *long) == stats(*long, *short) + parts
    # a few rows past the band in every sequence: as many segments as each needs, as many rows as it has
    mixed = (32768,) + (700,) * 63
    assert size(*mixed) == stats(*mixed) + parts + 63 * 8 * 2 * 700 * 2 * 128 * 4
    fp32 = dict(dtype=0, n_q_heads=8)
    assert size(*long, *short, **fp32) - size(*long, **fp32) == stats(*long, *short) - stats(*long)
