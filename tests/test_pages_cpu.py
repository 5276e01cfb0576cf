"""Refusals of the paged-cache entry points: all are found on the host before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

OK, INVALID, SHAPE, CAPACITY = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2505_24544_b200 import build
    from paper_2505_24544_b200.binding import load_library
    build.build()
    return load_library()


def pages(lib, **kw):
    from paper_2505_24544_b200.binding import BeaglePages
    p = BeaglePages()
    base = dict(k=1 << 20, v=2 << 20, table=3 << 20, length=4 << 20, refs=5 << 20, ws=6 << 20, n_pages=40, page_size=16, n_kv_heads=2, head_dim=64,
                dtype=1, max_slots=4, max_pages=8)
    base.update(kw)
    for n, x in base.items():
        setattr(p, n, x)
    n = C.c_size_t()
    if "ws_bytes" not in kw:
        lib.beagle_pages_workspace_bytes(C.byref(p), C.byref(n))
        p.ws_bytes = n.value
    return p


def arr(*v):
    return (C.c_int32 * max(1, len(v)))(*v)


def test_structure_matches_header():
    from paper_2505_24544_b200.binding import BeaglePages
    assert C.sizeof(BeaglePages) == 7 * 8 + 7 * 4 + 4            # six pointers, one size, seven int32, tail padding


def test_workspace_bytes(lib):
    p = pages(lib)
    n = C.c_size_t()
    assert lib.beagle_pages_workspace_bytes(C.byref(p), C.byref(n)) == OK and n.value % 256 == 0 and n.value >= 40 * 12
    assert lib.beagle_pages_workspace_bytes(None, C.byref(n)) == INVALID
    assert lib.beagle_pages_workspace_bytes(C.byref(p), None) == INVALID
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(p), 8, 0, 0, C.byref(n)) == OK and n.value == 0              # 128 positions at most: nothing to join
    wide = pages(lib, max_pages=100)
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(wide), 8, 0, 0, C.byref(n)) == OK and n.value > 0
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(wide), 8, 300, 4, C.byref(n)) == OK and n.value == 0            # 6 tiles of 64 and one
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(wide), 8, 600, 4, C.byref(n)) == OK and n.value > 0
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(wide), 8, -1, 4, C.byref(n)) == INVALID
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(p), 0, 0, 0, C.byref(n)) == INVALID
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(p), 3, 0, 0, C.byref(n)) == SHAPE             # not a multiple of the K/V heads
    assert lib.beagle_paged_attn_workspace_bytes(C.byref(p), 18, 0, 0, C.byref(n)) == SHAPE            # nine grouped heads


@pytest.mark.parametrize("kw, want", [
    (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(table=0), INVALID), (dict(length=0), INVALID), (dict(refs=0), INVALID), (dict(ws=0), INVALID),
    (dict(k=8 + (1 << 20)), INVALID), (dict(refs=4 + (1 << 20)), INVALID), (dict(table=2 + (1 << 20)), INVALID),
    (dict(n_pages=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(max_slots=0), INVALID), (dict(max_pages=-1), INVALID), (dict(dtype=2), INVALID),
    (dict(page_size=4), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=512), SHAPE), (dict(head_dim=48), SHAPE),
    (dict(head_dim=256, dtype=0), SHAPE), (dict(head_dim=16, dtype=1), SHAPE),
    (dict(ws_bytes=16), CAPACITY), (dict(n_pages=1 << 27), CAPACITY), (dict(max_slots=1 << 29), CAPACITY), (dict(max_pages=1 << 27), CAPACITY),
])
def test_bad_cache(lib, kw, want):
    p = C.byref(pages(lib, **kw))
    one, q = arr(0), 1 << 21
    assert lib.beagle_pages_reset(p, None) == want
    assert lib.beagle_pages_append(p, 1, one, 1, None, q, 128, q, 128, None, None) == want
    assert lib.beagle_pages_truncate(p, 1, one, None, None) == want
    assert lib.beagle_pages_fork(p, 1, one, arr(1), None) == want
    assert lib.beagle_pages_copy(p, 1, one, arr(1), None, None) == want
    assert lib.beagle_pages_compact(p, None) == want
    assert lib.beagle_paged_attn(p, 1, one, 4, q, 256, 0, 0, q, None, q, 1 << 30, None) == want


def test_bad_slots(lib):
    p = C.byref(pages(lib))
    q = 1 << 21
    many = arr(*range(65))
    for bad, want in ((arr(4), INVALID), (arr(-1), INVALID), (None, INVALID)):
        assert lib.beagle_pages_append(p, 1, bad, 1, None, q, 128, q, 128, None, None) == want
        assert lib.beagle_pages_truncate(p, 1, bad, None, None) == want
        assert lib.beagle_pages_fork(p, 1, bad, arr(1), None) == want
        assert lib.beagle_pages_fork(p, 1, arr(1), bad, None) == want
        assert lib.beagle_pages_copy(p, 1, bad, arr(1), None, None) == want
        assert lib.beagle_paged_attn(p, 1, bad, 4, q, 256, 0, 0, q, None, q, 1 << 30, None) == want
    twice = arr(1, 1)
    assert lib.beagle_pages_append(p, 2, twice, 1, None, q, 128, q, 128, None, None) == INVALID
    assert lib.beagle_pages_truncate(p, 2, twice, None, None) == INVALID
    assert lib.beagle_pages_fork(p, 2, arr(0, 0), twice, None) == INVALID
    assert lib.beagle_pages_fork(p, 2, arr(0, 1), arr(1, 2), None) == INVALID           # a slot in both lists
    assert lib.beagle_pages_copy(p, 1, arr(2), arr(2), None, None) == INVALID
    assert lib.beagle_pages_append(p, 65, many, 1, None, q, 128, q, 128, None, None) == CAPACITY
    assert lib.beagle_paged_attn(p, 65, many, 4, q, 256, 0, 0, q, None, q, 1 << 30, None) == CAPACITY
    assert lib.beagle_pages_truncate(p, -1, arr(0), None, None) == INVALID
    # nothing to do
    assert lib.beagle_pages_append(p, 0, None, 1, None, None, 0, None, 0, None, None) == OK
    assert lib.beagle_pages_truncate(p, 0, None, None, None) == OK
    assert lib.beagle_pages_fork(p, 0, None, None, None) == OK
    assert lib.beagle_paged_attn(p, 0, None, 4, None, 0, 0, 0, None, None, None, 0, None) == OK


def test_bad_rows(lib):
    p = C.byref(pages(lib))
    q, one = 1 << 21, arr(0)
    for a in ((None, 128, q, 128), (q, 128, None, 128), (q + 8, 128, q, 128), (q, 127, q, 128), (q, 132, q, 128), (q, 128, q, 64)):
        assert lib.beagle_pages_append(p, 1, one, 1, None, *a, None, None) == INVALID
    assert lib.beagle_pages_append(p, 1, one, -1, None, q, 128, q, 128, None, None) == INVALID
    assert lib.beagle_pages_append(p, 1, one, 0x7fffffff, None, q, 128, q, 128, None, None) == CAPACITY
    big = 1 << 30
    for hq, qp, st, w, k, o, ws, n, want in (
            (4, None, 256, 0, 0, q, q, big, INVALID), (4, q, 255, 0, 0, q, q, big, INVALID), (4, q, 260, 0, 0, q, q, big, INVALID),
            (4, q, 256, -1, 0, q, q, big, INVALID), (4, q, 256, 0, -1, q, q, big, INVALID), (4, q, 256, 0, 0, None, q, big, INVALID),
            (4, q + 2, 256, 0, 0, q, q, big, INVALID),
            (5, q, 512, 0, 0, q, q, big, SHAPE), (18, q, 2048, 0, 0, q, q, big, SHAPE)):
        assert lib.beagle_paged_attn(p, 1, one, hq, qp, st, w, k, o, None, ws, n, None) == want
    long = C.byref(pages(lib, max_pages=100))
    assert lib.beagle_paged_attn(long, 1, one, 4, q, 256, 0, 0, q, None, None, big, None) == INVALID
    assert lib.beagle_paged_attn(long, 1, one, 4, q, 256, 0, 0, q, None, q, 64, None) == CAPACITY
    wide = C.byref(pages(lib, head_dim=256))
    assert lib.beagle_paged_attn(wide, 1, one, 16, q, 4096, 0, 0, q, None, q, big, None) == SHAPE


def test_binding_checks_tensors():
    """The binding refuses tensors on another device, of another type or shape before the library sees their addresses."""
    torch = pytest.importorskip("torch")
    from paper_2505_24544_b200 import binding as b
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    i32 = dict(dtype=torch.int32)
    with pytest.raises(ValueError):
        b.PagedCache.from_tensors(k, k.clone(), torch.zeros(2, 3, **i32), torch.zeros(2, **i32), torch.zeros(4, **i32))       # host tensors
    with pytest.raises(ValueError):
        b.PagedCache.from_tensors(k.half(), k.half(), torch.zeros(2, 3, **i32), torch.zeros(2, **i32), torch.zeros(4, **i32))
    x = torch.zeros(3, 5, 4, 8)
    assert b._row_stride("x", x, 2) == 32
    fused = torch.zeros(3, 5, 96)
    assert b._row_stride("x", fused[:, :, 32:64].unflatten(2, (4, 8)), 2) == 96
    assert b._row_stride("x", fused[:, :1, 32:64].unflatten(2, (4, 8)), 2) == 480
    with pytest.raises(ValueError):
        b._row_stride("x", fused[:, :4, 32:64].unflatten(2, (4, 8)), 2)
    with pytest.raises(ValueError):
        b._row_stride("x", x.transpose(2, 3), 2)


def test_head_over_pages_refusals(lib):
    """What the paged prefill and step refuse before any launch, and the state they leave: a context over addresses nobody reads."""
    from paper_2505_24544_b200.binding import BeagleConfig, BeagleWeights
    assert lib.beagle_draft_step_pages(None, None, 0, None, None, 1, 0, 0, None, 1, None, None, None, None) == INVALID
    assert lib.beagle_prefill_pages(None, None, 0, None, None, None, None, None, 0, None) == INVALID

    def context(theta=0.0):
        cfg = BeagleConfig(512, 8, 2, 64, 1024, 4096, 1, 1e-5, 1, 1, 6, 64, 8, theta)
        w = BeagleWeights()
        for name, _ in BeagleWeights._fields_:
            setattr(w, name, 4096)
        w.w_lm_fp8 = w.w_lm_scale = None
        h = C.c_void_p()
        assert lib.beagle_create(C.byref(cfg), C.byref(w), 256, 1 << 40, 256, 1 << 40, C.byref(h)) == OK
        return h

    n = C.c_size_t()
    cfg = BeagleConfig(512, 8, 2, 64, 1024, 4096, 1, 1e-5, 1, 1, 6, 64, 8, 0.0)
    assert lib.beagle_prefill_pages_workspace_bytes(C.byref(cfg), 3, C.byref(n)) == OK and n.value == 2 * 768
    assert lib.beagle_prefill_pages_workspace_bytes(C.byref(cfg), 0, C.byref(n)) == OK and n.value == 0
    assert lib.beagle_prefill_pages_workspace_bytes(C.byref(cfg), -1, C.byref(n)) == INVALID
    assert lib.beagle_prefill_pages_workspace_bytes(C.byref(cfg), (1 << 24) + 1, C.byref(n)) == CAPACITY
    assert lib.beagle_prefill_pages_workspace_bytes(C.byref(cfg), 3, None) == INVALID
    h = context()

    def step(p, slots=(0,), tokens=4096, window=0, sinks=0, ctx=h):
        return lib.beagle_draft_step_pages(ctx, C.byref(p), len(slots), arr(*slots), tokens, 1, window, sinks, 1 << 30, 1, None, None, None, None)

    def prefill(p, slots=(0,), lens=(3,), hidden=1 << 30, ws=1 << 29, size=1 << 20, ctx=h):
        return lib.beagle_prefill_pages(ctx, C.byref(p), len(slots), arr(*slots), arr(*lens), hidden, None, ws, size, None)

    for call in (step, prefill):
        assert call(pages(lib, head_dim=128)) == SHAPE
        assert call(pages(lib, n_kv_heads=4)) == SHAPE
        assert call(pages(lib, dtype=0)) == SHAPE
        assert call(pages(lib, k=0)) == INVALID
        assert call(pages(lib, ws_bytes=16)) == CAPACITY
        assert call(pages(lib), slots=(4,)) == INVALID                       # the context has six slots, the cache four
        assert call(pages(lib, max_slots=8), slots=(6,)) == INVALID          # and the other way round
        assert call(pages(lib), slots=(1, 1)) == INVALID
        turned = context(10000.0)
        assert call(pages(lib), ctx=turned) == 5                             # UNSUPPORTED
        lib.beagle_destroy(turned)
    assert step(pages(lib), window=-1) == INVALID and step(pages(lib), sinks=-1) == INVALID
    assert step(pages(lib), tokens=None) == 4                                # no previous token: STATE
    assert step(pages(lib), slots=()) == OK
    assert prefill(pages(lib), lens=(-1,)) == INVALID
    assert prefill(pages(lib), lens=(1 << 25,)) == CAPACITY
    assert prefill(pages(lib), hidden=None) == INVALID and prefill(pages(lib), hidden=(1 << 30) + 2) == INVALID
    assert prefill(pages(lib), ws=None) == INVALID and prefill(pages(lib), ws=(1 << 29) + 16) == INVALID
    assert prefill(pages(lib), size=2 * 768 - 1) == CAPACITY
    assert prefill(pages(lib), lens=(0,), hidden=None, ws=None, size=0) == OK and prefill(pages(lib), slots=()) == OK
    lib.beagle_destroy(h)


class RefusingHead:
    """A head and a cache in the binding's eyes, of hidden size 512 and 4096 tokens; a call that reaches the library fails the test."""

    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was reached")

    def __init__(self):
        from paper_2505_24544_b200.binding import BeagleConfig
        self.cfg = BeagleConfig(512, 8, 2, 64, 1024, 4096, 1, 1e-5, 1, 1, 6, 64, 8, 0.0)
        self.lib, self.handle, self.ref = self.Library(), None, None

    def check(self, status):
        assert status == OK


@pytest.mark.parametrize("new_len", [[], [3], [3, 4, 5]])
def test_prefill_pages_wants_one_length_per_slot(new_len):
    """The library reads as many lengths as there are slots: a list of another length is refused before it sees them."""
    from paper_2505_24544_b200 import binding as b
    with pytest.raises(ValueError, match="new_len"):
        b.beagle_prefill_pages(RefusingHead(), RefusingHead(), [0, 1], new_len, None)


def test_draft_step_pages_checks_its_tensors(monkeypatch):
    """Type, shape, layout and device of every tensor of the paged step (host tensors stand for device ones where the device is
    not what is wrong)."""
    torch = pytest.importorskip("torch")
    from paper_2505_24544_b200 import binding as b
    i32, f32, bf16 = torch.int32, torch.float32, torch.bfloat16
    good = dict(tokens_in=((2,), i32), tokens_out=((2,), i32), logits_out=((2, 4096), f32), hidden_out=((2, 512), bf16), ok=((2,), i32))
    bad = dict(tokens_in=[((2,), torch.int64), ((3,), i32), ((2, 1), i32)], tokens_out=[((2,), f32), ((1,), i32), ((2, 1), i32)],
               logits_out=[((2, 4096), bf16), ((2, 4095), f32), ((1, 4096), f32)], hidden_out=[((2, 512), f32), ((2, 511), bf16), ((3, 512), bf16)],
               ok=[((2,), torch.int64), ((1,), i32)])

    def call(**kw):
        x = {n: torch.zeros(s, dtype=t) for n, (s, t) in good.items()}
        x.update(kw)
        b.beagle_draft_step_pages(RefusingHead(), RefusingHead(), [0, 1], x["tokens_in"], True, x["tokens_out"], x["logits_out"], x["hidden_out"], 0, 0, x["ok"])
    with pytest.raises(ValueError, match="device"):
        call()                                                               # host memory
    check = b._check
    monkeypatch.setattr(b, "_check", lambda name, t, dtype, shape, dense=True:
                        check(name, t, dtype, shape, dense) if t.dtype != dtype or t.shape != shape or (dense and not t.is_contiguous()) else t.data_ptr())
    with pytest.raises(AssertionError, match="beagle_draft_step_pages was reached"):
        call()                                                               # nothing wrong: on to the library
    for name, cases in bad.items():
        for shape, dtype in cases:
            with pytest.raises(ValueError, match=name):
                call(**{name: torch.zeros(shape, dtype=dtype)})
    for name in ("logits_out", "hidden_out"):
        shape, dtype = good[name]
        with pytest.raises(ValueError, match=name):
            call(**{name: torch.zeros(shape[1], shape[0], dtype=dtype).t()})


def test_paged_attn_checks_its_workspace(monkeypatch):
    """A workspace in host memory, or with gaps, is refused like any other tensor."""
    torch = pytest.importorskip("torch")
    from paper_2505_24544_b200 import binding as b
    cache, q = RefusingHead(), torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    cache.struct, cache.k, cache.attn_ws_bytes, cache.on_current_device = b.BeaglePages(head_dim=64), q, {(4, 0, 0): 64}, lambda: 0
    monkeypatch.setattr(b, "_check", lambda name, t, *_: t.data_ptr())           # q and out stand for tensors on the device
    with pytest.raises(ValueError, match="ws.*device"):
        b.beagle_paged_attn(cache, [0], q, q, ws=torch.zeros(64, dtype=torch.uint8))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    with pytest.raises(ValueError, match="ws.*contiguous"):
        b.beagle_paged_attn(cache, [0], q, q, ws=torch.zeros(64, 2, dtype=torch.uint8)[:, 0])
    with pytest.raises(AssertionError, match="beagle_paged_attn was reached"):
        b.beagle_paged_attn(cache, [0], q, q, ws=torch.zeros(64, dtype=torch.uint8))
