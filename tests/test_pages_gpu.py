"""Paged key/value cache on the GPU: book-keeping against a step-by-step model of it, attention against the definition in 64 bits."""
import random

import pytest
import torch

from paper_2505_24544_b200 import binding as b

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


class Model:
    """The documented behaviour, one slot after the other, on the host."""

    def __init__(self, cache):
        self.ps, self.width = cache.struct.page_size, cache.struct.max_pages
        self.k, self.v = cache.k.cpu(), cache.v.cpu()
        self.refs, self.length = [0] * cache.struct.n_pages, [0] * cache.struct.max_slots
        self.pages = [[] for _ in self.length]

    def append(self, slots, k, v, n):
        at_entry = list(self.refs)
        free, ok = [p for p, r in enumerate(at_entry) if r == 0], []
        want = []
        for s, m in zip(slots, n):
            L = self.length[s]
            shared = L % self.ps != 0 and m > 0 and at_entry[self.pages[s][-1]] > 1
            fits = L + m <= self.width * self.ps
            want.append((-(-(L + m) // self.ps) - -(-L // self.ps) + shared if fits else 0, shared, fits))
        taken = 0
        for i, (s, m) in enumerate(zip(slots, n)):
            need, shared, fits = want[i]
            taken += need
            good = fits and (need == 0 or taken <= len(free))
            ok.append(int(good))
            if not good:
                continue
            mine = free[taken - need:taken]
            L = self.length[s]
            for p in mine:
                self.refs[p] = 1
            if shared:
                old, new = self.pages[s][-1], mine.pop(0)
                self.k[new, :, :L % self.ps], self.v[new, :, :L % self.ps] = self.k[old, :, :L % self.ps], self.v[old, :, :L % self.ps]
                self.refs[old] -= 1
                self.pages[s][-1] = new
            self.pages[s] += mine
            for t in range(m):
                p, r = self.pages[s][(L + t) // self.ps], (L + t) % self.ps
                self.k[p, :, r], self.v[p, :, r] = k[i, t].cpu(), v[i, t].cpu()
            self.length[s] = L + m
        return ok

    def truncate(self, slots, keep):
        for s, n in zip(slots, keep):
            n = max(0, min(n, self.length[s]))
            have = -(-n // self.ps)
            for p in self.pages[s][have:]:
                self.refs[p] -= 1
            self.pages[s], self.length[s] = self.pages[s][:have], n

    def fork(self, src, dst):
        self.truncate(dst, [0] * len(dst))
        for x, y in zip(src, dst):
            self.pages[y], self.length[y] = list(self.pages[x]), self.length[x]
            for p in self.pages[x]:
                self.refs[p] += 1

    def copy(self, src, dst):
        self.truncate(dst, [0] * len(dst))
        free, taken, ok = [p for p, r in enumerate(self.refs) if r == 0], 0, []
        for x, y in zip(src, dst):
            need = len(self.pages[x])
            taken += need
            ok.append(int(need == 0 or taken <= len(free)))
            if ok[-1]:
                mine = free[taken - need:taken]
                for p, q in zip(self.pages[x], mine):
                    self.refs[q] = 1
                    self.k[q], self.v[q] = self.k[p], self.v[p]
                self.pages[y], self.length[y] = mine, self.length[x]
        return ok

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        move = dict(zip([p for p, r in enumerate(self.refs) if r > 0 and p >= live], [p for p, r in enumerate(self.refs) if r == 0 and p < live]))
        for x, y in move.items():
            self.k[y], self.v[y] = self.k[x], self.v[x]
            self.refs[y], self.refs[x] = self.refs[x], 0
        self.pages = [[move.get(p, p) for p in row] for row in self.pages]

    def same(self, cache):
        assert cache.length.tolist() == self.length
        assert cache.refs.tolist() == self.refs
        assert cache.table.tolist() == [row + [-1] * (self.width - len(row)) for row in self.pages]
        assert torch.equal(cache.k.cpu().view(torch.uint8), self.k.view(torch.uint8)) and torch.equal(cache.v.cpu().view(torch.uint8), self.v.view(torch.uint8))


def new_cache(n_pages, ps, hkv, dh, slots, width, dtype):
    cache = b.PagedCache(n_pages, ps, hkv, dh, slots, width, dtype)
    cache.k.normal_()
    cache.v.normal_()
    return cache


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,hkv,dh,ps,n_pages,slots,width", [
    ("bf16", 2, 64, 16, 60, 9, 8), ("bf16", 8, 128, 64, 40, 12, 6), ("fp32", 3, 16, 8, 100, 20, 9), ("bf16", 1, 256, 32, 24, 5, 7),
    ("fp32", 2, 128, 256, 12, 6, 3), ("bf16", 5, 32, 128, 17, 70, 2),
])
def test_random_book_keeping_cases(dtype, hkv, dh, ps, n_pages, slots, width):
    random_book_keeping(dtype, hkv, dh, ps, n_pages, slots, width)


def random_book_keeping(dtype, hkv, dh, ps, n_pages, slots, width):
    """Two hundred random calls, pages running out among them, follow the model exactly: table, counts, lengths and contents."""
    cache = new_cache(n_pages, ps, hkv, dh, slots, width, dtype)
    m, r = Model(cache), random.Random(n_pages)
    g = torch.Generator(device="cuda").manual_seed(5)
    failed = 0
    for i in range(200):
        kind = r.choice(["append"] * 4 + ["truncate", "truncate", "fork", "copy", "compact"])
        n = r.randint(1, min(slots // 2, 8))
        picked = r.sample(range(slots), 2 * n)
        if kind == "append":
            T = r.choice([0, 1, 1, 5, ps, 2 * ps + 3])
            rows = picked[:n]
            k, v = (torch.randn(n, T, hkv, dh, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
            counts = [r.randint(-2, T + 2) for _ in rows] if r.random() < 0.5 else None
            ok = i32([7] * n)
            b.beagle_pages_append(cache, rows, k, v, None if counts is None else i32(counts), ok)
            want = m.append(rows, k, v, [T] * n if counts is None else [min(max(c, 0), T) for c in counts])
            assert ok.tolist() == want
            failed += want.count(0)
        elif kind == "truncate":
            keep = [r.randint(-1, width * ps) for _ in range(n)] if r.random() < 0.6 else None
            b.beagle_pages_truncate(cache, picked[:n], None if keep is None else i32(keep))
            m.truncate(picked[:n], [0] * n if keep is None else keep)
        elif kind == "fork":
            src = [r.choice(picked[:n]) for _ in range(n)]
            b.beagle_pages_fork(cache, src, picked[n:])
            m.fork(src, picked[n:])
        elif kind == "copy":
            ok = i32([7] * n)
            b.beagle_pages_copy(cache, picked[:n], picked[n:], ok)
            want = m.copy(picked[:n], picked[n:])
            assert ok.tolist() == want
            failed += want.count(0)
        else:
            b.beagle_pages_compact(cache)
            m.compact()
        if i % 10 == 9:
            m.same(cache)
    m.same(cache)
    return failed


def test_random_book_keeping_in_a_small_pool():
    """Twenty pages for twelve slots of up to eight: calls run out of pages again and again."""
    assert random_book_keeping("bf16", 2, 64, 16, 20, 12, 8) > 10


def test_append_from_a_fused_projection():
    """Rows that are slices of a wider matrix, one row per slot and several, are read where they lie."""
    cache = new_cache(20, 16, 2, 64, 4, 8, "bf16")
    m = Model(cache)
    fused = torch.randn(3, 5, 12 * 64, device="cuda").bfloat16()
    k, v = (fused[:, :, i * 128:(i + 1) * 128].unflatten(2, (2, 64)) for i in (4, 5))
    b.beagle_pages_append(cache, [2, 0, 3], k, v)
    m.append([2, 0, 3], k, v, [5] * 3)
    b.beagle_pages_append(cache, [0, 3, 1], k[:, 2:3], v[:, 2:3])
    m.append([0, 3, 1], k[:, 2:3], v[:, 2:3], [1] * 3)
    m.same(cache)
    with pytest.raises((ValueError, b.BeagleError)):
        b.beagle_pages_append(cache, [0, 1, 2], k[:, :1].expand(3, 4, 2, 64), v[:, :1].expand(3, 4, 2, 64))       # one row for all: refused


def test_many_pages():
    """More pages than one step of the scan over the counts covers (16384), with holes everywhere."""
    n = 40000
    cache = new_cache(n, 8, 1, 32, 4, 20000, "bf16")
    rows = torch.randn(1, 8 * 18000, 1, 32, device="cuda").bfloat16()
    b.beagle_pages_append(cache, [0], rows, rows)
    b.beagle_pages_append(cache, [1], rows, rows)
    assert cache.table[1, :3].tolist() == [18000, 18001, 18002] and int(cache.table[1, 17999]) == 35999
    b.beagle_pages_truncate(cache, [0])
    b.beagle_pages_append(cache, [2], rows[:, :24], rows[:, :24])
    assert cache.table[2, :4].tolist() == [0, 1, 2, -1]
    b.beagle_pages_compact(cache)
    t = cache.table[1, :18000]
    assert int((cache.refs > 0).sum()) == 18003 and bool((cache.refs[:18003] == 1).all())
    # pages below the new count stay, the others fill the holes 3 .. in ascending order
    old = torch.arange(18000, 36000, device="cuda")
    assert torch.equal(t, torch.where(old < 18003, old, old - 18003 + 3).int())
    got = cache.k[t.long()].permute(1, 0, 2, 3).reshape(-1, 32)
    assert torch.equal(got, rows[0, :, 0])


def reference(cache, slots, q, window, sinks):
    """(o, lse, sum of p |v|, largest sum |q k| / sqrt(dh)) in 64 bits."""
    B, hq, dh = q.shape
    hkv = cache.struct.n_kv_heads
    G = hq // hkv
    o, mass = torch.zeros(B, hq, dh, dtype=torch.float64), torch.zeros(B, hq, dh, dtype=torch.float64)
    lse, size = torch.full((B, hq), -torch.inf, dtype=torch.float64), torch.zeros(B, hq, dtype=torch.float64)
    K, V, table, length = cache.k.cpu().double(), cache.v.cpu().double(), cache.table.cpu(), cache.length.tolist()
    for i, s in enumerate(slots):
        n = length[s]
        if n == 0:
            continue
        pages = table[s, : -(-n // cache.struct.page_size)].long()
        j = torch.arange(n)
        seen = ((j >= n - window) | (j < sinks)) if window > 0 else j >= 0
        for h in range(hq):
            k, v = (x[pages, h // G].reshape(-1, dh)[:n][seen] for x in (K, V))
            z = k @ q[i, h].cpu().double() / dh ** 0.5
            lse[i, h] = torch.logsumexp(z, 0)
            p = torch.exp(z - lse[i, h])
            o[i, h], mass[i, h] = p @ v, p @ v.abs()
            size[i, h] = (k.abs() @ q[i, h].cpu().double().abs()).max() / dh ** 0.5
    return o, lse, mass, size


def check_attn(cache, slots, q, window, sinks, dtype, out=None, lse=None):
    if out is None:
        out, lse = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 9.0, device="cuda")
        b.beagle_paged_attn(cache, slots, q, out, lse, window=window, sinks=sinks)
    o, l, mass, size = reference(cache, slots, q, window, sinks)
    dh, n = q.shape[2], cache.struct.max_pages * cache.struct.page_size
    # scores: fp32 products and sums; weights: the score's error, 2^-21 for the exponential and its argument's roundings;
    # sums over at most n terms; lse: the same plus its own roundings
    score = (dh + 8) * 2.0 ** -24 * size + 2.0 ** -21 * (1 + size)
    got_l = lse.cpu().double()
    empty = torch.isinf(l)
    assert torch.equal(empty, torch.isinf(got_l))
    assert bool(((got_l - l).abs()[~empty] <= (score + n * 2.0 ** -24 + 2.0 ** -21 * (1 + l.abs()))[~empty]).all())
    weight = 2 * score + 2 * n * 2.0 ** -24 + (HALF["bf16"] if dtype == "bf16" else 0.0)      # bf16: the product takes rounded weights
    err = (out.cpu().double() - o).abs()
    # (+ 2^-20: products of subnormal size)
    assert bool((err <= weight[..., None] * mass + HALF[dtype] * (o.abs() + weight[..., None] * mass) + 2.0 ** -40).all()), float(err.max())


def filled(lens, ps, hkv, dh, dtype, seed, nan=True, width=None):
    """A cache whose slots hold these lengths in shuffled pages; every position that holds nothing is NaN."""
    r = random.Random(seed)
    width = width or max(1, -(-max(lens) // ps)) + 1
    need = [-(-n // ps) for n in lens]
    cache = b.PagedCache(sum(need) + 3, ps, hkv, dh, len(lens), width, dtype)
    cache.k.fill_(float("nan") if nan else 0.0)
    cache.v.fill_(float("nan") if nan else 0.0)
    ids = r.sample(range(sum(need) + 3), sum(need))
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = [[-1] * width for _ in lens]
    at = 0
    for s, n in enumerate(lens):
        for i in range(need[s]):
            p, rows = ids[at], min(ps, n - i * ps)
            at += 1
            table[s][i] = p
            cache.k[p, :, :rows] = (torch.randn(hkv, rows, dh, generator=g, device="cuda")).to(DT[dtype])
            cache.v[p, :, :rows] = (torch.randn(hkv, rows, dh, generator=g, device="cuda")).to(DT[dtype])
    cache.table.copy_(i32(table))
    cache.length.copy_(i32(lens))
    used = torch.zeros(cache.struct.n_pages, dtype=torch.int32)
    used[ids] = 1
    cache.refs.copy_(used)
    return cache


LENS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 0, 1000, 7]


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 16, 2, 64), ("bf16", 3, 1, 128), ("bf16", 7, 1, 64),
                                            ("bf16", 4, 2, 32), ("bf16", 4, 1, 256), ("fp32", 4, 4, 64), ("fp32", 8, 1, 128), ("fp32", 6, 2, 16),
                                            ("fp32", 4, 2, 32), ("fp32", 5, 1, 64)])
@pytest.mark.parametrize("ps", [8, 16, 64, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (64, 4), (100, 70), (17, 1000), (600, 5)])
def test_attention(dtype, hq, hkv, dh, ps, window, sinks):
    """Lengths around every tile and page border, empty slots among them; whatever is not visible is NaN or Inf.  (The small
    windows are divided by pairs, the others into runs that are joined.)"""
    cache = filled(LENS, ps, hkv, dh, dtype, 11)
    r = random.Random(3)
    slots = list(range(len(LENS))) + [14, 12]            # a slot may serve several rows
    r.shuffle(slots)
    if window > 0:                                       # positions outside the window hold no finite number either
        for s, n in enumerate(LENS):
            for j in range(min(sinks, n), max(0, n - window)):
                p = int(cache.table[s, j // ps])
                cache.k[p, :, j % ps] = float("inf")
                cache.v[p, :, j % ps] = float("nan")
    q = (torch.randn(len(slots), hq, dh, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") * 2).to(DT[dtype])
    check_attn(cache, slots, q, window, sinks, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens", [[20000], [9000, 1, 0, 4000], [1] * 64, [130] * 64, [1]])
def test_attention_splits(dtype, lens):
    """One long sequence over many runs, many short ones inside one run, and rising scores (the reference point moves)."""
    cache = filled(lens, 32, 2, 64, dtype, 4)
    for s, n in enumerate(lens):                         # scores rise along the sequence by far more than the slack of the kernel
        for i in range(-(-n // 32)):
            cache.k[int(cache.table[s, i])] *= 1 + 0.01 * i
    q = (torch.randn(len(lens), 8, 64, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") * 2).to(DT[dtype])
    slots = list(range(len(lens)))
    check_attn(cache, slots, q, 0, 0, dtype)
    check_attn(cache, slots, q, 5000, 4, dtype)


def test_attention_strided_queries_and_another_stream():
    cache = filled([77, 300, 5], 16, 2, 128, "bf16", 9)
    fused = torch.randn(3, 20 * 128, device="cuda").bfloat16()
    q = fused[:, 512:512 + 8 * 128].unflatten(1, (8, 128))
    ref_out, ref_lse = torch.empty(3, 8, 128, device="cuda").bfloat16(), torch.empty(3, 8, device="cuda")
    b.beagle_paged_attn(cache, [2, 0, 1], q, ref_out, ref_lse)
    check_attn(cache, [2, 0, 1], q, 0, 0, "bf16", ref_out, ref_lse)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out, lse = torch.empty_like(ref_out), torch.empty_like(ref_lse)
    with torch.cuda.stream(side):
        b.beagle_paged_attn(cache, [2, 0, 1], q, out, lse)
    side.synchronize()
    assert torch.equal(out, ref_out) and torch.equal(lse, ref_lse)
    b.beagle_paged_attn(cache, [2, 0, 1], q, out, None)
    assert torch.equal(out, ref_out)
    with pytest.raises(b.BeagleError):
        b.beagle_paged_attn(cache, [2, 0, 9], q, out)
    with pytest.raises(ValueError):
        b.beagle_paged_attn(cache, [2, 0, 1], q, out.cpu())
    cache = filled([77, 300, 5], 16, 2, 128, "bf16", 9, width=200)
    with pytest.raises(b.BeagleError):
        b.beagle_paged_attn(cache, [2, 0, 1], q, out, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_damaged_table_stays_inside_the_pools():
    """Entries, lengths and counts out of range: contents are undefined, but every access stays inside the cache's buffers (the
    rows next to the pools are untouched) and the calls return."""
    hkv, dh, ps, n_pages = 2, 64, 16, 10
    rows = n_pages * hkv * ps * dh
    guard = torch.full((3 * rows,), 5.0, dtype=torch.bfloat16, device="cuda")
    k = guard[rows:2 * rows].view(n_pages, hkv, ps, dh)
    v = torch.zeros(n_pages, hkv, ps, dh, dtype=torch.bfloat16, device="cuda")
    table = i32([[3, 99, -7], [1 << 30, 2, 0], [-1, -1, -1]])
    cache = b.PagedCache.from_tensors(k, v, table, i32([48, 100000, -5]), i32([0] * n_pages))
    new = torch.ones(3, 2, hkv, dh, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(3, 4, dh, dtype=torch.bfloat16, device="cuda")
    b.beagle_paged_attn(cache, [0, 1, 2], torch.ones_like(out), out)
    b.beagle_pages_append(cache, [0, 1, 2], new, new)
    b.beagle_pages_fork(cache, [0], [2])
    b.beagle_pages_compact(cache)
    b.beagle_pages_copy(cache, [1], [2])
    b.beagle_pages_truncate(cache, [0, 1, 2])
    torch.cuda.synchronize()
    assert bool((guard[:rows] == 5).all()) and bool((guard[2 * rows:] == 5).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_serving_run(dtype):
    """The calls together, as a server makes them: prompts, steps with a window, a fork that diverges, rejected drafts rolled
    back, a sequence ended and the pool compacted; then the same steps from a captured graph.  Every attention against the
    definition over what the model says the slots hold."""
    hkv, dh, ps = 2, 64, 16
    cache = new_cache(64, ps, hkv, dh, 6, 16, dtype)
    m = Model(cache)
    g = torch.Generator(device="cuda").manual_seed(1)

    def rows(B, T):
        return [torch.randn(B, T, hkv, dh, generator=g, device="cuda").to(DT[dtype]) for _ in range(2)]

    def attend(slots, window=0, sinks=0):
        q = torch.randn(len(slots), 8, dh, generator=g, device="cuda").to(DT[dtype])
        check_attn(cache, slots, q, window, sinks, dtype)
        m.same(cache)

    k, v = rows(3, 100)
    n = [100, 37, 64]
    b.beagle_pages_append(cache, [0, 1, 2], k, v, i32(n))
    m.append([0, 1, 2], k, v, n)
    attend([0, 1, 2])
    b.beagle_pages_fork(cache, [0, 1], [3, 4])
    m.fork([0, 1], [3, 4])
    for step in range(20):
        k, v = rows(5, 3)
        b.beagle_pages_append(cache, [0, 1, 2, 3, 4], k, v)
        m.append([0, 1, 2, 3, 4], k, v, [3] * 5)
        keep = [x - (step + i) % 3 for i, x in enumerate(m.length[:5])]
        b.beagle_pages_truncate(cache, [0, 1, 2, 3, 4], i32(keep))
        m.truncate([0, 1, 2, 3, 4], keep)
    attend([0, 1, 2, 3, 4], 40, 4)
    b.beagle_pages_truncate(cache, [0])
    m.truncate([0], [0])
    b.beagle_pages_compact(cache)
    m.compact()
    attend([4, 3, 2, 1, 0], 0, 0)
    # one step from a graph: append, then attention, replayed with new rows; lengths move on the device
    k, v = rows(4, 1)
    q = torch.randn(4, 8, dh, generator=g, device="cuda").to(DT[dtype])
    out, lse = torch.empty_like(q), torch.empty(4, 8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.beagle_pages_append(cache, [1, 2, 3, 4], k, v)
            b.beagle_paged_attn(cache, [1, 2, 3, 4], q, out, lse, window=50, sinks=2)
    torch.cuda.synchronize()
    for _ in range(ps + 2):
        a, c = rows(4, 1)
        k.copy_(a)
        v.copy_(c)
        graph.replay()
        m.append([1, 2, 3, 4], k, v, [1] * 4)
    torch.cuda.synchronize()
    m.same(cache)
    check_attn(cache, [1, 2, 3, 4], q, 50, 2, dtype, out, lse)


@pytest.mark.parametrize("dtype,dh,group", [("fp32", d, g) for d in (16, 32, 64, 128) for g in (1, 2, 3, 8)] +
                         [("bf16", 32, g) for g in (1, 2, 4, 8)] + [("bf16", 256, g) for g in (1, 2, 4)])
@pytest.mark.parametrize("ps,window,sinks", [(8, 0, 0), (64, 0, 0), (256, 700, 90)])
def test_every_group_size_off_the_tensor_cores(dtype, dh, group, ps, window, sinks):
    """Every width and number of query heads a K/V head of the CUDA-core kernel, on sequences that are cut and joined."""
    cache = filled([3000, 1, 0, 257, 64, 1100], ps, 2, dh, dtype, 17)
    q = (torch.randn(6, 2 * group, dh, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") * 2).to(DT[dtype])
    check_attn(cache, [5, 0, 1, 2, 3, 4], q, window, sinks, dtype)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 256), ("fp32", 64)])
@pytest.mark.parametrize("width", [2, 200])
def test_an_empty_slot_gives_zero_and_minus_infinity(dtype, dh, width):
    """Whether pairs are divided whole or cut into runs."""
    cache = filled([0, 40, 0], 32, 2, dh, dtype, 6, width=width)
    q = torch.ones(3, 4, dh, dtype=DT[dtype], device="cuda")
    out, lse = torch.full_like(q, 9.0), torch.full((3, 4), 9.0, device="cuda")
    b.beagle_paged_attn(cache, [0, 1, 2], q, out, lse)
    assert bool(torch.isneginf(lse[[0, 2]]).all()) and bool(torch.isfinite(lse[1]).all())
    assert bool((out[[0, 2]] == 0).all()) and bool(torch.isfinite(out[1]).all())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 256), ("fp32", 128)])
def test_pools_past_32_bit_offsets(dtype, dh):
    """Pools of more than 2^31 elements: rows appended to the last pages, read, copied, moved and forked there as anywhere else."""
    hkv, ps = 8, 64
    n_pages = 2 ** 31 // (hkv * ps * dh) + 40
    cache = b.PagedCache(n_pages, ps, hkv, dh, 4, n_pages, dtype)
    g = torch.Generator(device="cuda").manual_seed(8)
    k, v = (torch.randn(1, 700, hkv, dh, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    q = torch.randn(1, 16, dh, generator=g, device="cuda").to(DT[dtype])

    def attend(slot):
        out, lse = torch.empty_like(q), torch.empty(1, 16, device="cuda")
        b.beagle_paged_attn(cache, [slot], q, out, lse, window=500, sinks=70)
        return out, lse

    def pages(slot):
        return cache.table[slot, :11].tolist()
    b.beagle_pages_append(cache, [0], k, v)
    want = attend(0)
    assert pages(0) == list(range(11))
    cache.refs[11:n_pages - 25] = 1                          # pages that another program holds: the free ones are the last
    b.beagle_pages_append(cache, [1], k, v)
    b.beagle_pages_copy(cache, [0], [2])
    top = n_pages - 25
    assert pages(1) == list(range(top, top + 11)) and pages(2) == list(range(top + 11, top + 22))
    for slot in (1, 2):
        at = torch.tensor(pages(slot), device="cuda")
        for pool, rows in ((cache.k, k), (cache.v, v)):
            assert torch.equal(pool[at].permute(0, 2, 1, 3).reshape(-1, hkv, dh)[:700], rows[0])
        assert all(torch.equal(x, y) for x, y in zip(attend(slot), want))
    b.beagle_pages_fork(cache, [2], [3])
    b.beagle_pages_append(cache, [3], k[:, :1], v[:, :1])    # the last page's rows are copied from one end of the pool to the other
    assert pages(3) == pages(2)[:10] + [top + 22]
    assert all(torch.equal(x, y) for x, y in zip(attend(2), want))
    cache.refs[11:top] = 0
    b.beagle_pages_compact(cache)
    assert pages(1) == list(range(11, 22)) and int(cache.table.max()) == 33
    for slot in (1, 2):
        assert all(torch.equal(x, y) for x, y in zip(attend(slot), want))
