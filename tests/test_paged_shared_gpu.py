"""Attention of groups that share a prefix, against the definition in 64 bits row by row; the steps of a sampled batch together."""
import random

import pytest
import torch

from paper_2505_24544_b200 import binding as b
from test_pages_gpu import HALF, check_attn, filled, i32, reference
from test_rotary_gpu import randn, reference as rotated

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def forked(groups, prefix, suffix, ps, hkv, dh, dtype, seed):
    """A cache of groups of slots that share their prefix's whole pages: prefix per group, suffix per slot; unused positions are NaN.
    (A prefix that ends inside a page lies once more in each slot's own page.)"""
    r = random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens = []
    for i, n in enumerate(groups):
        lens += [prefix[i] + suffix[len(lens) + x] for x in range(n)]
    width = max(1, -(-max(lens) // ps)) + 1
    n_pages = sum(-(-n // ps) for n in prefix) + sum(-(-n // ps) for n in lens) + 3
    cache = b.PagedCache(n_pages, ps, hkv, dh, len(lens), width, dtype)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    free = r.sample(range(n_pages), n_pages)
    table, refs, slot = [[-1] * width for _ in lens], [0] * n_pages, 0

    def rows(n, i):
        x = torch.randn(2, n, hkv, dh, generator=g, device="cuda")
        x[0] *= 1 + 0.02 * i                             # scores rise along the sequence: the reference points move
        return x.to(DT[dtype]).transpose(1, 2)

    shared = []
    for i, n in enumerate(groups):
        whole, rest = prefix[i] // ps, prefix[i] % ps
        pages = [free.pop() for _ in range(whole)]
        for x, p in enumerate(pages):
            cache.k[p], cache.v[p] = rows(ps, x)
        tail = rows(rest, whole)
        for _ in range(n):
            at = prefix[i] + suffix[slot]
            for x in range(whole):
                table[slot][x] = pages[x]
                refs[pages[x]] += 1
            for x in range(whole, -(-at // ps)):
                p, used = free.pop(), min(ps, at - x * ps)
                new = rows(used, x)
                if x == whole:
                    new[:, :, :min(rest, used)] = tail[:, :, :min(rest, used)]
                cache.k[p, :, :used], cache.v[p, :, :used] = new
                table[slot][x] = p
                refs[p] += 1
            slot += 1
        shared.append(whole * ps if n > 1 else 0)
    cache.table.copy_(i32(table))
    cache.length.copy_(i32(lens))
    cache.refs.copy_(i32(refs))
    return cache, shared


def attend(cache, slots, groups, shared, q, dtype):
    out, lse = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 9.0, device="cuda")
    b.beagle_paged_attn_shared(cache, slots, groups, shared, q, out, lse)
    check_attn(cache, slots, q, 0, 0, dtype, out, lse)
    again, lse2 = torch.empty_like(out), torch.empty_like(lse)
    b.beagle_paged_attn_shared(cache, slots, groups, shared, q, again, lse2)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    return out


KINDS = [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 16, 2, 64), ("bf16", 3, 1, 128), ("bf16", 7, 1, 64), ("bf16", 4, 2, 32), ("bf16", 4, 1, 256), ("bf16", 8, 1, 128),
         ("fp32", 4, 4, 64), ("fp32", 8, 1, 128), ("fp32", 6, 2, 16), ("fp32", 4, 2, 32), ("fp32", 5, 1, 64)]


@pytest.mark.parametrize("dtype,hq,hkv,dh", KINDS)
@pytest.mark.parametrize("ps", [8, 16, 64, 256])
def test_groups(dtype, hq, hkv, dh, ps):
    """Groups of one row to many, prefixes around tile and page borders, slots that end with their prefix, rows in any order of slots."""
    groups = [1, 5, 2, 33, 3, 4, 9]
    prefix = [70, 0, 64, 700, 63, 300, 1024]
    r = random.Random(ps)
    suffix = [r.choice([0, 1, 5, 63, 64, 65, 130]) for _ in range(sum(groups))]
    cache, shared = forked(groups, prefix, suffix, ps, hkv, dh, dtype, 5)
    slots = list(range(sum(groups)))
    got = torch.full((len(groups),), -5, dtype=torch.int32, device="cuda")
    b.beagle_pages_shared(cache, slots, groups, got)
    want = []
    for i, n in enumerate(groups):                       # what the table says: a slot may end before the shared pages do
        rows = cache.table[sum(groups[:i]):sum(groups[:i + 1])].tolist()
        least = min(prefix[i] + x for x in suffix[sum(groups[:i]):sum(groups[:i + 1])]) // ps
        same = 0
        while n > 1 and same < least and len({x[same] for x in rows}) == 1:
            same += 1
        want.append(same * ps)
    assert got.tolist() == want and all(x >= y for x, y in zip(want, shared) if y)
    q = (randn(len(slots), hq, dh, dtype=dtype, seed=1) * 2).to(DT[dtype])
    out = attend(cache, slots, groups, got, q, dtype)
    # smaller and larger numbers (clamped to the shortest slot only: the prompt's last page holds the same rows in every slot), none
    attend(cache, slots, groups, i32([max(0, x - 70) for x in want]), q, dtype)
    attend(cache, slots, groups, i32(prefix), q, dtype)
    attend(cache, slots, groups, i32([-3] * len(groups)), q, dtype)
    plain = torch.empty_like(out)
    b.beagle_paged_attn(cache, slots, q, plain)
    # both are within their bounds of the definition
    order = [1, 0] + list(range(2, len(groups)))
    start = [sum(groups[:i]) for i in range(len(groups))]
    mixed = [s for i in order for s in range(start[i], start[i] + groups[i])]
    attend(cache, mixed, [groups[i] for i in order], i32([want[i] for i in order]), q, dtype)


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 32, 8, 128), ("bf16", 8, 8, 64), ("bf16", 8, 1, 128), ("fp32", 4, 4, 64)])
@pytest.mark.parametrize("groups,prefix,suffix", [([64], [5000], 200), ([2], [20000], 0), ([1], [300], 7), ([16, 16, 16, 16], [1000, 64, 2500, 0], 90), ([2] * 32, [130] * 32, 3),
                                                  ([40, 1, 23], [100, 900, 9000], 1000)])
def test_sizes(dtype, hq, hkv, dh, groups, prefix, suffix):
    r = random.Random(3)
    own = [r.randint(0, suffix) for _ in range(sum(groups))]
    cache, shared = forked(groups, prefix, own, 32, hkv, dh, dtype, 6)
    q = (randn(sum(groups), hq, dh, dtype=dtype, seed=2) * 2).to(DT[dtype])
    attend(cache, list(range(sum(groups))), groups, i32(shared), q, dtype)


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 32), ("fp32", 64)])
def test_empty_slots(dtype, dh):
    cache, _ = forked([3, 1, 2], [0, 0, 64], [0, 5, 0, 0, 0, 9], 16, 2, dh, dtype, 7)
    q = randn(6, 4, dh, dtype=dtype, seed=3)
    out = attend(cache, list(range(6)), [3, 1, 2], i32([0, 0, 64]), q, dtype)
    assert bool((out[[0, 2, 3]] == 0).all())


def test_a_slot_twice_strided_queries_another_stream_and_own_workspace():
    cache, shared = forked([4, 4], [640, 100], [9, 70, 0, 1, 2, 3, 4, 5], 16, 2, 128, "bf16", 8)
    slots, groups = [0, 1, 1, 3, 4, 5, 4, 7], [4, 4]
    fused = randn(8, 20 * 128, dtype="bf16", seed=4)
    q = fused[:, 512:512 + 8 * 128].unflatten(1, (8, 128))
    ref = attend(cache, slots, groups, i32(shared), q, "bf16")
    ws = torch.full((b.beagle_paged_attn_shared_workspace_bytes(cache, 8, 8, groups),), 255, dtype=torch.uint8, device="cuda")
    sh, out = i32(shared).cuda(), torch.empty_like(ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.beagle_paged_attn_shared(cache, slots, groups, sh, q, out, ws=ws)
    side.synchronize()
    assert torch.equal(out, ref)
    with pytest.raises(b.BeagleError):
        b.beagle_paged_attn_shared(cache, slots, groups, sh, q, out, ws=ws[:-512])
    with pytest.raises(b.BeagleError):
        b.beagle_paged_attn_shared(cache, slots, [4, 3], sh, q, out)


def test_damaged_table_stays_inside_the_pools():
    """Page ids out of range and lengths past the table: wrong rows at most, and the other group's as they were."""
    cache, shared = forked([3, 3], [320, 200], [5, 70, 0, 1, 2, 3], 16, 2, 64, "bf16", 9)
    q = randn(6, 4, 64, dtype="bf16", seed=5)
    sh = i32(shared).cuda()
    ref, out = torch.empty_like(q), torch.empty_like(q)
    b.beagle_paged_attn_shared(cache, list(range(6)), [3, 3], sh, q, ref)
    cache.table[0, 2] = cache.struct.n_pages
    cache.table[0, 5] = 2 ** 31 - 1
    cache.table[1, 20] = -7
    cache.length[2] = 2 ** 31 - 1
    sh[0] = 2 ** 31 - 1
    b.beagle_paged_attn_shared(cache, list(range(6)), [3, 3], sh, q, out)
    b.beagle_pages_shared(cache, list(range(6)), [3, 3], sh)
    torch.cuda.synchronize()
    assert torch.equal(out[3:], ref[3:])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_sampling_from_a_forked_prompt(dtype):
    """A prompt's keys go in rotated, the slot is forked, and every step appends rotated keys (queries along), attends over the shared
    prefix, forms logits and draws a token, captured once and replayed: each step against the operators' definitions on the tensors it read."""
    hq, hkv, dh, ps, B, vocab, n0 = 8, 2, 64, 16, 6, 500, 150
    rot = b.Rotary(dh, 32, theta=5000.0, interleaved=True, scaling="bands", factor=4.0, original=100)
    cache = b.PagedCache(80, ps, hkv, dh, B, 20, dtype)
    pk, pv = randn(1, n0, hkv, dh, dtype=dtype, seed=1), randn(1, n0, hkv, dh, dtype=dtype, seed=2)
    b.beagle_pages_append_rotary(cache, [0], rot, pk, pv)
    b.beagle_pages_fork(cache, [0] * (B - 1), list(range(1, B)))
    shared = torch.empty(1, dtype=torch.int32, device="cuda")
    slots = list(range(B))
    emb = randn(vocab, (hq + 2 * hkv) * dh, dtype=dtype, seed=3)
    head = (randn(vocab, hq * dh, dtype=dtype, seed=4) * 0.2).to(DT[dtype])
    tokens, u, temp = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda"), torch.full((B,), 0.9, device="cuda")
    top_k = torch.full((B,), 40, dtype=torch.int32, device="cuda")
    q_out, out, logp = torch.empty(B, 1, hq, dh, dtype=DT[dtype], device="cuda"), torch.empty(B, hq, dh, dtype=DT[dtype], device="cuda"), torch.empty(B, device="cuda")
    x, logits, prev = torch.empty(B, (hq + 2 * hkv) * dh, dtype=DT[dtype], device="cuda"), torch.empty(B, vocab, device="cuda"), torch.zeros_like(tokens)

    def step():
        prev.copy_(tokens)
        x.copy_(emb[tokens.long()])
        q, k, v = x.unflatten(1, (1, -1, dh)).split([hq, hkv, hkv], 2)
        b.beagle_pages_append_rotary(cache, slots, rot, k, v, None, None, q, q_out)
        b.beagle_pages_shared(cache, slots, [B], shared)
        b.beagle_paged_attn_shared(cache, slots, [B], shared, q_out[:, 0], out)
        torch.matmul(out.flatten(1).float(), head.float().t(), out=logits)
        b.beagle_sample(logits, u, tokens, temperature=temp, top_k=top_k, logp=logp)

    step()
    assert shared.tolist() == [n0 // ps * ps]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    keep, was = cache.length.clone(), tokens.clone()
    with torch.cuda.graph(graph):
        step()
    assert torch.equal(cache.length, keep) and torch.equal(tokens, was)       # capturing runs nothing
    from test_sample_gpu import check
    for i in range(1, 25):
        u.copy_(torch.rand(B, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        pos = torch.full((B,), n0 + i, dtype=torch.int32)
        q, k, v = x.unflatten(1, (-1, dh)).split([hq, hkv, hkv], 1)
        assert torch.equal(x, emb[prev.long()])
        want, bound = rotated(rot, q, pos)
        assert bool(((q_out[:, 0].cpu().double() - want).abs() <= bound + HALF[dtype] * (want.abs() + bound)).all())
        want, bound = rotated(rot, k, pos)
        at = [(int(cache.table[s, (n0 + i) // ps]), (n0 + i) % ps) for s in slots]
        got = torch.stack([cache.k[p, :, r] for p, r in at]).cpu().double()
        assert bool(((got - want).abs() <= bound + HALF[dtype] * (want.abs() + bound)).all())
        assert torch.equal(torch.stack([cache.v[p, :, r] for p, r in at]), v)
        o, _, mass, size = reference(cache, slots, q_out[:, 0], 0, 0)
        score = (dh + 8) * 2.0 ** -24 * size + 2.0 ** -21 * (1 + size)
        weight = (2 * score + 2 * 320 * 2.0 ** -24 + (HALF["bf16"] if dtype == "bf16" else 0.0))[..., None] * mass
        assert bool(((out.cpu().double() - o).abs() <= weight + HALF[dtype] * (o.abs() + weight) + 2.0 ** -40).all())
        assert tokens.tolist() == check(logits, u.tolist(), temperature=[0.9] * B, top_k=[40] * B)
    assert cache.length.tolist() == [n0 + 25] * B and shared.tolist() == [n0 // ps * ps]
    assert len({tuple(r[n0 // ps:]) for r in cache.table.tolist()}) == B       # every sample has its own tail


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("fp32", 128)])
def test_pools_past_32_bit_offsets(dtype, dh):
    """Common and own pages at the end of pools of more than 2^31 elements."""
    ps, hkv = 256, 2
    n_pages = 2 ** 31 // (ps * hkv * dh) + 16
    cache = b.PagedCache(n_pages, ps, hkv, dh, 5, 4, dtype)
    lens = [600, 512, 700, 1000, 513]
    g = torch.Generator(device="cuda").manual_seed(3)
    free, table = list(range(n_pages - 1, n_pages - 14, -1)), [[-1] * 4 for _ in lens]
    common = [free.pop(0), free.pop(0)]
    for s, n in enumerate(lens):
        for i in range(-(-n // ps)):
            table[s][i] = common[i] if i < 2 else free.pop(0)
    for p in {x for row in table for x in row if x >= 0}:
        for pool in (cache.k, cache.v):
            pool[p] = torch.randn(hkv, ps, dh, generator=g, device="cuda").to(DT[dtype])
    cache.table.copy_(i32(table))
    cache.length.copy_(i32(lens))
    q = randn(5, 8, dh, dtype=dtype, seed=4)
    attend(cache, [0, 1, 2, 3, 4], [5], i32([512]).cuda(), q, dtype)
    shared = torch.empty(1, dtype=torch.int32, device="cuda")
    b.beagle_pages_shared(cache, [0, 1, 2, 3, 4], [5], shared)
    assert shared.tolist() == [512]


def test_two_streams_and_two_graphs_at_once():
    """Calls with workspaces of their own, on two streams and in two captured graphs, give what one alone gives."""
    cache, shared = forked([20, 5], [900, 300], list(range(25)), 16, 2, 128, "bf16", 10)
    groups, slots, sh = [20, 5], list(range(25)), i32(shared).cuda()
    qs = [randn(25, 8, 128, dtype="bf16", seed=s) for s in (1, 2)]
    want = [attend(cache, slots, groups, sh, q, "bf16") for q in qs]
    n = b.beagle_paged_attn_shared_workspace_bytes(cache, 25, 8, groups)
    ws, outs, graphs = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in qs], [torch.empty_like(q) for q in qs], []
    torch.cuda.synchronize()
    for q, w, o in zip(qs, ws, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            b.beagle_paged_attn_shared(cache, slots, groups, sh, q, o, ws=w)
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, x) for o, x in zip(outs, want))


def test_rows_behind_the_batch_stay():
    cache, shared = forked([3, 2], [128, 64], [5, 6, 7, 8, 9], 16, 2, 64, "bf16", 11)
    q = randn(9, 4, 64, dtype="bf16", seed=6)
    out, lse = torch.full_like(q, 7.0), torch.full((9, 4), 7.0, device="cuda")
    b.beagle_paged_attn_shared(cache, list(range(5)), [3, 2], i32(shared).cuda(), q[:5], out[:5], lse[:5])
    assert bool((out[5:] == 7.0).all()) and bool((lse[5:] == 7.0).all()) and not bool((out[:5] == 7.0).all())


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("bf16", 7, 1, 64), ("bf16", 4, 1, 256), ("fp32", 4, 4, 64)])
@pytest.mark.parametrize("off", [16, 32, 48, 128, 240, 256])
def test_workspace_at_any_16_byte_border(dtype, hq, hkv, dh, off):
    """A piece of a larger buffer as workspace: the same attention, and the bytes around the piece stay."""
    cache, shared = forked([20, 5, 2], [900, 300, 130], list(range(27)), 16, hkv, dh, dtype, 12)
    groups, slots, sh = [20, 5, 2], list(range(27)), i32(shared).cuda()
    q = randn(27, hq, dh, dtype=dtype, seed=8)
    ref = attend(cache, slots, groups, sh, q, dtype)
    n = b.beagle_paged_attn_shared_workspace_bytes(cache, 27, hq, groups)
    buf = torch.full((n + 1024,), 0x5a, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    b.beagle_paged_attn_shared(cache, slots, groups, sh, q, out, ws=buf[off:off + n])
    assert torch.equal(out, ref)
    assert bool((buf[:off] == 0x5a).all()) and bool((buf[off + n:] == 0x5a).all())


@pytest.mark.parametrize("dh", [64, 128])
def test_between_draft_steps_on_the_tensor_cores(dh):
    """Draft steps and shared attention one behind the other, each begun while the one before still runs, both with tensor memory: what
    each gives alone, eager and replayed from a graph."""
    from test_pages_head_gpu import GQA, WL, build, to_dev
    w = GQA.scaled(batch=20, gamma=3, ctx_max=100)
    head, _, own = build(w, ps=16)
    rng = WL.data_rng(w, 5)
    lengths, slots = [int(n) for n in WL.make_context_lengths(w, rng)], list(range(20))
    head.prefill_pages(own, slots, lengths, to_dev(WL.make_hidden(w, rng, sum(lengths)), w.dtype))
    first = to_dev(WL.make_tokens(w, rng, (20,)), w.dtype)
    cache, shared = forked([20, 5], [900, 300], list(range(25)), 16, 2, dh, "bf16", 13)
    groups, rows, sh = [20, 5], list(range(25)), i32(shared).cuda()
    qs = [randn(25, 8, dh, dtype="bf16", seed=s) for s in (1, 2, 3)]
    want = [attend(cache, rows, groups, sh, q, "bf16") for q in qs]
    keep = own.length.clone()

    def chain(draft, outs):
        keep.copy_(own.length)
        for s in range(w.gamma):
            b.beagle_draft_step_pages(head.ctx, own, slots, first if s == 0 else None, True, draft[:, s])
            if outs is not None:
                b.beagle_paged_attn_shared(cache, rows, groups, sh, qs[s], outs[s])
        b.beagle_pages_truncate(own, slots, keep)

    alone, both = (torch.zeros(20, w.gamma, dtype=torch.int32, device="cuda") for _ in range(2))
    outs = [torch.empty_like(q) for q in qs]
    chain(alone, None)
    head.rollback(slots)
    chain(both, outs)
    torch.cuda.synchronize()
    assert torch.equal(alone, both) and all(torch.equal(x, y) for x, y in zip(outs, want))
    head.rollback(slots)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(both, outs)
    for _ in range(20):
        both.zero_()
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(alone, both) and all(torch.equal(x, y) for x, y in zip(outs, want))


@pytest.mark.parametrize("dtype,hq,hkv,dh", KINDS)
@pytest.mark.parametrize("ps", [8, 64, 256])
def test_one_row_at_a_time_over_forked_slots(dtype, hq, hkv, dh, ps):
    """The attention of rows on their own over the same kind of cache, pages in several slots at once and NaN behind every length."""
    groups, prefix = [1, 5, 2, 20, 9], [70, 0, 64, 700, 1024]
    r = random.Random(ps + 1)
    cache, _ = forked(groups, prefix, [r.choice([0, 1, 5, 63, 64, 65, 130]) for _ in range(sum(groups))], ps, hkv, dh, dtype, 14)
    slots = r.sample(range(sum(groups)), sum(groups))
    q = (randn(len(slots), hq, dh, dtype=dtype, seed=9) * 2).to(DT[dtype])
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
    b.beagle_paged_attn(cache, slots, q, out, lse=lse)
    check_attn(cache, slots, q, 0, 0, dtype, out, lse)
