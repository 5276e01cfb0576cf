"""Measured cases of the operators around a paged key/value cache.

Four groups, as a serving or training program calls them:

* ``decode``  attention of one new token per sequence over the pages of its cache, whole or through a sliding window with a
  few first tokens (sinks) that stay visible;
* ``append``  roll back the rejected draft tokens, then append the new keys and values (pages are taken as needed);
* ``pages``   fork, append to the forks (copy on write), free, deep copy, compact;
* ``window``  causal attention over whole sequences with the same window and sinks, forward or forward and backward.

``run`` computes them with elementary torch operations, or, where ``own`` is true, through the package's entry points.
"""
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the tiny fp32 head right after its prompt: the smallest call, all latency
        {"name": "decode_tiny_fp32", "kind": "decode", "dtype": "fp32", "hq": 4, "hkv": 4, "dh": 64, "ps": 16, "batch": 1, "lo": 64, "hi": 64, "window": 0, "sinks": 0, "lens": 1},
        # batched serving of a Llama-3-8B shaped head, ragged contexts
        {"name": "decode_serve_b32", "kind": "decode", "dtype": "bf16", "hq": 32, "hkv": 8, "dh": 128, "ps": 64, "batch": 32, "lo": 512, "hi": 8192, "window": 0, "sinks": 0, "lens": 2},
        # long documents: 6 GB of cache, pools past 2^31 elements
        {"name": "decode_long_b16", "kind": "decode", "dtype": "bf16", "hq": 32, "hkv": 8, "dh": 128, "ps": 64, "batch": 16, "lo": 65000, "hi": 131072, "window": 0, "sinks": 0, "lens": 3},
        # a Llama-2-7B shaped head (MHA) that keeps a window and four sinks of chats of any length
        {"name": "decode_window_b64", "kind": "decode", "dtype": "bf16", "hq": 32, "hkv": 32, "dh": 128, "ps": 32, "batch": 64, "lo": 1, "hi": 6000, "window": 1024, "sinks": 4, "lens": 4},
        # one speculative step: seven rows per sequence appended after the roll-back
        {"name": "append_step_b32", "kind": "append", "dtype": "bf16", "hkv": 8, "dh": 128, "ps": 64, "batch": 32, "lo": 512, "hi": 8192, "t": 7, "lens": 5},
        # prompts of up to 8192 tokens enter the cache (padded batch)
        {"name": "append_prompt_b8", "kind": "append", "dtype": "bf16", "hkv": 8, "dh": 128, "ps": 64, "batch": 8, "lo": 0, "hi": 100, "t": 8192, "lens": 6},
        # a tiny fp32 head's four sequences forked, copied and compacted
        {"name": "pages_tiny_fp32", "kind": "pages", "dtype": "fp32", "hkv": 4, "dh": 64, "ps": 16, "batch": 4, "lo": 20, "hi": 300, "lens": 7},
        # the serving cache: sixteen sequences of up to 8192 tokens forked, copied and compacted
        {"name": "pages_serve_b16", "kind": "pages", "dtype": "bf16", "hkv": 8, "dh": 128, "ps": 64, "batch": 16, "lo": 512, "hi": 8192, "lens": 8},
        # training step of the tiny fp32 head's attention, strictly earlier keys (the first row sees nothing)
        {"name": "window_train_tiny_fp32", "kind": "window", "train": True, "dtype": "fp32", "hq": 4, "hkv": 4, "dh": 64, "batch": 3, "lo": 50, "hi": 333, "past": 0, "window": 64, "sinks": 2, "strict": True, "lens": 9},
        # training step at the block workload's size: 8 x 2048, 32 heads
        {"name": "window_train_8x2048", "kind": "window", "train": True, "dtype": "bf16", "hq": 32, "hkv": 32, "dh": 128, "batch": 8, "lo": 2048, "hi": 2048, "past": 0, "window": 512, "sinks": 4, "strict": True, "lens": 10},
        # training step on long ragged sequences with grouped heads
        {"name": "window_train_long", "kind": "window", "train": True, "dtype": "bf16", "hq": 32, "hkv": 8, "dh": 128, "batch": 2, "lo": 4001, "hi": 8191, "past": 0, "window": 2048, "sinks": 4, "strict": False, "lens": 12},
        # a prompt's next chunk over what the cache holds already
        {"name": "window_chunk_fwd", "kind": "window", "train": False, "dtype": "bf16", "hq": 32, "hkv": 8, "dh": 128, "batch": 4, "lo": 300, "hi": 1024, "past": 7000, "window": 4096, "sinks": 4, "strict": False, "lens": 13},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "append", "pages", "window", "window"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    lens = rng.randrange(1 << 30)
    hkv = rng.choice([1, 2, 4, 8, 8, 32])
    ps = rng.choice([16, 32, 64, 128])
    dh = rng.choice([64, 128])
    if kind == "decode":
        hq = hkv * rng.choice([1, 2, 4, 8] if hkv <= 4 else [1, 4] if hkv == 8 else [1])
        batch = _log_int(rng, 1, 64)
        # keys of all sequences and heads together stay below the largest listed case
        hi = _log_int(rng, 1, max(1, min(131072, 8_000_000 // (batch * hkv))))
        window = rng.choice([0, _log_int(rng, 1, 4096)])
        return {"kind": kind, "dtype": dtype, "hq": hq, "hkv": hkv, "dh": dh, "ps": ps, "batch": batch, "lo": rng.randint(1, hi), "hi": hi,
                "window": window, "sinks": rng.choice([0, 1, 4, 70]) if window else 0, "lens": lens}
    if kind == "append":
        batch = _log_int(rng, 1, 64)
        t = _log_int(rng, 1, max(1, min(8192, 500_000 // (batch * hkv))))
        hi = _log_int(rng, 1, max(1, min(8192, 1_000_000 // (batch * hkv))))
        return {"kind": kind, "dtype": dtype, "hkv": hkv, "dh": dh, "ps": ps, "batch": batch, "lo": rng.randint(0, hi), "hi": hi, "t": t, "lens": lens}
    if kind == "pages":
        batch = _log_int(rng, 1, 21)
        hi = _log_int(rng, 1, max(1, min(8192, 1_000_000 // (batch * hkv))))
        return {"kind": kind, "dtype": dtype, "hkv": hkv, "dh": dh, "ps": ps, "batch": batch, "lo": rng.randint(0, hi), "hi": hi, "lens": lens}
    hq = hkv * rng.choice([1, 2, 4, 8] if hkv <= 4 else [1, 4] if hkv == 8 else [1])
    # scores of the padded batch stay below the largest listed case; fp32 sequences are the tiny head's
    batch = _log_int(rng, 1, 8)
    most = 2 ** 20 * 512 if dtype == "bf16" else 2 ** 20 * 32
    past = rng.choice([0, 0, _log_int(rng, 1, 4000)])
    hi = _log_int(rng, 2, 8192 if dtype == "bf16" else 1500)
    while batch * hq * hi * (hi + past) > most:
        hi = max(2, hi * 3 // 4)
        past = past * 3 // 4
    return {"kind": kind, "train": rng.random() < 0.6, "dtype": dtype, "hq": hq, "hkv": hkv, "dh": dh, "batch": batch, "lo": rng.randint(2, hi), "hi": hi,
            "past": past, "window": rng.choice([0, _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)]), "sinks": rng.choice([0, 1, 4, 70]),
            "strict": rng.random() < 0.5, "lens": lens}


def _lengths(c):
    r = random.Random(c["lens"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["batch"])]


def _new_rows(c):
    r = random.Random(c["lens"] + 1)
    return [r.randint((c["t"] + 1) // 2, c["t"]) for _ in range(c["batch"])]


def _kv_lengths(c):
    r = random.Random(c["lens"] + 2)
    return [n + (r.randint(0, c["past"]) if c["past"] else 0) for n in _lengths(c)]


# ------------------------------------------------------------------------------------------------------------ preparing

def _pool(c, g, lens, max_slots, max_pages, spare):
    """A cache whose first len(lens) slots hold sequences of these lengths, their pages in a random order."""
    ps, dt = c["ps"], TYPES[c["dtype"]]
    need = [-(-n // ps) for n in lens]
    live = sum(need)
    n_pages = live + spare
    shape = (n_pages, c["hkv"], ps, c["dh"])
    k = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    v = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    ids = torch.randperm(live, generator=g, device=DEV).to(torch.int32)
    col = torch.arange(max_pages, device=DEV)[None, :]
    count = torch.tensor(need + [0] * (max_slots - len(need)), device=DEV)
    start = torch.cumsum(count, 0) - count
    at = (start[:, None] + col).clamp(max=max(live - 1, 0))
    table = torch.where(col < count[:, None], ids[at] if live else torch.full_like(at, -1, dtype=torch.int32), -1).to(torch.int32)
    length = torch.tensor(list(lens) + [0] * (max_slots - len(lens)), dtype=torch.int32, device=DEV)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[:live] = 1
    return {"k": k, "v": v, "table": table.contiguous(), "length": length, "refs": refs}


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[c["dtype"]]
    lens = _lengths(c)
    B, ps = c["batch"], c.get("ps")

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dt)

    if c["kind"] == "window":
        kv = _kv_lengths(c)
        n, m = sum(lens), sum(kv)
        s = {"case": c, "q_len": lens, "kv_len": kv, "q": normal(n, c["hq"], c["dh"], std=1.5), "k": normal(m, c["hkv"], c["dh"]), "v": normal(m, c["hkv"], c["dh"])}
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(n, c["hq"], dtype=torch.float32, device=DEV)
        if c["train"]:
            s["dout"] = normal(n, c["hq"], c["dh"])
            s.update(dq=torch.empty_like(s["q"]), dk=torch.empty_like(s["k"]), dv=torch.empty_like(s["v"]))
        return s
    slots = list(range(B))
    if c["kind"] == "decode":
        s = _pool(c, g, lens, B, -(-max(lens) // ps) + 1, 2)
        s["q"] = normal(B, c["hq"], c["dh"], std=1.5)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(B, c["hq"], dtype=torch.float32, device=DEV)
    elif c["kind"] == "append":
        new = _new_rows(c)
        s = _pool(c, g, lens, B, -(-(max(lens) + c["t"]) // ps), sum(-(-x // ps) + 1 for x in new))
        s["k_new"], s["v_new"] = normal(B, c["t"], c["hkv"], c["dh"]), normal(B, c["t"], c["hkv"], c["dh"])
        s["n_new"] = torch.tensor(new, dtype=torch.int32, device=DEV)
        s["keep"] = s["length"].clone()
        s["ok"] = torch.empty(B, dtype=torch.int32, device=DEV)
    else:
        # slots: B sequences, B forks, B copies
        live = sum(-(-n // ps) for n in lens)
        s = _pool(c, g, lens, 3 * B, -(-(max(lens) + 1) // ps), live + 2 * B)
        s["k_new"], s["v_new"] = normal(B, 1, c["hkv"], c["dh"]), normal(B, 1, c["hkv"], c["dh"])
        s["forks"], s["copies"] = list(range(B, 2 * B)), list(range(2 * B, 3 * B))
        s["ok"], s["ok2"], s["ok3"] = (torch.empty(B, dtype=torch.int32, device=DEV) for _ in range(3))
    s["case"], s["slots"] = c, slots
    if own:
        from paper_2505_24544_b200 import binding
        s["cache"] = binding.PagedCache.from_tensors(s["k"], s["v"], s["table"], s["length"], s["refs"])
    return s


# ---------------------------------------------------------------------------------------------------------- plain forms

def _softmax_parts(s):
    """exp(s - rowmax), its row sums and the row's log-sum-exp; a row without a finite score gives zeros and -inf."""
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    l = e.sum(-1, keepdim=True)
    return e, l, (m + torch.log(l))[..., 0]


def _plain_decode(s):
    c = s["case"]
    B, ps, hkv, dh = c["batch"], c["ps"], c["hkv"], c["dh"]
    G = c["hq"] // hkv
    n = s["length"][:B].long()
    width = max(1, -(-max(_lengths(c)) // ps))
    pages = s["table"][:B, :width].long().clamp(min=0)
    K = s["k"][pages].to(torch.float32).permute(0, 2, 1, 3, 4).reshape(B, hkv, width * ps, dh)
    V = s["v"][pages].to(torch.float32).permute(0, 2, 1, 3, 4).reshape(B, hkv, width * ps, dh)
    q = s["q"].to(torch.float32).view(B, hkv, G, dh)
    j = torch.arange(width * ps, device=DEV)[None, :]
    seen = j < n[:, None]
    if c["window"] > 0:
        seen &= (j >= n[:, None] - c["window"]) | (j < c["sinks"])
    sc = torch.matmul(q, K.transpose(-1, -2)) * dh ** -0.5
    sc = sc.masked_fill(~seen[:, None, None, :], float("-inf"))
    e, l, lse = _softmax_parts(sc)
    o = torch.matmul(e, V) / torch.where(l > 0, l, torch.ones_like(l))
    return [o.reshape(B, c["hq"], dh).to(s["q"].dtype), lse.reshape(B, c["hq"])]


def _plain_truncate(s, rows, keep):
    """Slots cut to `keep` positions (None: nothing); the pages behind are given back."""
    ps = s["k"].shape[2]
    rows = torch.tensor(rows, device=DEV)
    n = s["length"][rows]
    keep = torch.zeros_like(n) if keep is None else torch.minimum(keep.clamp(min=0), n)
    t = s["table"][rows]
    col = torch.arange(t.shape[1], device=DEV)[None, :]
    drop = (col >= ((keep + ps - 1) // ps)[:, None]) & (t >= 0)
    s["refs"].index_add_(0, t.clamp(min=0).reshape(-1).long(), -drop.reshape(-1).to(torch.int32))
    s["table"][rows] = torch.where(drop, -1, t)
    s["length"][rows] = keep


def _free_ids(s):
    """All page ids, the free ones first, lowest first; and how many are free."""
    free = s["refs"] == 0
    ids = torch.arange(free.numel(), device=DEV)
    return torch.sort(torch.where(free, ids, ids + free.numel())).values % free.numel(), free.sum()


def _plain_append(s, rows, k_new, v_new, n_new):
    ps = s["k"].shape[2]
    B, T = k_new.shape[:2]
    rows = torch.tensor(rows, device=DEV)
    t, L = s["table"][rows], s["length"][rows].long()
    width = t.shape[1]
    n = torch.full_like(L, T) if n_new is None else n_new.long().clamp(0, T)
    have, want = (L + ps - 1) // ps, (L + n + ps - 1) // ps
    tail = t.gather(1, (L // ps).clamp(max=width - 1)[:, None])[:, 0].long().clamp(min=0)
    shared = ((L % ps != 0) & (s["refs"][tail] > 1) & (n > 0)).long()
    fits = L + n <= width * ps
    need = (want - have + shared) * fits
    ids, n_free = _free_ids(s)
    ok = fits & ((need == 0) | (torch.cumsum(need, 0) <= n_free))
    need, n, shared = need * ok, n * ok, shared * ok
    start = torch.cumsum(need, 0) - need
    # a shared, partly filled last page is copied before it is written
    at = torch.nonzero(shared)[:, 0]
    if at.numel():
        old, new, r = tail[at], ids[start[at]], (L % ps)[at]
        part = (torch.arange(ps, device=DEV)[None, :] < r[:, None])[:, None, :, None]
        for pool in (s["k"], s["v"]):
            pool[new] = torch.where(part, pool[old], pool[new])
        s["refs"].index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
        s["refs"][new] = 1
        t[at, (L // ps)[at]] = new.to(torch.int32)
    col = torch.arange(width, device=DEV)[None, :]
    fresh = (col >= have[:, None]) & (col < (have + need - shared)[:, None])
    page = ids[(start + shared)[:, None].add(col - have[:, None]).clamp(0, ids.numel() - 1)]
    s["refs"].index_add_(0, page.reshape(-1), fresh.reshape(-1).to(torch.int32))
    t = torch.where(fresh, page.to(torch.int32), t)
    s["table"][rows] = t
    b, i = torch.nonzero(torch.arange(T, device=DEV)[None, :] < n[:, None], as_tuple=True)
    pos = L[b] + i
    page = t[b, pos // ps].long()
    s["k"][page, :, pos % ps] = k_new[b, i]
    s["v"][page, :, pos % ps] = v_new[b, i]
    s["length"][rows] = (L + n).to(torch.int32)
    return ok.to(torch.int32)


def _plain_fork(s, src, dst):
    _plain_truncate(s, dst, None)
    src, dst = torch.tensor(src, device=DEV), torch.tensor(dst, device=DEV)
    t = s["table"][src]
    s["refs"].index_add_(0, t.clamp(min=0).reshape(-1).long(), (t >= 0).reshape(-1).to(torch.int32))
    s["table"][dst] = t
    s["length"][dst] = s["length"][src]


def _plain_copy(s, src, dst):
    _plain_truncate(s, dst, None)
    ps = s["k"].shape[2]
    src, dst = torch.tensor(src, device=DEV), torch.tensor(dst, device=DEV)
    t, L = s["table"][src], s["length"][src].long()
    need = (L + ps - 1) // ps
    ids, n_free = _free_ids(s)
    ok = (need == 0) | (torch.cumsum(need, 0) <= n_free)
    need = need * ok
    start = torch.cumsum(need, 0) - need
    col = torch.arange(t.shape[1], device=DEV)[None, :]
    b, i = torch.nonzero(col < need[:, None], as_tuple=True)
    new, old = ids[start[b] + i], t[b, i].long()
    s["k"][new] = s["k"][old]
    s["v"][new] = s["v"][old]
    s["refs"][new] = 1
    s["table"][dst[b], i] = new.to(torch.int32)
    s["length"][dst] = (L * ok).to(torch.int32)
    return ok.to(torch.int32)


def _plain_compact(s):
    live = s["refs"] > 0
    n = live.sum()
    ids = torch.arange(live.numel(), device=DEV)
    old, new = torch.nonzero(live & (ids >= n))[:, 0], torch.nonzero(~live & (ids < n))[:, 0]
    s["k"][new] = s["k"][old]
    s["v"][new] = s["v"][old]
    s["refs"][new] = s["refs"][old]
    s["refs"][old] = 0
    to = ids.to(torch.int32)
    to[old] = new.to(torch.int32)
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].long().clamp(min=0)], s["table"]))


def _pad_index(lens):
    """[B, longest] row numbers of packed sequences, and which of them exist."""
    n = torch.tensor(lens, device=DEV)
    i = torch.arange(max(lens), device=DEV)[None, :]
    return ((torch.cumsum(n, 0) - n)[:, None] + i).clamp(max=sum(lens) - 1), i < n[:, None]


def _plain_window(s):
    c = s["case"]
    hq, hkv, dh, B = c["hq"], c["hkv"], c["dh"], c["batch"]
    G = hq // hkv
    qi, qv = _pad_index(s["q_len"])
    ki, kv = _pad_index(s["kv_len"])

    def rows_of(x, idx, heads):          # packed rows -> [B, heads, positions, dh] in 32 bits
        return x[idx].to(torch.float32).view(B, idx.shape[1], heads, dh).transpose(1, 2)

    def grouped(x):                      # [B, hq, n, dh] -> [B, hkv, G * n, dh]: the heads that share keys lie side by side
        return x.reshape(B, hkv, G * x.shape[2], dh)

    nq, nk = qi.shape[1], ki.shape[1]
    q, k, v = grouped(rows_of(s["q"], qi, hq)), rows_of(s["k"], ki, hkv), rows_of(s["v"], ki, hkv)
    last = torch.arange(nq, device=DEV)[None, :] + (torch.tensor(s["kv_len"], device=DEV) - torch.tensor(s["q_len"], device=DEV))[:, None] - int(c["strict"])
    j = torch.arange(nk, device=DEV)
    seen = (j <= last[..., None]) & kv[:, None, :]
    if c["window"] > 0:
        seen &= (j > last[..., None] - c["window"]) | (j < c["sinks"])
    seen &= qv[..., None]
    hidden = ~seen[:, None].expand(B, G, nq, nk).reshape(B, 1, G * nq, nk)
    scale = dh ** -0.5
    e, l, lse = _softmax_parts((torch.matmul(q, k.transpose(-1, -2)) * scale).masked_fill_(hidden, float("-inf")))
    p = e.div_(torch.where(l > 0, l, torch.ones_like(l)))
    o = torch.matmul(p, v)

    def packed(x, idx, exists, heads):   # [B, heads, n, ...] -> packed rows
        return x.reshape(B, heads, idx.shape[1], -1).transpose(1, 2)[exists]

    dt = s["q"].dtype
    out = [packed(o, qi, qv, hq).to(dt), packed(lse, qi, qv, hq)[..., 0]]
    if c["train"]:
        do = grouped(rows_of(s["dout"], qi, hq) * qv[:, None, :, None])
        dv = torch.matmul(p.transpose(-1, -2), do)
        dp = torch.matmul(do, v.transpose(-1, -2))
        ds = dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p)
        dq = torch.matmul(ds, k) * scale
        dk = torch.matmul(ds.transpose(-1, -2), q) * scale
        out += [packed(dq, qi, qv, hq).to(dt), packed(dk, ki, kv, hkv).to(dt), packed(dv, ki, kv, hkv).to(dt)]
    return out


# ------------------------------------------------------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    if own:
        from paper_2505_24544_b200 import binding as b
    if c["kind"] == "decode":
        if not own:
            return _plain_decode(s)
        b.beagle_paged_attn(s["cache"], s["slots"], s["q"], s["out"], s["lse"], window=c["window"], sinks=c["sinks"])
        return [s["out"], s["lse"]]
    if c["kind"] == "append":
        if own:
            b.beagle_pages_truncate(s["cache"], s["slots"], s["keep"])
            b.beagle_pages_append(s["cache"], s["slots"], s["k_new"], s["v_new"], s["n_new"], s["ok"])
            ok = s["ok"]
        else:
            _plain_truncate(s, s["slots"], s["keep"])
            ok = _plain_append(s, s["slots"], s["k_new"], s["v_new"], s["n_new"])
        return [s["k"], s["v"], s["table"], s["length"], s["refs"], ok]
    if c["kind"] == "pages":
        S, F, C = s["slots"], s["forks"], s["copies"]
        if own:
            p = s["cache"]
            b.beagle_pages_fork(p, S, F)
            b.beagle_pages_append(p, F, s["k_new"], s["v_new"], None, s["ok"])
            b.beagle_pages_truncate(p, F)
            b.beagle_pages_copy(p, S, C, s["ok2"])
            b.beagle_pages_truncate(p, S)
            b.beagle_pages_compact(p)
            b.beagle_pages_copy(p, C, S, s["ok3"])
            b.beagle_pages_truncate(p, C)
            b.beagle_pages_compact(p)
            ok = [s["ok"], s["ok2"], s["ok3"]]
        else:
            _plain_fork(s, S, F)
            ok = [_plain_append(s, F, s["k_new"], s["v_new"], None)]
            _plain_truncate(s, F, None)
            ok.append(_plain_copy(s, S, C))
            _plain_truncate(s, S, None)
            _plain_compact(s)
            ok.append(_plain_copy(s, C, S))
            _plain_truncate(s, C, None)
            _plain_compact(s)
        return [s["k"], s["v"], s["table"], s["length"], s["refs"], *ok]
    if not own:
        return _plain_window(s)
    b.beagle_window_attn_forward(s["q"], s["k"], s["v"], s["q_len"], s["kv_len"], s["out"], s["lse"], window=c["window"], sinks=c["sinks"], strict=c["strict"])
    if not c["train"]:
        return [s["out"], s["lse"]]
    b.beagle_window_attn_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["q_len"], s["kv_len"], s["dq"], s["dk"], s["dv"],
                                  window=c["window"], sinks=c["sinks"], strict=c["strict"])
    return [s["out"], s["lse"], s["dq"], s["dk"], s["dv"]]


def _pairs(n_q, n_kv, c):
    """Visible (query, key) pairs of one sequence, and how many of its keys anyone sees."""
    pairs, w, k0 = 0, c["window"], c["sinks"]
    first = n_kv - n_q - int(c["strict"])
    for last in range(max(first, 0), first + n_q):
        n = last + 1
        pairs += n if w <= 0 else min(n, w) + min(k0, max(0, n - w))
    low = max(0, max(first, 0) - w + 1) if w > 0 else 0
    return pairs, max(0, first + n_q - low) + min(k0, low)


def work(case):
    c = dict(case)
    e = 2 if c["dtype"] == "bf16" else 4
    lens, dh = _lengths(c), c["dh"]
    if c["kind"] == "decode":
        w, k0 = c["window"], c["sinks"]
        seen = sum(n if w <= 0 else min(n, w) + min(k0, max(0, n - w)) for n in lens)
        return {"bytes": 2 * seen * c["hkv"] * dh * e + c["batch"] * c["hq"] * (2 * dh * e + 4), "flops": 4 * seen * c["hq"] * dh}
    if c["kind"] == "append":
        return {"bytes": 2 * 2 * sum(_new_rows(c)) * c["hkv"] * dh * e + 32 * c["batch"], "flops": 0}
    if c["kind"] == "pages":
        # four whole copies of the sequences' pages (two deep copies, two compactions), each read and written
        pages = sum(-(-n // c["ps"]) for n in lens)
        return {"bytes": 4 * 2 * 2 * pages * c["hkv"] * c["ps"] * dh * e + 100 * c["batch"], "flops": 0}
    kv = _kv_lengths(c)
    got = [_pairs(a, b, c) for a, b in zip(lens, kv)]
    pairs, keys = sum(x[0] for x in got), sum(x[1] for x in got)
    nq = sum(lens)
    flops = 4 * pairs * c["hq"] * dh
    bytes_ = 2 * nq * c["hq"] * dh * e + 2 * keys * c["hkv"] * dh * e + 4 * nq * c["hq"]
    if c["train"]:
        flops += 10 * pairs * c["hq"] * dh
        bytes_ += 4 * nq * c["hq"] * dh * e + 4 * nq * c["hq"] + 2 * keys * c["hkv"] * dh * e + 2 * sum(kv) * c["hkv"] * dh * e
    return {"bytes": bytes_, "flops": flops}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_rows(q, k, v, seen, scale):
    """softmax over the seen keys, one head: q [n, dh], k and v [m, dh], seen [n, m]."""
    s = (q @ k.T * scale).masked_fill(~seen, -torch.inf)
    lse = torch.logsumexp(s, -1)
    some = seen.any(-1)
    p = torch.exp(s - torch.where(some, lse, 0.0)[:, None])
    return p @ v, lse


def _exact_decode(s):
    c = s["case"]
    G, ps, dh = c["hq"] // c["hkv"], c["ps"], c["dh"]
    out, lse = s["q"].double() * 0, torch.empty_like(s["lse"], dtype=torch.float64)
    for b, n in enumerate(_lengths(c)):
        pages = s["table"][b, : -(-n // ps)].long()
        j = torch.arange(n, device=DEV)
        seen = (j >= n - c["window"]) | (j < c["sinks"]) if c["window"] > 0 else j >= 0
        for h in range(c["hkv"]):
            k, v = (x[pages, h].reshape(-1, dh)[:n].double() for x in (s["k"], s["v"]))
            out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = _exact_rows(s["q"][b, h * G:(h + 1) * G].double(), k, v, seen.expand(G, n), dh ** -0.5)
    return [out, lse]


def _exact_window(s):
    c = s["case"]
    G, dh = c["hq"] // c["hkv"], c["dh"]
    res = [torch.zeros_like(s["q"], dtype=torch.float64), torch.zeros_like(s["lse"], dtype=torch.float64)]
    if c["train"]:
        res += [torch.zeros_like(s[x], dtype=torch.float64) for x in ("q", "k", "v")]
    a = b = 0
    for n, m in zip(s["q_len"], s["kv_len"]):
        last = torch.arange(n, device=DEV)[:, None] + (m - n - int(c["strict"]))
        j = torch.arange(m, device=DEV)[None, :]
        seen = j <= last
        if c["window"] > 0:
            seen = seen & ((last - j < c["window"]) | (j < c["sinks"]))
        for h in range(c["hq"]):
            q, k, v = (x.double().detach().requires_grad_(c["train"]) for x in (s["q"][a:a + n, h], s["k"][b:b + m, h // G], s["v"][b:b + m, h // G]))
            with torch.set_grad_enabled(c["train"]):
                o, lse = _exact_rows(q, k, v, seen, dh ** -0.5)
            res[0][a:a + n, h], res[1][a:a + n, h] = o.detach(), lse.detach()
            if c["train"]:
                # rows that see nothing have no gradient: their -inf stays out of the graph
                dq, dk, dv = torch.autograd.grad(_exact_rows(q, k, v, seen | ~seen.any(-1, keepdim=True), dh ** -0.5)[0], (q, k, v),
                                                 s["dout"][a:a + n, h].double() * seen.any(-1, keepdim=True))
                res[2][a:a + n, h] = dq
                res[3][b:b + m, h // G] += dk
                res[4][b:b + m, h // G] += dv
        a, b = a + n, b + m
    return res


class _Book:
    """The cache's bookkeeping and contents, one step after the other."""

    def __init__(self, s):
        self.k, self.v, self.ps = s["k"].double(), s["v"].double(), s["k"].shape[2]
        self.length, self.refs = s["length"].tolist(), s["refs"].tolist()
        self.width = s["table"].shape[1]
        self.pages = [[p for p in row if p >= 0] for row in s["table"].tolist()]

    def take(self, count):
        return [p for p, r in enumerate(self.refs) if r == 0][:count]

    def truncate(self, rows, keep):
        for r, n in zip(rows, keep):
            self.length[r] = min(n, self.length[r])
            have = -(-self.length[r] // self.ps)
            for p in self.pages[r][have:]:
                self.refs[p] -= 1
            self.pages[r] = self.pages[r][:have]

    def append(self, rows, k_new, v_new, counts):
        before, done = list(self.refs), []
        free = [p for p, r in enumerate(before) if r == 0]
        for b, (r, n) in enumerate(zip(rows, counts)):
            L = self.length[r]
            cow = L % self.ps != 0 and n > 0 and before[self.pages[r][-1]] > 1
            need = -(-(L + n) // self.ps) - -(-L // self.ps) + cow
            done.append(int(L + n <= self.width * self.ps and (need == 0 or need <= len(free))))
            if not done[-1]:
                if L + n <= self.width * self.ps:
                    free = []
                continue
            mine, free = free[:need], free[need:]
            for p in mine:
                self.refs[p] = 1
            if cow:
                old, new = self.pages[r][-1], mine.pop(0)
                self.k[new, :, : L % self.ps], self.v[new, :, : L % self.ps] = self.k[old, :, : L % self.ps], self.v[old, :, : L % self.ps]
                self.refs[old] -= 1
                self.pages[r][-1] = new
            self.pages[r] += mine
            if n:
                pos = torch.arange(L, L + n, device=DEV)
                page = torch.tensor(self.pages[r], device=DEV)[pos // self.ps]
                self.k[page, :, pos % self.ps], self.v[page, :, pos % self.ps] = k_new[b, :n].double(), v_new[b, :n].double()
            self.length[r] = L + n
        return done

    def copy(self, src, dst):
        self.truncate(dst, [0] * len(dst))
        free, done = self.take(len(self.refs)), []
        for a, b in zip(src, dst):
            need = len(self.pages[a])
            done.append(int(need <= len(free)))
            if not done[-1]:
                free = []
                continue
            mine, free = free[:need], free[need:]
            for p in mine:
                self.refs[p] = 1
            to, of = torch.tensor(mine, dtype=torch.long, device=DEV), torch.tensor(self.pages[a], dtype=torch.long, device=DEV)
            self.k[to], self.v[to] = self.k[of], self.v[of]
            self.pages[b], self.length[b] = mine, self.length[a]
        return done

    def fork(self, src, dst):
        self.truncate(dst, [0] * len(dst))
        for a, b in zip(src, dst):
            self.pages[b], self.length[b] = list(self.pages[a]), self.length[a]
            for p in self.pages[a]:
                self.refs[p] += 1

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        move = dict(zip([p for p, r in enumerate(self.refs) if r > 0 and p >= n], [p for p, r in enumerate(self.refs) if r == 0 and p < n]))
        if move:
            of, to = torch.tensor(list(move), device=DEV), torch.tensor(list(move.values()), device=DEV)
            self.k[to], self.v[to] = self.k[of], self.v[of]
        for a, b in move.items():
            self.refs[a], self.refs[b] = 0, self.refs[a]
        self.pages = [[move.get(p, p) for p in row] for row in self.pages]

    def outputs(self, ok):
        table = [row + [-1] * (self.width - len(row)) for row in self.pages]
        return [self.k, self.v, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, self.length, self.refs, *ok))]


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "decode":
        return _exact_decode(s)
    if c["kind"] == "window":
        return _exact_window(s)
    book = _Book(s)
    if c["kind"] == "append":
        book.truncate(s["slots"], s["keep"].tolist())
        return book.outputs([book.append(s["slots"], s["k_new"], s["v_new"], _new_rows(c))])
    S, F, C = s["slots"], s["forks"], s["copies"]
    none = [0] * len(S)
    book.fork(S, F)
    ok = [book.append(F, s["k_new"], s["v_new"], [1] * len(F))]
    book.truncate(F, none)
    ok.append(book.copy(S, C))
    book.truncate(S, none)
    book.compact()
    ok.append(book.copy(C, S))
    book.truncate(C, none)
    book.compact()
    return book.outputs(ok)
