"""Measured cases of the operators that decode many samples of one prompt over rotary keys.

Four groups, as a serving or training program calls them:

* ``rotary``  rotation of queries and keys by their positions, for whole rows, and its transpose for their gradients;
* ``append``  roll back the rejected draft tokens, then append new keys and values to the paged cache, the keys (and the queries that
  go with them) rotated on the way;
* ``shared``  attention of one new token per sequence where groups of sequences share a long prefix, which is read once;
* ``sample``  one token per row of logits: temperature, top-k, top-p, min-p and a given uniform number.

``run`` computes them with elementary torch operations, or, where ``own`` is true, through the package's entry points.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    wide = {"dtype": "bf16", "dh": 128, "rot": 128, "inter": False, "theta": 500000.0, "scaling": "bands", "factor": 8.0, "original": 8192}
    tiny = {"dtype": "fp32", "dh": 64, "rot": 64, "inter": False, "theta": 10000.0, "scaling": "none", "factor": 1.0, "original": 0}
    return [
        # queries and keys of one step of batched serving, at positions of long contexts: latency
        {"name": "rotary_step_b32", "kind": "rotary", **wide, "hq": 32, "hk": 8, "rows": 32, "span": 131072, "packed": False, "train": False, "lens": 1},
        # a chunk of prompts, a quarter of the head rotated in adjacent pairs, context stretched by a ramp over the frequencies
        {"name": "rotary_prompt_part", "kind": "rotary", **wide, "rot": 32, "inter": True, "scaling": "ramp", "factor": 4.0, "hq": 32, "hk": 8,
         "rows": 8191, "span": 40000, "packed": False, "train": False, "lens": 2},
        # training step at the block workload's size, 8 x 2048 positions, forward and backward
        {"name": "rotary_train_8x2048", "kind": "rotary", **wide, "theta": 10000.0, "scaling": "none", "factor": 1.0, "hq": 32, "hk": 32, "rows": 16384,
         "span": 2048, "packed": True, "train": True, "lens": 3},
        # one token of the tiny fp32 head enters its cache: the smallest call
        {"name": "append_tiny_fp32", "kind": "append", **tiny, "hq": 4, "hkv": 4, "ps": 16, "batch": 1, "lo": 64, "hi": 64, "t": 1, "after": 0, "lens": 4},
        # one speculative step of batched serving: seven keys, values and queries per sequence
        {"name": "append_step_b32", "kind": "append", **wide, "hq": 32, "hkv": 8, "ps": 64, "batch": 32, "lo": 512, "hi": 8192, "t": 7, "after": 1, "lens": 5},
        # prompts of up to 8192 tokens enter the cache (padded batch)
        {"name": "append_prompt_b8", "kind": "append", **wide, "hq": 0, "hkv": 8, "ps": 64, "batch": 8, "lo": 0, "hi": 100, "t": 8192, "after": 0, "lens": 6},
        # four samples of a short prompt of the tiny fp32 head
        {"name": "shared_tiny_fp32", "kind": "shared", "dtype": "fp32", "hq": 4, "hkv": 4, "dh": 64, "ps": 16, "groups": 1, "batch": 4, "plo": 64, "phi": 64,
         "slo": 1, "shi": 40, "lens": 7},
        # 32 samples of one prompt of 8192 tokens, some hundred tokens in
        {"name": "shared_b32_8k", "kind": "shared", "dtype": "bf16", "hq": 32, "hkv": 8, "dh": 128, "ps": 64, "groups": 1, "batch": 32, "plo": 8192, "phi": 8192,
         "slo": 1, "shi": 512, "lens": 8},
        # four prompts with sixteen samples each, heads not grouped
        {"name": "shared_4x16_mha", "kind": "shared", "dtype": "bf16", "hq": 32, "hkv": 32, "dh": 128, "ps": 32, "groups": 4, "batch": 64, "plo": 1000, "phi": 4000,
         "slo": 0, "shi": 300, "lens": 9},
        # 64 questions about one long document
        {"name": "shared_b64_64k", "kind": "shared", "dtype": "bf16", "hq": 32, "hkv": 8, "dh": 128, "ps": 64, "groups": 1, "batch": 64, "plo": 65536, "phi": 65536,
         "slo": 100, "shi": 2048, "lens": 10},
        # one row of a Llama-2-7B shaped head, the 50 best of them
        {"name": "sample_b1_topk", "kind": "sample", "dtype": "fp32", "rows": 1, "v": 32000, "std": 3.0, "params": "k", "lens": 11},
        # every position of a speculative step, 64 sequences of seven, each with the filters of its request
        {"name": "sample_b448_mixed", "kind": "sample", "dtype": "bf16", "rows": 448, "v": 128256, "std": 3.0, "params": "mixed", "lens": 12},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _draw_rotary(rng, dh):
    part = rng.choice([dh, dh, dh // 2, dh // 4, 2 * rng.randint(1, dh // 2)])
    scaling = rng.choice(["none", "linear", "base", "bands", "ramp"])
    return {"dh": dh, "rot": part, "inter": rng.random() < 0.5, "theta": rng.choice([10000.0, 500000.0, 1000000.0]),
            "scaling": scaling if part > 2 or scaling != "base" else "none", "factor": 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
            "original": rng.choice([2048, 4096, 8192])}


def draw(rng):
    kind = rng.choice(["rotary", "append", "shared", "shared", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    lens = rng.randrange(1 << 30)
    hkv = rng.choice([1, 2, 4, 8, 8, 32])
    dh = rng.choice([64, 128])
    ps = rng.choice([16, 32, 64, 128])
    hq = hkv * rng.choice([1, 2, 4, 8] if hkv <= 4 else [1, 4] if hkv == 8 else [1])
    if kind == "rotary":
        train = rng.random() < 0.5
        rows = _log_int(rng, 1, max(1, min(16384, 500_000 // (hq + hkv))))
        return {"kind": kind, "dtype": dtype, **_draw_rotary(rng, dh), "hq": hq, "hk": hkv, "rows": rows, "span": _log_int(rng, 1, 1_000_000),
                "packed": rng.random() < 0.5, "train": train, "lens": lens}
    if kind == "append":
        batch = _log_int(rng, 1, 64)
        t = _log_int(rng, 1, max(1, min(8192, 300_000 // (batch * hkv))))
        hi = _log_int(rng, 1, max(1, min(8192, 1_000_000 // (batch * hkv))))
        with_q = batch * t * hq <= 500_000 and rng.random() < 0.6
        return {"kind": kind, "dtype": dtype, **_draw_rotary(rng, dh), "hq": hq if with_q else 0, "hkv": hkv, "ps": ps, "batch": batch, "lo": rng.randint(0, hi),
                "hi": hi, "t": t, "after": rng.choice([0, 1]), "lens": lens}
    if kind == "shared":
        batch = _log_int(rng, 1, 64)
        groups = min(batch, rng.choice([1, 1, 2, 4, 7]))
        # keys of all sequences and heads, the shared ones for every row that reads them, stay below the largest listed case
        phi = _log_int(rng, 1, max(1, min(65536, 30_000_000 // (batch * hq))))
        shi = _log_int(rng, 1, max(1, min(4096, 1_000_000 // (batch * hkv))))
        return {"kind": kind, "dtype": dtype, "hq": hq, "hkv": hkv, "dh": dh, "ps": ps, "groups": groups, "batch": batch, "plo": rng.randint(1, phi), "phi": phi,
                "slo": rng.randint(0, shi), "shi": shi, "lens": lens}
    rows = _log_int(rng, 1, 448)
    v = _log_int(rng, 1000, min(131072, 20_000_000 // rows))
    return {"kind": kind, "dtype": dtype, "rows": rows, "v": v, "std": rng.choice([1.0, 3.0, 3.0, 6.0]), "params": rng.choice(["temp", "k", "p", "minp", "mixed", "mixed"]), "lens": lens}


def _lengths(c):
    r = random.Random(c["lens"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["batch"])]


def _new_rows(c):
    r = random.Random(c["lens"] + 1)
    return [r.randint((c["t"] + 1) // 2, c["t"]) for _ in range(c["batch"])]


def _groups(c):
    """Rows of every group, its prefix, and the rows' own positions behind it."""
    r = random.Random(c["lens"])
    sizes = [c["batch"] // c["groups"] + (i < c["batch"] % c["groups"]) for i in range(c["groups"])]
    return sizes, [r.randint(c["plo"], c["phi"]) for _ in sizes], [r.randint(c["slo"], c["shi"]) for _ in range(c["batch"])]


# ------------------------------------------------------------------------------------------------------------ preparing

def _table(need, max_slots, width, first_id, g):
    """Pages of sequences that need so many each, in a random order from id `first_id` on; [max_slots, width], -1 = none."""
    live = sum(need)
    ids = torch.randperm(live, generator=g, device=DEV) + first_id
    col = torch.arange(width, device=DEV)[None, :]
    count = torch.tensor(need + [0] * (max_slots - len(need)), device=DEV)
    at = ((torch.cumsum(count, 0) - count)[:, None] + col).clamp(max=max(live - 1, 0))
    return torch.where(col < count[:, None], ids[at] if live else torch.full_like(at, -1), -1).to(torch.int32)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(TYPES[c["dtype"]])

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    s = {"case": c}
    if c["kind"] == "rotary":
        n = c["rows"]
        s["q"], s["k"] = normal(n, c["hq"], c["dh"], std=1.5), normal(n, c["hk"], c["dh"])
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["pos"] = torch.arange(n, device=DEV, dtype=torch.int32) % c["span"] if c["packed"] else \
            torch.randint(0, c["span"], (n,), generator=g, device=DEV, dtype=torch.int32)
        if c["train"]:
            s["gq"], s["gk"] = normal(n, c["hq"], c["dh"]), normal(n, c["hk"], c["dh"])
            s["dq"], s["dk"] = torch.empty_like(s["gq"]), torch.empty_like(s["gk"])
    elif c["kind"] == "append":
        lens, new, B, ps = _lengths(c), _new_rows(c), c["batch"], c["ps"]
        width = -(-(max(lens) + c["t"]) // ps)
        need = [-(-n // ps) for n in lens]
        n_pages = sum(need) + sum(-(-x // ps) + 1 for x in new)
        s["k"], s["v"] = normal(n_pages, c["hkv"], ps, c["dh"]), normal(n_pages, c["hkv"], ps, c["dh"])
        s["table"] = _table(need, B, width, 0, g)
        s["length"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["refs"] = (torch.arange(n_pages, device=DEV) < sum(need)).to(torch.int32)
        s["k_new"], s["v_new"] = normal(B, c["t"], c["hkv"], c["dh"]), normal(B, c["t"], c["hkv"], c["dh"])
        s["n_new"] = torch.tensor(new, dtype=torch.int32, device=DEV)
        s["keep"], s["ok"] = s["length"].clone(), torch.empty(B, dtype=torch.int32, device=DEV)
        s["q"] = s["q_out"] = None
        if c["hq"]:
            s["q"] = normal(B, c["t"], c["hq"], c["dh"], std=1.5)
            s["q_out"] = torch.zeros_like(s["q"])
        s["slots"] = list(range(B))
    elif c["kind"] == "shared":
        sizes, pre, suf = _groups(c)
        B, ps = c["batch"], c["ps"]
        whole = [p // ps for p in pre]                          # pages that the group's rows have in common
        group_of = [i for i, n in enumerate(sizes) for _ in range(n)]
        lens = [pre[group_of[b]] + suf[b] for b in range(B)]
        own_pages = [-(-lens[b] // ps) - whole[group_of[b]] for b in range(B)]
        width = -(-max(lens) // ps) + 1
        n_pages = sum(whole) + sum(own_pages) + 1
        s["k"], s["v"] = normal(n_pages, c["hkv"], ps, c["dh"]), normal(n_pages, c["hkv"], ps, c["dh"])
        common = _table(whole, len(sizes), width, 0, g)
        mine = _table(own_pages, B, width, sum(whole), g)
        gi = torch.tensor(group_of, device=DEV)
        col = torch.arange(width, device=DEV)[None, :] - torch.tensor(whole, device=DEV)[gi][:, None]
        s["table"] = torch.where(col < 0, common[gi], mine.gather(1, col.clamp(min=0))).to(torch.int32).contiguous()
        s["length"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        at = s["table"].clamp(min=0).reshape(-1).long()
        s["refs"].index_add_(0, at, (s["table"] >= 0).reshape(-1).to(torch.int32))
        s["shared"] = torch.tensor([w * ps for w in whole], dtype=torch.int32, device=DEV)
        s["sizes"], s["whole"], s["slots"] = sizes, whole, list(range(B))
        s["q"] = normal(B, c["hq"], c["dh"], std=1.5)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(B, c["hq"], dtype=torch.float32, device=DEV)
    else:
        n, v, r = c["rows"], c["v"], random.Random(c["lens"])
        s["logits"] = normal(n, v, std=c["std"])
        s["u"] = uniform(n)
        some = {"temp": ("temp",), "k": ("temp", "k"), "p": ("temp", "p"), "minp": ("temp", "minp"), "mixed": ("temp", "k", "p", "minp")}[c["params"]]
        # requests as they come: some greedy, some with one filter, some with several
        mixed = c["params"] == "mixed"
        temp = [0.0 if mixed and r.random() < 0.1 else r.uniform(0.5, 1.3) for _ in range(n)]
        k = [0 if mixed and r.random() < 0.4 else 50 if not mixed else r.choice([1, 20, 50, 400, 3000]) for _ in range(n)]
        p = [1.0 if mixed and r.random() < 0.4 else r.uniform(0.5, 0.99) for _ in range(n)]
        mp = [0.0 if mixed and r.random() < 0.6 else r.uniform(0.001, 0.2) for _ in range(n)]
        s["temp"] = torch.tensor(temp, device=DEV)
        s["top_k"] = torch.tensor(k, dtype=torch.int32, device=DEV) if "k" in some else None
        s["top_p"] = torch.tensor(p, device=DEV) if "p" in some else None
        s["min_p"] = torch.tensor(mp, device=DEV) if "minp" in some else None
        s["tokens"], s["logp"] = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)
    if own:
        from paper_2505_24544_b200 import binding
        if c["kind"] in ("append", "shared"):
            s["cache"] = binding.PagedCache.from_tensors(s["k"], s["v"], s["table"], s["length"], s["refs"])
        if c["kind"] in ("rotary", "append"):
            s["rot"] = binding.Rotary(c["dh"], c["rot"], theta=c["theta"], interleaved=c["inter"], scaling=c["scaling"], factor=c["factor"], original=c["original"])
    return s


# ---------------------------------------------------------------------------------------------------------- plain forms

LOW, HIGH = {"bands": 1.0, "ramp": 1.0}, {"bands": 4.0, "ramp": 32.0}       # turns inside the original context


def _frequencies(c):
    """Radians per position of every pair, and the factor of cosine and sine."""
    r, theta, kind, factor = c["rot"], c["theta"], c["scaling"], c["factor"]
    if kind == "base":
        theta = theta * factor ** (r / (r - 2))
    f = [theta ** (-2 * i / r) for i in range(r // 2)]
    if kind == "linear":
        return [x / factor for x in f], 1.0
    if kind == "bands":
        out = []
        for x in f:
            turns = c["original"] * x / (2 * math.pi)
            t = min(max((turns - LOW[kind]) / (HIGH[kind] - LOW[kind]), 0.0), 1.0)
            out.append(x * (t + (1 - t) / factor))
        return out, 1.0
    if kind == "ramp":
        at = [r * math.log(c["original"] / (2 * math.pi * n)) / (2 * math.log(theta)) for n in (HIGH[kind], LOW[kind])]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        t = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(r // 2)]
        return [x * (1 - y + y / factor) for x, y in zip(f, t)], 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _plain_rotate(c, x, pos, inverse=False):
    """x [..., heads, dh] at positions pos [...]."""
    f, m = _frequencies(c)
    angle = pos.to(torch.float64)[..., None] * torch.tensor(f, dtype=torch.float64, device=DEV)
    cos, sin = (torch.cos(angle) * m).to(torch.float32)[..., None, :], (torch.sin(angle) * (-m if inverse else m)).to(torch.float32)[..., None, :]
    y = x.to(torch.float32).clone()
    r = c["rot"]
    first = slice(0, r, 2) if c["inter"] else slice(0, r // 2)
    second = slice(1, r, 2) if c["inter"] else slice(r // 2, r)
    a, b = y[..., first].clone(), y[..., second].clone()
    y[..., first] = a * cos - b * sin
    y[..., second] = b * cos + a * sin
    return y.to(x.dtype)


def _plain_append(s):
    """The slots cut back to `keep`, then their new rows, the keys rotated at the positions that they take."""
    c = s["case"]
    ps, T, width = c["ps"], c["t"], s["table"].shape[1]
    # roll back
    col = torch.arange(width, device=DEV)[None, :]
    L = torch.minimum(s["keep"], s["length"]).long()
    drop = (col >= ((L + ps - 1) // ps)[:, None]) & (s["table"] >= 0)
    s["refs"].index_add_(0, s["table"].clamp(min=0).reshape(-1).long(), -drop.reshape(-1).to(torch.int32))
    t = torch.where(drop, -1, s["table"])
    # free pages, lowest id first, in the order of the rows (no page has two holders here)
    n = s["n_new"].long().clamp(0, T)
    have, want = (L + ps - 1) // ps, (L + n + ps - 1) // ps
    free = s["refs"] == 0
    all_ids = torch.arange(free.numel(), device=DEV)
    ids = torch.sort(torch.where(free, all_ids, all_ids + free.numel())).values % free.numel()
    ok = (L + n <= width * ps) & ((want == have) | (torch.cumsum(want - have, 0) <= free.sum()))
    need = (want - have) * ok
    start = torch.cumsum(need, 0) - need
    fresh = (col >= have[:, None]) & (col < (have + need)[:, None])
    page = ids[(start[:, None] + col - have[:, None]).clamp(0, ids.numel() - 1)]
    s["refs"].index_add_(0, page.reshape(-1), fresh.reshape(-1).to(torch.int32))
    t = torch.where(fresh, page.to(torch.int32), t)
    s["table"].copy_(t)
    s["length"].copy_((L + n * ok).to(torch.int32))
    # rows
    i = torch.arange(T, device=DEV)[None, :]
    pos = L[:, None] + i
    b, j = torch.nonzero((i < n[:, None]) & ok[:, None], as_tuple=True)
    at, row = t[b, pos[b, j] // ps].long(), pos[b, j] % ps
    s["k"][at, :, row] = _plain_rotate(c, s["k_new"][b, j], pos[b, j])
    s["v"][at, :, row] = s["v_new"][b, j]
    if s["q"] is not None:
        b, j = torch.nonzero(i < n[:, None], as_tuple=True)
        s["q_out"][b, j] = _plain_rotate(c, s["q"][b, j], pos[b, j] + c["after"])
    return ok.to(torch.int32)


def _parts(x):
    """Maximum (0 where there is nothing), weights and their sum over the last dimension."""
    m = x.amax(-1, keepdim=True) if x.shape[-1] else x.new_full((*x.shape[:-1], 1), float("-inf"))
    e = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    return m, e, e.sum(-1, keepdim=True)


def _plain_shared(s):
    c = s["case"]
    ps, hkv, dh, G = c["ps"], c["hkv"], c["dh"], c["hq"] // c["hkv"]
    width = s["table"].shape[1]
    outs, lses, b0 = [], [], 0
    for size, whole in zip(s["sizes"], s["whole"]):
        R = size
        q = s["q"][b0:b0 + R].to(torch.float32).view(R, hkv, G, dh)
        # the common pages, once: all rows and grouped heads against each K/V head
        pages = s["table"][b0, :whole].long()
        K, V = (x[pages].to(torch.float32).transpose(0, 1).reshape(hkv, whole * ps, dh) for x in (s["k"], s["v"]))
        m0, e0, l0 = _parts(torch.matmul(q.permute(1, 0, 2, 3).reshape(hkv, R * G, dh), K.transpose(-1, -2)) * dh ** -0.5)
        o0 = torch.matmul(e0, V).view(hkv, R, G, dh).transpose(0, 1)
        m0, l0 = (x.view(hkv, R, G, 1).transpose(0, 1) for x in (m0, l0))
        # every row's own pages
        rest = s["table"][b0:b0 + R, whole:].long().clamp(min=0)
        K, V = (x[rest].to(torch.float32).permute(0, 2, 1, 3, 4).reshape(R, hkv, (width - whole) * ps, dh) for x in (s["k"], s["v"]))
        seen = torch.arange((width - whole) * ps, device=DEV)[None, :] + whole * ps < s["length"][b0:b0 + R, None]
        m1, e1, l1 = _parts((torch.matmul(q, K.transpose(-1, -2)) * dh ** -0.5).masked_fill(~seen[:, None, None, :], float("-inf")))
        o1 = torch.matmul(e1, V)
        m = torch.maximum(m0, m1)
        f0, f1 = torch.exp(m0 - m), torch.exp(m1 - m)
        l = l0 * f0 + l1 * f1
        outs.append(((o0 * f0 + o1 * f1) / l).reshape(R, c["hq"], dh))
        lses.append((m + torch.log(l)).reshape(R, c["hq"]))
        b0 += R
    return [torch.cat(outs).to(s["q"].dtype), torch.cat(lses)]


def _plain_sample(s):
    z = s["logits"]
    n, v = z.shape
    greedy = s["temp"] <= 0
    T = torch.where(greedy, torch.ones_like(s["temp"]), s["temp"]).to(torch.float64)[:, None]
    zs, ids = torch.sort(z, dim=-1, descending=True, stable=True)              # ties: the lower id first
    d = (zs.to(torch.float64) - zs[:, :1].to(torch.float64)) / T
    w = torch.exp(d)
    rank = torch.arange(v, device=DEV)[None, :]
    kept = rank >= 0
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        kept = kept & ((k <= 0) | (rank < k))
    if s["top_p"] is not None:
        p = s["top_p"].to(torch.float64)[:, None]
        wk = w * kept
        before = torch.cumsum(wk, -1) - wk
        kept = kept & ((p >= 1) | (before < p * wk.sum(-1, keepdim=True)) | (rank == 0))
    if s["min_p"] is not None:
        kept = kept & (d >= torch.log(s["min_p"].to(torch.float64))[:, None])
    w = torch.zeros_like(w).scatter_(1, ids, w * kept)
    cum = torch.cumsum(w, -1)
    total = cum[:, -1:]
    token = (cum <= s["u"].to(torch.float64)[:, None] * total).sum(-1).clamp(max=v - 1)
    logp = torch.log(w.gather(1, token[:, None]) / total)[:, 0]
    return [torch.where(greedy, ids[:, 0], token).to(torch.int32), torch.where(greedy, torch.zeros_like(logp), logp).to(torch.float32)]


# ------------------------------------------------------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    if own:
        from paper_2505_24544_b200 import binding as b
    if c["kind"] == "rotary":
        if own:
            b.beagle_rotary_apply(s["rot"], s["q"], s["q_out"], s["k"], s["k_out"], s["pos"])
            out = [s["q_out"], s["k_out"]]
            if c["train"]:
                b.beagle_rotary_apply(s["rot"], s["gq"], s["dq"], s["gk"], s["dk"], s["pos"], inverse=True)
                out += [s["dq"], s["dk"]]
            return out
        out = [_plain_rotate(c, s["q"], s["pos"]), _plain_rotate(c, s["k"], s["pos"])]
        if c["train"]:
            out += [_plain_rotate(c, s["gq"], s["pos"], True), _plain_rotate(c, s["gk"], s["pos"], True)]
        return out
    if c["kind"] == "append":
        if own:
            b.beagle_pages_truncate(s["cache"], s["slots"], s["keep"])
            b.beagle_pages_append_rotary(s["cache"], s["slots"], s["rot"], s["k_new"], s["v_new"], s["n_new"], s["ok"], s["q"], s["q_out"], q_offset=c["after"])
            ok = s["ok"]
        else:
            ok = _plain_append(s)
        return [s["k"], s["v"], s["table"], s["length"], s["refs"], ok] + ([] if s["q"] is None else [s["q_out"]])
    if c["kind"] == "shared":
        if not own:
            return _plain_shared(s)
        b.beagle_paged_attn_shared(s["cache"], s["slots"], s["sizes"], s["shared"], s["q"], s["out"], s["lse"])
        return [s["out"], s["lse"]]
    if not own:
        return _plain_sample(s)
    b.beagle_sample(s["logits"], s["u"], s["tokens"], temperature=s["temp"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], logp=s["logp"])
    return [s["tokens"], s["logp"]]


def work(case):
    c = dict(case)
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rotary":
        n = c["rows"] * (c["hq"] + c["hk"]) * (2 if c["train"] else 1)
        return {"bytes": 2 * n * c["dh"] * e + 4 * c["rows"], "flops": 3 * n * c["rot"]}
    if c["kind"] == "append":
        n = sum(_new_rows(c))
        return {"bytes": 2 * n * (2 * c["hkv"] + c["hq"]) * c["dh"] * e + 32 * c["batch"], "flops": 3 * n * (c["hkv"] + c["hq"]) * c["rot"]}
    if c["kind"] == "shared":
        sizes, pre, suf = _groups(c)
        whole = [p // c["ps"] * c["ps"] for p in pre]
        rows = sum(suf) + sum(n * (p - w) for n, p, w in zip(sizes, pre, whole))
        return {"bytes": 2 * (sum(whole) + rows) * c["hkv"] * c["dh"] * e + c["batch"] * c["hq"] * (2 * c["dh"] * e + 4),
                "flops": 4 * (sum(n * w for n, w in zip(sizes, whole)) + rows) * c["hq"] * c["dh"]}
    return {"bytes": c["rows"] * (c["v"] * e + 24), "flops": 2 * c["rows"] * c["v"]}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_rotate(c, x, pos, inverse=False):
    """Pairs as complex numbers, turned by exp(i pos f)."""
    r, i = c["rot"], np.arange(c["rot"] // 2)
    theta, factor, kind, m = c["theta"], c["factor"], c["scaling"], 1.0
    f = np.exp(-2.0 * i / r * math.log(theta))
    turns = c["original"] * f / (2 * np.pi)
    if kind == "linear":
        f = f / factor
    elif kind == "base":
        f = np.exp(-2.0 * i / r * (math.log(theta) + r / (r - 2) * math.log(factor)))
    elif kind == "bands":
        f = np.where(turns > 4.0, f, np.where(turns < 1.0, f / factor, f * ((turns - 1.0) / 3.0 + (4.0 - turns) / 3.0 / factor)))
    elif kind == "ramp":
        where = [r / 2 * math.log(c["original"] / (n * 2 * math.pi), theta) for n in (32, 1)]
        lo, hi = max(math.floor(where[0]), 0), min(math.ceil(where[1]), r - 1)
        f = f * np.interp(i, [lo, max(hi, lo + 0.001)], [1.0, 1.0 / factor])
        m = 1.0 + math.log(factor) / 10
    turn = torch.polar(torch.full((pos.numel(), r // 2), m, dtype=torch.float64, device=DEV), (-1 if inverse else 1) * pos.double()[:, None] * torch.from_numpy(f).to(DEV))
    y = x.double()
    z = y[..., :r].reshape(*y.shape[:-1], r // 2, 2) if c["inter"] else y[..., :r].reshape(*y.shape[:-1], 2, r // 2).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None, :])
    y[..., :r] = z.reshape(*y.shape[:-1], r) if c["inter"] else z.transpose(-1, -2).reshape(*y.shape[:-1], r)
    return y


def _exact_append(s):
    c = s["case"]
    ps, width = c["ps"], s["table"].shape[1]
    k, v, refs = s["k"].double(), s["v"].double(), s["refs"].tolist()
    lens, new, ok = _lengths(c), _new_rows(c), []
    q_out = None if s["q"] is None else s["q_out"].double()
    free = [p for p, r in enumerate(refs) if r == 0]
    pages = [[p for p in row if p >= 0] for row in s["table"].tolist()]
    for b, (n, t) in enumerate(zip(lens, new)):
        need = -(-(n + t) // ps) - len(pages[b])
        pos = torch.arange(n, n + t, device=DEV)
        if q_out is not None:
            q_out[b, :t] = _exact_rotate(c, s["q"][b, :t], pos + c["after"])
        ok.append(int(n + t <= width * ps and need <= len(free)))
        if not ok[-1]:
            continue
        mine, free = free[:need], free[need:]
        for p in mine:
            refs[p] = 1
        pages[b] += mine
        at = torch.tensor(pages[b], device=DEV)[pos // ps]
        k[at, :, pos % ps] = _exact_rotate(c, s["k_new"][b, :t], pos)
        v[at, :, pos % ps] = s["v_new"][b, :t].double()
        lens[b] = n + t
    table = [row + [-1] * (width - len(row)) for row in pages]
    out = [k, v, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, lens, refs, ok))]
    return out if q_out is None else out + [q_out]


def _exact_shared(s):
    c = s["case"]
    G, ps, dh = c["hq"] // c["hkv"], c["ps"], c["dh"]
    out, lse = s["q"].double() * 0, s["lse"].double() * 0
    lens, b0 = s["length"].tolist(), 0
    for size, whole in zip(s["sizes"], s["whole"]):
        for h in range(c["hkv"]):
            pk, pv = (x[s["table"][b0, :whole].long(), h].reshape(-1, dh).double() for x in (s["k"], s["v"]))
            q = s["q"][b0:b0 + size, h * G:(h + 1) * G].double()
            first = q.reshape(-1, dh) @ pk.T * dh ** -0.5
            lp = torch.logsumexp(first, -1).view(size, G)
            op = (torch.exp(first - lp.reshape(-1, 1)) @ pv if whole else torch.zeros_like(q)).view(size, G, dh)
            for i in range(size):
                n = lens[b0 + i] - whole * ps
                if n > 0:
                    pages = s["table"][b0 + i, whole:whole - (-n // ps)].long()
                    k, v = (x[pages, h].reshape(-1, dh)[:n].double() for x in (s["k"], s["v"]))
                    sc = q[i] @ k.T * dh ** -0.5
                    lr = torch.logsumexp(sc, -1)
                    both = torch.logaddexp(lp[i], lr)
                    out[b0 + i, h * G:(h + 1) * G] = torch.exp(lp[i] - both)[:, None] * op[i] + torch.exp(sc - both[:, None]) @ v
                    lse[b0 + i, h * G:(h + 1) * G] = both
                else:
                    out[b0 + i, h * G:(h + 1) * G], lse[b0 + i, h * G:(h + 1) * G] = op[i], lp[i]
        b0 += size
    return [out, lse]


def _exact_sample(s):
    z = s["logits"].double().cpu().numpy()
    get = lambda x, none: [none] * z.shape[0] if x is None else x.double().tolist()
    tokens, logp = [], []
    for row, t, k, p, mp, u in zip(z, s["temp"].double().tolist(), get(s["top_k"], 0), get(s["top_p"], 1.0), get(s["min_p"], 0.0), s["u"].double().tolist()):
        order = np.argsort(-row, kind="stable")
        if t <= 0:
            tokens.append(int(order[0]))
            logp.append(0.0)
            continue
        if 0 < k < len(order):
            order = order[:int(k)]
        d = (row[order] - row[order[0]]) / t
        if p < 1:
            run_sum = np.cumsum(np.exp(d))
            order = order[:max(1, int(np.searchsorted(run_sum, p * run_sum[-1], side="left")) + 1)]
            d = d[:len(order)]
        if mp > 0:
            order = order[d >= math.log(mp)]
        ids = np.sort(order)
        weight = np.exp((row[ids] - row[order[0]]) / t)
        run_sum = np.cumsum(weight)
        at = min(int(np.searchsorted(run_sum, u * run_sum[-1], side="right")), len(ids) - 1)
        tokens.append(int(ids[at]))
        logp.append(math.log(weight[at] / run_sum[-1]))
    return [torch.tensor(tokens, dtype=torch.int32, device=DEV), torch.tensor(logp, dtype=torch.float64, device=DEV)]


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "rotary":
        out = [_exact_rotate(c, s["q"], s["pos"]), _exact_rotate(c, s["k"], s["pos"])]
        return out + [_exact_rotate(c, s["gq"], s["pos"], True), _exact_rotate(c, s["gk"], s["pos"], True)] if c["train"] else out
    return {"append": _exact_append, "shared": _exact_shared, "sample": _exact_sample}[c["kind"]](s)
