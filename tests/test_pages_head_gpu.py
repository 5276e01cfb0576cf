"""The draft head over a paged cache: prefill, draft chains, verification and rollback against the oracle in 64 bits, whole and
through a window with sinks; the pages run out, the chain is captured, the head's own cache is left alone."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import beagle_oracle
from paper_2505_24544_b200 import binding as b
from paper_2505_24544_b200 import workloads as WL
from parity_utils import oracle_head, run_chain_parity, to_dev

pytestmark = pytest.mark.gpu

GQA = WL.WORKLOADS["c3_llama3_8b_b1"].scaled(name="paged_gqa", hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=64, mlp_dim=1416, vocab=4099,
                                             batch=3, ctx_min=1, ctx_max=500, gamma=4, seed=2101)
MHA = WL.WORKLOADS["c2_llama2_7b_b1"].scaled(name="paged_mha", hidden=768, n_q_heads=6, n_kv_heads=6, head_dim=128, mlp_dim=2048, vocab=5000,
                                             batch=2, ctx_min=100, ctx_max=300, gamma=4, seed=2102)
FP32 = WL.WORKLOADS["c1_tiny_fp32"].scaled(name="paged_fp32", batch=3, ctx_min=1, ctx_max=90, seed=2103)


class PagedHead:
    """The head with its paged calls in the shape that run_chain_parity drives."""

    def __init__(self, head, cache, window, sinks):
        self.head, self.cache, self.window, self.sinks = head, cache, window, sinks

    def draft_step(self, slots, tokens_in=None, concat=True, want_logits=False, want_hidden=False):
        return self.head.draft_step_pages(self.cache, slots, tokens_in, concat, want_logits, want_hidden, self.window, self.sinks)


def visible(kv, window, sinks):
    k, v = kv
    j = np.arange(len(k))
    seen = (j >= len(k) - window) | (j < sinks) if window > 0 else j >= 0
    return k[seen], v[seen]


def build(w, ps=16, pages=None):
    weights = WL.make_weights(w)
    # the head's own cache holds one position a slot: nothing of these runs fits in it
    head = b.BeagleHead.from_workload(w, weights, max_ctx=1, max_draft=1)
    width = -(-(w.ctx_max + 64) // ps)
    return head, oracle_head(w, weights), head.paged_cache(pages or w.batch * width, ps, w.batch, width)


def prefill_both(head, cpu, cache, w, rng, slots, seqs, lengths):
    hidden = WL.make_hidden(w, rng, int(np.sum(lengths)))
    head.prefill_pages(cache, slots, [int(n) for n in lengths], to_dev(hidden, w.dtype) if len(hidden) else None)
    r = 0
    for s, n in zip(seqs, lengths):
        O.prefill_kv(cpu, s, hidden[r:r + n])
        r += n


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
@pytest.mark.parametrize("w,batch,ps", [(GQA, 3, 16), (GQA, 1, 64), (GQA, 12, 8), (GQA, 20, 64), (GQA, 40, 16), (MHA, 2, 32), (FP32, 3, 8), (FP32, 20, 8)],
                         ids=lambda x: getattr(x, "name", str(x)))
def test_chains_against_the_oracle(w, batch, ps, window, sinks, monkeypatch):
    """Decoding iterations: prefill, a chain of drafted tokens, verification, the draft tail cut off, the accepted states appended."""
    block = beagle_oracle.draft_block
    monkeypatch.setattr(beagle_oracle, "draft_block", lambda head, toks, kv, pos: block(head, toks, [visible(x, window, sinks) for x in kv], pos))
    w = w.scaled(batch=batch)
    head, cpu, cache = build(w, ps)
    rng = WL.data_rng(w, batch)
    slots = [int(s) for s in rng.permutation(batch)]
    lengths = WL.make_context_lengths(w, rng)
    lengths[0] = 0                                           # a slot without a state: the first step's attention reads nothing
    seqs = [O.OracleSequence(cpu) for _ in slots]
    before = head.ctx.kv_buf.clone()
    prefill_both(head, cpu, cache, w, rng, slots, seqs, lengths)
    first = WL.make_tokens(w, rng, (batch,))
    for it in range(2):
        drafted, drafted_ref, _ = run_chain_parity(PagedHead(head, cache, window, sinks), cpu, w, slots, seqs, first, w.gamma)
        torch.cuda.synchronize()
        assert [cache.length.tolist()[s] for s in slots] == [q.n_true + w.gamma - 1 for q in seqs]
        target = WL.make_target_stream(w, rng, drafted_ref)
        acc, out = O.verify_greedy(drafted_ref, target_ids=target)
        acc_gpu, out_gpu = head.verify_greedy(to_dev(drafted_ref.astype(np.int32), w.dtype), target_ids=to_dev(target, w.dtype))
        np.testing.assert_array_equal(acc_gpu.cpu().numpy(), acc)
        keep = torch.tensor([q.n_true for q in seqs], dtype=torch.int32, device="cuda")
        b.beagle_pages_truncate(cache, slots, keep)
        prefill_both(head, cpu, cache, w, rng, slots, seqs, acc + 1)
        torch.cuda.synchronize()
        assert [cache.length.tolist()[s] for s in slots] == [q.n_true for q in seqs]
        first = np.array([out[r, acc[r]] for r in range(batch)])
    b.beagle_check_device(head.ctx)
    assert torch.equal(head.ctx.kv_buf, before)


@pytest.mark.parametrize("w,rows", [(GQA, 700), (GQA, 400), (GQA, 65), (GQA, 9), (GQA, 8), (MHA, 513), (FP32, 64), (FP32, 17), (FP32, 16)],
                         ids=lambda x: getattr(x, "name", str(x)))
def test_prefill_rows(w, rows):
    """Every kernel that forms the rows, ragged sequences, an empty one among them: each cached value against the definition.  bf16:
    one rounding of the sum (half a step, 2^-8) and fp32 accumulation over the hidden size; the same bound in fp32 with 2^-24."""
    w = w.scaled(batch=3, ctx_max=rows)
    head, cpu, cache = build(w)
    rng = WL.data_rng(w, rows)
    lengths = [rows // 3 + 1, 0, rows - rows // 3 - 1]
    hidden = WL.make_hidden(w, rng, rows)
    ok = torch.full((3,), 7, dtype=torch.int32, device="cuda")
    head.prefill_pages(cache, [2, 0, 1], lengths, to_dev(hidden, w.dtype), ok)
    torch.cuda.synchronize()
    assert ok.tolist() == [1, 1, 1] and cache.length.tolist() == [0, lengths[2], lengths[0]]
    k, v = O.project_kv(cpu, hidden)
    half = 2.0 ** -8 if w.dtype == "bf16" else 2.0 ** -24
    r = 0
    for slot, n in zip([2, 0, 1], lengths):
        t = cache.table[slot, : -(-n // 16)].long()
        for pool, want, weight in ((cache.k, k, "w_k"), (cache.v, v, "w_v")):
            got = pool[t].permute(0, 2, 1, 3).reshape(-1, w.n_kv_heads * w.head_dim)[:n].double().cpu().numpy()
            ref = want[r:r + n].reshape(n, w.n_kv_heads * w.head_dim)
            mass = np.abs(hidden[r:r + n]).astype(np.float64) @ np.abs(getattr(cpu, weight)).T.astype(np.float64)
            assert np.all(np.abs(got - ref) <= half * np.abs(ref) + (w.hidden + 8) * 2.0 ** -24 * 1.01 * mass + 1e-30)
        r += n


def test_concat_off_rollback_and_a_full_pool():
    w = GQA.scaled(batch=2, ctx_max=64)
    head, _, cache = build(w, ps=16, pages=4)
    rng = WL.data_rng(w, 5)
    hidden = to_dev(WL.make_hidden(w, rng, 64), w.dtype)
    tok = to_dev(WL.make_tokens(w, rng, (2,)), w.dtype)
    ok = torch.full((2,), 7, dtype=torch.int32, device="cuda")
    head.prefill_pages(cache, [0, 1], [32, 31], hidden[:63], ok)
    a = head.draft_step_pages(cache, [0, 1], tok, want_logits=True, ok=ok)[1]
    head.draft_step_pages(cache, [0, 1], tok, concat=False, ok=ok)                     # the states are not appended
    torch.cuda.synchronize()
    assert cache.length.tolist() == [32, 31] and ok.tolist() == [1, 1]
    head.draft_step_pages(cache, [0, 1], tok, want_logits=True, ok=ok)                 # slot 0 needs a page, there is none; slot 1 has room
    torch.cuda.synchronize()
    assert cache.length.tolist() == [32, 32] and ok.tolist() == [0, 1]
    b.beagle_pages_truncate(cache, [0, 1], torch.tensor([32, 31], dtype=torch.int32, device="cuda"))
    head.rollback([0, 1])
    c = head.draft_step_pages(cache, [0, 1], tok, want_logits=True)[1]
    assert torch.equal(a, c)
    head.prefill_pages(cache, [1], [2], hidden[:2], ok[:1])                            # 31 + 2 positions want a third page
    torch.cuda.synchronize()
    assert ok.tolist()[0] == 0 and cache.length.tolist() == [32, 31]
    head.rollback([0])
    with pytest.raises(b.BeagleError) as e:
        head.draft_step_pages(cache, [0])                                              # no previous token
    assert e.value.status == 4


def test_chain_from_a_captured_graph():
    """A chain, the tail cut off, replayed: the same tokens as the eager chain, whatever the lengths on the device have become."""
    w = GQA.scaled(batch=12, gamma=4)
    head, _, cache = build(w)
    rng = WL.data_rng(w, 77)
    lengths = [int(n) for n in WL.make_context_lengths(w, rng)]
    slots = list(range(12))
    hidden = to_dev(WL.make_hidden(w, rng, sum(lengths)), w.dtype)
    first = to_dev(WL.make_tokens(w, rng, (12,)), w.dtype)
    keep = cache.length.clone()

    def chain(draft):
        keep.copy_(cache.length)
        for s in range(w.gamma):
            b.beagle_draft_step_pages(head.ctx, cache, slots, first if s == 0 else None, True, draft[:, s], window=100, sinks=4)
        b.beagle_pages_truncate(cache, slots, keep)

    head.prefill_pages(cache, slots, lengths, hidden)
    eager, captured = (torch.zeros(12, w.gamma, dtype=torch.int32, device="cuda") for _ in range(2))
    chain(eager)
    torch.cuda.synchronize()
    head.rollback(slots)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(captured)
    for _ in range(2):
        captured.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, captured) and cache.length.tolist() == lengths
    head.prefill_pages(cache, slots, [3] * 12, hidden[:36])                            # longer sequences: the graph reads the new lengths
    graph.replay()
    longer = captured.clone()
    head.rollback(slots)
    chain(eager)
    torch.cuda.synchronize()
    assert torch.equal(eager, longer) and cache.length.tolist() == [n + 3 for n in lengths]


@pytest.mark.parametrize("w", [GQA, FP32], ids=lambda x: x.name)
def test_a_reused_slot_starts_a_chain_of_its_own(w):
    """A slot whose old sequence is freed and that becomes a fork: with its old chain dropped it drafts what the slot it was forked
    from drafts, and the old chain's last state is not appended to it."""
    w = w.scaled(batch=2, ctx_max=40)
    head, _, cache = build(w, ps=8)
    rng = WL.data_rng(w, 9)
    hidden = to_dev(WL.make_hidden(w, rng, 70), w.dtype)
    first = to_dev(WL.make_tokens(w, rng, (2,)), w.dtype)
    head.prefill_pages(cache, [0, 1], [37, 33], hidden)
    head.draft_step_pages(cache, [1], first[1:])                       # slot 1 has a chain, its last state pending
    b.beagle_pages_truncate(cache, [1])
    b.beagle_pages_fork(cache, [0], [1])
    head.rollback([1])
    both = first[:1].expand(2).contiguous()
    tok, logits, _ = head.draft_step_pages(cache, [0, 1], both, want_logits=True)
    assert cache.length.tolist() == [37, 37] and torch.equal(logits[0], logits[1]) and int(tok[0]) == int(tok[1])
    tok, logits, _ = head.draft_step_pages(cache, [0, 1], want_logits=True)      # both append their first state, to pages of their own
    assert cache.length.tolist() == [38, 38] and torch.equal(logits[0], logits[1]) and int(tok[0]) == int(tok[1])
    assert cache.table[0, :4].tolist() == cache.table[1, :4].tolist() and int(cache.table[0, 4]) != int(cache.table[1, 4])
    b.beagle_check_device(head.ctx)
