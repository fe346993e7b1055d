"""Steps whose plan holds absent sequences and such that wait: nothing of theirs is
written or read, and the others' tokens go where the plan says."""
import numpy as np
import pytest

import kv_plain
from test_gpu_decode import GROUP, PAGE, D
from test_gpu_step import SEQS, Server, ints, sq  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F16 = torch.float16


def grow(s, sq, targets, T, mask=None):  # noqa: F811
    """A step in which each sequence is to reach its target, T tokens on or none."""
    old = s.lengths.tolist()
    plan = sq.kv_plan(s.pages, s.lengths, ints(targets), SEQS * T)
    X = s.x(SEQS, T)
    y = s.net.step(X, s.pages.table, s.lengths, mask, slots=plan)
    torch.cuda.synchronize()
    new = plan.lengths.tolist()
    there = [b for b in range(SEQS) if new[b] > max(old[b], 0)]
    s.check_heads(X.view(SEQS * T, -1), [(max(n, 0) if b in there else n) + t for b, n in enumerate(old) for t in range(T)])
    k, v = s.net.k.double().cpu().numpy(), s.net.v.double().cpu().numpy()
    for b in there:
        s.k[b], s.v[b] = np.concatenate([s.k[b], k[b]]), np.concatenate([s.v[b], v[b]])
    held = [[kv_plain.values(lay, rows[b], F16) if b in there else rows[b] for b in range(SEQS)]
            for lay, rows in ((s.net.cache.k, s.k), (s.net.cache.v, s.v))]
    lens = [max(n, 0) if b in there else -1 for b, n in enumerate(old)]
    if there:
        ref, mag, dscore, total = kv_plain.attend(s.net.q.double().cpu().numpy(), *held, lens, None, GROUP, D ** -0.5)
        tol = kv_plain.tolerance(ref, mag, dscore, total, max(lens) + T, max(np.abs(held[1][b]).max() for b in there), F16)
        assert (np.abs(s.net.o.double().cpu().numpy() - ref) <= tol).all()
    absent = [b for b in range(SEQS) if b not in there]
    assert (s.net.o[absent] == 0).all()
    s.check_projection(1, s.net.o.flatten(0, 1).flatten(1), y.view(SEQS * T, -1))
    s.lengths = plan.lengths
    s.check_cache()
    assert sq.sync_status() == 0
    return plan


def test_absent_sequences_in_front(sq):  # noqa: F811
    s = Server(sq, 91, 30)
    s.prompts(sq, [None, 33, None, 60, 15])
    for _ in range(3):
        grow(s, sq, [-1, *(n + 1 if n >= 0 else -1 for n in s.lengths.tolist()[1:])], 1)
    # pieces of three tokens, in which some sequences add nothing
    n = s.lengths.tolist()
    grow(s, sq, [3, n[1], -1, n[3] + 3, n[4]], 3)


def waiting_pool(sq, seed):  # noqa: F811
    """Sequence 0 gave back a page that sequence 1 has since taken, the pool is empty, and
    the table still names it behind sequence 0's context."""
    s = Server(sq, seed, 5)
    s.prompts(sq, [33, 20, None, None, None])
    s.lengths = sq.kv_plan(s.pages, s.lengths, ints([32, 20, -1, -1, -1]), 0).lengths
    s.k[0], s.v[0] = s.k[0][:32], s.v[0][:32]
    grow(s, sq, [32, 33, -1, -1, -1], 13)
    assert s.pages.count.tolist() == [0, 0] and s.pages.table[0, 2] == s.pages.table[1, 2] and PAGE == 16
    return s


def test_a_sequence_that_waits_is_absent(sq):  # noqa: F811
    s = waiting_pool(sq, 92)
    for T in (1, 2):
        n = s.lengths.tolist()
        grow(s, sq, [32 + T, n[1] + T, -1, -1, -1], T)
        assert s.lengths.tolist() == [32, n[1] + T, -1, -1, -1]
    # the other leaves, and it goes on
    s.lengths = sq.kv_plan(s.pages, s.lengths, ints([32, -1, -1, -1, -1]), 0).lengths
    s.k[1], s.v[1] = s.k[1][:0], s.v[1][:0]
    grow(s, sq, [33, -1, -1, -1, -1], 1)
    assert s.lengths.tolist() == [33, -1, -1, -1, -1]


def test_another_number_of_tokens_is_reported(sq):  # noqa: F811
    s = Server(sq, 93, 30)
    s.prompts(sq, [16, 20, None, None, None])
    plan = sq.kv_plan(s.pages, s.lengths, ints([18, 23, -1, -1, -1]), 15)
    s.net.step(s.x(SEQS, 3), s.pages.table, s.lengths, slots=plan)
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
    assert (s.net.o[0] == 0).all() and (s.net.o[1] != 0).any()


def test_a_captured_step(sq):  # noqa: F811
    """Plan and step in one graph: every replay is the next token of what is there."""
    a, b = Server(sq, 94, 30), Server(sq, 94, 30)
    for s in (a, b):
        s.prompts(sq, [None, 14, None, 29, 1])
    X = a.x(SEQS, 1)
    b.x(SEQS, 1)
    lengths = b.lengths.clone()
    out = sq.KVStep(*(torch.zeros(n, dtype=d, device="cuda") for n, d in ((SEQS + 1, torch.int32), (SEQS, torch.int32), (SEQS, torch.int64),
                                                                          (SEQS, torch.int32))))
    before = torch.empty_like(lengths)

    def run():
        before.copy_(lengths)
        sq.kv_plan(b.pages, before, before + (before >= 0).int(), SEQS, out=out)
        y = b.net.step(X, b.pages.table, before, slots=out)
        lengths.copy_(out.lengths)
        return y

    warm = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=warm):
        got = run()
    for _ in range(20):
        n = a.lengths.tolist()
        plan = sq.kv_plan(a.pages, a.lengths, ints([x + 1 if x >= 0 else -1 for x in n]), SEQS)
        want = a.net.step(X, a.pages.table, a.lengths, slots=plan)
        a.lengths = plan.lengths
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(lengths, a.lengths)
    assert sq.sync_status() == 0


@pytest.mark.parametrize("T", [1, 3])
def test_a_sequence_that_waits_accepts_nothing(sq, T):  # noqa: F811
    """Its drafts have no slots, and the page behind its context is another's."""
    s = waiting_pool(sq, 95)
    n = s.lengths.tolist()
    plan = sq.kv_plan(s.pages, s.lengths, ints([n[0] + T, n[1] + T, -1, -1, -1]), SEQS * T)
    s.net.step(s.x(SEQS, T), s.pages.table, s.lengths, slots=plan)
    path = torch.tensor([list(range(T))] * SEQS, device="cuda")
    path[1, 1:] = -1
    new = s.net.accept(path, s.pages.table, s.lengths)
    assert new.tolist() == [n[0], n[1] + 1, -1, -1, -1]
    k, v = s.net.k.double().cpu().numpy(), s.net.v.double().cpu().numpy()
    s.k[1], s.v[1] = np.concatenate([s.k[1], k[1, :1]]), np.concatenate([s.v[1], v[1, :1]])
    s.lengths = sq.kv_plan(s.pages, plan.lengths, new, 0).lengths
    s.check_cache()
    assert sq.sync_status() == 0
