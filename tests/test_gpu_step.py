"""The operators of a step together, as a server runs them: pages planned, prompts
packed, queries and keys normed and turned, prompts attended to, tokens decoded over
what the cache holds, sequences that leave and others in their pages."""
import numpy as np
import pytest

import kv_plain
import step_plain
from test_gpu_decode import DV, GROUP, HEADS, K, PAGE, D, Layer

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
SEQS, WIDTH = 5, 12


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import build, soniq
    build.build()
    soniq.lib()
    return soniq


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server(Layer):
    """A layer with norms and a rotation, its pages, and each sequence's rows as the cache was given them."""

    def __init__(self, sq, seed, n_pages):
        super().__init__(sq, seed, 1)
        from paper_2311_14114_gb300.decode import CachedAttention
        old = self.net
        self.rotary = sq.Rotary(D // 2 * 2, base=5000.0, scaling=("linear", 2.0))
        self.gains = tuple(torch.from_numpy((1 + 0.2 * self.rng.standard_normal(D)).astype(np.float32)).cuda() for _ in range(2))
        self.net = CachedAttention(self.lays[0], self.lays[1], self.q_heads, old.cache.k, old.cache.v, n_pages, PAGE,
                                   rotary=self.rotary, gains=self.gains, eps=1e-5)
        self.pages = sq.KVPages(n_pages, PAGE, SEQS, WIDTH)
        self.lengths = ints([-1] * SEQS)
        self.k = [np.zeros((0, HEADS, D)) for _ in range(SEQS)]
        self.v = [np.zeros((0, HEADS, DV)) for _ in range(SEQS)]

    def check_heads(self, X, positions):
        """Projection against the oracle through the cuda projection's own rows, norms and rotation against fp64."""
        plain = self.net._project(0, X)
        self.check_projection(0, X, plain)
        q, k, _ = plain.split(self.net.widths, -1)
        for got, x, gain in ((self.net.q, q, self.gains[0]), (self.net.k, k, self.gains[1])):
            x = x.reshape(len(X), -1, D)
            ref, mag = step_plain.rotate(x.double().cpu().numpy(), self.rotary.frequencies, positions, False, gain.double().cpu().numpy(), 1e-5)
            err = np.abs(got.reshape(x.shape).double().cpu().numpy() - ref)
            assert (err <= step_plain.rotate_tolerance(ref, mag, torch.float16)).all()

    def check_cache(self):
        for b in range(SEQS):
            n = max(self.lengths.tolist()[b], 0)
            assert len(self.k[b]) == n
            got = self.net.context(self.pages.table, self.lengths, b)
            for g, rows, lay in zip(got, (self.k[b], self.v[b]), (self.net.cache.k, self.net.cache.v)):
                assert np.array_equal(g.cpu().numpy(), kv_plain.values(lay, rows, torch.float16).astype(np.float16))

    def prompts(self, sq, lens, pad=0):
        """Sequences with a length in `lens` are admitted, None: left as they are."""
        old = self.lengths.tolist()
        targets = [o if n is None else n for o, n in zip(old, lens)]
        cap = sum(n or 0 for n in lens) + pad
        step = sq.kv_plan(self.pages, self.lengths, ints(targets), cap)
        X = self.x(1, cap)[0]
        y = self.net.prompt(X, step)
        torch.cuda.synchronize()
        starts = step.starts.tolist()
        self.check_heads(X[:starts[-1]] if pad == 0 else X, step.positions.tolist())
        self.lengths = step.lengths
        q, k, v = (t[:starts[-1]].double() for t in (self.net.q, self.net.k, self.net.v))
        ref = step_plain.attend(q, k, v, starts, True, D ** -0.5)
        tol = step_plain.attend_tolerance(*ref, max(cap, 1), torch.float16)
        assert ((self.net.o[:starts[-1]].double() - ref[0]).abs() <= tol).all() and (self.net.o[starts[-1]:] == 0).all()
        self.check_projection(1, self.net.o.flatten(1), y)
        for b in range(SEQS):
            if starts[b + 1] > starts[b] and self.lengths.tolist()[b] > 0:
                self.k[b] = k[starts[b]:starts[b + 1]].cpu().numpy()
                self.v[b] = v[starts[b]:starts[b + 1]].cpu().numpy()
        self.check_cache()
        return step

    def decode(self, sq):
        """One token of every sequence that is there."""
        old = self.lengths.tolist()
        step = sq.kv_plan(self.pages, self.lengths, ints([n + 1 if n >= 0 else -1 for n in old]), SEQS)
        X = self.x(SEQS, 1)
        slots = torch.full((SEQS,), -1, dtype=torch.int64, device="cuda")
        there = [b for b in range(SEQS) if old[b] >= 0]
        slots[there] = step.slots[:len(there)]
        y = self.net.step(X, self.pages.table, self.lengths, slots=slots)
        torch.cuda.synchronize()
        self.check_heads(X[:, 0], old)
        k, v = self.net.k[:, 0].double().cpu().numpy(), self.net.v[:, 0].double().cpu().numpy()
        for b in there:
            self.k[b], self.v[b] = np.concatenate([self.k[b], k[b:b + 1]]), np.concatenate([self.v[b], v[b:b + 1]])
        held = [[kv_plain.values(lay, rows[b], torch.float16) if b in there else rows[b] for b in range(SEQS)]
                for lay, rows in ((self.net.cache.k, self.k), (self.net.cache.v, self.v))]
        ref, mag, dscore, total = kv_plain.attend(self.net.q.double().cpu().numpy(), *held, old, None, GROUP, D ** -0.5)
        tol = kv_plain.tolerance(ref, mag, dscore, total, max(old) + 1, max(np.abs(held[1][b]).max() for b in there), torch.float16)
        assert (np.abs(self.net.o.double().cpu().numpy() - ref) <= tol).all()
        self.check_projection(1, self.net.o.flatten(0, 1).flatten(1), y[:, 0])
        self.lengths = step.lengths
        self.check_cache()


def test_prompts_decoding_and_reused_pages(sq):
    s = Server(sq, 81, 30)
    s.prompts(sq, [33, None, 100, None, 1])
    for _ in range(3):
        s.decode(sq)
    # sequence 2 leaves, 1 and 3 come into its pages, in a padded buffer
    left = s.lengths.clone()
    left[2] = -1
    s.lengths = sq.kv_plan(s.pages, s.lengths, left, 0).lengths
    s.k[2], s.v[2] = s.k[2][:0], s.v[2][:0]
    s.check_cache()
    s.prompts(sq, [None, 64, None, 120, None], pad=9)
    for _ in range(14):
        s.decode(sq)
    assert sq.sync_status() == 0


def test_a_prompt_that_waits(sq):
    """The pool holds two of three prompts: the third's rows are attended to but not kept."""
    s = Server(sq, 82, 9)
    s.prompts(sq, [60, 70, 50, None, None])
    assert s.lengths.tolist() == [60, 70, -1, -1, -1]
    s.decode(sq)
    assert sq.sync_status() == 0


def test_trees_turn_by_depth(sq):
    """Drafts of one depth share a position; the accepted ones stay as they were turned."""
    s = Server(sq, 83, 30)
    s.prompts(sq, [20, 35, None, None, None])
    B, n = 2, s.lengths.tolist()[:2]
    step = sq.kv_plan(s.pages, s.lengths, ints([26, 41, -1, -1, -1]), 12)
    depth = [0, 1, 1, 2, 2, 2]
    parent = [-1, 0, 0, 1, 1, 2]
    mask = np.zeros((6, 6), dtype=bool)
    for t, p in enumerate(parent):
        mask[t] = mask[p] if p >= 0 else False
        mask[t, t] = True
    X, table, lens = s.x(B, 6), s.pages.table[:B], s.lengths[:B].contiguous()
    positions = lens[:, None] + ints(depth)
    s.net.step(X, table, lens, torch.from_numpy(mask).cuda(), positions=positions, slots=step.slots)
    torch.cuda.synchronize()
    s.check_heads(X.view(12, K), positions.view(-1).tolist())
    k, v = s.net.k.double().cpu().numpy(), s.net.v.double().cpu().numpy()
    new = s.net.accept(torch.tensor([[0, 2, 5], [0, 1, -1]], device="cuda"), table, lens)
    assert new.tolist() == [23, 37]
    s.k[0], s.v[0] = np.concatenate([s.k[0], k[0, [0, 2, 5]]]), np.concatenate([s.v[0], v[0, [0, 2, 5]]])
    s.k[1], s.v[1] = np.concatenate([s.k[1], k[1, [0, 1]]]), np.concatenate([s.v[1], v[1, [0, 1]]])
    # the rejected drafts' pages go back
    s.lengths = sq.kv_plan(s.pages, step.lengths, torch.cat([new, ints([-1] * 3)]), 0).lengths
    s.check_cache()
    s.decode(sq)
    assert sq.sync_status() == 0
