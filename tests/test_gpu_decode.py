"""An attention layer over the quantized cache, run as a decoder with drafted
tokens runs it: prompt pieces, trees, acceptance.  Projections against the
oracle, the cache's bytes and the attention against their definitions in fp64."""
import numpy as np
import pytest

import kv_plain
import oracle
from helpers import assert_y_close
from paper_2311_14114_gb300 import workloads as wl

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HEADS, GROUP, D, DV, K, PAGE = 2, 4, 64, 48, 264, 16
SEEN_MAX = 200


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import build, soniq
    build.build()
    soniq.lib()
    return soniq


class Layer:
    def __init__(self, sq, seed, B):
        from paper_2311_14114_gb300.decode import CachedAttention
        rng = np.random.default_rng(seed)
        self.rng, self.q_heads = rng, HEADS * GROUP

        def weights(N, K, bits):
            perm, count, _ = wl.assignment(rng, K, 0.25, 0)
            return dict(W=(rng.standard_normal((N, K)) / np.sqrt(K)).astype(np.float32), perm=perm, count=count,
                        bits=list(bits))

        def side(D, n_hi, bits):
            perm = np.stack([rng.permutation(D) for _ in range(HEADS)])
            return sq.KVLayout(perm, (D - n_hi, n_hi), bits)

        self.lays = [weights(self.q_heads * D + HEADS * (D + DV), K, (4, 8)), weights(K, self.q_heads * DV, (4, 8))]
        per_seq = -(-SEEN_MAX // PAGE)
        self.table = torch.from_numpy(rng.permutation(B * per_seq).reshape(B, per_seq).astype(np.int32)).cuda()
        self.net = CachedAttention(self.lays[0], self.lays[1], self.q_heads, side(D, 16, (4, 8)), side(DV, 8, (4, 8)),
                                   B * per_seq, PAGE)

    def x(self, B, T):
        return torch.from_numpy(self.rng.standard_normal((B, T, K)).astype(np.float16)).cuda()

    def check_projection(self, which, x, y):
        lay = self.lays[which]
        r = oracle.linear_variant(x.cpu().numpy(), lay["W"], lay["perm"], lay["count"], lay["bits"], lay["bits"],
                                  kind=(1, 1), act_mode="row")
        assert_y_close(y.cpu().numpy().astype(np.float64), r["Y64"].astype(np.float16), r["terms"], f"projection {which}")

    def check(self, X, y, ks, vs, lens, mask):
        """The last step: ks, vs are each sequence's 16-bit rows, context and drafts."""
        net, (B, T) = self.net, X.shape[:2]
        self.check_projection(0, X.view(B * T, K), torch.cat([t.flatten(2) for t in (net.q, net.k, net.v)], -1).view(B * T, -1))
        self.check_projection(1, net.o.view(B * T, -1), y.view(B * T, -1))
        k = [kv_plain.values(net.cache.k, t.double().cpu().numpy(), torch.float16) for t in ks]
        v = [kv_plain.values(net.cache.v, t.double().cpu().numpy(), torch.float16) for t in vs]
        ref, mag, dscore, total = kv_plain.attend(net.q.double().cpu().numpy(), k, v, lens, mask, GROUP, D ** -0.5)
        tol = kv_plain.tolerance(ref, mag, dscore, total, max(lens) + T, max(np.abs(t).max() for t in v), torch.float16)
        assert (np.abs(net.o.double().cpu().numpy() - ref) <= tol).all()


def test_prompt_drafts_and_acceptance(sq):
    B = 3
    L = Layer(sq, 71, B)
    net = L.net
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    ks, vs = [None] * B, [None] * B

    def keep(n, rows):
        for b in range(B):
            for to, new in ((ks, net.k[b, rows[b]]), (vs, net.v[b, rows[b]])):
                to[b] = new.clone() if to[b] is None else torch.cat([to[b][:n[b]], new])

    # two pieces of a prompt
    for T in (70, 37):
        X = L.x(B, T)
        y = net.step(X, L.table, lens)
        keep(lens.tolist(), [list(range(T))] * B)
        L.check(X, y, ks, vs, lens.tolist(), None)
        lens += T
    # a tree of drafts: 0 -> {1, 2}, 1 -> {3, 4}, 2 -> 5, 5 -> 6
    parent = [-1, 0, 0, 1, 1, 2, 5]
    mask = np.zeros((7, 7), dtype=bool)
    for t, p in enumerate(parent):
        mask[t] = mask[p] if p >= 0 else False
        mask[t, t] = True
    for paths in ([[0, 2, 5, 6], [0, 1, 4, -1], [0, -1, -1, -1]], [[0, 2, -1, -1], [-1, -1, -1, -1], [0, 1, 3, -1]]):
        X = L.x(B, 7)
        y = net.step(X, L.table, lens, torch.from_numpy(mask).cuda())
        n = lens.tolist()
        drafts = [[torch.cat([old[b][:n[b]], new[b]]) for b in range(B)] for old, new in ((ks, net.k), (vs, net.v))]
        L.check(X, y, drafts[0], drafts[1], n, np.broadcast_to(mask, (B, 7, 7)))
        taken = [[t for t in p if t >= 0] for p in paths]
        keep(n, taken)
        lens = net.accept(torch.tensor(paths, device="cuda"), L.table, lens)
        assert lens.tolist() == [a + len(t) for a, t in zip(n, taken)]
    # the next token of each, and what the cache holds by then
    X = L.x(B, 1)
    y = net.step(X, L.table, lens)
    n = lens.tolist()
    keep(n, [[0]] * B)
    L.check(X, y, ks, vs, n, None)
    for b in range(B):
        k, v = net.context(L.table, lens + 1, b)
        for got, rows, lay in ((k, ks[b], net.cache.k), (v, vs[b], net.cache.v)):
            want = kv_plain.values(lay, rows.double().cpu().numpy(), torch.float16).astype(np.float16)
            assert np.array_equal(got.cpu().numpy(), want)
    assert sq.sync_status() == 0


def test_absent_sequences_and_full_tables(sq):
    L = Layer(sq, 72, 2)
    lens = torch.tensor([-1, 5], dtype=torch.int32, device="cuda")
    y = L.net.step(L.x(2, 3), L.table, lens)
    assert sq.sync_status() == 0
    assert (L.net.o[0] == 0).all() and (y[0] == 0).all()
    assert L.net.accept(torch.tensor([[0], [0]], device="cuda"), L.table, lens).tolist() == [-1, 6]
    full = L.table.shape[1] * PAGE
    L.net.step(L.x(2, 3), L.table, torch.tensor([0, full - 1], dtype=torch.int32, device="cuda"))
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
    assert sq.sync_status() == 0


def test_sizes_that_differ_are_refused(sq):
    from paper_2311_14114_gb300.decode import CachedAttention
    L = Layer(sq, 73, 1)
    c = L.net.cache
    for q_heads in (HEADS * GROUP - 1, HEADS):
        with pytest.raises(ValueError):
            CachedAttention(L.lays[0], L.lays[1], q_heads, c.k, c.v, 4, PAGE)
