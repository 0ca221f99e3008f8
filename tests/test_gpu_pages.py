"""Page operators on the GPU: random histories of a pool against the plain restatement (everything exactly equal), what the device
flags, and sequences forked and compacted under the verify path."""
import numpy as np
import pytest
import torch

from oracle import tok_oracle as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2609_24698_b200 import binding, pages, tokens
    return binding, tokens, pages


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """The pool on the device and its restatement."""

    def __init__(self, pg, slots, max_pages, n_pages, page_tokens, widths, row_widths, seed=0):
        rng = self.rng = np.random.default_rng(seed)
        self.pg = pg
        planes = [torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (n_pages, w), dtype=np.int64).astype(np.int32)).cuda() for w in widths]
        rows = [torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (slots, w), dtype=np.int64).astype(np.int32)).cuda() for w in row_widths]
        self.L = torch.zeros(slots, dtype=torch.int32, device="cuda")
        self.pool = pg.PagePool(torch.full((slots, max_pages), -1, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda"),
                                page_tokens, planes, [self.L] + rows)
        self.ws = pg.alloc_workspace(self.pool)
        self.ws.fill_(0xff)
        self.ref = T.Pool(self.pool.page_table.cpu().numpy(), self.pool.ref.cpu().numpy(), page_tokens, [p.cpu().numpy() for p in planes],
                          [r.cpu().numpy() for r in self.pool.rows])

    def check(self, status, exp):
        assert status.tolist() == exp
        self.same()

    def same(self):
        assert np.array_equal(self.pool.page_table.cpu().numpy(), self.ref.table)
        assert np.array_equal(self.pool.ref.cpu().numpy(), self.ref.ref)
        for a, b in zip(self.pool.planes + self.pool.rows, self.ref.planes + self.ref.rows):
            assert np.array_equal(a.cpu().numpy(), b)

    def call(self, what, *lists):
        n = len(lists[0])
        status = torch.zeros(max(n, 1), dtype=torch.int32, device="cuda")[:n]
        dev = [i32(*x) if n else torch.zeros(0, dtype=torch.int32, device="cuda") for x in lists]
        if what == "assign":
            self.pg.pages_assign(self.pool, *dev, self.ws, status)
            self.check(status, self.ref.assign(*lists))
        elif what == "free":
            self.pg.pages_free(self.pool, *dev, status)
            self.check(status, self.ref.free(*lists))
        else:
            L = self.L.tolist()
            self.pg.pages_fork(self.pool, *dev, self.L, self.ws, status)
            self.check(status, self.ref.fork(*lists, L))

    def set_lengths(self, L):
        self.L.copy_(i32(*L))
        self.ref.rows[0][:] = np.asarray(L, np.int32).reshape(self.ref.rows[0].shape)

    def compact(self):
        n = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        self.pg.pages_compact(self.pool, n, self.ws)
        assert int(n) == self.ref.compact()
        self.same()


# planes of one 16-byte vector, of less and more than a copy's chunk, of no round number of them; odd and large row arrays
@pytest.mark.parametrize("slots,max_pages,n_pages,page_tokens,widths,row_widths,seed", [
    (1, 1, 1, 1, [4], [], 0), (5, 7, 23, 4, [4, 4096 + 12, 40], [1, 3, 5000], 1), (40, 33, 500, 16, [8], [2], 2), (12, 70, 40000, 128, [4], [4], 3), (6, 40, 64, 3, [], [1], 4),
    (300, 3, 1000, 8, [16], [16], 5)])
def test_random_histories(api, slots, max_pages, n_pages, page_tokens, widths, row_widths, seed):
    _, _, pg = api
    x = Both(pg, slots, max_pages, n_pages, page_tokens, widths, row_widths, seed)
    rng = x.rng
    for step in range(14):
        k = int(rng.integers(1, min(slots, 24) + 1))
        pick = [int(s) for s in rng.permutation(slots)[:k]]
        lo = [int(v) for v in rng.integers(0, max_pages, k)]
        hi = [int(rng.integers(a, max_pages + 1)) for a in lo]
        x.call("assign", pick, [0] * k if step % 3 else lo, hi)
        x.set_lengths([int(rng.integers(0, max_pages * page_tokens + 1)) for _ in range(slots)])
        used = [s for s in range(slots) if (x.ref.table[s] >= 0).any()]
        empty = [s for s in range(slots) if (x.ref.table[s] < 0).all()]
        if used and empty:
            m = min(len(empty), 9)
            x.call("fork", [int(rng.choice(used)) for _ in range(m)], [int(s) for s in rng.permutation(empty)[:m]])
        if step % 2:
            x.call("free", [int(s) for s in rng.integers(0, slots, k)], lo, hi)
        if step % 4 == 3:
            x.compact()
    x.call("free", list(range(min(slots, 1024))), [0] * min(slots, 1024), [max_pages] * min(slots, 1024))
    assert not x.ref.ref.any()
    x.compact()


def test_flags(api):
    _, _, pg = api
    x = Both(pg, 6, 4, 9, 4, [8], [2], 0)
    x.call("assign", [0, 0, -1, 6, 1, 2, 3], [0, 0, 0, 0, 3, -1, 0], [3, 4, 1, 1, 2, 2, 5])
    x.set_lengths([10, 0, 0, 0, -1, 17])
    x.call("fork", [0, 0, 0, 6, -1, 4, 5, 1], [1, 1, 0, 2, 2, 2, 2, 6])      # a second copy into 1; onto itself; no such slot; bad lengths; into a source
    x.call("assign", [2, 3], [0, 0], [4, 4])                                 # the pool has five left: the second entry gets none
    x.call("fork", [0, 1], [4, 5], )
    x.call("free", [0, 7, 1, 0], [0, 0, 2, 0], [4, 1, 1, 4])
    x.compact()


def test_the_largest_list_and_none(api):
    _, _, pg = api
    x = Both(pg, 1500, 2, 3000, 4, [4], [1], 7)
    x.call("assign", list(range(1024)), [0] * 1024, [1] * 1024)
    x.set_lengths([3] * 1500)
    x.call("fork", [7] * 400, list(range(1024, 1424)))
    x.call("free", [])if False else x.call("free", [5], [0], [0])
    for f in ("assign", "free"):
        x.call(f, [], [], [])
    x.call("fork", [], [])
    tsv = api[0]
    with pytest.raises(tsv.TsvError) as e:
        x.call("free", list(range(1025)), [0] * 1025, [1] * 1025)
    assert e.value.code == tsv.ERR_LIMIT


@pytest.mark.parametrize("n_pages", [16384, 16385])       # (as many as stay in one CTA's registers, and one more)
def test_compaction_of_a_large_pool(api, n_pages):
    _, _, pg = api
    x = Both(pg, 256, 64, n_pages, 4, [4], [], 9)
    for half in (0, 1):
        x.call("assign", list(range(128 * half, 128 * half + 128)), [0] * 128, [64] * 128)
    gone = [int(v) for v in x.rng.permutation(256)[:150]]
    x.call("free", gone, [int(v) for v in x.rng.integers(0, 30, 150)], [int(v) for v in x.rng.integers(30, 65, 150)])
    x.compact()
    x.compact()                                           # (nothing moves)


def test_pages_beyond_32_bits(api):
    """A fork's copy and a compaction's move between pages that lie 6 GB apart."""
    _, _, pg = api
    n_pages, words = 6000, 1 << 18
    plane = torch.empty(n_pages, words, dtype=torch.int32, device="cuda")
    L = i32(5, 0, 0)
    pool = pg.PagePool(torch.full((3, 2), -1, dtype=torch.int32, device="cuda"), torch.ones(n_pages, dtype=torch.int32, device="cuda"), 4, [plane], [L])
    pool.page_table[0] = i32(7, 5990)
    pool.ref[5995] = 0
    plane[7], plane[5990] = 7, torch.arange(words, dtype=torch.int32, device="cuda")
    ws, status = pg.alloc_workspace(pool), i32(0)
    pg.pages_fork(pool, i32(0), i32(2), L, ws, status)
    assert not status.any() and pool.page_table[2].tolist() == [7, 5995] and torch.equal(plane[5995], plane[5990]) and L.tolist() == [5, 0, 5]
    pool.ref.zero_()
    pool.ref[7], pool.ref[5990], pool.ref[5995] = 2, 1, 1
    plane[5995] += 1
    n = i32(0)
    pg.pages_compact(pool, n, ws)
    assert n.tolist() == [3] and pool.ref[:3].tolist() == [2, 1, 1] and not pool.ref[3:].any()
    a, b = pool.page_table[0].tolist(), pool.page_table[2].tolist()
    assert a[0] == b[0] and sorted({a[0], a[1], b[1]}) == [0, 1, 2]
    assert (plane[a[0]] == 7).all() and torch.equal(plane[a[1]], torch.arange(words, dtype=torch.int32, device="cuda")) and torch.equal(plane[b[1]], plane[a[1]] + 1)


def test_many_planes(api):
    """More arrays than one launch's parameters hold."""
    _, _, pg = api
    x = Both(pg, 5, 6, 40, 4, [4 + 4 * (i % 5) for i in range(190)], [1 + i % 7 for i in range(150)], 8)
    x.call("assign", [0, 1, 2], [0, 0, 0], [6, 3, 1])
    x.set_lengths([21, 10, 4, 0, 0])
    x.call("fork", [0, 1], [3, 4])
    x.call("free", [0], [0], [6])
    x.compact()


def test_graph_and_stream(api):
    """Fork and free captured and replayed: the same children again."""
    _, _, pg = api
    x = Both(pg, 6, 5, 60, 8, [64], [3], 9)
    x.call("assign", [0, 1], [0, 0], [4, 5])
    x.set_lengths([27, 33, 0, 0, 0, 0])
    src, dst, zero, five, st = i32(0, 0, 1), i32(2, 3, 4), i32(0, 0, 0), i32(5, 5, 5), i32(0, 0, 0)
    x.call("fork", [0, 0, 1], [2, 3, 4])
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        pg.pages_free(x.pool, dst, zero, five, st)
        pg.pages_fork(x.pool, src, dst, x.L, x.ws, st)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert not st.any()
    x.same()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_forked_sequences_verify_alike(api, dtype):
    """The verify path over a forked sequence and over a compacted pool: with the same inputs parent and child give the same bits, cycle
    after cycle, each writing pages of its own; and what a child commits does not touch its parent."""
    tsv, _, pg = api
    from paper_2609_24698_b200 import harness as hz, synth
    from tests.helpers import oracle_states, state_arrays
    sh = synth.Shape("bf16", 3, 8, 64, 512, 4, 512, 4, 128, 128, 128) if dtype == "bf16" else synth.Shape("fp32", 3, 8, 16, 128, 4, 64, 1, 64, 128, 128)
    cfg = synth.Config("fork", 230, sh, layers=2, L_min=0, L_max=1000, seed=4)
    lengths = np.asarray([1000, 0, 300])
    states = oracle_states(cfg, lengths)
    ccap, hcap = hz.capacities(sh, [1000, 1000, 300], 64)
    eng = hz.VerifyEngine(sh, 2, ccap, hcap, 1200, page_tokens=128)
    for c in eng.caches[1:]:
        c.page_table = eng.caches[0].page_table           # one table for the stack (the pools have the same sizes)
    for l in range(2):
        for b in range(3):
            hz.fill_cache(eng.caches[l], sh, b, int(lengths[b]), state_arrays(states[l][b]))
    pool = pg.PagePool.of_layers(eng.caches)
    ws, st, n_used = pg.alloc_workspace(pool), i32(0), i32(-1)
    mp = pool.c.max_pages
    pg.pages_free(pool, i32(1), i32(0), i32(mp), st)
    pg.pages_fork(pool, i32(0), i32(1), eng.caches[0].L, ws, st)
    assert not st.any()
    table = eng.caches[0].page_table.cpu().numpy()
    assert (table[0, :7] == table[1, :7]).all() and table[0, 7] != table[1, 7] and pool.ref.max() == 2
    for cyc in range(5):
        nodes = [synth.node_inputs(cfg, l, cyc) for l in range(2)]
        parent, n_nodes = synth.trees(cfg, cyc)
        draft, target = synth.tokens(cfg, cyc, parent, n_nodes)
        for a in [parent, n_nodes, draft, target] + [x for nd in nodes for x in nd.values()]:
            a[1] = a[0]
        if cyc == 3:                                       # the child goes its own way: its parent must not notice
            target[1] = (target[1] + 1) % 32000
        eng.launch_cycle(hz.InputSet.from_numpy(sh, nodes, parent, n_nodes, draft, target))
        assert not eng.status.any()
        for o in eng.out:
            if cyc < 4:
                assert torch.equal(o[0], o[1]) and o[0].any()
        if cyc < 3:
            assert eng.accept_len[0] == eng.accept_len[1] and eng.caches[0].L[0] == eng.caches[0].L[1]
            for c in eng.caches:
                for name in ("csa_mx", "csa_s", "csa_acc_kv", "csa_acc_ik", "hca_mx", "hca_s", "hca_acc_kv"):
                    assert torch.equal(getattr(c, name)[0], getattr(c, name)[1])
        if cyc == 1:
            pg.pages_compact(pool, n_used, ws)
            assert int(n_used) == int((pool.ref > 0).sum()) and int(eng.caches[0].page_table.max()) == int(n_used) - 1
    # a fresh engine with the parent's history alone gives the parent's last outputs
    solo = hz.VerifyEngine(sh, 2, ccap, hcap, 1200)
    for l in range(2):
        for b in range(3):
            hz.fill_cache(solo.caches[l], sh, b, int(lengths[b]), state_arrays(states[l][b]))
    for cyc in range(5):
        nodes = [synth.node_inputs(cfg, l, cyc) for l in range(2)]
        parent, n_nodes = synth.trees(cfg, cyc)
        draft, target = synth.tokens(cfg, cyc, parent, n_nodes)
        solo.launch_cycle(hz.InputSet.from_numpy(sh, nodes, parent, n_nodes, draft, target))
    tol = 2e-2 if dtype == "bf16" else 1e-5              # (the parity tests' bounds: chunks of a paged list differ)
    for l in range(2):
        a, b = eng.out[l][0].float(), solo.out[l][0].float()
        assert (a - b).abs().max() <= tol * b.abs().max()
