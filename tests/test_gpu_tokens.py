"""Token-level operators on the GPU against the fp64 restatement: types, head layouts, lengths from none to long, windows, sinks,
rings and pages, chains and trees, strided rows, values that are not finite in places that are not seen, what the device flags.

Tolerances, per value (es: half a rounding step of the storage type relative to the value, 2^-8 or 2^-24):
  attention  |err| <= es |out| + A (ew + 2 es_score), A = sum_j p_j |v_j|: the weights are rounded to bf16 (ew = 2^-8; fp32: exp and
             the sums, 2^-20) and a score is off by at most (d + 4) 2^-24 times its sum of magnitudes (fp32 accumulation), which moves
             a weight by twice that relative to their sum.
  rotation   |err| <= es |y| + (|a| + |b|) (d 2^-24 + 2^-20): the sum of squares (at most d roundings, half of it after the root),
             the products, and cosines and sines to 2^-22.
"""
import numpy as np
import pytest
import torch

from oracle import tok_oracle as T

pytestmark = pytest.mark.gpu

STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


@pytest.fixture(scope="module")
def api():
    from paper_2609_24698_b200 import binding, pages, tokens
    return binding, tokens, pages


def f64(t):
    return t.double().cpu().numpy()


class Layer:
    """A random batch and cache.  Rows of no sequence and cache rows that no query sees hold NaN."""

    def __init__(self, tk, dtype, H, Hk, d, shared, window, sinks, L, n, tree=False, page=0, seed=0, gap=2, holes=False, fused=False, scale=0.0, extra_n=0):
        rng = self.rng = np.random.default_rng(seed)
        B = len(L)
        self.L, self.n, self.B = list(L), list(n), B
        self.shape = tk.TokenShape(dtype, B, H, Hk, d, window, sinks, max_L=max(a + b for a, b in zip(L, n)) + 3, max_n=max(max(n), 1) + extra_n, sm_scale=scale)
        dt = self.shape.torch_dtype
        order = rng.permutation(B)                       # sequences lie in the packed arrays in any order, with rows between them
        row0, at = [0] * B, gap
        for b in order:
            row0[b] = at
            at += n[b] + int(rng.integers(0, gap + 1))
        self.row0, self.rows = row0, at + gap
        self.parents = [[-1] + [int(rng.integers(0, i)) for i in range(1, k)] if k else [] for k in n] if tree else None
        par = None
        if tree:
            p = np.full(self.rows, 7, np.int32)
            for b in range(B):
                p[row0[b]:row0[b] + n[b]] = self.parents[b]
            par = torch.from_numpy(p).cuda()
        self.batch = tk.TokenBatch(torch.tensor(row0, dtype=torch.int64).cuda(), torch.tensor(n, dtype=torch.int32).cuda(), par)
        mine = np.zeros(self.rows, bool)
        for b in range(B):
            mine[row0[b]:row0[b] + n[b]] = True

        def packed(heads):
            x = rng.standard_normal((self.rows, heads, d)).astype(np.float32)
            x[~mine] = np.nan
            return torch.from_numpy(x).cuda().to(dt)
        if fused:
            w = (H + 2 * Hk) * d
            proj = torch.cat([packed(H).flatten(1), packed(Hk).flatten(1), packed(Hk).flatten(1)], 1).contiguous()
            assert proj.shape[1] == w
            self.q, self.k = proj[:, :H * d].unflatten(1, (H, d)), proj[:, H * d:(H + Hk) * d].unflatten(1, (Hk, d))
            self.v = None if shared else proj[:, (H + Hk) * d:].unflatten(1, (Hk, d))
        else:
            self.q, self.k, self.v = packed(H), packed(Hk), None if shared else packed(Hk)
        # history by position, then into the rows that some query sees
        self.hist_k = [torch.from_numpy(rng.standard_normal((l, Hk, d)).astype(np.float32)).to(dt) for l in L]
        self.hist_v = self.hist_k if shared else [torch.from_numpy(rng.standard_normal((l, Hk, d)).astype(np.float32)).to(dt) for l in L]
        if page:
            need = [max(1, -(-(a + b) // page)) for a, b in zip(L, n)]
            n_pages = sum(need) + 3
            ids = list(rng.permutation(n_pages))
            table = np.full((B, max(need) + 1), -1, np.int32)
            for b in range(B):
                for lp in range(need[b]):
                    lo, hi = lp * page, lp * page + page - 1
                    if holes and hi < L[b] - window + 1 and lo >= sinks:
                        continue                         # a page between sinks and window, given back
                    table[b, lp] = ids.pop()
            crows = n_pages * page
        else:
            table, crows = None, B * (sinks + window)
        ck = torch.full((crows, Hk, d), float("nan"), dtype=dt)
        cv = None if shared else ck.clone()
        for b in range(B):
            for pos in range(L[b]):
                if pos >= sinks and pos <= L[b] - window:
                    continue
                r = table[b, pos // page] * page + pos % page if page else T.ring_row(b, pos, sinks, window)
                ck[r] = self.hist_k[b][pos]
                if cv is not None:
                    cv[r] = self.hist_v[b][pos]
        self.cache = tk.TokenCache(torch.tensor(L, dtype=torch.int32).cuda(), ck.cuda(), None if cv is None else cv.cuda(),
                                   None if table is None else torch.from_numpy(table).cuda(), page)
        self.table, self.page = table, page
        self.scale = scale if scale > 0 else d ** -0.5
        self.status = torch.zeros(B, dtype=torch.int32, device="cuda")

    def run(self, tk, out=None):
        out = torch.full((self.rows, self.shape.H, self.shape.d), 3.0, dtype=self.shape.torch_dtype, device="cuda") if out is None else out
        ws = tk.alloc_workspace(self.shape, self.rows)
        tk.window_sink_attn(self.shape, self.cache, self.batch, self.q, self.k, self.v, out, ws, self.status)
        return out

    def ref(self, b):
        r = slice(self.row0[b], self.row0[b] + self.n[b])
        v = self.k if self.v is None else self.v
        return T.attend(f64(self.q[r]), f64(self.k[r]), f64(v[r]), f64(self.hist_k[b]), f64(self.hist_v[b]), self.shape.window, self.shape.n_sink,
                        self.scale, self.parents[b] if self.parents else None)

    def check(self, out, status=0):
        es, d = STEP[self.shape.dtype], self.shape.d
        got, used = f64(out), np.zeros(self.rows, bool)
        for b in range(self.B):
            r = slice(self.row0[b], self.row0[b] + self.n[b])
            used[r] = True
            if not self.n[b]:
                continue
            ref, mag, reach = self.ref(b)
            tol = es * np.abs(ref) + mag * (2.0 ** -8 if self.shape.dtype == "bf16" else 2.0 ** -20) + mag * 2 * ((d + 4) * 2.0 ** -24 * reach)[..., None] + 1e-30
            err = np.abs(got[r] - ref)
            assert (np.isfinite(ref) == np.isfinite(got[r])).all()
            assert (err <= tol)[np.isfinite(ref)].all(), f"sequence {b}: {np.nanmax(err / tol):.3g} of the tolerance"
        assert (got[~used] == 3.0).all(), "rows of no sequence were written"
        assert (self.status.cpu().numpy() == status).all()


HEADS = [("bf16", 64, 1, 512, True), ("bf16", 8, 2, 128, False), ("fp32", 16, 1, 128, True)]
ODD_HEADS = [("bf16", 3, 1, 8, True), ("bf16", 5, 5, 72, False), ("bf16", 12, 2, 96, False), ("bf16", 7, 1, 200, True), ("bf16", 6, 2, 264, False),
             ("bf16", 4, 1, 512, False), ("fp32", 6, 3, 40, False), ("fp32", 5, 1, 264, True), ("fp32", 4, 2, 512, False), ("bf16", 20, 4, 80, False),
             ("bf16", 64, 64, 64, False), ("bf16", 256, 1, 64, True)]


@pytest.mark.parametrize("heads", HEADS + ODD_HEADS, ids=lambda h: "_".join(map(str, h)))
@pytest.mark.parametrize("tree", [False, True])
def test_head_layouts(api, heads, tree):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=37, sinks=3, L=[0, 1, 36, 90], n=[5, 1, 7, 4], tree=tree, page=16 if tree else 0, seed=hash(heads) % 1000)
    lay.check(lay.run(tk))


# the same heads with more rows for a key head than a small tile has
@pytest.mark.parametrize("heads", [h for h in HEADS + ODD_HEADS if h[0] == "bf16"], ids=lambda h: "_".join(map(str, h)))
@pytest.mark.parametrize("tree", [False, True])
def test_head_layouts_with_more_rows(api, heads, tree):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=37, sinks=3, L=[0, 1, 36, 90], n=[18, 1, 32 if tree else 47, 0], tree=tree, page=0 if tree else 24, seed=hash(heads) % 1000)
    lay.check(lay.run(tk))


# window, sinks: one position; no sinks; sinks that reach into the window, into the new tokens, beyond everything; a window beyond everything
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 2), (5, 0), (16, 40), (33, 4), (64, 1), (500, 0), (500, 600), (2 ** 30, 0)])
@pytest.mark.parametrize("heads", [("bf16", 8, 2, 64, False), ("bf16", 4, 1, 512, True), ("fp32", 4, 1, 64, True)], ids=lambda h: "_".join(map(str, h)))
def test_windows_and_sinks(api, window, sinks, heads):
    _, tk, _ = api
    for tree in (False, True):
        lay = Layer(tk, *heads, window=window, sinks=sinks, L=[0, 3, 70, 130, 200], n=[9, 1, 12, 0, 31], tree=tree, page=8 if tree or window > 1000 else 0,
                    seed=window + sinks)
        lay.check(lay.run(tk))


# pages that end inside a block of keys, pages of one token, pages given back between sinks and window
@pytest.mark.parametrize("page", [1, 3, 16, 64, 100])
@pytest.mark.parametrize("heads", [HEADS[1], HEADS[2], ("bf16", 8, 1, 512, True)], ids=lambda h: "_".join(map(str, h)))
def test_pages(api, page, heads):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=50, sinks=2, L=[300, 49, 128, 7], n=[3, 66, 1, 20], page=page, seed=page, holes=True)
    lay.check(lay.run(tk))


# a token or two of many sequences, some of them of none; lists of many keys
@pytest.mark.parametrize("heads,L,n,window", [
    (("bf16", 16, 1, 512, True), [3 * i for i in range(70)], [(1, 2, 1, 0)[i % 4] for i in range(70)], 60),
    (("bf16", 6, 2, 264, False), [5 * i % 97 for i in range(40)], [1] * 40, 33),
    (("bf16", 3, 1, 256, True), [i for i in range(66)], [(1, 4)[i % 2] for i in range(66)], 128), (("bf16", 2, 1, 200, True), [17000, 50], [1, 2], 16900),
    (("bf16", 4, 1, 512, False), [16700], [1], 16500)], ids=lambda x: "" if isinstance(x, list) else str(x))
@pytest.mark.parametrize("page", [0, 16])
def test_single_tokens(api, heads, L, n, window, page):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=window, sinks=4, L=L, n=n, page=page, seed=len(L))
    lay.check(lay.run(tk))


# the same pages at the end of a pool of more than 2^32 elements
@pytest.mark.parametrize("heads", [("bf16", 64, 1, 512, True), ("bf16", 8, 2, 128, False), ("fp32", 4, 1, 256, True)], ids=lambda h: "_".join(map(str, h)))
@pytest.mark.parametrize("n", [[1, 1], [40, 90]])
def test_pages_beyond_32_bits(api, heads, n):
    _, tk, _ = api
    page = 32
    lay = Layer(tk, *heads, window=50, sinks=2, L=[300, 45], n=n, page=page, seed=6)
    want = lay.run(tk)
    small = [t for t in (lay.cache.k, lay.cache.v) if t is not None]
    rows, row = small[0].shape[0], lay.shape.Hk * lay.shape.d
    first = ((1 << 32) // row // page + 1) * page
    big = []
    for t in small:
        x = torch.empty(first + rows, *t.shape[1:], dtype=t.dtype, device="cuda")
        x[first:] = t
        big.append(x)
    assert first * row >= 1 << 32
    table = torch.where(lay.cache.page_table >= 0, lay.cache.page_table + first // page, -1).int()
    lay.cache = tk.TokenCache(lay.cache.L, big[0], big[1] if len(big) > 1 else None, table, page)
    assert torch.equal(lay.run(tk).nan_to_num(9), want.nan_to_num(9))
    tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status)
    assert not lay.status.any()
    for b, L in enumerate(lay.L):
        pos = torch.arange(L, L + n[b])
        at = (table[b].cpu()[pos // page].long() * page + pos % page).cuda()
        for x, src in zip(big, (lay.k, lay.v)):
            assert torch.equal(x[at], src[lay.row0[b]:lay.row0[b] + n[b]])


# many tokens: tiles of queries that begin and end inside tokens, prompts with and without history
@pytest.mark.parametrize("heads,window,L,n", [
    (("bf16", 6, 2, 64, False), 70, [0, 45, 200], [333, 130, 257]), (("bf16", 5, 1, 128, True), 129, [0, 5], [300, 201]),
    (("bf16", 64, 1, 512, True), 20, [0, 33], [21, 9]), (("bf16", 4, 4, 128, False), 400, [10, 0], [450, 128]),
    (("bf16", 3, 1, 256, False), 90, [100, 0], [140, 127]), (("fp32", 4, 2, 64, False), 60, [0, 30], [130, 65])], ids=str)
@pytest.mark.parametrize("page", [0, 32])
def test_prompts(api, heads, window, L, n, page):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=window, sinks=4, L=L, n=n, page=page, seed=window, fused=True)
    lay.check(lay.run(tk))


# long windows at a few rows: keys split over CTAs and joined, some shares empty
@pytest.mark.parametrize("heads,window,L,n,tree", [
    (("bf16", 8, 2, 128, False), 5000, [6000, 100], [1, 2], False), (("bf16", 16, 1, 512, True), 3000, [2900], [5], True),
    (("bf16", 64, 1, 512, True), 2000, [2500, 64, 0], [1, 3, 1], False), (("fp32", 16, 1, 128, True), 2000, [1900, 3], [1, 4], False),
    (("bf16", 4, 1, 64, True), 3500, [4000], [3], False)], ids=str)
def test_long_windows(api, heads, window, L, n, tree):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=window, sinks=5, L=L, n=n, tree=tree, page=64, seed=window)
    lay.check(lay.run(tk))


@pytest.mark.parametrize("heads", [("bf16", 8, 2, 64, False), ("bf16", 8, 1, 512, True), ("fp32", 4, 1, 64, True), ("bf16", 16, 1, 128, False)],
                         ids=lambda h: "_".join(map(str, h)))
@pytest.mark.parametrize("n", [6, 150])
def test_what_is_not_seen_has_no_influence(api, heads, n):
    """NaN and infinities in the keys and values of a token: earlier tokens (same tile) and those beyond its window are as without; those that see it
    have what the formula gives."""
    _, tk, _ = api
    for bad in (float("nan"), float("inf"), -float("inf")):
        lay = Layer(tk, *heads, window=40, sinks=1, L=[20, 0], n=[n, 3], seed=n)
        at = n // 2
        clean = lay.run(tk).clone()
        lay.k[lay.row0[0] + at, -1, 1] = bad
        if lay.v is not None:
            lay.v[lay.row0[0] + at, :, 3] = bad
        out = lay.run(tk)
        got, was = f64(out), f64(clean)
        r0 = lay.row0[0]
        assert (got[r0:r0 + at] == was[r0:r0 + at]).all()
        if n > at + 40:
            assert (got[r0 + at + 40:r0 + n] == was[r0 + at + 40:r0 + n]).all()
        ref, _, _ = lay.ref(0)
        assert (np.isfinite(ref) == np.isfinite(got[r0:r0 + n])).all()
        ok = np.isfinite(ref)
        assert np.abs(got[r0:r0 + n] - ref)[ok].max() < 0.1


@pytest.mark.parametrize("heads", [("bf16", 64, 1, 512, True), ("bf16", 8, 1, 512, False), ("bf16", 32, 1, 128, True)], ids=lambda h: "_".join(map(str, h)))
def test_infinite_scores_in_split_keys(api, heads):
    """A key with an infinite value: some rows' score of it is -infinity (no weight), others' is +infinity, and all shares of a row's keys agree."""
    _, tk, _ = api
    for bad in (float("inf"), -float("inf")):
        lay = Layer(tk, *heads, window=3000, sinks=1, L=[3100], n=[8], seed=5)
        lay.k[lay.row0[0] + 2, -1, 1] = bad
        got = f64(lay.run(tk))[lay.row0[0]:lay.row0[0] + 8]
        ref, mag, _ = lay.ref(0)
        ok = np.isfinite(ref)
        assert (ok == np.isfinite(got)).all()
        assert not ok[2:].all() and ok[2:].any()
        # (a rounding of each weight, of the result, and of fp32 sums of 3 k terms)
        assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -8 * mag + 1e-3 * mag)[ok].all()
        assert not lay.status.any()


# rows computed one by one, some tenths of a second of them in front of a CTA's next tile
@pytest.mark.parametrize("heads,L,n", [(("bf16", 16, 1, 64, False), 0, 4900), (("bf16", 64, 1, 512, True), 7000, 310)], ids=str)
def test_nan_that_all_rows_of_a_long_window_see(api, heads, L, n):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=20000, sinks=0, L=[L], n=[n], seed=1)
    clean = lay.run(tk).clone()
    (lay.k if lay.v is None else lay.v)[lay.row0[0], 0, 3] = float("nan")
    out = lay.run(tk)
    r = slice(lay.row0[0], lay.row0[0] + n)
    assert not lay.status.any()
    got, was = out[r].float(), clean[r].float()
    assert got[..., 3].isnan().all()
    if lay.v is None:
        assert got.isnan().all()                          # (every score of that key)
    else:
        got[..., 3] = was[..., 3]
        # two results, each within a rounding of the weights and of itself (values of up to 6)
        assert ((got - was).abs() <= 2 * (2.0 ** -8 * 6 + 2.0 ** -8 * was.abs())).all()


def test_large_scores(api):
    """Scores far apart: one key decides, and the reference of the softmax moves from block to block."""
    _, tk, _ = api
    for heads in (("bf16", 8, 2, 64, False), ("bf16", 8, 1, 512, True), ("fp32", 4, 1, 64, True)):
        lay = Layer(tk, *heads, window=300, sinks=4, L=[400, 90], n=[5, 130], seed=5, scale=3.0)
        lay.check(lay.run(tk))


def test_a_row_whose_scores_are_all_minus_infinity(api):
    _, tk, _ = api
    lay = Layer(tk, "bf16", 4, 2, 64, False, window=9, sinks=0, L=[0], n=[4], seed=1)
    lay.q[lay.row0[0]] = 1.0
    lay.k[lay.row0[0], :, 0] = -float("inf")
    got = f64(lay.run(tk))
    assert np.isnan(got[lay.row0[0]]).all()              # exp(-inf - -inf)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [0, 4])
def test_flags(api, dtype, page):
    """What the device finds wrong with a sequence: its rows are zeros (where they can be), the others' results stand."""
    tsv, tk, _ = api
    mk = lambda: Layer(tk, dtype, 4, 2, 64, False, window=20, sinks=2, L=[30, 8, 15, 40], n=[5, 4, 6, 3], tree=True, page=page, seed=3)
    lay = mk()
    good = f64(lay.run(tk))
    lay.check(lay.run(tk))
    for b, change, flag, rows in [(1, "n", tsv.ST_NODES, "left"), (2, "neg", tsv.ST_NODES, "left"), (0, "row0", tsv.ST_NODES, "left"), (3, "far", tsv.ST_NODES, "left"),
                                  (2, "L", tsv.ST_LENGTH, "zero"), (3, "longL", tsv.ST_LENGTH, "zero"), (0, "parent", tsv.ST_PARENT, "zero"), (1, "root", tsv.ST_PARENT, "zero")]:
        lay = mk()
        if change == "n":
            lay.batch.n[b] = lay.shape.max_n + 1
        elif change == "neg":
            lay.batch.n[b] = -1
        elif change == "row0":
            lay.batch.row0[b] = -1
        elif change == "far":
            lay.batch.row0[b] = lay.rows - 1
        elif change == "L":
            lay.cache.L[b] = -5
        elif change == "longL":
            lay.cache.L[b] = lay.shape.max_L
        elif change == "parent":
            lay.batch.parent[lay.row0[b] + 2] = 2
        else:
            lay.batch.parent[lay.row0[b]] = 0
        got = f64(lay.run(tk))
        st = lay.status.cpu().numpy()
        assert st[b] == flag and (np.delete(st, b) == 0).all(), (change, st)
        r = slice(lay.row0[b], lay.row0[b] + lay.n[b])
        assert (got[r] == (3.0 if rows == "left" else 0.0)).all(), change
        others = np.ones(lay.rows, bool)
        others[r] = False
        assert (got[others] == good[others]).all(), change
        # the rotation finds the same, and the commit leaves the sequence alone
        st2, q, k = torch.zeros_like(lay.status), torch.full_like(lay.q, 3.0), torch.full_like(lay.k, 3.0)
        inv = 10000.0 ** -torch.arange(0, 1, 2 / 32, device="cuda")
        tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, lay.k, q, k, None, None, 1e-6, inv, 0, False, st2)
        assert st2[b] == flag and (f64(q)[r] == (3.0 if rows == "left" else 0.0)).all() and (f64(k)[r] == (3.0 if rows == "left" else 0.0)).all(), change
        if "arent" not in change and change != "root":   # (a commit does not look at the tree)
            st3, L0 = torch.zeros_like(lay.status), lay.cache.L.clone()
            tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, st3)
            assert st3[b] == flag and lay.cache.L[b] == L0[b] and (lay.cache.L - L0).sum() == sum(lay.n) - lay.n[b], change


def test_missing_pages(api):
    tsv, tk, _ = api
    for dtype in ("bf16", "fp32"):
        for bad in (-1, 10 ** 6, -7):
            lay = Layer(tk, dtype, 4, 2, 64, False, window=20, sinks=2, L=[30, 38], n=[2, 2], page=8, seed=4)
            lay.cache.page_table[1, 3] = bad             # positions 24 .. 31
            out = lay.run(tk)
            assert lay.status.tolist() == [0, 64]
            # what is there decides: as a sequence whose history has a gap
            got = f64(out)
            hk, hv = f64(lay.hist_k[1]), f64(lay.hist_v[1])
            for i in range(2):
                p = 38 + i
                js = [j for j in range(38) if (j > p - 20 or j < 2) and not 24 <= j < 32]
                K = np.concatenate([hk[js], f64(lay.k)[lay.row0[1]:lay.row0[1] + i + 1]])
                V = np.concatenate([hv[js], f64(lay.v)[lay.row0[1]:lay.row0[1] + i + 1]])
                for h in range(4):
                    s = K[:, h // 2] @ f64(lay.q)[lay.row0[1] + i, h] / 8
                    w = np.exp(s - s.max())
                    assert np.abs(got[lay.row0[1] + i, h] - (w[:, None] * V[:, h // 2]).sum(0) / w.sum()).max() < 0.03
            L0 = lay.cache.L.clone()
            lay.status.zero_()
            lay.cache.page_table[1, 4] = bad             # the page of positions 38, 39
            tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status)
            assert lay.status.tolist() == [0, 64] and (lay.cache.L - L0).tolist() == [2, 0]


def test_no_tokens_at_all(api):
    _, tk, _ = api
    lay = Layer(tk, "bf16", 4, 2, 64, False, window=20, sinks=2, L=[3, 0], n=[0, 0], gap=0)
    lay.q = lay.q.new_empty(0, 4, 64)
    lay.k, lay.v, lay.rows = lay.k.new_empty(0, 2, 64), lay.v.new_empty(0, 2, 64), 0
    lay.run(tk)
    assert lay.status.tolist() == [0, 0]


def test_many_sequences(api):
    """More sequences than a warp looks over at a time, many of them without tokens."""
    _, tk, _ = api
    rng = np.random.default_rng(8)
    n = [int(x) for x in rng.integers(0, 3, 150)]
    lay = Layer(tk, "bf16", 4, 2, 64, False, window=12, sinks=1, L=[int(x) for x in rng.integers(0, 40, 150)], n=n, seed=9, extra_n=70)
    lay.check(lay.run(tk))


# more tiles than SMs, of one and of two halves, with a block of keys or several, in any order
@pytest.mark.parametrize("heads,window", [(("bf16", 32, 1, 64, True), 20), (("bf16", 64, 2, 128, False), 150), (("bf16", 64, 1, 128, True), 200),
                                          (("bf16", 40, 1, 72, False), 140), (("bf16", 32, 2, 256, False), 150), (("bf16", 64, 1, 512, True), 160)], ids=str)
@pytest.mark.parametrize("tree", [False, True])
def test_many_tiles(api, heads, window, tree):
    _, tk, _ = api
    rng = np.random.default_rng(window)
    B = 260 if heads[3] <= 128 else 170
    n = [int(x) for x in rng.integers(0, 12, B)]
    lay = Layer(tk, *heads, window=window, sinks=2, L=[int(x) for x in rng.integers(0, 300, B)], n=n, tree=tree, page=32 if tree else 0, seed=9)
    out = lay.run(tk)
    pick = sorted(int(b) for b in rng.permutation(B)[:40])           # (the restatement takes its time)
    es = STEP["bf16"]
    got = f64(out)
    assert not lay.status.any() and np.isfinite(got[~np.isnan(f64(lay.q)).any((1, 2))]).all()
    for b in pick:
        if n[b]:
            r = slice(lay.row0[b], lay.row0[b] + n[b])
            ref, mag, reach = lay.ref(b)
            tol = es * np.abs(ref) + mag * 2.0 ** -8 + mag * 2 * ((heads[3] + 4) * 2.0 ** -24 * reach)[..., None] + 1e-30
            assert (np.abs(got[r] - ref) <= tol).all(), b


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1], HEADS[2]], ids=lambda h: "_".join(map(str, h)))
def test_repeated_overlapping_and_replayed_calls(api, heads):
    """Bits do not depend on the run, on what is in the workspace, on the stream, on another call at the same time, or on a graph."""
    _, tk, _ = api
    mk = lambda s: Layer(tk, *heads, window=600, sinks=3, L=[700, 20], n=[3, 140], seed=s)
    a, b = mk(1), mk(2)
    ra, rb = a.run(tk).clone(), b.run(tk).clone()
    ws = [tk.alloc_workspace(x.shape, x.rows) for x in (a, b)]
    for w in ws:
        w.fill_(0xff)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.full_like(r, 3.0) for r in (ra, rb)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, w, s, o in zip((a, b), ws, streams, outs):
            tk.window_sink_attn(x.shape, x.cache, x.batch, x.q, x.k, x.v, o, w, x.status, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0].nan_to_num(9), ra.nan_to_num(9)) and torch.equal(outs[1].nan_to_num(9), rb.nan_to_num(9))
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        tk.window_sink_attn(a.shape, a.cache, a.batch, a.q, a.k, a.v, outs[0], ws[0], a.status)
    outs[0].fill_(3.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0].nan_to_num(9), ra.nan_to_num(9))
    a.cache.L.fill_(25)                                   # the graph reads the lengths of its replay
    a.L = [25, 25]
    g.replay()
    torch.cuda.synchronize()
    assert not torch.equal(outs[0].nan_to_num(9), ra.nan_to_num(9))


# ----------------------------------------------------------------------------- norms and rotation
@pytest.mark.parametrize("dtype,H,Hk,d,rot,first", [
    ("bf16", 64, 1, 512, 64, 448), ("bf16", 8, 2, 128, 128, 0), ("bf16", 3, 1, 72, 64, 8), ("bf16", 5, 5, 40, 16, 16), ("bf16", 9, 3, 8, 0, 0), ("bf16", 2, 1, 200, 32, 96),
    ("bf16", 256, 4, 64, 64, 0), ("fp32", 16, 1, 128, 128, 0), ("fp32", 5, 1, 72, 32, 40), ("fp32", 3, 3, 512, 512, 0), ("fp32", 2, 1, 264, 16, 248), ("fp32", 4, 2, 16, 16, 0)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("form", ["tree", "chain", "fused"])
def test_norm_rope(api, dtype, H, Hk, d, rot, first, pairs, form):
    _, tk, _ = api
    L = [0, 1, 131071, 77] if form != "tree" else [5, 2 ** 29, 0, 1]
    lay = Layer(tk, dtype, H, Hk, d, form != "fused", window=1, sinks=0, L=[0] * 4, n=[3, 0, 19, 6], tree=form == "tree", seed=d + rot, fused=form == "fused")
    lay.shape = tk.TokenShape(dtype, 4, H, Hk, d, 1, max_L=1 << 30, max_n=19)
    lay.cache.L.copy_(torch.tensor(L, dtype=torch.int32))
    rng = np.random.default_rng(d)
    wq, wk = (torch.from_numpy(rng.uniform(0.5, 1.5, d).astype(np.float32)).cuda() for _ in range(2))
    inv = torch.from_numpy((10000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))).astype(np.float32)).cuda() if rot else None
    lay.q[lay.row0[2] + 1] *= 1e-4                        # (where eps counts)
    qo, ko = torch.full((lay.rows, H, d), 3.0, dtype=lay.shape.torch_dtype, device="cuda"), torch.full((lay.rows, Hk, d), 3.0, dtype=lay.shape.torch_dtype, device="cuda")
    q0, k0 = lay.q.clone(), lay.k.clone()
    tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, lay.k, qo, ko, wq, None if form == "chain" else wk, 1e-6, inv, first, pairs, lay.status)
    es = STEP[dtype]
    used = np.zeros(lay.rows, bool)
    for b in range(4):
        r = slice(lay.row0[b], lay.row0[b] + lay.n[b])
        used[r] = True
        depth, _ = T.depths_and_kin(lay.n[b], lay.parents[b] if lay.parents else None)
        for got, x, w in ((qo, q0, wq), (ko, k0, None if form == "chain" else wk)):
            if not lay.n[b]:
                continue
            ref, mag = T.norm_rope(f64(x[r]), None if w is None else f64(w), float(np.float32(1e-6)), [L[b] + e for e in depth], f64(inv) if rot else np.zeros(0), first, pairs)
            err, tol = np.abs(f64(got[r]) - ref), es * np.abs(ref) + mag * (d * 2.0 ** -24 + 2.0 ** -20) + 1e-30
            assert (err <= tol).all(), f"{(err / tol).max():.3g} of the tolerance"
    assert (f64(qo)[~used] == 3.0).all() and (f64(ko)[~used] == 3.0).all() and not lay.status.any()
    # in place, queries alone, keys alone: the same bits
    tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, None, lay.q, None, wq, None, 1e-6, inv, first, pairs, lay.status)
    tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, None, lay.k, None, lay.k, None, None if form == "chain" else wk, 1e-6, inv, first, pairs, lay.status)
    assert torch.equal(lay.q[torch.from_numpy(used).cuda()], qo[torch.from_numpy(used).cuda()]) and torch.equal(lay.k[torch.from_numpy(used).cuda()], ko[torch.from_numpy(used).cuda()])


def test_norm_rope_of_many_tokens(api):
    """Enough tokens that a CTA takes eight of them; lengths that leave its last one short."""
    _, tk, _ = api
    for dtype, H, Hk, d in (("bf16", 4, 2, 64), ("fp32", 2, 1, 128)):
        lay = Layer(tk, dtype, H, Hk, d, True, window=1, sinks=0, L=[0, 0, 0], n=[2501, 3, 2700], seed=3)
        lay.shape = tk.TokenShape(dtype, 3, H, Hk, d, 1, max_L=1 << 20, max_n=4000)
        inv = (10000.0 ** -torch.arange(0, 1, 2 / d, device="cuda")).float()
        qo, ko = torch.full_like(lay.q, 3.0), torch.full_like(lay.k, 3.0)
        tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, lay.k, qo, ko, None, None, 1e-6, inv, 0, True, lay.status)
        for b in range(3):
            for i in [0, 1, 2, 1250, 2499, 2500, 2699]:
                if i >= lay.n[b]:
                    continue
                r = slice(lay.row0[b] + i, lay.row0[b] + i + 1)
                for got, x in ((qo, lay.q), (ko, lay.k)):
                    ref, mag = T.norm_rope(f64(x[r]), None, float(np.float32(1e-6)), [i], f64(inv), 0, True)
                    assert (np.abs(f64(got[r]) - ref) <= STEP[dtype] * np.abs(ref) + mag * (d * 2.0 ** -24 + 2.0 ** -20)).all()


# ----------------------------------------------------------------------------- commit
@pytest.mark.parametrize("dtype,Hk,d,shared", [("bf16", 1, 512, True), ("bf16", 2, 72, False), ("fp32", 1, 8, False)])
@pytest.mark.parametrize("page", [0, 1, 7, 32])
@pytest.mark.parametrize("n,window", [([4, 0, 6, 1], 5), ([130, 0, 3, 64], 20)])
@pytest.mark.parametrize("paths", [False, True])
def test_commit(api, dtype, Hk, d, shared, page, n, window, paths):
    _, tk, _ = api
    L, sinks = [0, 9, 30, 2], 3
    lay = Layer(tk, dtype, Hk, Hk, d, shared, window=window, sinks=sinks, L=L, n=n, page=page, seed=sum(n) + page, fused=True)
    rng = np.random.default_rng(1)
    path = count = None
    if paths:
        want = [sorted(rng.choice(k, size=int(rng.integers(0, k + 1)), replace=False)) if k else [] for k in n]
        path = torch.tensor([w + [-1] * (max(n) - len(w)) for w in [[int(x) for x in w] for w in want]], dtype=torch.int32).cuda()
        count = torch.tensor([len(w) for w in want], dtype=torch.int32).cuda()
    else:
        want = [range(k) for k in n]
    bufs = [lay.cache.k] + ([] if shared else [lay.cache.v])
    exp = [b.clone() for b in bufs]
    for b in range(4):
        for i, node in enumerate(want[b]):
            pos = L[b] + i
            row = lay.table[b, pos // page] * page + pos % page if page else T.ring_row(b, pos, sinks, window)
            for e, src in zip(exp, [lay.k, lay.v]):
                e.view(-1, Hk, d)[row] = src[lay.row0[b] + int(node)]
    tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status, path=path, count=count)
    for x, e in zip(bufs, exp):
        assert torch.equal(x.nan_to_num(9), e.nan_to_num(9))
    assert lay.cache.L.tolist() == [a + len(w) for a, w in zip(L, want)] and not lay.status.any()


@pytest.mark.parametrize("Hk,shared", [(48, False), (24, True)])
def test_commit_of_wide_rows(api, Hk, shared):
    """Rows of keys and values that a CTA's shared memory holds none of, or one."""
    _, tk, _ = api
    lay = Layer(tk, "fp32", Hk, Hk, 512, shared, window=4, sinks=0, L=[3, 0, 9], n=[70, 0, 2], page=16, seed=1)
    exp = [x.clone() for x in [lay.cache.k] + ([] if shared else [lay.cache.v])]
    for b in range(3):
        for i in range(lay.n[b]):
            pos = lay.L[b] + i
            for e, src in zip(exp, [lay.k, lay.v]):
                e[lay.table[b, pos // 16] * 16 + pos % 16] = src[lay.row0[b] + i]
    tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status)
    for x, e in zip([lay.cache.k] + ([] if shared else [lay.cache.v]), exp):
        assert torch.equal(x.nan_to_num(9), e.nan_to_num(9))
    assert lay.cache.L.tolist() == [73, 0, 11] and not lay.status.any()


@pytest.mark.parametrize("big", [False, True])
def test_commit_flags(api, big):
    tsv, tk, _ = api
    n = [80, 5, 0] if big else [4, 5, 0]
    for what in ("count", "negative", "wide", "node", "low", "early", "none"):
        lay = Layer(tk, "bf16", 2, 2, 64, False, window=10, sinks=1, L=[4, 9, 2], n=n, seed=2)
        path = torch.arange(90, dtype=torch.int32, device="cuda").expand(3, 90).contiguous()
        count = torch.tensor([2, 3, 0], dtype=torch.int32, device="cuda")
        bad = 1
        if what == "count":
            count[1] = 6
        elif what == "negative":
            count[1] = -1
        elif what == "wide":
            path, count[1] = path[:, :3].contiguous(), 4
        elif what == "node":
            path[1, 2] = 5
        elif what == "low":
            path[1, 0] = -1
        elif what == "early":
            lay.status[1] = tsv.ST_CSA_CAP
        else:
            count[2], bad = 1, 2
        before = lay.cache.k.clone()
        tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status, path=path, count=count)
        grow = [2, 3, 0]
        grow[bad] = 0
        assert lay.cache.L.tolist() == [4 + grow[0], 9 + grow[1], 2 + grow[2]], what
        st = lay.status.tolist()
        assert st[bad] == (tsv.ST_CSA_CAP if what == "early" else tsv.ST_NODES) and sum(st) == st[bad], what
        assert torch.equal(lay.cache.k.view(3, -1)[bad].nan_to_num(9), before.view(3, -1)[bad].nan_to_num(9)), what


# ----------------------------------------------------------------------------- a run of them
@pytest.mark.parametrize("dtype,H,Hk,d,shared,page", [("bf16", 8, 2, 64, False, 8), ("bf16", 16, 1, 128, True, 0), ("fp32", 4, 1, 64, True, 4)])
def test_a_drafter_layer(api, dtype, H, Hk, d, shared, page):
    """Prompts, single tokens and a draft tree with its accepted path through one layer, as a server runs them: norms and rotation from the
    fused projection, attention, commit, with pages handed out as the sequences grow and given back behind the window.  Against the fp64
    restatement of the whole history (on the device's own rotated vectors)."""
    _, tk, pg = api
    rng = np.random.default_rng(6)
    B, window, sinks, steps = 3, 24, 2, [[37, 5, 0], [1, 1, 1], [1, 1, 9], "tree", [1, 30, 1], "tree", [2, 0, 1]]
    shape = tk.TokenShape(dtype, B, H, Hk, d, window, sinks, max_L=256, max_n=40)
    dt = shape.torch_dtype
    inv = (10000.0 ** -torch.arange(0, 1, 2 / 32, device="cuda")).float()
    w = torch.from_numpy(rng.uniform(0.5, 1.5, d).astype(np.float32)).cuda()
    ones = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    if page:
        cache = tk.alloc_token_pool(shape, 40, page, 64, values=not shared)
        pool = pg.PagePool(cache.page_table, torch.zeros(40, dtype=torch.int32, device="cuda"), page, [cache.k] + ([] if shared else [cache.v]), [cache.L])
        pws = pg.alloc_workspace(pool)
    else:
        cache = tk.alloc_token_cache(shape, values=not shared)
    hk, hv = [[] for _ in range(B)], [[] for _ in range(B)]
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    es = STEP[dtype]
    for step in steps:
        tree = step == "tree"
        n = [6, 4, 7] if tree else step
        L = cache.L.tolist()
        rows = sum(n)
        row0 = [sum(n[:b]) for b in range(B)]
        parents = [[-1] + [int(rng.integers(0, i)) for i in range(1, k)] for k in n] if tree else None
        batch = tk.TokenBatch(torch.tensor(row0, dtype=torch.int64).cuda(), ones(*n), ones(*sum(parents, [])) if tree else None)
        if page:
            need = ones(*[-(-(a + b) // page) for a, b in zip(L, n)])
            first = ones(*[a // page for a in L])
            pg.pages_assign(pool, ones(0, 1, 2), first, need, pws, status)
        proj = torch.from_numpy(rng.standard_normal((rows, (H + 2 * Hk) * d)).astype(np.float32)).cuda().to(dt)
        q, k, v = (x.unflatten(1, (-1, d)) for x in proj.split([H * d, Hk * d, Hk * d], 1))
        v = None if shared else v
        tk.qk_norm_rope(shape, cache.L, batch, q, k, q, k, w, w, 1e-6, inv, d - 32, False, status)
        out = torch.empty(rows, H, d, dtype=dt, device="cuda")
        tk.window_sink_attn(shape, cache, batch, q, k, v, out, tk.alloc_workspace(shape, rows), status)
        path = count = None
        picks = [list(range(x)) for x in n]
        if tree:
            picks = []
            for p in parents:
                at, way = 0, [0]
                while True:
                    below = [i for i in range(len(p)) if p[i] == at]
                    if not below:
                        break
                    at = below[0]
                    way.append(at)
                picks.append(way)
            path, count = ones(*[x for wy in picks for x in wy + [-1] * (8 - len(wy))]).view(B, 8), ones(*[len(x) for x in picks])
        tk.token_commit(shape, cache, batch, k, v, status, path=path, count=count)
        assert not status.any()
        for b in range(B):
            if not n[b]:
                continue
            r = slice(row0[b], row0[b] + n[b])
            K, V = f64(k[r]), f64((k if v is None else v)[r])
            old = lambda h: np.array(h).reshape(len(h), Hk, d)
            ref, mag, reach = T.attend(f64(q[r]), K, V, old(hk[b]), old(hv[b]), window, sinks, d ** -0.5, parents[b] if tree else None)
            tol = es * np.abs(ref) + mag * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) + mag * 2 * ((d + 4) * 2.0 ** -24 * reach)[..., None]
            assert (np.abs(f64(out[r]) - ref) <= tol).all()
            hk[b] += [K[i] for i in picks[b]]
            hv[b] += [V[i] for i in picks[b]]
        assert cache.L.tolist() == [len(h) for h in hk]
        if page:                                          # pages wholly between the sinks and the window go back
            lo = [-(-sinks // page)] * B
            hi = [max(l, (len(h) - window + 1) // page) for l, h in zip(lo, hk)]
            pg.pages_free(pool, ones(0, 1, 2), ones(*lo), ones(*hi), status)
            assert not status.any() and int(pool.ref.sum()) == int((cache.page_table >= 0).sum()) <= B * (2 + (window + 40) // page)
