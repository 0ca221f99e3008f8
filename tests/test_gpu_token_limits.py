"""Token-level operators at the ends of their ranges: values near the largest of the type, lengths and rows that no sequence can have, sequences
without tokens, other lengths under one captured call."""
import numpy as np
import pytest
import torch

from oracle import tok_oracle as T
from tests.test_gpu_tokens import Layer, api, f64  # noqa: F401

pytestmark = pytest.mark.gpu


def set_history(lay, b, k, v):
    """Other committed keys and values of sequence b, in the rows where they are visible."""
    lay.hist_k[b], lay.hist_v[b] = k, v
    pos = torch.tensor([p for p in range(lay.L[b]) if p < lay.shape.n_sink or p > lay.L[b] - lay.shape.window])
    if not len(pos):
        return
    if lay.page:
        at = torch.from_numpy(lay.table)[b][pos // lay.page].long() * lay.page + pos % lay.page
    else:
        at = torch.tensor([T.ring_row(b, int(p), lay.shape.n_sink, lay.shape.window) for p in pos])
    lay.cache.k[at.cuda()] = k[pos].cuda()
    if lay.cache.v is not None:
        lay.cache.v[at.cuda()] = v[pos].cuda()


def fill(lay, big, rise):
    """Scores that rise with the position, by `rise` powers of two over a sequence (the first dim's product; the others' is zero), and values of
    magnitudes from big / 2 to big, of one sign in a column."""
    rng = np.random.default_rng(3)
    H, Hk, d, dt = lay.shape.H, lay.shape.Hk, lay.shape.d, lay.shape.torch_dtype
    lay.q.zero_()
    lay.q[:, :, 0] = 1.0
    for b in range(lay.B):
        total = lay.L[b] + lay.n[b]
        v = rng.uniform(0.5, 1.0, (total, Hk, d)) * big * np.where(np.arange(d) % 2, -1.0, 1.0)
        k = v.copy() if lay.v is None else rng.standard_normal((total, Hk, d))
        k[:, :, 0] = (np.arange(total) * (rise * np.log(2.0) / max(1, total - 1)))[:, None]
        k = torch.from_numpy(k).float().to(dt)
        v = k if lay.v is None else torch.from_numpy(v).float().to(dt)
        r = slice(lay.row0[b], lay.row0[b] + lay.n[b])
        lay.k[r] = k[lay.L[b]:].cuda()
        if lay.v is not None:
            lay.v[r] = v[lay.L[b]:].cuda()
        set_history(lay, b, k[:lay.L[b]], v[:lay.L[b]])


# every kernel: tiles of 128 rows of each width, with shares joined afterwards and without; tiles of 16 rows, shares joined in a cluster and afterwards;
# fp32.  Sums over the keys go beyond what fp32 holds: 700 keys, weights of up to 2^9 beside the first block's, of 1e36; or equal weights of 3e38
@pytest.mark.parametrize("big,rise", [(1e36, 9.5), (3e38, 0.0), (3e38, 3.0)])
@pytest.mark.parametrize("heads,L,n", [
    (("bf16", 2, 1, 64, False), [0, 40], [250, 20]), (("bf16", 4, 2, 128, True), [300], [40]), (("bf16", 2, 1, 256, False), [500], [20]),
    (("bf16", 2, 1, 200, True), [0], [140]), (("bf16", 2, 1, 512, True), [430], [70]), (("bf16", 2, 1, 512, False), [300], [20]),
    (("bf16", 20, 1, 128, False), [9000], [1]), (("bf16", 2, 1, 512, True), [17000], [1]), (("bf16", 2, 1, 256, False), [17000], [1]),
    (("bf16", 2, 1, 64, False), [700], [1]), (("bf16", 2, 1, 128, True), [90, 3], [1, 2]), (("bf16", 2, 1, 128, False), [9000], [1]),
    (("bf16", 2, 1, 256, False), [700], [1]), (("bf16", 2, 1, 512, True), [1200], [3]), (("bf16", 2, 1, 512, False), [9000], [1]),
    (("fp32", 2, 1, 64, False), [700], [30]), (("fp32", 2, 1, 264, True), [700], [1]), (("fp32", 2, 1, 512, False), [9000], [1])], ids=str)
def test_sums_beyond_the_range(api, heads, L, n, big, rise):
    _, tk, _ = api
    lay = Layer(tk, *heads, window=20000, sinks=4, L=L, n=n, page=64, seed=len(L), scale=1.0)
    fill(lay, big, rise)
    lay.check(lay.run(tk))


@pytest.mark.parametrize("dtype,d,rot,pairs", [("bf16", 128, 64, True), ("bf16", 72, 32, False), ("fp32", 64, 64, False), ("fp32", 512, 16, True)])
def test_norms_of_vectors_at_the_ends_of_the_range(api, dtype, d, rot, pairs):
    """Vectors whose squares fp32 does not hold, or holds as zero, beside ordinary ones, in one call; eps zero, so that it does not count."""
    _, tk, _ = api
    lay = Layer(tk, dtype, 3, 1, d, True, window=1, sinks=0, L=[0, 0], n=[9, 40], seed=d)
    scales = [1.0, 1e30, 3e37, 1e-30, 1e18, 1e-24, 1e-37, 1.0, 1e20]
    for b in range(2):
        for i in range(lay.n[b]):
            lay.q[lay.row0[b] + i] *= scales[i % 9]
            lay.k[lay.row0[b] + i] *= scales[(i + 4) % 9]
    w = torch.from_numpy(np.random.default_rng(d).uniform(0.5, 1.5, d).astype(np.float32)).cuda()
    inv = torch.from_numpy((10000.0 ** (-np.arange(rot // 2) * 2 / rot)).astype(np.float32)).cuda()
    qo, ko = torch.zeros_like(lay.q), torch.zeros_like(lay.k)
    first = 8 if d > rot else 0
    tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, lay.k, qo, ko, w, w, 0.0, inv, first, pairs, lay.status)
    for b in range(2):
        r = slice(lay.row0[b], lay.row0[b] + lay.n[b])
        for got, x in ((qo, lay.q), (ko, lay.k)):
            ref, mag = T.norm_rope(f64(x[r]), f64(w), 0.0, range(lay.n[b]), f64(inv), first, pairs)
            tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref) + mag * (d * 2.0 ** -24 + 2.0 ** -20) + 1e-30
            assert (np.abs(f64(got[r]) - ref) <= tol).all()


def test_a_flagged_sequence_has_zeros_whatever_the_weights(api):
    _, tk, _ = api
    for bad in (float("nan"), float("inf")):
        lay = Layer(tk, "bf16", 4, 2, 64, True, window=1, sinks=0, L=[0, 0], n=[5, 3], seed=1)
        lay.cache.L[0] = -1
        w = torch.full((64,), bad, device="cuda")
        inv = (10000.0 ** -torch.arange(0, 1, 2 / 32, device="cuda")).float()
        qo, ko = torch.full_like(lay.q, 3.0), torch.full_like(lay.k, 3.0)
        tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, lay.k, qo, ko, w, w, 1e-6, inv, 16, False, lay.status)
        r = slice(lay.row0[0], lay.row0[0] + 5)
        assert lay.status.tolist() == [api[0].ST_LENGTH, 0] and (qo[r] == 0).all() and (ko[r] == 0).all()


@pytest.mark.parametrize("max_n", [8, 64, 65, 300])
@pytest.mark.parametrize("page", [0, 16])
def test_commit_flags_lengths_of_sequences_without_tokens(api, max_n, page):
    """A length that no sequence can have is flagged whether or not there are tokens to commit, and whatever the shape's bounds."""
    tsv, tk, _ = api
    lay = Layer(tk, "bf16", 2, 2, 64, False, window=10, sinks=1, L=[4, 9, 2, 5, 0], n=[3, 0, 0, 0, 2], page=page, seed=2, extra_n=max_n - 3)
    assert lay.shape.max_n == max_n
    lay.cache.L[1], lay.cache.L[2] = -1, lay.shape.max_L + 1
    tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status)
    assert lay.status.tolist() == [0, tsv.ST_LENGTH, tsv.ST_LENGTH, 0, 0]
    assert lay.cache.L.tolist() == [7, -1, lay.shape.max_L + 1, 5, 2]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [[3, 4], [40, 90]])
def test_first_rows_at_the_ends_of_64_bits(api, dtype, n):
    """row0[b] + n[b] passes 64 bits: outside the packed arrays like any other such row, in every call."""
    tsv, tk, _ = api
    for row0 in (2 ** 63 - 1, 2 ** 63 - n[0], 2 ** 63 - n[0] - 1, -2 ** 63):
        lay = Layer(tk, dtype, 4, 2, 64, False, window=20, sinks=2, L=[30, 8], n=n, page=4, seed=3, extra_n=5)
        was = lay.row0[0]
        good, q = lay.run(tk).clone(), torch.full_like(lay.q, 3.0)
        lay.batch.row0[0] = row0
        mine = slice(lay.row0[1], lay.row0[1] + n[1])
        out = lay.run(tk)
        assert lay.status.tolist() == [tsv.ST_NODES, 0] and torch.equal(out[mine], good[mine]) and (out[was:was + n[0]] == 3.0).all()
        st = torch.zeros_like(lay.status)
        tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, None, q, None, None, None, 1e-6, None, 0, False, st)
        assert st.tolist() == [tsv.ST_NODES, 0] and (q[was:was + n[0]] == 3.0).all() and not (q[mine] == 3.0).any()
        st.zero_()
        tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, st)
        assert st.tolist() == [tsv.ST_NODES, 0] and lay.cache.L.tolist() == [30, 8 + n[1]]


@pytest.fixture
def tries(api):
    """Sets how often the waits inside the kernels try before they give up, for the launches of one test."""
    import ctypes as C
    f = api[0]._lib.tsv_set_wait_tries
    f.argtypes, f.restype = [C.c_int64], C.c_int
    yield f
    torch.cuda.synchronize()
    f(-1)


@pytest.mark.parametrize("n", [[70, 0, 300], [4000, 3, 65]])
def test_commit_whose_copies_do_not_come(api, tries, n):
    """Waits that give up at once: the sequences are flagged and keep their lengths, the next call does everything."""
    tsv, tk, _ = api
    lay = Layer(tk, "bf16", 2, 2, 128, False, window=20, sinks=1, L=[3, 9, 5], n=n, page=16, seed=1)
    tries(0)
    tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status)
    assert lay.status.tolist() == [tsv.ST_INTERNAL if k else 0 for k in n] and lay.cache.L.tolist() == [3, 9, 5]
    tries(-1)
    lay.status.zero_()
    tk.token_commit(lay.shape, lay.cache, lay.batch, lay.k, lay.v, lay.status)
    assert not lay.status.any() and lay.cache.L.tolist() == [3 + n[0], 9 + n[1], 5 + n[2]]
    for b in range(3):
        pos = np.arange(lay.L[b], lay.L[b] + n[b])
        at = torch.from_numpy(lay.table[b][pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
        assert torch.equal(lay.cache.k[at], lay.k[lay.row0[b]:lay.row0[b] + n[b]]) and torch.equal(lay.cache.v[at], lay.v[lay.row0[b]:lay.row0[b] + n[b]])


@pytest.mark.parametrize("words", [8, 5000, 300000])
def test_page_copies_that_do_not_come(api, tries, words):
    """A fork and a compaction whose waits give up at once tell so, and the next call on the same pool works."""
    tsv, _, pg = api
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    plane = torch.arange(40, dtype=torch.int32, device="cuda")[:, None].expand(40, words).contiguous()
    L = i32(10, 0, 0, 9, 0)
    pool = pg.PagePool(torch.full((5, 4), -1, dtype=torch.int32, device="cuda"), torch.zeros(40, dtype=torch.int32, device="cuda"), 4, [plane], [L])
    ws, st, used = pg.alloc_workspace(pool), i32(0, 0), i32(7)
    pool.page_table[0, :3], pool.page_table[3, :3] = i32(30, 31, 32), i32(33, 34, 35)
    pool.ref[30:36] = 1
    tries(0)
    pg.pages_fork(pool, i32(0, 3), i32(1, 2), L, ws, st)
    assert st.tolist() == [tsv.ST_INTERNAL] * 2
    tries(-1)
    st.zero_()
    pg.pages_free(pool, i32(1, 2), i32(0, 0), i32(4, 4), st)
    pg.pages_fork(pool, i32(0, 3), i32(1, 2), L, ws, st)
    assert not st.any() and pool.page_table[1].tolist() == [30, 31, 0, -1] and pool.page_table[2].tolist() == [33, 34, 1, -1]
    assert (plane[0] == 32).all() and (plane[1] == 35).all()
    tries(0)
    pg.pages_compact(pool, used, ws)
    assert used.tolist() == [-1]
    tries(-1)
    pg.pages_compact(pool, used, ws)                      # (nothing left to move)
    assert used.tolist() == [8]


@pytest.mark.parametrize("heads,L,n", [
    (("bf16", 8, 2, 64, False), [700, 20], [30, 140]), (("bf16", 32, 1, 128, True), [900], [300]), (("bf16", 6, 1, 256, False), [300, 4], [20, 300]),
    (("bf16", 64, 1, 512, True), [700, 20, 3], [3, 140, 50]), (("bf16", 64, 1, 512, True), [17000], [1])], ids=str)
def test_attention_whose_waits_give_up(api, tries, heads, L, n):
    """After any number of tries: the sequences are flagged, or the result is whole (no wait was longer than its first try, of 4 us); other rows stay
    as they were, and the next call is right."""
    tsv, tk, _ = api
    lay = Layer(tk, *heads, window=20000, sinks=3, L=L, n=n, page=64, seed=1)
    good = lay.run(tk).clone()
    assert not lay.status.any()
    mine = torch.zeros(lay.rows, dtype=torch.bool)
    for r, k in zip(lay.row0, n):
        mine[r:r + k] = True
    seen = set()
    for k in [0, 0, 0, 1, 1, 2, 3, 5, 8, 13, 40, 1 << 20]:
        tries(k)
        lay.status.zero_()
        out = lay.run(tk)
        st = set(lay.status.tolist())
        assert st <= {0, tsv.ST_INTERNAL} and len(st) == 1 and (out[~mine.cuda()] == 3.0).all()
        seen |= st
        if st == {0}:
            assert torch.equal(out.nan_to_num(9), good.nan_to_num(9))
        tries(-1)
        lay.status.zero_()
        assert torch.equal(lay.run(tk).nan_to_num(9), good.nan_to_num(9)) and not lay.status.any()
    assert 0 in seen


# (more than two tiles for every CTA, and a first position that all rows see)
@pytest.mark.parametrize("heads,n", [(("bf16", 16, 1, 64, False), 9000), (("bf16", 16, 1, 128, True), 9000), (("bf16", 32, 1, 256, False), 2400),
                                     (("bf16", 64, 1, 512, True), 500), (("bf16", 64, 1, 512, False), 500)], ids=str)
def test_rows_one_by_one_that_outlast_the_waits(api, tries, heads, n):
    """Rows that see a NaN take longer than the others wait for them: the call is flagged, and the items that are being worked on stay as they are."""
    tsv, tk, _ = api
    lay = Layer(tk, *heads, window=200, sinks=1, L=[0], n=[n], seed=1)
    (lay.k if lay.v is None else lay.v)[lay.row0[0], 0, 3] = float("nan")
    want = lay.run(tk).clone()
    assert not lay.status.any()
    for k in (0, 1, 3, 10, 30, 100):
        tries(k)
        lay.run(tk)
        assert lay.status.tolist() == [tsv.ST_INTERNAL]
        tries(-1)
        lay.status.zero_()
        assert torch.equal(lay.run(tk).nan_to_num(9), want.nan_to_num(9)) and not lay.status.any()


@pytest.mark.parametrize("page_tokens", [0, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_over_a_verify_layers_window(api, dtype, page_tokens):
    """New tokens attend to the token-level KV that a verify layer holds, after cycles of it, and the layer goes on as without that."""
    tsv, tk, _ = api
    from paper_2609_24698_b200 import harness as hz, synth
    from tests.helpers import oracle_states, state_arrays
    from tests.test_gpu_tokens import STEP
    sh = synth.Shape("bf16", 3, 8, 64, 512, 4, 512, 4, 128, 128, 128) if dtype == "bf16" else synth.Shape("fp32", 3, 8, 16, 128, 4, 64, 1, 64, 128, 128)
    cfg = synth.Config("tokens", 230, sh, layers=1, L_min=0, L_max=1000, seed=4)
    lengths = np.asarray([1000, 3, 300])
    states = oracle_states(cfg, lengths)
    ccap, hcap = hz.capacities(sh, [1000, 1000, 300], 64)
    eng = hz.VerifyEngine(sh, 1, ccap, hcap, 1200, page_tokens=page_tokens)
    for b in range(3):
        hz.fill_cache(eng.caches[0], sh, b, int(lengths[b]), state_arrays(states[0][b]))
    for cyc in range(2):
        parent, n_nodes = synth.trees(cfg, cyc)
        draft, target = synth.tokens(cfg, cyc, parent, n_nodes)
        eng.launch_cycle(hz.InputSet.from_numpy(sh, [synth.node_inputs(cfg, 0, cyc)], parent, n_nodes, draft, target))
    layer = eng.caches[0]
    L = layer.L.tolist()
    cache = tk.TokenCache.of_layer(layer)
    n, d, H = [2, 40, 1], sh.d, 8
    row0, rows = [0, 2, 42], 43
    shape = tk.TokenShape(dtype, 3, H, 1, d, sh.window, max_L=2000, max_n=40)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k = (torch.randn(rows, h, d, device="cuda", generator=gen).to(shape.torch_dtype) for h in (H, 1))
    batch = tk.TokenBatch(torch.tensor(row0, dtype=torch.int64).cuda(), torch.tensor(n, dtype=torch.int32).cuda())
    out, st = torch.zeros_like(q), torch.zeros(3, dtype=torch.int32, device="cuda")
    before = layer.win_kv.clone()
    tk.window_sink_attn(shape, cache, batch, q, k, None, out, tk.alloc_workspace(shape, rows), st)
    assert not st.any() and layer.L.tolist() == L and torch.equal(layer.win_kv, before)
    flat = layer.win_kv.view(-1, d)
    for b in range(3):
        first = max(0, L[b] - sh.window)
        hist = np.zeros((L[b], 1, d))
        hist[first:, 0] = f64(flat[layer.tok_row_index(sh, b, torch.arange(first, L[b], device="cuda"))])
        r = slice(row0[b], row0[b] + n[b])
        ref, mag, reach = T.attend(f64(q[r]), f64(k[r]), f64(k[r]), hist, hist, sh.window, 0, d ** -0.5)
        tol = STEP[dtype] * np.abs(ref) + mag * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) + mag * 2 * ((d + 4) * 2.0 ** -24 * reach)[..., None]
        assert (np.abs(f64(out[r]) - ref) <= tol).all()
    with pytest.raises(tsv.TsvError):
        tk.token_commit(shape, cache, batch, k, None, st)
    assert layer.L.tolist() == L


def test_a_pool_of_layers_whose_table_names_pages_that_are_none(api):
    """Counts are made without such words, and the sequences that hold them are flagged where they are forked."""
    tsv, _, pg = api
    from paper_2609_24698_b200 import harness as hz, synth
    sh = synth.Shape("fp32", 3, 8, 16, 128, 4, 64, 1, 64, 128, 128)
    ccap, hcap = hz.capacities(sh, [1000, 1000, 300], 64)
    eng = hz.VerifyEngine(sh, 2, ccap, hcap, 1200, page_tokens=128)
    eng.caches[1].page_table = eng.caches[0].page_table
    table = eng.caches[0].page_table
    n = eng.caches[0].win_kv.shape[0] // 128
    table.fill_(-1)
    table[0, :3] = torch.tensor([4, n, 5], dtype=torch.int32)
    table[2, :2] = torch.tensor([4, -9], dtype=torch.int32)
    pool = pg.PagePool.of_layers(eng.caches)
    want = [0] * n
    want[4], want[5] = 2, 1
    assert pool.ref.tolist() == want
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    pg.pages_fork(pool, i32(0), i32(1), eng.caches[0].L, pg.alloc_workspace(pool), st)
    assert st.tolist() == [pg.ST_PAGE] and (table[1] == -1).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rope_among_column_ranges(api, dtype):
    """Outputs in column ranges of the array that holds the inputs, in place and beside them, with the bits of outputs of their own; one row; and what
    would share rows is refused."""
    tsv, tk, _ = api
    H, Hk, d, rows = 4, 2, 64, 70
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    shape = tk.TokenShape(dtype, 1, H, Hk, d, 1, max_L=1000, max_n=rows)
    gen = torch.Generator(device="cuda").manual_seed(1)
    L, st = torch.tensor([7], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    inv = (10000.0 ** -torch.arange(0, 1, 2 / 64, device="cuda")).float()
    for n in (rows, 1):
        batch = tk.TokenBatch(torch.zeros(1, dtype=torch.int64, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"))
        big = torch.randn(n, 2 * (H + Hk) * d, device="cuda", generator=gen).to(dt)
        part = lambda a, heads: big[:, a * d:(a + heads) * d].unflatten(1, (heads, d))
        q, k, q2, k2 = part(0, H), part(H, Hk), part(H + Hk, H), part(2 * H + Hk, Hk)
        call = lambda *x: tk.qk_norm_rope(shape, L, batch, *x, None, None, 1e-6, inv, 0, False, st)
        qo, ko = torch.empty(n, H, d, dtype=dt, device="cuda"), torch.empty(n, Hk, d, dtype=dt, device="cuda")
        call(q, k, qo, ko)
        call(q, k, q2, k2)
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
        call(q, k, q, k)
        assert torch.equal(q, qo) and torch.equal(k, ko) and not st.any()
        for bad in ((q, k, part(1, H), k2), (q, k, part(H - 1, H), k2), (q, k, q2, part(H - 1, Hk)), (q, k, q2, part(H + Hk + 1, Hk))):
            with pytest.raises(tsv.TsvError) as e:
                call(*bad)
            assert e.value.code == tsv.ERR_SHAPE


@pytest.mark.parametrize("n", [[5, 4], [5, 70]])
def test_commit_does_not_look_at_parents(api, n):
    """As the header says: the path decides; a flag of an earlier call of the same tokens stops the sequence."""
    tsv, tk, _ = api
    for flagged in (False, True):
        lay = Layer(tk, "bf16", 2, 2, 64, False, window=10, sinks=1, L=[4, 9], n=n, page=4, seed=2)
        par = torch.full((lay.rows,), 7, dtype=torch.int32, device="cuda")
        batch = tk.TokenBatch(lay.batch.row0, lay.batch.n, par)
        path, count = torch.tensor([[0, 2, 4, -1], [0, 1, 3, 2]], dtype=torch.int32, device="cuda"), torch.tensor([3, 4], dtype=torch.int32, device="cuda")
        if flagged:
            tk.qk_norm_rope(lay.shape, lay.cache.L, batch, lay.q, None, lay.q.clone(), None, None, None, 1e-6, None, 0, False, lay.status)
            assert lay.status.tolist() == [tsv.ST_PARENT] * 2
        before = lay.cache.k.clone()
        tk.token_commit(lay.shape, lay.cache, batch, lay.k, lay.v, lay.status, path=path, count=count)
        assert lay.status.tolist() == [tsv.ST_PARENT * flagged] * 2 and lay.cache.L.tolist() == ([4, 9] if flagged else [7, 13])
        for b, nodes in enumerate([[0, 2, 4], [0, 1, 3, 2]]):
            pos = np.arange(lay.L[b], lay.L[b] + len(nodes))
            at = torch.from_numpy(lay.table[b][pos // 4].astype(np.int64) * 4 + pos % 4).cuda()
            want = before[at] if flagged else lay.k[[lay.row0[b] + i for i in nodes]]
            assert torch.equal(lay.cache.k[at].nan_to_num(9), want.nan_to_num(9))



@pytest.mark.parametrize("heads", [("bf16", 64, 1, 512, True), ("bf16", 8, 2, 128, False), ("fp32", 16, 1, 128, True)], ids=lambda h: "_".join(map(str, h)))
@pytest.mark.parametrize("n", [[3, 140], [1, 2]])
def test_a_replay_at_other_lengths(api, heads, n):
    """A captured call replayed at other lengths, shorter and longer ones, has the bits of a call made at them."""
    _, tk, _ = api
    lay = Layer(tk, *heads, window=600, sinks=3, L=[700, 20], n=n, page=64, seed=1)
    lay.cache.k.nan_to_num_(0.5)                          # (rows of the pages that the captured lengths do not reach)
    if lay.cache.v is not None:
        lay.cache.v.nan_to_num_(0.5)
    ws, out = tk.alloc_workspace(lay.shape, lay.rows), torch.zeros(lay.rows, *lay.q.shape[1:], dtype=lay.q.dtype, device="cuda")
    call = lambda o, st: tk.window_sink_attn(lay.shape, lay.cache, lay.batch, lay.q, lay.k, lay.v, o, ws, st)
    call(out, lay.status)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        call(out, lay.status)
    for L in ([25, 20], [0, 1], [640, 22], [700, 20]):
        lay.cache.L.copy_(torch.tensor(L, dtype=torch.int32))
        out.zero_()
        g.replay()
        want = torch.zeros_like(out)
        call(want, lay.status)
        torch.cuda.synchronize()
        assert torch.equal(out.nan_to_num(9), want.nan_to_num(9)) and not lay.status.any()


@pytest.mark.parametrize("heads", [("bf16", 8, 2, 64, False), ("bf16", 8, 1, 512, True), ("fp32", 4, 1, 64, True), ("bf16", 16, 1, 128, False), ("bf16", 8, 1, 256, False)],
                         ids=lambda h: "_".join(map(str, h)))
@pytest.mark.parametrize("n", [6, 150])
def test_rows_that_see_an_infinite_value(api, heads, n):
    """An infinity in a value, and a score with it (without values of their own): what stays finite is within the bounds of any other result."""
    _, tk, _ = api
    for bad in (float("inf"), -float("inf")):
        lay = Layer(tk, *heads, window=40, sinks=1, L=[20, 0], n=[n, 3], seed=n)
        if lay.v is None:
            lay.k[lay.row0[0] + n // 2, -1, 1] = bad
        else:
            lay.v[lay.row0[0] + n // 2, :, 3] = bad
        got = f64(lay.run(tk))[lay.row0[0]:lay.row0[0] + n]
        ref, mag, reach = lay.ref(0)
        ok = np.isfinite(ref)
        assert (ok == np.isfinite(got)).all() and ok.any() and not ok.all()
        es, d = 2.0 ** -8 if heads[0] == "bf16" else 2.0 ** -24, heads[3]
        with np.errstate(all="ignore"):
            # (a row whose score of the key is -infinity gives it no weight, and its bound comes from the others: at most the largest of them)
            top = np.where(np.isfinite(mag), mag, 0) if lay.v is not None else np.full_like(ref, np.abs(f64(lay.k)[np.isfinite(f64(lay.k))]).max())
            far = np.where(np.isfinite(reach), reach, np.nanmax(np.where(np.isfinite(reach), reach, 0)))
            tol = es * np.abs(ref) + top * (2.0 ** -8 if heads[0] == "bf16" else 2.0 ** -20) + top * 2 * ((d + 4) * 2.0 ** -24 * far)[..., None] + 1e-30
            assert (np.abs(got - ref) <= tol)[ok].all()


# a share of split keys, joined in a cluster or afterwards, that holds nothing but keys with an infinite value, which no other share has
@pytest.mark.parametrize("heads,L,first,last", [
    (("bf16", 16, 1, 64, True), 500, 128, 192), (("bf16", 16, 1, 512, True), 1200, 320, 480), (("bf16", 16, 1, 128, True), 9000, 2048, 2560),
    (("bf16", 8, 1, 512, True), 17000, 2640, 3168), (("bf16", 24, 1, 128, True), 6000, 1024, 1536), (("fp32", 16, 1, 72, True), 500, 128, 192),
    (("fp32", 4, 1, 512, True), 9000, 2048, 2560), (("fp32", 16, 1, 128, True), 64, 63, 64)], ids=str)
def test_shares_of_infinite_keys(api, heads, L, first, last):
    """Rows whose score of those keys is -infinity give them no weight, and 0 times infinity is NaN in that column alone; where it is +infinity, all is."""
    _, tk, _ = api
    lay = Layer(tk, *heads, window=20000, sinks=0, L=[L], n=[1], page=64, seed=4)
    k = lay.hist_k[0].clone()
    k[first:last, :, 3] = float("inf")
    set_history(lay, 0, k, k)
    lay.q[:, ::2, 3] = -lay.q[:, ::2, 3].abs() - 0.1
    lay.q[:, 1::2, 3] = lay.q[:, 1::2, 3].abs() + 0.1
    got = f64(lay.run(tk))[lay.row0[0]]
    ref, mag, _ = lay.ref(0)
    ref, mag = ref[0], mag[0]
    assert np.isnan(ref[::2, 3]).all() and np.isfinite(np.delete(ref[::2], 3, 1)).all() and np.isnan(ref[1::2]).all()
    assert (np.isnan(got) == np.isnan(ref)).all() and not np.isinf(got).any() and not lay.status.any()
    ok = np.isfinite(ref)
    # (a rounding of each weight, of the result, and of fp32 sums)
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 1e-3) * mag)[ok].all()


@pytest.mark.parametrize("dtype,H,Hk,d", [("bf16", 40, 8, 128), ("bf16", 100, 1, 512), ("fp32", 9, 3, 512), ("fp32", 6, 2, 64)])
@pytest.mark.parametrize("tokens", [3, 300])
def test_norms_in_place_at_the_ends_of_the_range(api, dtype, H, Hk, d, tokens):
    """Heads that are done once more beside heads whose results are as far out as those: weights of 1e-25 bring every result there.  In place every head is
    done once, with the bits of outputs of their own."""
    _, tk, _ = api
    lay = Layer(tk, dtype, H, Hk, d, True, window=1, sinks=0, L=[0], n=[tokens], seed=d)
    rng = np.random.default_rng(H)
    for x in (lay.q, lay.k):
        x *= torch.from_numpy(10.0 ** rng.choice([0, 0, 0, 30, -30], size=(*x.shape[:2], 1))).to(x)
    w = torch.full((d,), 1e-25, device="cuda")
    inv = (10000.0 ** -torch.arange(0, 1, 2 / 32, device="cuda")).float()
    qo, ko = torch.empty_like(lay.q), torch.empty_like(lay.k)
    call = lambda qo, ko: tk.qk_norm_rope(lay.shape, lay.cache.L, lay.batch, lay.q, lay.k, qo, ko, w, w, 0.0, inv, 16, False, lay.status)
    call(qo, ko)
    r = slice(lay.row0[0], lay.row0[0] + tokens)
    ref, mag = T.norm_rope(f64(lay.q[r]), f64(w), 0.0, range(tokens), f64(inv), 16, False)
    assert (np.abs(f64(qo[r]) - ref) <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref) + mag * (d * 2.0 ** -24 + 2.0 ** -20)).all()
    call(lay.q, lay.k)
    assert torch.equal(lay.q[r], qo[r]) and torch.equal(lay.k[r], ko[r]) and not lay.status.any()


def test_one_row_in_place_under_a_larger_output(api):
    """A call of one row, whose output is its input by address: the strides of neither count."""
    _, tk, _ = api
    H, d = 4, 64
    shape = tk.TokenShape("bf16", 1, H, 1, d, 1, max_L=1000, max_n=1)
    L, st = torch.tensor([7], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    batch = tk.TokenBatch(torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"))
    inv = (10000.0 ** -torch.arange(0, 1, 2 / 64, device="cuda")).float()
    big = torch.randn(5, 2 * H * d, device="cuda").to(torch.bfloat16)
    q = big[:, :H * d].unflatten(1, (H, d))
    out = torch.empty(1, H, d, dtype=torch.bfloat16, device="cuda")
    rest = big.clone()
    tk.qk_norm_rope(shape, L, batch, q[:1], None, out, None, None, None, 1e-6, inv, 0, False, st)
    tk.qk_norm_rope(shape, L, batch, q[:1], None, q, None, None, None, 1e-6, inv, 0, False, st)
    assert torch.equal(q[:1], out) and torch.equal(big[1:], rest[1:]) and torch.equal(big[0, H * d:], rest[0, H * d:]) and not st.any()
