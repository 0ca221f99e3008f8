"""Token-level and page operators without a GPU: what the host refuses before any launch, and the 64-bit restatement by its own
invariants."""
import ctypes as C

import numpy as np
import pytest

from oracle import tok_oracle as T

FAKE = 0x10000            # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def api():
    from paper_2609_24698_b200.build import build_library
    build_library()
    from paper_2609_24698_b200 import binding, pages, tokens
    return binding, tokens, pages


def _shape(tk, **kw):
    base = dict(dtype=1, B=2, H=8, Hk=2, d=64, window=16, n_sink=2, max_n=8, max_L=4096, sm_scale=0.0, reserved=0)
    base.update(kw)
    return tk.CTokShape(**base)


BAD_SHAPES = [dict(dtype=2), dict(B=0), dict(H=0), dict(H=257), dict(Hk=3), dict(Hk=0), dict(d=12), dict(d=520), dict(d=0), dict(window=0),
              dict(n_sink=-1), dict(max_n=0), dict(max_n=(1 << 22) + 1), dict(max_L=0), dict(max_L=(1 << 30) + 1)]


def test_workspace_of_shapes(api):
    tsv, tk, _ = api
    f = tsv._lib.tsv_tok_workspace_bytes
    s = _shape(tk)
    sizes = [f(C.addressof(s), r) for r in (0, 1, 7, 100, 10000, 1 << 22)]
    assert all(n > 0 and n % 256 == 0 for n in sizes) and sizes == sorted(sizes)
    for bad in BAD_SHAPES:
        assert f(C.addressof(_shape(tk, **bad)), 10) == 0, bad
    assert f(None, 10) == 0 and f(C.addressof(s), -1) == 0


def _structs(tk, ring_rows=36, **kw):
    cache = tk.CTokCache(FAKE, FAKE, FAKE, ring_rows, None, 0, 0)
    batch = tk.CTokBatch(FAKE, FAKE, None, 8)
    rows = tk.CTokRows(FAKE, FAKE, FAKE, 512, 128, 128)
    for k, v in kw.items():
        for st in (cache, batch, rows):
            if any(k == n for n, _ in st._fields_) and not (k == "rows" and st is batch):
                setattr(st, k, v)
    return cache, batch, rows


@pytest.mark.parametrize("change,code", [
    (dict(), "ERR_WORKSPACE"), (dict(L=None), "ERR_NULL"), (dict(k=None), "ERR_NULL"), (dict(row0=None), "ERR_NULL"), (dict(n=None), "ERR_NULL"),
    (dict(q=None), "ERR_NULL"), (dict(v=None), "ERR_WORKSPACE"), (dict(q=FAKE + 8), "ERR_ALIGN"), (dict(k=FAKE + 2), "ERR_ALIGN"),
    (dict(q_ld=511), "ERR_SHAPE"), (dict(q_ld=516), "ERR_ALIGN"), (dict(k_ld=64), "ERR_SHAPE"), (dict(v_ld=132), "ERR_ALIGN"),
    (dict(ring_rows=35), "ERR_SHAPE"), (dict(page_table=FAKE), "ERR_SHAPE"), (dict(page_table=FAKE, page_tokens=4), "ERR_SHAPE"),
    (dict(page_table=FAKE, page_tokens=4, max_pages=3), "ERR_WORKSPACE")])
def test_attention_refusals(api, change, code):
    tsv, tk, _ = api
    cache, batch, rows = _structs(tk, **change)
    s = _shape(tk)
    f = tsv._lib.window_sink_attn
    a = C.addressof
    assert f(a(s), a(cache), a(batch), a(rows), FAKE, None, 0, FAKE, None) == getattr(tsv, code)
    assert f(a(s), a(cache), a(batch), a(rows), None, FAKE, 1 << 40, FAKE, None) == tsv.ERR_NULL
    assert f(a(s), a(cache), a(batch), a(rows), FAKE, FAKE, 1 << 40, None, None) == tsv.ERR_NULL
    assert f(None, a(cache), a(batch), a(rows), FAKE, FAKE, 1 << 40, FAKE, None) == tsv.ERR_NULL


def test_one_of_values_only_is_refused(api):
    tsv, tk, _ = api
    s, a = _shape(tk), C.addressof
    cache, batch, rows = _structs(tk)
    rows.v = None
    assert tsv._lib.window_sink_attn(a(s), a(cache), a(batch), a(rows), FAKE, FAKE, 1 << 40, FAKE, None) == tsv.ERR_NULL
    cache.v, rows.v = None, FAKE
    assert tsv._lib.token_commit(a(s), a(cache), a(batch), a(rows), None, 0, None, FAKE, None) == tsv.ERR_NULL


def test_more_attention_refusals(api):
    tsv, tk, _ = api
    cache, batch, rows = _structs(tk)
    f, a = tsv._lib.window_sink_attn, C.addressof
    for bad in BAD_SHAPES:
        assert f(a(_shape(tk, **bad)), a(cache), a(batch), a(rows), FAKE, FAKE, 1 << 40, FAKE, None) == tsv.ERR_SHAPE, bad
    s = _shape(tk)
    assert f(a(s), a(cache), a(batch), a(rows), FAKE + 8, FAKE, 1 << 40, FAKE, None) == tsv.ERR_ALIGN
    assert f(a(s), a(cache), a(batch), a(rows), FAKE, FAKE + 16, 1 << 40, FAKE, None) == tsv.ERR_WORKSPACE
    assert f(a(s), a(cache), a(batch), a(rows), FAKE, FAKE, 16, FAKE, None) == tsv.ERR_WORKSPACE
    batch.rows = -1
    assert f(a(s), a(cache), a(batch), a(rows), FAKE, FAKE, 1 << 40, FAKE, None) == tsv.ERR_SHAPE


def test_output_over_inputs_is_refused(api):
    tsv, tk, _ = api
    cache, batch, rows = _structs(tk)
    f, a, s = tsv._lib.window_sink_attn, C.addressof, _shape(tk)
    es, n = 2 if s.dtype == tsv.TSV_BF16 else 4, batch.rows
    out_bytes = n * s.H * s.d * es
    rows.q, rows.k, rows.v = 1 << 30, 2 << 30, 3 << 30
    for base, ld, heads in ((rows.q, rows.q_ld, s.H), (rows.k, rows.k_ld, s.Hk), (rows.v, rows.v_ld, s.Hk)):
        span = ((n - 1) * ld + heads * s.d) * es
        for out in (base, base + 16, base + span - 16, base - out_bytes + 16):
            assert f(a(s), a(cache), a(batch), a(rows), out, FAKE, 1 << 40, FAKE, None) == tsv.ERR_SHAPE


def test_rope_refusals(api):
    tsv, tk, _ = api
    _, batch, rows = _structs(tk)
    a = C.addressof

    def call(s=_shape(tk), io=rows, inv=FAKE, rot=32, first=0, q=FAKE, ldq=512, k=FAKE, ldk=128, status=FAKE, L=FAKE):
        return tsv._lib.qk_norm_rope(a(s), L, a(batch), a(io), None, None, 1e-6, inv, rot, first, 0, q, ldq, k, ldk, status, None)
    assert call(L=None) == tsv.ERR_NULL and call(status=None) == tsv.ERR_NULL and call(inv=None) == tsv.ERR_NULL
    assert call(q=None) == tsv.ERR_NULL and call(k=None) == tsv.ERR_NULL and call(io=tk.CTokRows(None, None, None, 0, 0, 0)) == tsv.ERR_NULL
    for kw in (dict(rot=8), dict(rot=-16), dict(rot=80), dict(first=4), dict(first=-8), dict(first=40), dict(ldq=500), dict(ldk=64)):
        assert call(**kw) == tsv.ERR_SHAPE, kw
    for kw in (dict(q=FAKE + 4), dict(k=FAKE + 8), dict(ldq=516), dict(ldk=132)):
        assert call(**kw) == tsv.ERR_ALIGN, kw
    for bad in BAD_SHAPES:
        assert call(s=_shape(tk, **bad)) == tsv.ERR_SHAPE, bad


def test_commit_refusals(api):
    tsv, tk, _ = api
    cache, batch, rows = _structs(tk)
    a, s = C.addressof, _shape(tk)
    f = tsv._lib.token_commit
    assert f(a(s), a(cache), a(batch), a(rows), FAKE, 0, None, FAKE, None) == tsv.ERR_SHAPE
    assert f(a(s), a(cache), a(batch), a(rows), None, 0, None, None, None) == tsv.ERR_NULL
    assert f(a(s), None, a(batch), a(rows), None, 0, None, FAKE, None) == tsv.ERR_NULL
    assert f(a(s), a(cache), None, a(rows), None, 0, None, FAKE, None) == tsv.ERR_NULL
    assert f(a(s), a(cache), a(batch), None, None, 0, None, FAKE, None) == tsv.ERR_NULL


def test_page_refusals(api):
    tsv, _, pg = api
    a, lib = C.addressof, tsv._lib

    def pool(plane=(FAKE, 64), row=(FAKE, 8), **kw):
        pl, rw = (pg.CPageArray * 1)(pg.CPageArray(*plane)), (pg.CPageArray * 1)(pg.CPageArray(*row))
        f = dict(page_table=FAKE, ref=FAKE, slots=4, max_pages=8, n_pages=16, page_tokens=4, planes=a(pl), rows=a(rw), n_planes=1, n_rows=1)
        f.update(kw)
        p = pg.CPagePool(*[f[n] for n, _ in pg.CPagePool._fields_])
        p.keep = (pl, rw)
        return p
    ok = pool()
    need = lib.tsv_pages_workspace_bytes(a(ok))
    assert need > 0
    for p, code in [(pool(page_table=None), tsv.ERR_NULL), (pool(ref=None), tsv.ERR_NULL), (pool(planes=None), tsv.ERR_NULL), (pool(slots=0), tsv.ERR_SHAPE),
                    (pool(max_pages=0), tsv.ERR_SHAPE), (pool(n_pages=0), tsv.ERR_SHAPE), (pool(page_tokens=0), tsv.ERR_SHAPE), (pool(n_planes=-1), tsv.ERR_SHAPE),
                    (pool(plane=(FAKE + 8, 64)), tsv.ERR_ALIGN), (pool(plane=(FAKE, 24)), tsv.ERR_ALIGN), (pool(plane=(FAKE, 0)), tsv.ERR_SHAPE),
                    (pool(plane=(None, 64)), tsv.ERR_NULL), (pool(row=(FAKE + 2, 8)), tsv.ERR_ALIGN), (pool(row=(FAKE, 6)), tsv.ERR_ALIGN)]:
        assert lib.tsv_pages_workspace_bytes(a(p)) == 0
        assert lib.pages_free(a(p), 1, FAKE, FAKE, FAKE, FAKE, None) == code
        assert lib.pages_assign(a(p), 1, FAKE, FAKE, FAKE, FAKE, need, FAKE, None) == code
        assert lib.pages_fork(a(p), 1, FAKE, FAKE, FAKE, FAKE, need, FAKE, None) == code
        assert lib.pages_compact(a(p), FAKE, FAKE, need, None) == code
    for n, code in [(-1, tsv.ERR_SHAPE), (pg.MAX_LIST + 1, tsv.ERR_LIMIT), (0, tsv.TsvError and 0)]:
        assert lib.pages_free(a(ok), n, None, None, None, None, None) == code
        assert lib.pages_assign(a(ok), n, None, None, None, FAKE, need, None, None) == code
        assert lib.pages_fork(a(ok), n, None, None, None, FAKE, need, None, None) == code
    assert lib.pages_free(a(ok), 1, None, FAKE, FAKE, FAKE, None) == tsv.ERR_NULL
    assert lib.pages_fork(a(ok), 1, FAKE, FAKE, FAKE, FAKE, need - 1, FAKE, None) == tsv.ERR_WORKSPACE
    assert lib.pages_assign(a(ok), 1, FAKE, FAKE, FAKE, FAKE + 4, need, FAKE, None) == tsv.ERR_WORKSPACE
    assert lib.pages_compact(a(ok), FAKE, None, need, None) == tsv.ERR_WORKSPACE
    assert lib.pages_compact(a(ok), None, FAKE, need, None) == tsv.ERR_NULL


def test_wrappers_refuse_what_the_library_cannot_see(api):
    """Types, shapes, strides and devices of tensors (all on the CPU here: the device check is the last)."""
    import torch
    tsv, tk, pg = api
    s = tk.TokenShape("bf16", 2, 4, 2, 16, window=8, max_L=64, max_n=4)
    z = lambda *sh, dt=torch.bfloat16: torch.zeros(*sh, dtype=dt)
    i32 = lambda *sh: torch.zeros(*sh, dtype=torch.int32)
    batch = tk.TokenBatch(torch.zeros(2, dtype=torch.int64), i32(2))
    for dt, rows, heads, t in [(torch.bfloat16, 5, 4, z(5, 4, 16, dt=torch.float32)), (torch.bfloat16, 5, 4, z(4, 4, 16)), (torch.bfloat16, 5, 4, z(5, 2, 16)),
                               (torch.bfloat16, 5, 4, z(5, 64)), (torch.bfloat16, 5, 4, z(5, 16, 4).transpose(1, 2)), (torch.bfloat16, 5, 4, z(5, 4, 16))]:
        with pytest.raises(tsv.TsvError) as e:
            tk._vectors("q", t, dt, rows, heads, 16, 0)
        assert e.value.code == tsv.ERR_SHAPE
    with pytest.raises(tsv.TsvError):
        tk.TokenBatch(i32(2), i32(2)).pack(2, 5, -1)
    with pytest.raises(tsv.TsvError):
        batch.pack(3, 5, -1)
    with pytest.raises(tsv.TsvError):
        batch.pack(2, 5, 0)
    with pytest.raises(tsv.TsvError):
        tk.alloc_token_cache(s, device="cpu").pack(s, 0)
    assert len(batch.pack(2, 5, -1)) == C.sizeof(tk.CTokBatch) and len(tk.alloc_token_cache(s, device="cpu").pack(s, -1)) == C.sizeof(tk.CTokCache)
    with pytest.raises(tsv.TsvError):
        tk.TokenShape("fp16", 1, 1, 1, 8, 1)
    with pytest.raises(tsv.TsvError):
        pg.PagePool(i32(2, 3), i32(4), 4, [z(4, 8)])


# ----------------------------------------------------------------------------- the restatement
def test_a_window_over_everything_is_causal_attention():
    rng = np.random.default_rng(0)
    import torch
    n, L, H, Hk, d = 7, 9, 4, 2, 8
    q, kn, vn, ko, vo = (rng.standard_normal(s) for s in [(n, H, d), (n, Hk, d), (n, Hk, d), (L, Hk, d), (L, Hk, d)])
    got, _, _ = T.attend(q, kn, vn, ko, vo, 100, 0, 0.3)
    K, V = (torch.from_numpy(np.concatenate(x)).repeat_interleave(2, 1).permute(1, 0, 2) for x in ([ko, kn], [vo, vn]))
    mask = torch.ones(n, L + n).tril(L).bool()
    ref = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).permute(1, 0, 2), K, V, attn_mask=mask, scale=0.3).permute(1, 0, 2)
    assert np.abs(got - ref.numpy()).max() < 1e-12


def test_a_path_of_a_tree_is_a_chain():
    rng = np.random.default_rng(1)
    parent = [-1, 0, 0, 2, 1, 3]
    q, kn, vn = (rng.standard_normal((6, 2, 8)) for _ in range(3))
    ko, vo = (rng.standard_normal((5, 2, 8)) for _ in range(2))
    tree, _, _ = T.attend(q, kn, vn, ko, vo, 4, 2, 0.3, parent)
    path = [0, 2, 3, 5]
    chain, _, _ = T.attend(q[path], kn[path], vn[path], ko, vo, 4, 2, 0.3)
    assert np.abs(tree[path] - chain).max() < 1e-13


def test_rotated_products_depend_on_distances():
    rng = np.random.default_rng(2)
    f = 10000.0 ** (-np.arange(8) / 8)
    q, k = rng.standard_normal((1, 1, 24)), rng.standard_normal((1, 1, 24))
    for pairs in (False, True):
        dots = [float((T.norm_rope(q, None, 0, [a + 5], f, 8, pairs)[0] * T.norm_rope(k, None, 0, [a], f, 8, pairs)[0]).sum()) for a in (0, 3, 1000)]
        assert np.ptp(dots) < 1e-9


def test_pool_operations_keep_counts():
    rng = np.random.default_rng(3)
    pool = T.Pool(np.full((6, 5), -1), np.zeros(12, int), 4, [np.arange(12)[:, None] * 10], [np.arange(6)[:, None]])
    assert pool.assign([0, 2], [0, 0], [3, 2]) == [0, 0] and list(pool.table[2, :2]) == [3, 4]
    assert pool.fork([0, 0, 2], [1, 3, 1], [10, 0, 8, 0, 0, 0]) == [0, 0, 64]
    assert list(pool.ref[:3]) == [3, 3, 1] and pool.table[1, 2] == 5 and pool.planes[0][5] == 20 and pool.rows[0][3] == 0
    assert pool.free([0, 0], [0, 0], [5, 5]) == [0, 0] and list(pool.ref[:3]) == [2, 2, 0]
    used = pool.compact()
    assert used == 6 and (pool.ref[:used] > 0).all() and (pool.ref[used:] == 0).all()
    assert pool.assign([4], [0], [5]) == [0] and pool.assign([5], [0], [5]) == [128]
    for s in range(6):
        for p in pool.table[s]:
            assert p < 0 or pool.ref[p] > 0


def test_a_verify_layers_cache_is_read_only(api):
    """Its lengths belong to the verify path; a ring is refused under another window than its own."""
    import torch
    tsv, tk, _ = api
    from types import SimpleNamespace
    layer = SimpleNamespace(L=torch.zeros(2, dtype=torch.int32), win_kv=torch.zeros(2, 8, 16, dtype=torch.bfloat16), page_table=None, page_tokens=0)
    cache = tk.TokenCache.of_layer(layer)
    batch = tk.TokenBatch(torch.zeros(2, dtype=torch.int64), torch.ones(2, dtype=torch.int32))
    shape = lambda window, sinks=0: tk.TokenShape("bf16", 2, 4, 1, 16, window=window, n_sink=sinks, max_L=64, max_n=4)
    with pytest.raises(tsv.TsvError, match="accept_and_refresh"):
        tk.token_commit(shape(8), cache, batch, torch.zeros(2, 1, 16, dtype=torch.bfloat16), None, torch.zeros(2, dtype=torch.int32))
    assert len(cache.pack(shape(8), -1)) == C.sizeof(tk.CTokCache)
    for bad in (shape(4), shape(7, 1)):
        with pytest.raises(tsv.TsvError) as e:
            cache.pack(bad, -1)
        assert e.value.code == tsv.ERR_SHAPE
        with pytest.raises(tsv.TsvError):
            tk.alloc_token_cache(shape(8), device="cpu").pack(bad, -1)


def _paged_layer(pages=6, page_tokens=4, table=None):
    import torch
    from types import SimpleNamespace
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    rows = {n: z(2, 3) for n in ("csa_mx", "csa_s", "csa_acc_kv", "csa_acc_ik", "hca_mx", "hca_s", "hca_acc_kv")}
    return SimpleNamespace(L=z(2, dt=torch.int32), csa_cap=z(2, dt=torch.int32), hca_cap=z(2, dt=torch.int32), page_tokens=page_tokens,
                           csa_kv=z(pages, 8), csa_ik=z(pages, 8), hca_kv=z(pages, 8), win_kv=z(pages * page_tokens, 8),
                           page_table=torch.tensor([[0, 1, -1], [2, -1, -1]], dtype=torch.int32) if table is None else table, **rows)


@pytest.mark.parametrize("word", [6, 1 << 30, -2, -(1 << 31)])
def test_counts_of_a_table_with_words_that_name_no_page(api, word):
    """Such words count for nothing.  (Everything is on the CPU here, which the pool itself refuses, last.)"""
    import torch
    tsv, _, pg = api
    table = torch.tensor([[0, word, -1], [2, 0, -1]], dtype=torch.int32)
    assert pg.counts_of(table, 6).tolist() == [2, 0, 1, 0, 0, 0]
    with pytest.raises(tsv.TsvError):
        pg.PagePool.of_layers([_paged_layer(table=table)])


def test_layers_whose_pools_differ_are_refused(api):
    """Pages of other sizes or another number of them behind the one table: the bytes of a page would be wrong in every plane of that layer."""
    tsv, _, pg = api
    a = _paged_layer()
    for b in (_paged_layer(pages=12, table=a.page_table), _paged_layer(page_tokens=8, table=a.page_table)):
        with pytest.raises(tsv.TsvError, match="page sizes"):
            pg.PagePool.of_layers([a, b])
    with pytest.raises(tsv.TsvError, match="one page table"):
        pg.PagePool.of_layers([a, _paged_layer(table=a.page_table.clone())])
    with pytest.raises(tsv.TsvError):
        pg.PagePool.of_layers([])


def test_missing_arguments_and_other_ranks_are_refused(api, monkeypatch):
    """None, numbers and tensors of another rank where a tensor is needed: the library's own error, before it is called.  (On the CPU, taken for the
    current device; a call that gets through would end in the library's refusal of a NULL pointer or of the workspace.)"""
    import torch
    tsv, tk, pg = api
    for m in (tk, pg):
        monkeypatch.setattr(m, "_device", lambda: -1)
        monkeypatch.setattr(m, "_on", lambda stream, dev: 0)
    s = tk.TokenShape("bf16", 2, 4, 2, 16, window=8, max_L=64, max_n=4)
    i32 = lambda *sh: torch.zeros(*sh, dtype=torch.int32)
    z = lambda h: torch.zeros(5, h, 16, dtype=torch.bfloat16)
    batch, st = tk.TokenBatch(torch.zeros(2, dtype=torch.int64), i32(2)), i32(2)
    cache = tk.alloc_token_cache(s, device="cpu")
    table = lambda t: tk.TokenCache(cache.L, cache.k, cache.v, t, 4)
    ws = torch.zeros(64, dtype=torch.uint8)
    rope = lambda L=st, q=z(4), k=z(2), qo=z(4), ko=z(2), w=None, inv=torch.zeros(8), status=st, b=batch: tk.qk_norm_rope(s, L, b, q, k, qo, ko, w, w, 1e-6, inv, 0, False, status)
    attn = lambda c=cache, b=batch, q=z(4), k=z(2), v=z(2), out=z(4), ws=ws, status=st: tk.window_sink_attn(s, c, b, q, k, v, out, ws, status)
    commit = lambda c=cache, b=batch, k=z(2), v=z(2), status=st, path=None, count=None: tk.token_commit(s, c, b, k, v, status, path=path, count=count)
    calls = [lambda x=x: rope(**{x: bad}) for x in ("L", "qo", "ko", "status") for bad in (None, 3)]
    calls += [lambda: rope(q=None, k=None), lambda: rope(q=3), lambda: rope(w=3), lambda: rope(inv=torch.zeros(8, dtype=torch.float64))]
    calls += [lambda x=x, bad=bad: attn(**{x: bad}) for x in ("q", "k", "out", "ws", "status") for bad in ((3,) if x == "ws" else (3, torch.zeros(())))]
    calls += [lambda: attn(k=None), lambda: attn(out=None), lambda: attn(ws=None), lambda: attn(status=None), lambda: attn(q=None)]
    calls += [lambda t=t: attn(c=table(t)) for t in (i32(6), i32(2, 3, 1), 3)] + [lambda: attn(c=tk.TokenCache(None, cache.k)), lambda: attn(c=tk.TokenCache(cache.L, None))]
    calls += [lambda b=b: attn(b=b) for b in (tk.TokenBatch(None, i32(2)), tk.TokenBatch(batch.row0, None), tk.TokenBatch(batch.row0, batch.n, 3))]
    calls += [lambda: commit(k=None), lambda: commit(status=None), lambda: commit(path=i32(8)), lambda: commit(path=3), lambda: commit(path=i32(1, 4)), lambda: commit(count=3)]
    pool = pg.PagePool.__new__(pg.PagePool)
    pool.device, pool.page_table, pool.c = -1, i32(2, 3), pg.CPagePool()
    one = i32(1)
    calls += [lambda: pg.pages_assign(pool, None, one, one, ws, one), lambda: pg.pages_assign(pool, one, None, one, ws, one), lambda: pg.pages_assign(pool, one, one, one, None, one),
              lambda: pg.pages_free(pool, None, one, one, one), lambda: pg.pages_free(pool, one, one, one, None), lambda: pg.pages_fork(pool, None, one, one, ws, one),
              lambda: pg.pages_fork(pool, one, one, None, ws, one), lambda: pg.pages_fork(pool, one, one, one, None, one), lambda: pg.pages_compact(pool, None, ws),
              lambda: pg.pages_compact(pool, one, None), lambda: pg.PagePool(i32(6), one, 4, []), lambda: pg.PagePool(None, one, 4, []), lambda: pg.PagePool(i32(2, 3), None, 4, [])]
    for i, call in enumerate(calls):
        with pytest.raises(tsv.TsvError):
            call()
            raise AssertionError(f"call {i} went through")


def test_rope_outputs_over_other_rows_are_refused(api):
    """Against marks of every element: any sharing but that of an output with its input at the same address and stride."""
    tsv, tk, _ = api
    a, s = C.addressof, _shape(tk, H=2, Hk=1, d=8)
    n, es = 3, 2
    batch = tk.CTokBatch(FAKE, FAKE, None, n)

    def marks(base, ld, heads):
        return {base + (r * ld + i) * es for r in range(n) for i in range(heads * 8)}
    rng = np.random.default_rng(0)
    refused = 0
    for _ in range(1500):
        ld = [int(x) * 8 for x in rng.integers(3, 6, 4)]
        if rng.random() < 0.6:
            ld = [ld[0]] * 4
        base = [FAKE + 16 * int(x) for x in rng.integers(0, 24, 4)]
        if rng.random() < 0.3:
            base[2] = base[0]
        if rng.random() < 0.3:
            base[3] = base[1]
        q, k, qo, ko = (marks(b, l, h) for b, l, h in zip(base, ld, (2, 1, 2, 1)))
        own = lambda out, i: base[out] == base[i] and ld[out] == ld[i]
        bad = (q & qo and not own(2, 0)) or (k & ko and not own(3, 1)) or (qo & k) or (ko & q) or (qo & ko)
        if not bad:
            continue
        io = tk.CTokRows(base[0], base[1], None, ld[0], ld[1], 0)
        assert tsv._lib.qk_norm_rope(a(s), FAKE, a(batch), a(io), None, None, 1e-6, None, 0, 0, 0, base[2], ld[2], base[3], ld[3], FAKE, None) == tsv.ERR_SHAPE, (base, ld)
        refused += 1
    assert refused > 500
