"""Host side of the latent cache, its attention and its pages: what is refused before any launch, scratch sizes."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def edg():
    from paper_2609_18063_b200 import build
    build.build()
    import paper_2609_18063_b200 as m
    return m


def _desc(edg, **kw):
    a = dict(heads=8, d_nope=64, d_rope=32, d_v=64, d_latent=256, page=64, n_pages=100, max_pages=10, scale=0.1)
    a.update(kw)
    return edg.make_latent_desc(**a)


@pytest.mark.parametrize("kw,code", [(dict(heads=0), -2), (dict(heads=257), -2), (dict(d_nope=8), -2), (dict(d_nope=144), -2), (dict(d_rope=0), -2),
                                     (dict(d_rope=80), -2), (dict(d_rope=40), -2), (dict(d_v=136), -2), (dict(d_latent=64), -2), (dict(d_latent=320), -2),
                                     (dict(d_latent=640), -2), (dict(page=8), -2), (dict(page=48), -2), (dict(page=512), -2), (dict(n_pages=0), -2),
                                     (dict(n_pages=2 ** 25), -2), (dict(max_pages=0), -2), (dict(max_pages=2 ** 26), -2), (dict(out_dtype="f32"), -1),
                                     (dict(form=3), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(ldkv=280), -2), (dict(ldkv=290), -2), (dict(ldq=760), -2), (dict(ldq=770), -2)])
def test_descriptors_that_are_refused(edg, kw, code):
    with pytest.raises(edg.EdgError) as e:
        edg.latent_workspace_bytes(_desc(edg, **kw), 1, 1, 1, 1)
    assert e.value.code == code


def test_scratch_never_falls(edg):
    for form in (edg.LATENT_AUTO, edg.LATENT_ABSORBED, edg.LATENT_EXPANDED):
        for heads in (1, 8, 33, 128):
            d = _desc(edg, form=form, heads=heads)
            for args in ([(n, 4096, 64, 50000) for n in range(1, 400, 7)], [(4, T, 1, 50000) for T in range(1, 700)],
                         [(4, 4096, m, 50000) for m in range(1, 900)], [(4, 1000, 700, k) for k in range(0, 9000, 50)]):
                size = [edg.latent_workspace_bytes(d, *a) for a in args]
                assert size[0] >= 4096 and all(a <= b for a, b in zip(size, size[1:]))


@pytest.mark.parametrize("args", [(0, 1, 1, 1), (65536, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, -1)])
def test_bounds_that_are_refused(edg, args):
    with pytest.raises(edg.EdgError):
        edg.latent_workspace_bytes(_desc(edg), *args)


def test_attention_calls_that_are_refused_before_any_launch(edg):
    d = _desc(edg)
    n = edg.latent_workspace_bytes(d, 2, 4, 3, 100)
    names = ("cu", "lens", "table", "q", "q_rope", "W_uk", "W_uv", "cache", "y", "ws")
    ok = dict(zip(names, [4096] * len(names)))

    def call(n_seqs=2, T=4, max_new=3, total=100, size=n, **kw):
        a = dict(ok, **kw)
        edg.latent_attention(d, n_seqs, T, max_new, total, *[a[k] for k in names], size, 0)
    for k in names:
        if k != "q_rope":
            with pytest.raises(edg.EdgError) as e:
                call(**{k: None})
            assert e.value.code == -1, k
        with pytest.raises(edg.EdgError) as e:
            call(**{k: 4096 + 2})
        assert e.value.code == (-7 if k == "ws" else -1), k
    for kw, code in [(dict(n_seqs=0), -1), (dict(T=0), -1), (dict(max_new=0), -1), (dict(max_new=5), -1), (dict(total=-1), -1), (dict(size=n - 1), -7)]:
        with pytest.raises(edg.EdgError) as e:
            call(**kw)
        assert e.value.code == code, kw
    with pytest.raises(TypeError):
        edg.latent_attention(edg.make_linear_desc(16, 32, group=32), 1, 1, 1, 1, *[4096] * 10, n, 0)


def test_append_calls_that_are_refused_before_any_launch(edg):
    d = _desc(edg)
    ok = dict(cu=4096, lens=4096, table=4096, kv=4096, gain=4096, eps=1e-6, inv_freq=4096, q=4096, q_rope=4096, cache=4096, ws=4096, size=4096)

    def call(n=1, T=1, **kw):
        a = dict(ok, **kw)
        edg.latent_append(d, n, T, *[a[k] for k in ok if k != "size"], a["size"], 0)
    for kw, code in [(dict(cu=None), -1), (dict(lens=None), -1), (dict(table=None), -1), (dict(kv=None), -1), (dict(inv_freq=None), -1), (dict(cache=None), -1),
                     (dict(ws=None), -1), (dict(q=None), -1), (dict(q_rope=None), -1), (dict(kv=4104), -1), (dict(cache=4104), -1), (dict(q=4104), -1),
                     (dict(gain=4098), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(n=0), -1), (dict(T=0), -1), (dict(size=4095), -7),
                     (dict(ws=4112), -7)]:
        with pytest.raises(edg.EdgError) as e:
            call(**kw)
        assert e.value.code == code, kw


def test_page_calls_that_are_refused_before_any_launch(edg):
    pool = edg.PagePool(100, 16, 8, 10, 4096, 4096, 4096)
    cache = edg.PageCache(4096, 100 * 16 * 64, 2, 100, 16, 64)
    n = edg.pages_workspace_bytes(pool)

    def changed(s, **kw):
        c = type(s).from_buffer_copy(s)
        for k, v in kw.items():
            setattr(c, k, v)
        return c
    for kw, code in [(dict(n_pages=0), -2), (dict(page=0), -2), (dict(n_seqs=0), -2), (dict(max_pages=0), -2), (dict(refs=None), -1), (dict(table=None), -1),
                     (dict(lens=4097), -1), (dict(max_pages=2 ** 30), -2)]:
        for f in (lambda p: edg.pages_fork(p, 1, 4096, 4096, 4096, n, 0), lambda p: edg.pages_free(p, 1, 4096, 4096, n, 0),
                  lambda p: edg.pages_reserve(p, cache, 1, 4096, 4096, 4096, n, 0), lambda p: edg.pages_compact(p, cache, 4096, n, 0),
                  edg.pages_workspace_bytes):
            with pytest.raises(edg.EdgError) as e:
                f(changed(pool, **kw))
            assert e.value.code == code, kw
    for kw, code in [(dict(base=None), -1), (dict(base=4104), -1), (dict(n_layers=0), -2), (dict(n_pages=99), -2), (dict(page=32), -2), (dict(row_bytes=24), -2),
                     (dict(layer_stride=64), -2), (dict(layer_stride=100 * 16 * 64 + 8), -2)]:
        for f in (lambda c: edg.pages_reserve(pool, c, 1, 4096, 4096, 4096, n, 0), lambda c: edg.pages_compact(pool, c, 4096, n, 0)):
            with pytest.raises(edg.EdgError) as e:
                f(changed(cache, **kw))
            assert e.value.code == code, kw
    for bad in (0, -1, 1025):
        for f in (lambda: edg.pages_fork(pool, bad, 4096, 4096, 4096, n, 0), lambda: edg.pages_free(pool, bad, 4096, 4096, n, 0),
                  lambda: edg.pages_reserve(pool, cache, bad, 4096, 4096, 4096, n, 0)):
            with pytest.raises(edg.EdgError) as e:
                f()
            assert e.value.code == -1
    for ws, size, code in [(None, n, -1), (4096, n - 1, -7), (4112, n, -7)]:
        for f in (lambda: edg.pages_fork(pool, 1, 4096, 4096, ws, size, 0), lambda: edg.pages_free(pool, 1, 4096, ws, size, 0),
                  lambda: edg.pages_reserve(pool, cache, 1, 4096, 4096, ws, size, 0), lambda: edg.pages_compact(pool, cache, ws, size, 0)):
            with pytest.raises(edg.EdgError) as e:
                f()
            assert e.value.code == code
    other = changed(cache, base=1 << 30)
    for d, s, k, code in [(cache, changed(other, page=32), 1, -2), (cache, changed(other, row_bytes=32), 1, -2), (cache, changed(other, n_layers=1), 1, -2),
                          (cache, changed(cache, n_pages=50), 1, -2), (cache, other, 0, -1), (cache, other, 65536, -1)]:
        with pytest.raises(edg.EdgError) as e:
            edg.pages_copy(d, s, k, 4096, 4096, 4096, 4096, 0)
        assert e.value.code == code
    with pytest.raises(TypeError):
        edg.pages_free(cache, 1, 4096, 4096, n, 0)


def test_structures_agree_with_the_header(edg):
    assert ctypes.sizeof(edg.LatentDesc) == 14 * 4 and ctypes.sizeof(edg.LinearDesc) == 8 * 4
    assert ctypes.sizeof(edg.PagePool) == 4 * 4 + 3 * 8 and ctypes.sizeof(edg.PageCache) == 8 + 8 + 4 * 4


def test_pools_from_tensors(edg):
    import torch
    refs, table, lens = torch.zeros(7, dtype=torch.int32), torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    p = edg.make_page_pool(refs, table, lens, page=16)
    assert (p.n_pages, p.page, p.n_seqs, p.max_pages, p.table) == (7, 16, 3, 4, table.data_ptr())
    with pytest.raises(ValueError):
        edg.make_page_pool(refs, table, lens[:2], page=16)
    with pytest.raises(ValueError):
        edg.make_page_pool(refs, table.t(), torch.zeros(4, dtype=torch.int32), page=16)
    c = edg.make_page_cache(torch.zeros((2, 7, 16, 24), dtype=torch.bfloat16))
    assert (c.n_layers, c.n_pages, c.page, c.row_bytes, c.layer_stride) == (2, 7, 16, 48, 7 * 16 * 48)
    with pytest.raises(ValueError):
        edg.make_page_cache(torch.zeros((7, 16, 24), dtype=torch.bfloat16))


def test_the_state_machine_itself(edg):
    """The oracle of the GPU tests: shared pages are copied by all growers but the last holder, and come back when nobody holds them."""
    from _latent_ref import Pages
    p = Pages(8, 4, 4, 4)
    assert p.reserve([0], [6]) == (False, False) and p.pages[0] == [0, 1]
    p.rows[0][1][0] = "a"
    assert not p.fork([0, 0], [1, 2]) and p.refs[:2].tolist() == [3, 3]
    assert p.reserve([1, 0, 2], [1, 1, 1]) == (False, False)
    assert [p.pages[i][-1] for i in range(3)] == [3, 2, 1] and p.rows[0][2][0] == p.rows[0][3][0] == "a" and p.refs[:4].tolist() == [3, 1, 1, 1]
    assert p.reserve([3], [17]) == (True, False) and p.reserve([3, 0], [16, 8]) == (False, True)
    p.free([0, 1])
    p.compact()
    assert p.pages[2] == [0, 1] and p.refs.tolist() == [1, 1] + [0] * 6
