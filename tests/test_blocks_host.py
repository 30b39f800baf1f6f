"""Decoder blocks: what is refused before anything is launched.  Tensors of this process's memory stand for device ones; no call gets them."""
import pytest
import torch

HEADS, DN, DR, DV, DL, H = 2, 32, 16, 32, 128, 64


@pytest.fixture(scope="module")
def edg():
    from paper_2609_18063_b200 import build
    build.build()
    import paper_2609_18063_b200 as m
    return m


def _desc(edg, **kw):
    return edg.make_latent_desc(**dict(dict(heads=HEADS, d_nope=DN, d_rope=DR, d_v=DV, d_latent=DL, page=16, n_pages=6, max_pages=4, scale=0.1), **kw))


def _projection(edg, N, K, out="bf16", rank=0, **kw):
    d = edg.make_linear_desc(N, K, group=32, rank=rank, out_dtype=out, **kw)
    w = (d, torch.zeros(edg.linear_record_bytes(d), dtype=torch.uint8))
    return w + (torch.zeros((rank, K), dtype=torch.bfloat16), torch.zeros((N, rank), dtype=torch.bfloat16)) if rank else w


def _parts(edg, **kw):
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16)      # noqa: E731
    a = dict(desc=_desc(edg), w_q=_projection(edg, HEADS * (DN + DR), H, rank=8), w_kv=_projection(edg, DL + DR, H), w_out=_projection(edg, H, HEADS * DV, "f32"),
             w_uk=b(HEADS, DN, DL), w_uv=b(HEADS, DV, DL), gain=b(DL), inv_freq=torch.zeros(DR // 2), max_rows=3, max_seqs=2, max_new=2, max_total=40)
    return dict(a, **kw)


def _block(edg, **kw):
    from paper_2609_18063_b200.decoder import LatentBlock
    return LatentBlock(**_parts(edg, **kw))


def test_a_block_of_fitting_parts(edg):
    b = _block(edg)
    assert b.q.dtype == b.kv.dtype == b.a.dtype == torch.bfloat16 and b.q.shape == (3, HEADS * (DN + DR)) and b.a.shape == (3, HEADS * DV)
    for out in ("f16", "bf16", "f32"):
        _block(edg, w_out=_projection(edg, H, HEADS * DV, out), gain=None)
    _block(edg, desc=_desc(edg, ldq=HEADS * (DN + DR), ldkv=DL + DR), w_kv=_projection(edg, DL + DR, H, ldx=H, ldy=DL + DR))


def test_attention_outputs_that_the_next_projection_would_misread_are_refused(edg):
    with pytest.raises(ValueError, match="bf16"):
        _block(edg, desc=_desc(edg, out_dtype="f16"))


@pytest.mark.parametrize("out", ["f16", "f32"])
def test_queries_and_rows_of_another_type_are_refused(edg, out):
    for kw in (dict(w_q=_projection(edg, HEADS * (DN + DR), H, out)), dict(w_kv=_projection(edg, DL + DR, H, out))):
        with pytest.raises(ValueError, match="bf16"):
            _block(edg, **kw)


def test_parts_of_other_sizes_are_refused(edg):
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16)      # noqa: E731
    short = _projection(edg, DL + DR, H)
    with_rank = _projection(edg, DL + DR, H, rank=8)
    for kw in (dict(w_q=_projection(edg, HEADS * (DN + DR) + 1, H)), dict(w_q=_projection(edg, HEADS * (DN + DR), 2 * H)), dict(w_kv=_projection(edg, DL, H)),
               dict(w_out=_projection(edg, H + 1, HEADS * DV)), dict(w_out=_projection(edg, H, 2 * HEADS * DV)), dict(w_kv=_projection(edg, DL + DR, H, ldy=DL + DR + 8)),
               dict(w_kv=_projection(edg, DL + DR, H, ldx=H + 8)), dict(desc=_desc(edg, ldq=HEADS * (DN + DR) + 8)), dict(desc=_desc(edg, ldkv=DL + DR + 8)),
               dict(w_kv=(short[0], short[1][:-1])), dict(w_kv=with_rank[:2]), dict(w_kv=short + with_rank[2:]), dict(w_kv=with_rank[:2] + (with_rank[2][:4], with_rank[3])),
               dict(w_kv=with_rank[:3] + (with_rank[3].float(),)), dict(w_uk=b(HEADS, DN, DL + 1)), dict(w_uk=b(HEADS, DN, DL).float()), dict(w_uv=b(HEADS, DN + 16, DL)),
               dict(gain=b(DL - 1)), dict(gain=torch.zeros(DL)), dict(inv_freq=torch.zeros(DR)), dict(inv_freq=b(DR // 2)),
               dict(w_kv=(short[0], short[1].to("meta")))):
        with pytest.raises(ValueError):
            _block(edg, **kw)


def _call(edg, **kw):
    """Arguments of a run of three rows of two sequences"""
    i = lambda v: torch.tensor(v, dtype=torch.int32)      # noqa: E731
    return dict(dict(x=torch.zeros((3, H), dtype=torch.bfloat16), y=torch.zeros((3, H)), cu=i([0, 1, 3]), lens=i([5, 9]),
                     table=torch.zeros((2, 4), dtype=torch.int32), rows=torch.zeros((6, 16, DL + DR), dtype=torch.bfloat16), max_new=2), **kw)


@pytest.fixture
def launched(edg, monkeypatch):
    """Names of the library's calls, none of which is made"""
    from paper_2609_18063_b200 import binding
    names = []
    for name in ("linear_int4_lora", "latent_append", "latent_attention"):
        monkeypatch.setattr(binding, name, lambda *a, _n=name, **k: names.append(_n))
    return names


def test_a_run_within_the_bounds_makes_its_calls(edg, launched):
    _block(edg).run(**_call(edg))
    assert launched == ["linear_int4_lora"] * 2 + ["latent_append", "latent_attention", "linear_int4_lora"]


def test_runs_beyond_the_bounds_launch_nothing(edg, launched):
    """The block is made for 3 rows of 2 sequences, 2 new ones each, 40 positions."""
    i = lambda v: torch.tensor(v, dtype=torch.int32)      # noqa: E731
    b = _block(edg)
    for T in (4, 8, 64):
        with pytest.raises(ValueError):
            b.run(**_call(edg, x=torch.zeros((T, H), dtype=torch.bfloat16), y=torch.zeros((T, H))))
    for kw in (dict(x=torch.zeros((0, H), dtype=torch.bfloat16), y=torch.zeros((0, H))), dict(cu=i([0])), dict(cu=i([0, 1, 2, 3]), lens=i([5, 9, 9]), table=torch.zeros((3, 4), dtype=torch.int32)),
               dict(max_new=3), dict(max_new=0), dict(total=41), dict(total=-1),
               dict(x=torch.zeros((1, H), dtype=torch.bfloat16), y=torch.zeros((1, H)), cu=i([0, 1, 1]))):          # (two new rows of one sequence, one in all)
        with pytest.raises(ValueError):
            b.run(**_call(edg, **kw))
    assert launched == []


def test_tensors_that_do_not_fit_launch_nothing(edg, launched):
    i = lambda v: torch.tensor(v, dtype=torch.int32)      # noqa: E731
    b = _block(edg)
    for kw in (dict(x=torch.zeros((3, H))), dict(x=torch.zeros((3, H + 8), dtype=torch.bfloat16)), dict(x=torch.zeros((3, 2 * H), dtype=torch.bfloat16)[:, :H]),
               dict(y=torch.zeros((3, H), dtype=torch.bfloat16)), dict(y=torch.zeros((2, H))), dict(y=torch.zeros((3, H), device="meta")), dict(y=torch.zeros((3, 2 * H))[:, :H]),
               dict(cu=torch.tensor([0, 1, 3])), dict(lens=torch.tensor([5, 9])), dict(lens=i([5])), dict(table=torch.zeros((2, 4), dtype=torch.int64)),
               dict(table=torch.zeros((1, 4), dtype=torch.int32)), dict(table=torch.zeros((2, 5), dtype=torch.int32)), dict(table=torch.zeros(8, dtype=torch.int32)),
               dict(rows=torch.zeros((5, 16, DL + DR), dtype=torch.bfloat16)), dict(rows=torch.zeros((6, 16, DL + DR))), dict(rows=torch.zeros((6, 16, DL), dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            b.run(**_call(edg, **kw))
    assert launched == []


@pytest.fixture
def stack(edg, monkeypatch):
    """BlockDecoder(blocks, cache, seq) over a stack of one layer that has no store"""
    from paper_2609_18063_b200 import decoder

    def base(self, desc, store, W_pre, prefetch=True):
        self.desc, self.store, self.W_pre, self.L = desc, store, W_pre, 1
    monkeypatch.setattr(decoder.StackDecoder, "__init__", base)

    def make(block=None, cache=None, seq=0, out="f32", **kw):
        d = edg.make_desc(None, out_dtype=out, **dict(dict(H=H, I=64, E=8, K=2, group=32, rank=8, n_adapters=1, n_slots=4, lora_scale=1.0), **kw))
        c = decoder.LatentCache(*(cache or (1, 6, 16, DL + DR, 2, 4)), device="cpu")
        return decoder.BlockDecoder(d, None, torch.zeros(1), [block or _block(edg)], c, seq=seq)
    return make


def test_stacks_whose_parts_do_not_fit_are_refused(edg, stack):
    assert stack().o.dtype == torch.float32 and stack(seq=1).o.shape == (H,)
    assert stack(_block(edg, w_out=_projection(edg, H, HEADS * DV, "f16")), out="f16").o.dtype == torch.float16
    for kw in (dict(out="bf16"), dict(out="f16"), dict(H=2 * H), dict(seq=2), dict(seq=-1), dict(cache=(2, 6, 16, DL + DR, 2, 4)), dict(cache=(1, 5, 16, DL + DR, 2, 4)),
               dict(cache=(1, 6, 32, DL + DR, 2, 4)), dict(cache=(1, 6, 16, DL, 2, 4)), dict(cache=(1, 6, 16, DL + DR, 2, 5))):
        with pytest.raises(ValueError):
            stack(**kw)


def test_a_state_that_is_no_state_is_refused_first(edg, stack):
    dec = stack()
    for x in (torch.zeros(H), torch.zeros(H - 1, dtype=torch.bfloat16), torch.zeros((2, H), dtype=torch.bfloat16), torch.zeros(2 * H, dtype=torch.bfloat16)[::2]):
        with pytest.raises(ValueError):
            dec.token(0, x)


def test_lists_that_are_no_lists_are_refused(edg, monkeypatch):
    """Of another type, on another device than the cache, or shorter than the one beside them: the kernels would read behind them."""
    from paper_2609_18063_b200 import binding, decoder
    names = []
    for name in ("pages_reserve", "pages_fork", "pages_free"):
        monkeypatch.setattr(binding, name, lambda *a, _n=name: names.append(_n))
    c = decoder.LatentCache(1, 6, 16, DL + DR, 2, 4, device="cpu")
    i = lambda v, **kw: torch.tensor(v, dtype=torch.int32, **kw)      # noqa: E731
    for bad in (torch.tensor([0, 1]), i([0, 1]).to("meta"), torch.tensor([0.0, 1.0])):
        for call in (lambda: c.reserve(bad, i([1, 1])), lambda: c.reserve(i([0, 1]), bad), lambda: c.fork(bad, i([1, 1])), lambda: c.fork(i([0, 0]), bad), lambda: c.free(bad)):
            with pytest.raises(ValueError):
                call()
    for call in (lambda: c.reserve(i([0, 1]), i([1])), lambda: c.fork(i([0]), i([0, 1]))):
        with pytest.raises(ValueError):
            call()
    assert names == []
    c.reserve(i([0, 1]), i([1, 5]))
    c.fork(i([0]), i([1]))
    c.free(i([0]))
    assert names == ["pages_reserve", "pages_fork", "pages_free"]
