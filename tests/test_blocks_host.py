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
