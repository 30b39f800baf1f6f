"""Decoder blocks where the cache has no room for a token: the token is refused, no row of any request changes, and it can be asked for again."""
import numpy as np
import pytest
import torch

import paper_2609_18063_b200 as edg
from paper_2609_18063_b200 import layer_io
from paper_2609_18063_b200.decoder import BlockDecoder, LatentBlock, LatentCache
from workloads import synth

from test_gpu_blocks import DL, DN, DR, DV, HEADS, _projection

pytestmark = pytest.mark.gpu

PAGE = 16


class World:
    """Two layers, a cache of n_pages, requests 0 and 1."""

    def __init__(self, n_pages, max_pages, max_total=None):
        cfg = synth.CONFIGS["cfg1"].with_(n_layers=2, n_slots=16)
        self.L, self.H = cfg.n_layers, cfg.H
        self.d = d = edg.make_desc(cfg)
        hosts = [layer_io.host_layer(d, lambda e, l=l: synth.expert_tensors(cfg, l, e)) for l in range(self.L)]
        loras, self.keep = zip(*[layer_io.lora_to_device(d, [synth.lora_tensors(cfg, l, 0)]) for l in range(self.L)])
        self.slots = torch.zeros((self.L, 16, edg.record_bytes(d)), dtype=torch.uint8, device="cuda")
        self.tables = torch.zeros((self.L, cfg.E), dtype=torch.int32, device="cuda")
        self.stream = torch.cuda.Stream()
        self.store = edg.Store(d, hosts, self.slots, self.tables, list(loras), self.stream)
        self.W_pre = torch.from_numpy(np.stack([synth.prerouter_weights(cfg, l) for l in range(self.L)])).cuda()
        rng, g = np.random.default_rng(3), torch.Generator().manual_seed(4)
        self.cache = LatentCache(self.L, n_pages=n_pages, page=PAGE, row=DL + DR, n_seqs=2, max_pages=max_pages)
        desc = edg.make_latent_desc(heads=HEADS, d_nope=DN, d_rope=DR, d_v=DV, d_latent=DL, page=PAGE, n_pages=n_pages, max_pages=max_pages, scale=(DN + DR) ** -0.5)
        inv_freq = (10000.0 ** (-torch.arange(0, DR, 2) / DR)).float().cuda()
        self.blocks = []
        for _ in range(self.L):
            w = [_projection(rng, *s)[0] for s in ((HEADS * (DN + DR), self.H, "bf16"), (DL + DR, self.H, "bf16"), (self.H, HEADS * DV, "f32"))]
            uk, uv = [(torch.randn((HEADS, k, DL), generator=g) * DL ** -0.5).bfloat16().cuda() for k in (DN, DV)]
            self.blocks.append(LatentBlock(desc, *w, uk, uv, None, inv_freq, max_rows=1, max_seqs=1, max_new=1, max_total=max_total or max_pages * PAGE))
        self.first = torch.randn(self.H, generator=g).bfloat16().cuda()

    def decoder(self, seq):
        dec = BlockDecoder(self.d, self.store, self.W_pre, self.blocks, self.cache, seq=seq)
        dec.prime(self.first.expand(self.L, self.H).contiguous())
        return dec

    def state(self):
        torch.cuda.synchronize()
        return [v.clone() for v in (self.cache.rows, self.cache.refs, self.cache.table, self.cache.lens)]

    def refuse(self, dec, t, x, code):
        before, out, misses = self.state(), dec.x_out.clone(), dec.misses
        for _ in range(2):                                     # (asked for twice: the routing that it takes is still there)
            with pytest.raises(edg.EdgError) as e:
                dec.token(t, x)
            assert e.value.code == code
        assert all(torch.equal(a, b) for a, b in zip(before, self.state())) and torch.equal(out, dec.x_out) and dec.misses == misses


def _one(v):
    return torch.tensor([v], dtype=torch.int32, device="cuda")


def test_a_sequence_that_is_full():
    w = World(n_pages=4, max_pages=1)
    dec, x = w.decoder(0), w.first
    for t in range(PAGE):
        x = dec.token(t, x).clone()
    assert w.cache.status() == 0
    w.refuse(dec, PAGE, x, -4)
    assert w.cache.lens.tolist() == [PAGE, 0]
    w.store.close()


def test_a_pool_without_a_page_for_the_copy_of_a_shared_one():
    """Request 1 is forked from 0 within a page; its next token needs a page of its own, and there is none.  The rows that 0 reads keep their bits; when 0
    is freed the token goes through, with the bits that it has where there was room all along."""
    results = []
    for n_pages in (2, 8):
        w = World(n_pages=n_pages, max_pages=2)
        dec, x = w.decoder(0), w.first
        for t in range(20):
            x = dec.token(t, x).clone()
        w.cache.fork(_one(0), _one(1))
        other, x2, got = w.decoder(1), w.first, []
        if n_pages == 2:
            w.refuse(other, 0, x2, -3)
            assert w.cache.lens.tolist() == [20, 20] and w.cache.refs.tolist() == [2, 2]
        got.append(dec.x_out.clone())
        w.cache.free(_one(0))
        for t in range(3):
            x2 = other.token(t, x2).clone()
            got.append(x2)
        assert w.cache.lens.tolist() == [0, 23] and w.cache.status() == 0 and all(edg.workspace_status(b.ws) == 0 for b in w.blocks)
        results.append(got)
        w.store.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_a_pool_that_is_empty_at_a_page_end():
    w = World(n_pages=1, max_pages=2)
    dec, x = w.decoder(0), w.first
    for t in range(PAGE):
        x = dec.token(t, x).clone()
    w.refuse(dec, PAGE, x, -3)
    w.store.close()


def test_more_positions_than_the_blocks_are_made_for():
    w = World(n_pages=4, max_pages=2, max_total=5)
    dec, x = w.decoder(0), w.first
    for t in range(5):
        x = dec.token(t, x).clone()
    w.refuse(dec, 5, x, -4)
    assert w.cache.status() == 0 and all(edg.workspace_status(b.ws) == 0 for b in w.blocks)
    w.store.close()
