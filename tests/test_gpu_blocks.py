"""Whole decoder blocks, token by token: int4 projections, latent attention over a paged cache and the MoE layer-step, against 64 bits from each
block's own input; a request that is forked halfway goes its own way."""
import numpy as np
import pytest
import torch

import paper_2609_18063_b200 as edg
from oracle import moe_oracle as orc
from paper_2609_18063_b200 import layer_io
from paper_2609_18063_b200.decoder import BlockDecoder, LatentBlock, LatentCache
from workloads import synth

from _gpu_util import TOL_MAX_ABS, TOL_REL_L2

pytestmark = pytest.mark.gpu

HEADS, DN, DR, DV, DL = 8, 64, 32, 64, 256


def _projection(rng, N, K, out, rank=0):
    d = edg.make_linear_desc(N, K, group=64, rank=rank, out_dtype=out, lora_scale=2.0)
    codes = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    sc, ze = np.full((N, K // 64), 0.2 * K ** -0.5, np.float16), np.full((N, K // 64), 7.5, np.float16)
    q = np.empty((N, K))
    q[:, 0::2], q[:, 1::2] = codes & 15, codes >> 4
    W = torch.from_numpy((q - 7.5) * float(sc[0, 0])).cuda()
    w = (d, torch.from_numpy(edg.pack_linear(d, codes, sc, ze)).cuda())
    if rank:
        g = torch.Generator().manual_seed(N)
        A, B = (torch.randn((rank, K), generator=g) * 0.02).bfloat16().cuda(), (torch.randn((N, rank), generator=g) * 0.05).bfloat16().cuda()
        return w + (A, B), W + 2.0 * B.double() @ A.double()
    return w, W


class Reference:
    """One layer's attention half in 64 bits, with the rows of a request so far."""

    def __init__(self, Wq, Wkv, Wo, uk, uv, gain, inv_freq, rows=()):
        self.w = (Wq, Wkv, Wo, uk, uv, gain, inv_freq)
        self.rows = list(rows)

    def fork(self):
        return Reference(*self.w, rows=self.rows)

    def step(self, x):
        Wq, Wkv, Wo, uk, uv, gain, inv_freq = self.w
        ang = len(self.rows) * inv_freq.double()
        co, si = ang.cos(), ang.sin()
        rot = lambda v: torch.stack([v[..., 0::2] * co - v[..., 1::2] * si, v[..., 0::2] * si + v[..., 1::2] * co], -1).flatten(-2)   # noqa: E731
        q, kv = (Wq @ x).view(HEADS, DN + DR), Wkv @ x
        c = kv[:DL] / torch.sqrt((kv[:DL] ** 2).mean() + 1e-6) * gain.double()
        self.rows.append((c, rot(kv[DL:])))
        C, P = torch.stack([a for a, _ in self.rows]), torch.stack([b for _, b in self.rows])
        s = torch.einsum("hn,hnl,jl->hj", q[:, :DN], uk.double(), C) + rot(q[:, DN:]) @ P.T
        p = torch.softmax(s * (DN + DR) ** -0.5, dim=-1)
        return Wo @ torch.einsum("hj,jl,hvl->hv", p, C, uv.double()).flatten()


def _norm(v):
    return v / torch.sqrt((v ** 2).mean() + 1e-6)


@pytest.mark.parametrize("n_slots", [4, 16])
def test_blocks_token_by_token(n_slots):
    cfg = synth.CONFIGS["cfg1"].with_(n_layers=2, n_slots=n_slots)
    L, H, K = cfg.n_layers, cfg.H, cfg.K
    d = edg.make_desc(cfg)
    experts = {}
    get = lambda l, e: experts.setdefault((l, e), synth.expert_tensors(cfg, l, e))      # noqa: E731
    hosts = [layer_io.host_layer(d, lambda e, l=l: get(l, e)) for l in range(L)]
    loras_np = [synth.lora_tensors(cfg, l, 0) for l in range(L)]
    loras, keep = zip(*[layer_io.lora_to_device(d, [ln]) for ln in loras_np])
    slots = torch.zeros((L, n_slots, edg.record_bytes(d)), dtype=torch.uint8, device="cuda")
    tables = torch.zeros((L, cfg.E), dtype=torch.int32, device="cuda")
    store = edg.Store(d, hosts, slots, tables, list(loras), torch.cuda.Stream())
    W_pre = torch.from_numpy(np.stack([synth.prerouter_weights(cfg, l) for l in range(L)])).cuda()

    rng, g = np.random.default_rng(11), torch.Generator().manual_seed(12)
    cache = LatentCache(L, n_pages=14, page=16, row=DL + DR, n_seqs=2, max_pages=4)
    desc = edg.make_latent_desc(heads=HEADS, d_nope=DN, d_rope=DR, d_v=DV, d_latent=DL, page=16, n_pages=14, max_pages=4, scale=(DN + DR) ** -0.5)
    inv_freq = (10000.0 ** (-torch.arange(0, DR, 2) / DR)).float().cuda()
    blocks, refs = [], []
    for l in range(L):
        wq, Wq = _projection(rng, HEADS * (DN + DR), H, "bf16", rank=8)
        wkv, Wkv = _projection(rng, DL + DR, H, "bf16")
        wo, Wo = _projection(rng, H, HEADS * DV, "f32", rank=8)
        uk = (torch.randn((HEADS, DN, DL), generator=g) * DL ** -0.5).bfloat16().cuda()
        uv = (torch.randn((HEADS, DV, DL), generator=g) * DL ** -0.5).bfloat16().cuda()
        gain = (1 + 0.1 * torch.randn(DL, generator=g)).bfloat16().cuda()
        blocks.append(LatentBlock(desc, wq, wkv, wo, uk, uv, gain, inv_freq, max_rows=1, max_seqs=1, max_new=1, max_total=64))
        refs.append(Reference(Wq, Wkv, Wo, uk, uv, gain, inv_freq))
    first = torch.randn(H, generator=g).bfloat16().cuda()

    def check(dec, refs, t, x):
        inds, gates = dec.inds[t % 2].cpu().numpy().copy(), dec.gates[t % 2].cpu().numpy().astype(np.float64)
        out = dec.token(t, x)
        torch.cuda.synchronize()
        for l in range(L):
            # five roundings to bf16 lie between a block's input and its attention output (queries, rows, one inside, weights, values), each at most
            # 2^-8 and mostly independent: six times sqrt 5 * 2^-8 / sqrt 3 in the norm; the state is rounded once more (half a step of each value)
            o = refs[l].step(x.double())
            want = _norm(x.double() + o)
            got = dec.x_moe[l].double()
            assert (got - want).norm() <= (6 * 5 ** 0.5 * 2.0 ** -8 / 3 ** 0.5 * o.norm() / (x.double() + o).norm() + 2.0 ** -8) * want.norm()
            bits = dec.x_moe[l].view(torch.int16).cpu().numpy().view(np.uint16)
            ref = orc.moe_ffn(bits, inds[l], gates[l], lambda e: get(l, e), lambda e: loras_np[l], cfg.lora_scale, cfg.group)
            y = dec.y[l].cpu().numpy()
            assert orc.max_abs(y, ref) <= TOL_MAX_ABS and orc.rel_l2(y, ref) <= TOL_REL_L2
            nxt = _norm(dec.x_moe[l].double() + dec.y[l].double())
            assert (dec.x_out[l].double() - nxt).abs().max() <= 2.0 ** -8 * nxt.abs().max()
            x = dec.x_out[l].clone()
        return out.clone()
    dec = BlockDecoder(d, store, W_pre, blocks, cache)
    dec.prime(first.expand(L, H).contiguous())
    x = first
    for t in range(20):                                        # over a page's end
        x = check(dec, refs, t, x)
    one = lambda v: torch.tensor([v], dtype=torch.int32, device="cuda")       # noqa: E731
    cache.fork(one(0), one(1))
    other = BlockDecoder(d, store, W_pre, blocks, cache, seq=1)
    other.prime(first.expand(L, H).contiguous())
    refs2, x2 = [r.fork() for r in refs], first
    for t in range(4):
        x, x2 = check(dec, refs, 20 + t, x), check(other, refs2, t, x2)
    assert cache.lens.tolist() == [24, 24] and cache.table[0, 0] == cache.table[1, 0] and cache.table[0, 1] != cache.table[1, 1]
    cache.free(one(0))
    cache.compact()
    for t in range(4, 6):
        x2 = check(other, refs2, t, x2)
    assert cache.status() == 0 and all(edg.workspace_status(b.ws) == 0 for b in blocks) and edg.workspace_status(dec.ws) == 0
    assert cache.refs.tolist() == [1, 1] + [0] * 12
    store.close()


def test_a_block_takes_prompts_and_batches():
    """The same rows one at a time (three requests beside one another) and as prompts: the same cache rows and outputs within their roundings."""
    H = 512
    rng, g = np.random.default_rng(5), torch.Generator().manual_seed(6)
    wq, _ = _projection(rng, HEADS * (DN + DR), H, "bf16")
    wkv, _ = _projection(rng, DL + DR, H, "bf16")
    wo, _ = _projection(rng, H, HEADS * DV, "f32")
    uk, uv = (torch.randn((HEADS, DN, DL), generator=g) * DL ** -0.5).bfloat16().cuda(), (torch.randn((HEADS, DV, DL), generator=g) * DL ** -0.5).bfloat16().cuda()
    inv_freq = (10000.0 ** (-torch.arange(0, DR, 2) / DR)).float().cuda()
    n, m = 3, 100
    x = torch.randn((n * m, H), generator=g).bfloat16().cuda()
    results = []
    for step in (1, m):
        cache = LatentCache(1, n_pages=30, page=16, row=DL + DR, n_seqs=n, max_pages=8)
        desc = edg.make_latent_desc(heads=HEADS, d_nope=DN, d_rope=DR, d_v=DV, d_latent=DL, page=16, n_pages=30, max_pages=8, scale=(DN + DR) ** -0.5)
        block = LatentBlock(desc, wq, wkv, wo, uk, uv, None, inv_freq, max_rows=n * m, max_seqs=n, max_new=m, max_total=n * m)
        seqs = torch.arange(n, dtype=torch.int32, device="cuda")
        y = torch.empty((n, m, H), device="cuda")
        for at in range(0, m, step):
            cache.reserve(seqs, torch.full_like(seqs, step))
            rows = x.view(n, m, H)[:, at:at + step].reshape(n * step, H).contiguous()
            out = torch.empty((n * step, H), device="cuda")
            block.run(rows, out, torch.arange(n + 1, dtype=torch.int32, device="cuda") * step, cache.lens, cache.table, cache.rows[0], max_new=step)
            y[:, at:at + step] = out.view(n, step, H)
        assert cache.status() == 0 and edg.workspace_status(block.ws) == 0 and cache.lens.tolist() == [m] * n
        latent = torch.stack([cache.rows[0][cache.table[i, :(m + 15) // 16].long()].flatten(0, 1)[:m] for i in range(n)])
        results.append((y.double(), latent))
    # A projection's fp32 sum is taken in an order that depends on the number of rows, so a value next to the middle of two bf16 numbers may
    # go to either: one step (2^-7) of kv.  The norm scales it, rounding to the cache adds at most another: 2^-6 of a latent value.  A rotated
    # value takes it from both of its pair, at most sqrt 2 times the pair's magnitude, and its own rounding: 2^-5 of that magnitude.
    (_, u), (_, v) = results
    u, v = u.double(), v.double()
    assert ((u - v)[..., :DL].abs() <= 2.0 ** -6 * u[..., :DL].abs()).all()
    pair = (u[..., DL::2] ** 2 + u[..., DL + 1::2] ** 2).sqrt().repeat_interleave(2, dim=-1)
    assert ((u - v)[..., DL:].abs() <= 2.0 ** -5 * pair).all()
    # four roundings to bf16 differ between the two forms and the output's input is one more: six times sqrt 5 * 2^-8 / sqrt 3 in the norm
    a, b = results[0][0], results[1][0]
    assert (a - b).norm() <= 6 * 5 ** 0.5 * 2.0 ** -8 / 3 ** 0.5 * a.norm()
