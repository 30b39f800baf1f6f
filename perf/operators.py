"""Performance cases of the operators around the MoE layer-step: int4 projections, attention over a paged cache of latent rows, and
the pages of that cache.

Kinds of work (``case["kind"]``):

* ``linear`` -- y = W x + lora_scale B (A x) for T tokens, W int4 with a scale and a zero point per group: the projections of a
  decoder block and its output head, in the format of the experts.
* ``append`` -- new rows of a latent cache: root-mean-square norm of the latent part, rotation of the positional part, write into
  the sequences' pages; the queries' positional parts are rotated with them.
* ``attend`` -- attention of new rows over the cache, keys and values of all heads coming from one latent row a token; one new row
  a sequence when decoding, many for prompts.
* ``fork``   -- sequences are forked (pages shared), grown (a shared last page is copied, new pages are taken) and some freed.
* ``compact`` -- pages in use are moved to the front of the pool.

A sequence i has ``new[i]`` rows that this step brings and ``lens[i]`` rows in all (texts of numbers in a case), the new ones last; new row r stands at position
``lens[i] - new[i] + r`` and sees every position up to its own.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# head layouts: small ones beside a layer of H = 1024, large ones beside H = 2048
SMALL = dict(heads=8, nope=64, rope=32, v=64, latent=256)
LARGE = dict(heads=32, nope=128, rope=64, v=128, latent=512)


def _text(numbers):
    return " ".join(str(n) for n in numbers)


def _ints(text):
    return [int(n) for n in text.split()]


def listed():
    return [
        # the smallest projection: a square one of the small model, one token
        dict(name="linear_small", kind="linear", T=1, N=1024, K=1024, group=32, rank=8, out="f32"),
        # output projection of an attention block of the large layer, one token
        dict(name="linear_out", kind="linear", T=1, N=2048, K=4096, group=64, rank=16, out="bf16"),
        # query projection of 64 concurrent requests
        dict(name="linear_batch", kind="linear", T=64, N=6144, K=2048, group=64, rank=16, out="bf16"),
        # an output head over an odd vocabulary, 16 requests
        dict(name="linear_head", kind="linear", T=16, N=64001, K=2048, group=64, rank=0, out="f32"),
        # new rows of 64 concurrent requests, one each
        dict(name="append_step", kind="append", new=_text([1] * 64), lens=_text(64 + 61 * i for i in range(64)), page=64, halves=False, **LARGE),
        # new rows of a prompt and of two chunks of others
        dict(name="append_prompt", kind="append", new="4096 333 1", lens="4096 2000 100001", page=64, halves=True, **LARGE),
        # one request of the small model, a short context
        dict(name="attend_small", kind="attend", new="1", lens="333", page=16, out="bf16", **SMALL),
        # 32 requests with contexts from one token to 8192
        dict(name="attend_batch", kind="attend", new=_text([1] * 32), lens=_text(1 + 8191 * i * i // 961 for i in range(32)), page=64, out="bf16", **LARGE),
        # eight long contexts with many heads
        dict(name="attend_long", kind="attend", new=_text([1] * 8), lens=_text(65536 - 17 * i for i in range(8)), page=64, out="bf16", **dict(LARGE, heads=128)),
        # a prompt, a chunk of another one, and a request that decodes beside them
        dict(name="attend_prompt", kind="attend", new="4096 333 1", lens="4096 2000 1007", page=64, out="bf16", **LARGE),
        # 64 continuations of one long prompt: fork, one token each, then half of them end
        dict(name="pages_fork", kind="fork", n_pages=4096, page=64, layers=4, row=576, parents=4, length=5000, children=64, grow=1),
        # a pool with holes between its pages
        dict(name="pages_compact", kind="compact", n_pages=4096, page=64, layers=1, row=576, seqs=48, fill=0.6),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "append", "attend", "attend", "attend", "fork", "compact"])
    if kind == "linear":
        T = _log_int(rng, 1, 64)
        group = rng.choice([32, 64, 128])
        K = 128 * _log_int(rng, 2, 64)
        top = min(64001, 64001 * 2048 // K, 6144 * 2048 * 64 * 4 // (K * T))
        return dict(kind=kind, T=T, N=_log_int(rng, 16, max(16, top)), K=K, group=group, rank=rng.choice([0, 0, 8, 16, 33, 64]),
                    out=rng.choice(["f32", "f16", "bf16"]))
    if kind == "compact":
        return dict(kind=kind, n_pages=_log_int(rng, 16, 4096), page=rng.choice([16, 32, 64]), layers=1, row=rng.choice([128, 288, 576]),
                    seqs=rng.randint(1, 64), fill=rng.uniform(0.1, 0.95))
    if kind == "fork":
        page = rng.choice([16, 32, 64])
        parents = rng.randint(1, 4)
        return dict(kind=kind, n_pages=4096, page=page, layers=rng.choice([1, 4]), row=rng.choice([128, 288, 576]), parents=parents,
                    length=_log_int(rng, 1, 600 * page), children=rng.randint(1, 64), grow=_log_int(rng, 1, 20 * page))
    heads = rng.choice([1, 5, 8, 12, 20, 32, 64, 128])
    lay = rng.choice([dict(SMALL, heads=heads), dict(LARGE, heads=heads), dict(LARGE, heads=heads, nope=64, v=96, latent=384)])
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        n = rng.randint(1, 64)
        new = [_log_int(rng, 1, 4096 // n + 1) for _ in range(n)]
        return dict(kind=kind, new=_text(new), lens=_text(m + _log_int(rng, 1, 4096) - 1 for m in new), page=page, halves=rng.random() < 0.5, **lay)
    if rng.random() < 0.6:                                  # decoding, a few rows at a time at most
        n = rng.randint(1, 64)
        rows = rng.choice([1, 1, 1, 2, 4])
        lens = [_log_int(rng, rows, max(rows + 1, 8 * 65536 * 32 // (n * max(heads, 32)))) for _ in range(n)]
        new = [rows] * n
    else:                                                   # prompts and chunks of them
        lay = dict(lay, heads=min(heads, 32))
        n = rng.randint(1, 4)
        lens = [_log_int(rng, 1, 4096 // n) for _ in range(n)]
        new = [rng.choice([m, rng.randint(1, m), 1]) for m in lens]
    return dict(kind="attend", new=_text(new), lens=_text(lens), page=page, out=rng.choice(["f16", "bf16", "bf16"]), **lay)


_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _numbers(case):
    """The case with its lists of numbers"""
    return dict(case, **{k: _ints(case[k]) for k in ("new", "lens") if k in case})


# ---------------------------------------------------------------- inputs

def _prep_linear(c, g):
    N, K, T, r = c["N"], c["K"], c["T"], c["rank"]
    s = dict(codes=torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8),
             scales=torch.rand((N, K // c["group"]), generator=g, device="cuda").mul_(0.015).add_(0.005).half(),
             zeros=torch.randint(0, 16, (N, K // c["group"]), generator=g, device="cuda").half(),
             x=_normal(g, (T, K)), lora_scale=2.0)
    if r:
        s["A"], s["B"] = _normal(g, (r, K), 0.02), _normal(g, (N, r), 0.01)
    if own:
        import paper_2609_18063_b200 as edg
        d = s["desc"] = edg.make_linear_desc(N, K, group=c["group"], rank=r, out_dtype=c["out"], lora_scale=2.0)
        s["record"] = torch.from_numpy(edg.pack_linear(d, s["codes"].cpu().numpy(), s["scales"].cpu().numpy(), s["zeros"].cpu().numpy())).cuda()
        s["ws"] = torch.zeros(edg.linear_workspace_bytes(d, T), dtype=torch.uint8, device="cuda")
        s["y"] = torch.empty((T, N), dtype=_DT[c["out"]], device="cuda")
    return s


def _tables(lens, page, g, spare=3):
    """Pages of the sequences, in random places of a pool with a few to spare: (table, pages in the pool)."""
    need = [(n + page - 1) // page for n in lens]
    total = sum(need) + spare
    perm = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    t = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        t[i, :n] = perm[at:at + n]
        at += n
    return t, total


def _cumulative(new):
    return torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")


def _latent_desc(c, n_pages, max_pages):
    import paper_2609_18063_b200 as edg
    return edg.make_latent_desc(heads=c["heads"], d_nope=c["nope"], d_rope=c["rope"], d_v=c["v"], d_latent=c["latent"], page=c["page"],
                                n_pages=n_pages, max_pages=max_pages, scale=(c["nope"] + c["rope"]) ** -0.5, out_dtype=c.get("out", "bf16"),
                                rope_halves=c.get("halves", False))


def _prep_append(c, g):
    T, row = sum(c["new"]), c["latent"] + c["rope"]
    table, n_pages = _tables(c["lens"], c["page"], g)
    s = dict(table=table, cu=_cumulative(c["new"]), lens=torch.tensor(c["lens"], dtype=torch.int32, device="cuda"),
             kv=_normal(g, (T, row)), q=_normal(g, (T, c["heads"], c["nope"] + c["rope"])), gain=_normal(g, (c["latent"],), 0.1) + 1,
             inv_freq=(10000.0 ** (-torch.arange(0, c["rope"], 2, dtype=torch.float64) / c["rope"])).float().cuda(),
             cache=_normal(g, (n_pages, c["page"], row)), eps=1e-6)
    if own:
        import paper_2609_18063_b200 as edg
        d = s["desc"] = _latent_desc(c, n_pages, table.shape[1])
        s["ws"] = torch.zeros(edg.latent_workspace_bytes(d, len(c["new"]), T, max(c["new"]), sum(c["lens"])), dtype=torch.uint8, device="cuda")
        s["q_rope"] = torch.empty((T, c["heads"], c["rope"]), dtype=torch.bfloat16, device="cuda")
    return s


def _prep_attend(c, g):
    T, row, h = sum(c["new"]), c["latent"] + c["rope"], c["heads"]
    table, n_pages = _tables(c["lens"], c["page"], g)
    s = dict(table=table, cu=_cumulative(c["new"]), lens=torch.tensor(c["lens"], dtype=torch.int32, device="cuda"), new_host=list(c["new"]),
             lens_host=list(c["lens"]), q=_normal(g, (T, h, c["nope"] + c["rope"])), q_rope=_normal(g, (T, h, c["rope"])),
             W_uk=_normal(g, (h, c["nope"], c["latent"]), c["latent"] ** -0.5), W_uv=_normal(g, (h, c["v"], c["latent"]), c["latent"] ** -0.5),
             cache=_normal(g, (n_pages, c["page"], row)))
    if own:
        import paper_2609_18063_b200 as edg
        d = s["desc"] = _latent_desc(c, n_pages, table.shape[1])
        s["ws"] = torch.zeros(edg.latent_workspace_bytes(d, len(c["new"]), T, max(c["new"]), sum(c["lens"])), dtype=torch.uint8, device="cuda")
        s["y"] = torch.empty((T, h, c["v"]), dtype=_DT[c["out"]], device="cuda")
    return s


def _prep_pages(c, g):
    P, page = c["n_pages"], c["page"]
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    if c["kind"] == "fork":
        n_seqs = c["parents"] + c["children"]
        lens_host = [max(1, c["length"] - 7 * i) for i in range(c["parents"])]
        need = [(n + page - 1) // page for n in lens_host]
        # (as many pages as the pool can hold: the largest children copy a page and take their new ones)
        grow = min(c["grow"], max(1, ((P - sum(need)) // c["children"] - 2) * page))
        max_pages = max(need) + grow // page + 2
        perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
        table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = perm[at:at + n]
            refs[perm[at:at + n].long()] = 1
            at += n
        lens = torch.tensor(lens_host + [0] * c["children"], dtype=torch.int32, device="cuda")
        kids = torch.arange(c["parents"], n_seqs, dtype=torch.int32, device="cuda")
        s = dict(parents=(kids - c["parents"]) % c["parents"], children=kids, counts=torch.full_like(kids, grow), ends=kids[::2].contiguous())
    else:
        used = max(1, int(c["fill"] * P))
        per = max(1, used // c["seqs"])
        n_seqs, max_pages = used // per, per
        perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
        table = perm[:n_seqs * per].view(n_seqs, per).clone()
        refs[perm[:n_seqs * per].long()] = 1
        lens = torch.full((n_seqs,), per * page - 3, dtype=torch.int32, device="cuda")
        s = {}
    s.update(cache=_normal(g, (c["layers"], P, page, c["row"])), table0=table, lens0=lens, refs0=refs, page=page,
             table=table.clone(), lens=lens.clone(), refs=refs.clone())
    if own:
        import paper_2609_18063_b200 as edg
        s["pool"] = edg.make_page_pool(s["refs"], s["table"], s["lens"], page=page)
        s["pages"] = edg.make_page_cache(s["cache"])
        s["ws"] = torch.zeros(edg.pages_workspace_bytes(s["pool"]), dtype=torch.uint8, device="cuda")
    return s


_PREP = {"linear": _prep_linear, "append": _prep_append, "attend": _prep_attend, "fork": _prep_pages, "compact": _prep_pages}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = _PREP[case["kind"]](_numbers(case), g)
    s["case"] = _numbers(case)
    return s


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2609_18063_b200 as edg
    c = s["case"]
    k = c["kind"]
    if k == "linear":
        edg.linear_int4_lora(s["desc"], s["record"], c["T"], s["x"], s.get("A"), s.get("B"), s["y"], s["ws"])
        return s["y"]
    if k == "append":
        edg.latent_append(s["desc"], len(c["new"]), sum(c["new"]), s["cu"], s["lens"], s["table"], s["kv"], s["gain"], s["eps"], s["inv_freq"],
                          s["q"], s["q_rope"], s["cache"], s["ws"])
        return s["q_rope"], s["cache"]
    if k == "attend":
        edg.latent_attention(s["desc"], len(c["new"]), sum(c["new"]), max(c["new"]), sum(c["lens"]), s["cu"], s["lens"], s["table"], s["q"],
                             s["q_rope"], s["W_uk"], s["W_uv"], s["cache"], s["y"], s["ws"])
        return s["y"]
    s["table"].copy_(s["table0"])
    s["lens"].copy_(s["lens0"])
    s["refs"].copy_(s["refs0"])
    if k == "fork":
        edg.pages_fork(s["pool"], len(s["children"]), s["parents"], s["children"], s["ws"])
        edg.pages_reserve(s["pool"], s["pages"], len(s["children"]), s["children"], s["counts"], s["ws"])
        edg.pages_free(s["pool"], len(s["ends"]), s["ends"], s["ws"])
    else:
        edg.pages_compact(s["pool"], s["pages"], s["ws"])
    return s["table"], s["lens"], s["refs"], s["cache"]


# ---------------------------------------------------------------- plain forms

def _weights(s, c, dtype):
    """[N][K] dequantised"""
    q = torch.stack([s["codes"] & 15, s["codes"] >> 4], dim=-1).view(c["N"], -1, c["group"]).to(dtype)
    return ((q - s["zeros"].to(dtype)[..., None]) * s["scales"].to(dtype)[..., None]).view(c["N"], c["K"])


def _plain_linear(s, c):
    x = s["x"].float()
    y = x @ _weights(s, c, torch.float32).T
    if c["rank"]:
        y = y + s["lora_scale"] * ((x @ s["A"].float().T) @ s["B"].float().T)
    return y.to(_DT[c["out"]])


def _positions(s, T):
    """Sequence and position of every new row."""
    t = torch.arange(T, device="cuda")
    seq = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    return seq, s["lens"][seq].long() - s["cu"][seq + 1].long() + t


def _rotate(x, cos, sin, halves):
    if halves:
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)


def _plain_append(s, c):
    T, dl = sum(c["new"]), c["latent"]
    seq, pos = _positions(s, T)
    angle = pos.double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    kv = s["kv"].float()
    lat = kv[:, :dl]
    lat = lat * torch.rsqrt((lat * lat).mean(dim=-1, keepdim=True) + s["eps"]) * s["gain"].float()
    rows = torch.cat([lat, _rotate(kv[:, dl:], cos, sin, c["halves"])], dim=-1).bfloat16()
    q = _rotate(s["q"][..., c["nope"]:].float(), cos[:, None], sin[:, None], c["halves"]).bfloat16()
    page = s["table"][seq, pos // c["page"]].long()
    s["cache"][page, pos % c["page"]] = rows
    return q, s["cache"]


def _context(s, c, i, dtype):
    """Cache rows of sequence i, in order: [len][latent + rope]"""
    n = s["lens_host"][i]
    pages = s["table"][i, :(n + c["page"] - 1) // c["page"]].long()
    return s["cache"][pages].flatten(0, 1)[:n].to(dtype)


def _plain_attend(s, c):
    out, at, dl, scale = [], 0, c["latent"], (c["nope"] + c["rope"]) ** -0.5
    W_uk, W_uv = s["W_uk"].float(), s["W_uv"].float()
    for i, (m, n) in enumerate(zip(s["new_host"], s["lens_host"])):
        row = _context(s, c, i, torch.float32)
        qn, qr = s["q"][at:at + m, :, :c["nope"]].float(), s["q_rope"][at:at + m].float()
        # few new rows: the queries are brought to the latent space; many: keys and values are expanded from it
        if m <= 128:
            ql = torch.einsum("thn,hnl->htl", qn, W_uk)
            sc = ql.flatten(0, 1) @ row[:, :dl].T + qr.transpose(0, 1).flatten(0, 1) @ row[:, dl:].T
            sc = sc.view(c["heads"], m, n)
        else:
            key = torch.einsum("jl,hnl->hjn", row[:, :dl], W_uk)
            sc = qn.transpose(0, 1) @ key.transpose(1, 2) + qr.transpose(0, 1) @ row[:, dl:].T
            del key
        j = torch.arange(n, device="cuda")
        sc.mul_(scale).masked_fill_(j[None] > (n - m + torch.arange(m, device="cuda"))[:, None], float("-inf"))
        sc = torch.exp(sc.sub_(sc.max(dim=-1, keepdim=True).values))
        sc.div_(sc.sum(dim=-1, keepdim=True))
        if m <= 128:
            lat = (sc.view(c["heads"] * m, n) @ row[:, :dl]).view(c["heads"], m, dl)
            out.append(torch.einsum("htl,hvl->thv", lat, W_uv))
        else:
            out.append((sc @ torch.einsum("jl,hvl->hjv", row[:, :dl], W_uv)).transpose(0, 1))
        at += m
    return torch.cat(out).to(_DT[c["out"]])


def _count_refs(refs, pages, by):
    """refs[p] += by for every p >= 0 among the pages"""
    refs.index_add_(0, pages.clamp(min=0).flatten().long(), (pages >= 0).flatten().to(torch.int32) * by)


def _plain_fork(s, c):
    table, lens, refs, page = s["table"], s["lens"], s["refs"], s["page"]
    par, kid = s["parents"].long(), s["children"].long()
    table[kid] = table[par]
    lens[kid] = lens[par]
    _count_refs(refs, table[par], 1)
    # grow
    old = lens[kid].long()
    new = old + s["counts"].long()
    p_old, p_new = (old + page - 1) // page, (new + page - 1) // page
    last = table[kid, (p_old - 1).clamp(min=0)].long().clamp(min=0)
    partial = old % page != 0
    same = (last[:, None] == last[None]) & partial[:, None] & partial[None]
    copy = partial & (same.tril(-1).sum(1) < refs[last] - 1)
    need = p_new - p_old + copy
    first = torch.cumsum(need, 0) - need
    free = torch.sort((refs > 0).to(torch.int8), stable=True).indices
    j = torch.arange(table.shape[1], device="cuda")[None]
    take = free[(first[:, None] + copy[:, None] + j - p_old[:, None]).clamp(0, free.numel() - 1)]
    is_new = (j >= p_old[:, None]) & (j < p_new[:, None])
    rows = torch.where(is_new, take.to(torch.int32), table[kid])
    target = torch.where(copy, free[first.clamp(max=free.numel() - 1)], last)
    rows = torch.where((j == p_old[:, None] - 1) & copy[:, None], target[:, None].to(torch.int32), rows)
    refs.index_add_(0, last, -copy.to(torch.int32))
    refs.index_add_(0, target, copy.to(torch.int32))
    _count_refs(refs, torch.where(is_new, rows, torch.full_like(rows, -1)), 1)
    table[kid] = rows
    lens[kid] = new.to(torch.int32)
    filled = (torch.arange(page, device="cuda")[None] < (old % page)[:, None]) & copy[:, None]
    src, dst = s["cache"][:, last], s["cache"][:, target]
    s["cache"][:, target] = torch.where(filled[None, :, :, None], src, dst)
    # the ones that end
    end = s["ends"].long()
    _count_refs(refs, table[end], -1)
    table[end] = -1
    lens[end] = 0


def _plain_compact(s, c):
    refs, P = s["refs"], s["refs"].numel()
    at = torch.arange(P, device="cuda")
    used = refs > 0
    n = used.sum()
    movers, holes = used & (at >= n), ~used & (at < n)
    m = int(movers.sum())
    src, dst = at[movers][:m], at[holes][:m]
    to = at.clone()
    to[src] = dst
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()].to(torch.int32), s["table"]))
    s["cache"][:, dst] = s["cache"][:, src]
    refs[dst] = refs[src]
    refs[src] = 0


def run(s):
    if own:
        return _own(s)
    c = s["case"]
    if c["kind"] == "linear":
        return _plain_linear(s, c)
    if c["kind"] == "append":
        return _plain_append(s, c)
    if c["kind"] == "attend":
        return _plain_attend(s, c)
    s["table"].copy_(s["table0"])
    s["lens"].copy_(s["lens0"])
    s["refs"].copy_(s["refs0"])
    (_plain_fork if c["kind"] == "fork" else _plain_compact)(s, c)
    return s["table"], s["lens"], s["refs"], s["cache"]


# ---------------------------------------------------------------- what a pass cannot do without

_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def work(case):
    c = _numbers(case)
    if c["kind"] == "linear":
        N, K, T, r = c["N"], c["K"], c["T"], c["rank"]
        return {"bytes": N * K // 2 + N * K // c["group"] * 4 + T * K * 2 + T * N * _SIZE[c["out"]] + r * (N + K) * 2,
                "flops": 2 * T * (N * K + r * (N + K))}
    if c["kind"] == "append":
        T = sum(c["new"])
        return {"bytes": T * ((c["latent"] + c["rope"]) * 4 + c["heads"] * c["rope"] * 4), "flops": T * (5 * c["latent"] + 3 * c["rope"] * (c["heads"] + 1))}
    if c["kind"] == "attend":
        h, dn, dr, dv, dl = (c[k] for k in ("heads", "nope", "rope", "v", "latent"))
        T, flops = sum(c["new"]), 0
        for m, n in zip(c["new"], c["lens"]):
            pairs = m * (n - m) + m * (m + 1) // 2
            flops += 2 * h * min(pairs * (2 * dl + dr) + m * dl * (dn + dv), pairs * (dn + dr + dv) + n * dl * (dn + dv))
        return {"bytes": sum(c["lens"]) * (dl + dr) * 2 + T * h * (dn + dr) * 2 + h * (dn + dv) * dl * 2 + T * h * dv * _SIZE[c["out"]], "flops": flops}
    if c["kind"] == "fork":
        pages = -(-c["length"] // c["page"])
        return {"bytes": c["children"] * (c["length"] % c["page"]) * c["layers"] * c["row"] * 4 + c["children"] * pages * 12 + c["n_pages"] * 4, "flops": 0}
    used = max(1, int(c["fill"] * c["n_pages"]))
    return {"bytes": int(used * (1 - c["fill"])) * c["layers"] * c["page"] * c["row"] * 4 + c["n_pages"] * 8, "flops": 0}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c = _numbers(case)
    if c["kind"] in ("fork", "compact"):
        return None                                          # whole numbers and copied rows
    s = prepare(case, seed)
    if c["kind"] == "linear":
        out = torch.empty((c["T"], c["N"]), dtype=torch.float64, device="cuda")
        x = s["x"].double()
        step = max(1, (1 << 26) // c["K"])
        for n in range(0, c["N"], step):                     # sum_k s (q - z) x, group by group
            sl = slice(n, min(c["N"], n + step))
            code = s["codes"][sl]
            q = torch.empty((code.shape[0], c["K"]), dtype=torch.float64, device="cuda")
            q[:, 0::2], q[:, 1::2] = (code % 16).double(), (code // 16).double()
            q -= s["zeros"][sl].double().repeat_interleave(c["group"], dim=1)
            q *= s["scales"][sl].double().repeat_interleave(c["group"], dim=1)
            out[:, sl] = x @ q.T
        if c["rank"]:
            out += s["lora_scale"] * (x @ (s["B"].double() @ s["A"].double()).T)
        return out
    if c["kind"] == "append":
        cache, q = s["cache"].double(), s["q"].double()[..., c["nope"]:].clone()
        dl, at, half = c["latent"], 0, c["rope"] // 2
        first = torch.arange(half, device="cuda") if c["halves"] else 2 * torch.arange(half, device="cuda")
        second = first + (half if c["halves"] else 1)
        for i, (m, n) in enumerate(zip(c["new"], c["lens"])):
            pos = torch.arange(n - m, n, device="cuda")
            turn = torch.polar(torch.ones((m, half), dtype=torch.float64, device="cuda"), pos.double()[:, None] * s["inv_freq"].double()[None])
            kv = s["kv"][at:at + m].double()
            norm = kv[:, :dl].pow(2).sum(dim=1).div(dl).add(s["eps"]).sqrt()
            rows = torch.empty_like(kv)
            rows[:, :dl] = kv[:, :dl] / norm[:, None] * s["gain"].double()[None]
            z = torch.complex(kv[:, dl + first], kv[:, dl + second]) * turn
            rows[:, dl + first], rows[:, dl + second] = z.real, z.imag
            zq = torch.complex(q[at:at + m][..., first], q[at:at + m][..., second]) * turn[:, None]
            q[at:at + m, :, first], q[at:at + m, :, second] = zq.real, zq.imag
            cache[s["table"][i][torch.div(pos, c["page"], rounding_mode="floor")].long(), torch.remainder(pos, c["page"])] = rows
            at += m
        return q, cache
    # scores and sums position by position block: a running maximum and sum for every row, keys and values written out per head
    out, at, dl = [], 0, c["latent"]
    if work(case)["flops"] > 4e11:
        return None
    for i, (m, n) in enumerate(zip(c["new"], c["lens"])):
        rows = _context(s, c, i, torch.float64)
        y = torch.empty((m, c["heads"], c["v"]), dtype=torch.float64, device="cuda")
        last = torch.arange(n - m, n, device="cuda")
        for h in range(c["heads"]):
            q = torch.cat([s["q"][at:at + m, h, :c["nope"]].double() @ s["W_uk"][h].double(), s["q_rope"][at:at + m, h].double()], dim=1)
            q = q / math.sqrt(c["nope"] + c["rope"])
            top = torch.full((m, 1), -math.inf, dtype=torch.float64, device="cuda")
            tot = torch.zeros((m, 1), dtype=torch.float64, device="cuda")
            acc = torch.zeros((m, dl), dtype=torch.float64, device="cuda")
            for j in range(0, n, 16384):
                blk = rows[j:j + 16384]
                e = q @ blk.T
                e[torch.arange(j, j + blk.shape[0], device="cuda")[None] > last[:, None]] = -math.inf
                t = torch.maximum(top, e.amax(dim=1, keepdim=True))
                fade = torch.exp(top - t)
                e = torch.exp(e - t)
                tot, acc, top = tot * fade + e.sum(dim=1, keepdim=True), acc * fade + e @ blk[:, :dl], t
            y[:, h] = (acc / tot) @ s["W_uv"][h].double().T
        out.append(y)
        at += m
    return torch.cat(out)
