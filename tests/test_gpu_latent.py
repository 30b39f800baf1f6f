"""Latent attention and the rows of its cache against their definitions in 64 bits.

Tolerance of attention: six standard deviations of what the bf16 roundings inside leave on an output (computed with the reference, row by row:
see _latent_ref.attention), half a step of the output's type, and 2^-16 of the largest value for sums in fp32."""
import numpy as np
import pytest
import torch

import paper_2609_18063_b200 as edg
from _latent_ref import append_rows, attention

pytestmark = pytest.mark.gpu

SMALL = dict(heads=8, dn=64, dr=32, dv=64, dl=256)
LARGE = dict(heads=4, dn=128, dr=64, dv=128, dl=512)
ODD = dict(heads=5, dn=48, dr=16, dv=96, dl=384)
ONE = dict(heads=1, dn=16, dr=64, dv=16, dl=128)
WIDE = dict(heads=72, dn=32, dr=32, dv=32, dl=128)
FORMS = [edg.LATENT_ABSORBED, edg.LATENT_EXPANDED]
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


class Batch:
    def __init__(self, lay, new, lens, page=64, seed=0, form=edg.LATENT_AUTO, out="bf16", behind=0, halves=False, spare=2, ldq=0, ldkv=0, sharp=1.0):
        self.lay, self.new, self.lens_host = lay, new, lens
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        H, dn, dr, dv, dl = (lay[k] for k in ("heads", "dn", "dr", "dv", "dl"))
        self.dn, self.dl, self.dr = dn, dl, dr
        n = lambda *s: torch.randn(s, generator=g, device="cuda")            # noqa: E731
        need = [-(-x // page) for x in lens]
        n_pages = sum(need) + spare
        perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), max(need + [1])), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, k in enumerate(need):
            self.table[i, :k] = perm[at:at + k]
            at += k
        self.cu_host = [0] + [int(x) for x in np.cumsum(new)]
        self.T = self.cu_host[-1] + behind
        self.cu = torch.tensor(self.cu_host, dtype=torch.int32, device="cuda")
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.scale = (dn + dr) ** -0.5
        self.cache = n(n_pages, page, dl + dr).bfloat16()
        wide = n(self.T, ldq or H * (dn + dr)) * sharp
        self.q_buf = wide.bfloat16()
        self.q = self.q_buf[:, :H * (dn + dr)].reshape(self.T, H, dn + dr)
        self.q_rope = (n(self.T, H, dr) * sharp).bfloat16()
        self.kv_buf = n(self.T, ldkv or dl + dr).bfloat16()
        self.kv = self.kv_buf[:, :dl + dr]
        self.W_uk, self.W_uv = (n(H, dn, dl) * dl ** -0.5).bfloat16(), (n(H, dv, dl) * dl ** -0.5).bfloat16()
        self.gain = (1 + 0.1 * n(dl)).bfloat16()
        self.inv_freq = (10000.0 ** (-torch.arange(0, dr, 2, dtype=torch.float64) / dr)).float().cuda()
        self.desc = edg.make_latent_desc(heads=H, d_nope=dn, d_rope=dr, d_v=dv, d_latent=dl, page=page, n_pages=n_pages, max_pages=self.table.shape[1],
                                         scale=self.scale, out_dtype=out, rope_halves=halves, form=form, ldq=ldq, ldkv=ldkv)
        self.out = out
        self.bounds = (len(lens), self.T, max(max(new), 1), sum(lens))
        self.ws = torch.zeros(edg.latent_workspace_bytes(self.desc, *self.bounds), dtype=torch.uint8, device="cuda")
        self.y = torch.full((self.T, H, dv), 7.0, dtype=DT[out], device="cuda")

    def attend(self, q_rope=True, ws=None):
        edg.latent_attention(self.desc, *self.bounds, self.cu, self.lens, self.table, self.q_buf, self.q_rope if q_rope else None, self.W_uk, self.W_uv,
                             self.cache, self.y, self.ws if ws is None else ws)

    def append(self, gain=True, q=True):
        edg.latent_append(self.desc, self.bounds[0], self.T, self.cu, self.lens, self.table, self.kv_buf, self.gain if gain else None, 1e-6,
                          self.inv_freq, self.q_buf if q else None, self.q_rope if q else None, self.cache, self.ws)

    def reference(self, q_rope=None):
        q_rope = self.q_rope if q_rope is None else q_rope
        y, sigma = attention(self.cache, self.table, self.cu_host, self.lens_host, self.q, q_rope, self.W_uk, self.W_uv, self.scale)
        top = torch.nan_to_num(y).abs().max()
        return y, 6 * sigma + HALF_STEP[self.out] * (y.abs() + 6 * sigma) + 2.0 ** -16 * top + (2.0 ** -25 if self.out == "f16" else 0.0)

    def check(self, status=0, **kw):
        torch.cuda.synchronize()
        assert edg.workspace_status(self.ws) == status
        y, tol = self.reference(**kw)
        n = self.cu_host[-1]
        got = self.y.double()
        assert torch.isfinite(got).all()
        off = (got - y).abs()[:n] - tol[:n]
        assert n == 0 or off.max() <= 0, (float((got - y)[:n].abs().max()), float(off.max()), int(off.flatten().argmax()))
        assert (got[n:] == 7.0).all()


LENS = [[1], [2], [15], [16], [17], [63], [64], [65], [127], [128], [129], [300]]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("lay", [SMALL, LARGE, ODD, ONE, WIDE])
@pytest.mark.parametrize("lens", LENS)
def test_one_new_row(form, lay, lens):
    b = Batch(lay, [1], lens, form=form, page=16)
    b.attend()
    b.check()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("lay", [SMALL, LARGE, ODD])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_ragged_batches(form, lay, page):
    b = Batch(lay, [1, 1, 1, 1, 1, 1, 1], [1, 700, 33, 64, 0, 257, 1500], page=page, form=form)
    b.attend()
    b.check()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("lay", [SMALL, LARGE, ODD, ONE])
@pytest.mark.parametrize("new,lens", [([5], [5]), ([1, 4, 2], [70, 4, 2]), ([128], [128]), ([129], [129]), ([300, 1, 77], [300, 500, 400]), ([257, 31], [700, 31])])
def test_several_new_rows(form, lay, new, lens):
    b = Batch(lay, new, lens, form=form)
    b.attend()
    b.check()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("out", ["f16", "bf16"])
def test_output_types_strides_and_rows_behind(form, out):
    lay = SMALL
    b = Batch(lay, [3, 0, 1, 20], [90, 50, 1, 20], form=form, out=out, behind=5, ldq=lay["heads"] * 96 + 24)
    b.attend()
    b.check()


@pytest.mark.parametrize("form", FORMS)
def test_rows_that_see_nothing_are_zero(form):
    """More new rows than positions: the first ones stand before position 0."""
    b = Batch(SMALL, [6, 3, 2], [2, 0, 40], form=form)
    b.attend()
    b.check()
    assert (b.y[:4] == 0).all() and (b.y[6:9] == 0).all()


@pytest.mark.parametrize("form", FORMS)
def test_queries_that_are_rotated_in_place(form):
    b = Batch(ODD, [2, 1], [40, 90], form=form)
    b.attend(q_rope=False)
    b.check(q_rope=b.q[..., b.dn:])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_what_lies_behind_a_sequence_does_not_reach_it(form, value):
    b = Batch(SMALL, [1, 140, 1], [33, 140, 64], page=64, form=form)
    used = torch.zeros(b.cache.shape[:2], dtype=torch.bool, device="cuda")
    for i, n in enumerate(b.lens_host):
        for j in range(n):
            used[int(b.table[i, j // 64]), j % 64] = True
    b.cache[~used] = value
    b.attend()
    b.check()


@pytest.mark.parametrize("form", FORMS)
def test_sharp_scores(form):
    """Scores of some hundreds: a row's weight sits on one position, and the running maximum moves by far more than an exponent."""
    b = Batch(SMALL, [1, 9], [900, 500], form=form, sharp=60.0)
    b.cache[:, :, :b.dl] *= torch.linspace(0.1, 3.0, 64, device="cuda")[None, :, None]
    b.attend()
    b.check()


@pytest.mark.parametrize("form", FORMS)
def test_a_row_of_the_cache_that_is_not_finite_reaches_its_sequence_alone(form):
    b = Batch(SMALL, [1, 1, 2], [100, 200, 150], form=form)
    b.cache[int(b.table[1, 1]), 3] = float("nan")
    b.attend()
    torch.cuda.synchronize()
    y, tol = b.reference()
    got = b.y.double()
    assert torch.isnan(got[1]).all()
    assert ((got - y).abs() <= tol)[[0, 2, 3]].all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new,length,where", [(5, 70, 67), (40, 40, 0), (40, 100, 99), (140, 300, 200), (150, 150, 127), (300, 300, 131)])
def test_a_new_row_that_is_not_finite_reaches_no_row_before_it(form, value, new, length, where):
    b = Batch(SMALL, [new, 1], [length, 50], form=form)
    b.cache[int(b.table[0, where // 64]), where % 64, 5:b.dl:7] = value
    b.attend()
    torch.cuda.synchronize()
    got = b.y.double()
    clean = where - (length - new)                        # rows of sequence 0 that stand before it
    before = [r for r in range(new + 1) if r < clean or r == new]
    clean_cache = b.cache.clone()
    clean_cache[int(b.table[0, where // 64]), where % 64] = 0
    y, sigma = attention(clean_cache, b.table, b.cu_host, b.lens_host, b.q, b.q_rope, b.W_uk, b.W_uv, b.scale)
    tol = 6 * sigma + HALF_STEP[b.out] * (y.abs() + 6 * sigma) + 2.0 ** -16 * y.abs().max()
    assert ((got - y).abs() <= tol)[before].all()
    if value != value:
        assert all(torch.isnan(got[r]).all() for r in range(max(clean, 0), new))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bad", [-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1])
def test_a_page_outside_the_cache_is_raised(form, bad):
    b = Batch(SMALL, [1, 1], [200, 100], form=form)
    b.table[0, 2] = bad
    b.attend()
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == -4
    y, tol = attention(b.cache, b.table[1:], [0, 1], [100], b.q[1:], b.q_rope[1:], b.W_uk, b.W_uv, b.scale)
    assert ((b.y[1:].double() - y).abs() <= 6 * tol + 2.0 ** -8 * y.abs() + 1e-3).all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("what", ["lens", "cu", "table"])
def test_bounds_that_do_not_hold_are_raised(form, what):
    b = Batch(SMALL, [4, 1], [200, 100], form=form)
    if what == "lens":
        b.lens[0] = 64 * b.table.shape[1] + 1000
    elif what == "cu":
        b.bounds = (2, 4, 3, 300)
    else:
        b.bounds = (2, 5, 4, 150)
        b.ws = torch.zeros(edg.latent_workspace_bytes(b.desc, *b.bounds), dtype=torch.uint8, device="cuda")
        if form == edg.LATENT_ABSORBED:
            return                                       # (its scratch does not depend on the sum of lens)
    b.attend()
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == -4


@pytest.mark.parametrize("form", FORMS)
def test_offsets_beyond_32_bits(form):
    """A cache of more than 2^32 bytes: the sequence lies in its last pages."""
    n_pages = 60000
    b = Batch(LARGE, [1, 150], [130, 150], form=form)
    big = torch.empty((n_pages, 64, 576), dtype=torch.bfloat16, device="cuda")
    assert big.numel() * 2 > 2 ** 32 and big.numel() > 2 ** 31
    k = b.cache.shape[0]
    big[-k:] = b.cache
    b.table = torch.where(b.table >= 0, b.table + (n_pages - k), b.table)
    b.desc.n_pages = n_pages
    b.cache = big
    b.attend()
    b.check()


@pytest.mark.parametrize("form", FORMS)
def test_same_bits_every_time_captured_and_on_another_stream(form):
    b = Batch(SMALL, [1, 1, 5], [700, 64, 300], form=form)
    b.attend()
    b.check()
    first = b.y.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.attend()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first, b.y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.attend()
    for lens in ([700, 64, 300], [650, 10, 299], [1, 0, 5]):
        b.lens_host = lens
        b.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        b.y.fill_(7.0)
        g.replay()
        b.check()


def test_two_sizes_through_one_workspace():
    a, b = Batch(SMALL, [1] * 9, [300 + 40 * i for i in range(9)]), Batch(SMALL, [200], [333], seed=1)
    ws = torch.zeros(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        a.attend(ws=ws)
        b.attend(ws=ws)
    a.check()
    b.check()


@pytest.mark.parametrize("lay", [SMALL, LARGE, ODD, ONE])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("new,lens,page", [([1], [1], 16), ([1, 0, 3, 5], [100, 7, 3, 70], 32), ([70, 1], [70, 20000], 64)])
def test_append(lay, halves, new, lens, page):
    """A value is rounded once (half a step); norms and rotations in fp32 add a few units of 2^-24, of the largest of a pair for rotated ones."""
    b = Batch(lay, new, lens, page=page, halves=halves, behind=2, ldkv=lay["dl"] + lay["dr"] + 8, ldq=lay["heads"] * (lay["dn"] + lay["dr"]) + 8)
    before = b.cache.clone()
    b.q_rope.fill_(7.0)
    want, qr = append_rows(before, b.table, b.cu_host, lens, b.kv, b.gain, 1e-6, b.inv_freq, b.q, b.dn, halves, b.dl)
    b.append()
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == 0
    n = b.cu_host[-1]
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -18
    assert ((b.cache.double() - want).abs() <= tol).all()
    assert ((b.q_rope[:n].double() - qr[:n]).abs() <= 2.0 ** -8 * qr[:n].abs() + 2.0 ** -18).all()
    assert (b.q_rope[n:] == 7.0).all()
    written = (want != before.double()).any(dim=-1)
    assert torch.equal(b.cache[~written], before[~written]) and int(written.sum()) == n


def test_append_without_gain_and_queries():
    b = Batch(SMALL, [2, 9], [30, 9])
    before = b.cache.clone()
    q_rope = b.q_rope.clone()
    want, _ = append_rows(before, b.table, b.cu_host, b.lens_host, b.kv, None, 1e-6, b.inv_freq, b.q, b.dn, False, b.dl)
    b.append(gain=False, q=False)
    torch.cuda.synchronize()
    assert ((b.cache.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all() and torch.equal(q_rope, b.q_rope)


def test_append_far_positions():
    """Angles of 10^6 and more keep their digits."""
    b = Batch(ONE, [1], [2 ** 20 + 77], page=256)
    before = b.cache.clone()
    want, qr = append_rows(before, b.table, b.cu_host, b.lens_host, b.kv, b.gain, 1e-6, b.inv_freq, b.q, b.dn, False, b.dl)
    b.append()
    torch.cuda.synchronize()
    assert ((b.cache.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all()
    assert ((b.q_rope.double() - qr).abs() <= 2.0 ** -8 * qr.abs() + 2.0 ** -18).all()


def test_append_skips_what_has_no_place():
    b = Batch(SMALL, [3, 2], [2, 100])
    b.table[1, 1] = b.cache.shape[0]                         # rows 98, 99 of sequence 1 would go there
    before = b.cache.clone()
    b.append()
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == -4
    changed = (b.cache != before).any(dim=-1)
    assert int(changed.sum()) == 2                            # the two rows of sequence 0 that have a position


def test_many_sequences_are_told_apart():
    n = 1500
    new = [i % 3 for i in range(n)]
    lens = [m + i % 7 for i, m in enumerate(new)]
    b = Batch(ONE, new, lens, page=16)
    want, qr = append_rows(b.cache, b.table, b.cu_host, lens, b.kv, b.gain, 1e-6, b.inv_freq, b.q, b.dn, False, b.dl)
    b.append()
    torch.cuda.synchronize()
    assert ((b.cache.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all()
    b.attend()
    b.check()


def test_together_as_a_decoder_uses_them():
    """Projections, new rows, attention and the output projection of one request, token by token, then a fork that goes its own way."""
    H, lay = 512, dict(SMALL, heads=4)
    rng = np.random.default_rng(0)
    dn, dr, dv, dl, heads = 64, 32, 64, 256, 4

    def linear(N, K, out):
        d = edg.make_linear_desc(N, K, group=64, out_dtype=out)
        codes = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
        sc, ze = np.full((N, K // 64), 0.2 * K ** -0.5, np.float16), np.full((N, K // 64), 7.5, np.float16)
        q = np.empty((N, K))
        q[:, 0::2], q[:, 1::2] = codes & 15, codes >> 4
        W = torch.from_numpy((q - 7.5) * float(sc[0, 0])).cuda()
        return d, torch.from_numpy(edg.pack_linear(d, codes, sc, ze)).cuda(), W
    Wq, Wkv, Wo = linear(heads * (dn + dr), H, "bf16"), linear(dl + dr, H, "bf16"), linear(H, heads * dv, "f32")
    page, n_pages = 16, 12
    cache = torch.zeros((1, n_pages, page, dl + dr), dtype=torch.bfloat16, device="cuda")
    refs, table = torch.zeros(n_pages, dtype=torch.int32, device="cuda"), torch.full((2, 5), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    pool, pc = edg.make_page_pool(refs, table, lens, page=page), edg.make_page_cache(cache)
    g = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(s, generator=g).cuda()                        # noqa: E731
    W_uk, W_uv = (n(heads, dn, dl) * dl ** -0.5).bfloat16(), (n(heads, dv, dl) * dl ** -0.5).bfloat16()
    inv_freq = (10000.0 ** (-torch.arange(0, dr, 2) / dr)).float().cuda()
    desc = edg.make_latent_desc(heads=heads, d_nope=dn, d_rope=dr, d_v=dv, d_latent=dl, page=page, n_pages=n_pages, max_pages=5, scale=(dn + dr) ** -0.5)
    ws = torch.zeros(max(edg.latent_workspace_bytes(desc, 2, 40, 40, 160), edg.pages_workspace_bytes(pool)), dtype=torch.uint8, device="cuda")
    seqs = [torch.tensor(s, dtype=torch.int32, device="cuda") for s in ([0], [0, 1])]
    length, history = [0, 0], [[], []]

    def step(x, ids, new):
        """x [T][H]: `new` rows of each sequence of `ids` -> output projection"""
        T, k = x.shape[0], len(ids)
        q, kv = torch.empty((T, heads * (dn + dr)), dtype=torch.bfloat16, device="cuda"), torch.empty((T, dl + dr), dtype=torch.bfloat16, device="cuda")
        qr, y, o = torch.empty((T, heads, dr), dtype=torch.bfloat16, device="cuda"), torch.empty((T, heads * dv), dtype=torch.bfloat16, device="cuda"), \
            torch.empty((T, H), device="cuda")
        cu = torch.arange(k + 1, dtype=torch.int32, device="cuda") * new
        edg.pages_reserve(pool, pc, k, seqs[k - 1], torch.full((k,), new, dtype=torch.int32, device="cuda"), ws)
        edg.linear_int4_lora(Wq[0], Wq[1], T, x, None, None, q, ws)
        edg.linear_int4_lora(Wkv[0], Wkv[1], T, x, None, None, kv, ws)
        edg.latent_append(desc, k, T, cu, lens, table, kv, None, 1e-6, inv_freq, q, qr, cache, ws)
        edg.latent_attention(desc, k, T, new, 2 * 80, cu, lens, table, q, qr, W_uk, W_uv, cache, y, ws)
        edg.linear_int4_lora(Wo[0], Wo[1], T, y, None, None, o, ws)
        # the same in 64 bits, from the inputs alone
        xd = x.double()
        qd, kvd = (xd @ Wq[2].T).view(T, heads, dn + dr), xd @ Wkv[2].T
        want = []
        for i, s in enumerate(ids):
            for r in range(new):
                t = i * new + r
                ang = length[s] * inv_freq.double()
                co, si = ang.cos(), ang.sin()
                rot = lambda v: torch.stack([v[..., 0::2] * co - v[..., 1::2] * si, v[..., 0::2] * si + v[..., 1::2] * co], -1).flatten(-2)  # noqa: E731
                c = kvd[t, :dl] / torch.sqrt((kvd[t, :dl] ** 2).mean() + 1e-6)
                history[s].append((c, rot(kvd[t, dl:])))
                length[s] += 1
                C, P = torch.stack([a for a, _ in history[s]]), torch.stack([b for _, b in history[s]])
                sc = torch.einsum("hn,hnl,jl->hj", qd[t, :, :dn], W_uk.double(), C) + rot(qd[t, :, dn:]) @ P.T
                p = torch.softmax(sc * (dn + dr) ** -0.5, dim=-1)
                want.append(torch.einsum("hj,jl,hvl->hv", p, C, W_uv.double()).flatten() @ Wo[2].T)
        return o.double(), torch.stack(want)
    # five roundings to bf16 lie between x and the output (q, rows, weights, y, and one inside attention), each at most 2^-8 of its value and mostly
    # independent: 5 * 2^-8 / sqrt 3 of the output's magnitude as a standard deviation, six of them in the norm
    def near(got, want):
        assert (got - want).norm() <= 6 * 5 ** 0.5 * 2.0 ** -8 / 3 ** 0.5 * want.norm()
    near(*step(n(20, H).bfloat16(), [0], 20))
    for _ in range(3):
        near(*step(n(1, H).bfloat16(), [0], 1))
    edg.pages_fork(pool, 1, torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"), ws)
    length[1], history[1] = length[0], list(history[0])
    for _ in range(12):
        near(*step(n(2, H).bfloat16(), [0, 1], 1))
    edg.pages_free(pool, 1, seqs[0], ws)
    edg.pages_compact(pool, pc, ws)
    length[0], history[0] = 0, []
    for _ in range(2):
        near(*step(n(2, H).bfloat16(), [0, 1], 1))
    assert edg.workspace_status(ws) == 0
    assert lens.tolist() == length and int((refs > 0).sum()) == sum(-(-k // page) for k in length)
