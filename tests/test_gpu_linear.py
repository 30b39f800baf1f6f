"""The int4 projection against its formula in 64 bits.

Tolerance: codes, activations (bf16 brought to fp16 by a power of two) and their products are exact; what rounds are fp32 additions.  A value
is a sum of Kd products through at most Kd / 16 + 64 consecutive additions, each off by at most 2^-23 of the magnitudes summed
(tensor cores truncate), S = sum s (q + z) |x|; the adapter adds Kd / 32 + rank + 8 of them over its own magnitudes.  fp16 activations
lose 2^-34 of the token's largest per product.  The output is rounded by half a step."""
import numpy as np
import pytest
import torch

import paper_2609_18063_b200 as edg

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


class Case:
    def __init__(self, N, K, group, rank, T, out="f32", scale=1.0, seed=0, ldx=0, ldy=0, whole_zeros=True):
        rng = np.random.default_rng([seed, N, K, T])
        self.N, self.K, self.T, self.out, self.rank = N, K, T, out, rank
        self.codes = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
        self.sc = rng.uniform(0.005, 0.02, (N, K // group)).astype(np.float16)
        z = rng.integers(0, 16, (N, K // group)) if whole_zeros else rng.integers(0, 2049, (N, K // group)) / 128
        self.ze = z.astype(np.float16)
        self.desc = edg.make_linear_desc(N, K, group=group, rank=rank, out_dtype=out, lora_scale=2.0, ldx=ldx, ldy=ldy)
        self.record = torch.from_numpy(edg.pack_linear(self.desc, self.codes, self.sc, self.ze)).cuda()
        g = torch.Generator().manual_seed(seed + N + K)
        lx = ldx or K
        self.x = (torch.randn((T, lx), generator=g) * scale).to(torch.bfloat16)
        self.A = (torch.randn((max(rank, 1), K), generator=g) * 0.02).to(torch.bfloat16)
        self.B = (torch.randn((N, max(rank, 1)), generator=g) * 0.01).to(torch.bfloat16)
        self.ws = torch.zeros(edg.linear_workspace_bytes(self.desc, T), dtype=torch.uint8, device="cuda")
        self.group = group
        self.dev = (self.x.cuda(), self.A.cuda(), self.B.cuda())
        self.y = torch.full((T, ldy or N), 7.0, dtype=DT[out], device="cuda")

    def run(self, stream=None):
        x, A, B = self.dev
        edg.linear_int4_lora(self.desc, self.record, self.T, x, A if self.rank else None, B if self.rank else None, self.y, self.ws, stream=stream)

    def reference(self):
        q = np.empty((self.N, self.K))
        q[:, 0::2], q[:, 1::2] = self.codes & 15, self.codes >> 4
        s = np.repeat(self.sc.astype(np.float64), self.group, axis=1)
        z = np.repeat(self.ze.astype(np.float64), self.group, axis=1)
        x = self.x[:, :self.K].double().numpy()
        y, mag = x @ (s * (q - z)).T, np.abs(x) @ (s * (q + z)).T
        tol = (self.K / 16 + 64) * 2.0 ** -23 * mag + 2.0 ** -34 * np.abs(x).max(axis=1, keepdims=True) * (s * 16).sum(axis=1)
        if self.rank:
            A, B = self.A.double().numpy(), self.B.double().numpy()
            y = y + 2.0 * (x @ A.T) @ B.T
            tol = tol + (self.K / 32 + self.rank + 8) * 2.0 ** -23 * 2.0 * (np.abs(x) @ np.abs(A).T) @ np.abs(B).T
        return y, tol + HALF_STEP[self.out] * (np.abs(y) + tol) + (2.0 ** -25 if self.out == "f16" else 0.0)

    def check(self):
        torch.cuda.synchronize()
        got = self.y[:, :self.N].double().cpu().numpy()
        y, tol = self.reference()
        off = np.abs(got - y) - tol
        assert np.isfinite(got).all() and off.max() <= 0, (float(np.abs(got - y).max()), float(tol.min()), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("N,K,group,rank", [(16, 32, 32, 0), (1, 128, 128, 1), (17, 96, 96, 0), (100, 160, 32, 5), (33, 384, 192, 64), (1024, 1024, 32, 8),
                                            (2048, 4096, 64, 16), (577, 2048, 64, 16), (130, 8192, 256, 0)])
@pytest.mark.parametrize("T", [1, 2, 8, 9, 16, 17, 33, 64, 65, 131])
def test_against_64_bits(N, K, group, rank, T):
    c = Case(N, K, group, rank, T)
    c.run()
    c.check()


@pytest.mark.parametrize("out", ["f16", "bf16"])
@pytest.mark.parametrize("T", [1, 24, 64])
def test_output_types(out, T):
    c = Case(300, 512, 64, 16, T, out=out)
    c.run()
    c.check()


@pytest.mark.parametrize("T,N", [(1, 40001), (16, 40001), (64, 20001)])
def test_many_row_tiles(T, N):
    c = Case(N, 512, 64, 0, T)
    c.run()
    c.check()


@pytest.mark.parametrize("K,T", [(65536, 1), (65536, 5), (32768, 16), (16384, 64)])
def test_long_input_dimension(K, T):
    c = Case(35, K, 128, 0, T)
    c.run()
    c.check()


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e4, 1e30])
def test_activations_of_any_magnitude(scale):
    c = Case(64, 512, 64, 0, 9, scale=scale)
    c.run()
    c.check()


def test_fractional_zero_points():
    c = Case(96, 256, 32, 0, 4, whole_zeros=False)
    c.run()
    c.check()


def test_rows_apart_and_what_lies_between_them():
    c = Case(50, 256, 64, 8, 11, ldx=264, ldy=61)
    c.run()
    c.check()
    assert (c.y[:, 50:] == 7.0).all()


def test_a_token_that_is_not_finite_stays_alone():
    c = Case(80, 256, 64, 8, 10)
    c.x[3, 17] = float("inf")
    c.x[7, 200] = float("nan")
    c.dev = (c.x.cuda(),) + c.dev[1:]
    c.run()
    torch.cuda.synchronize()
    got = c.y.cpu().double().numpy()
    keep = [t for t in range(10) if t not in (3, 7)]
    c.x[3], c.x[7] = 0, 0
    y, tol = c.reference()
    assert (np.abs(got - y) <= tol)[keep].all()
    assert not np.isfinite(got[3]).any() and np.isnan(got[7]).all()


def test_a_token_of_zeros():
    c = Case(80, 256, 64, 8, 3)
    c.x[1] = 0
    c.dev = (c.x.cuda(),) + c.dev[1:]
    c.run()
    c.check()
    assert (c.y[1] == 0).all()


def test_same_bits_every_time_whatever_else_is_in_the_batch():
    a = Case(577, 2048, 64, 16, 8)
    a.run()
    first = a.y.clone()
    a.run()
    assert torch.equal(first, a.y)


def test_captured_replayed_and_on_another_stream():
    c = Case(256, 1024, 64, 16, 7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.run()
    torch.cuda.current_stream().wait_stream(s)
    c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for k in range(3):
        c.x = (torch.randn(c.x.shape, generator=torch.Generator().manual_seed(50 + k))).to(torch.bfloat16)
        c.dev[0].copy_(c.x)
        c.y.fill_(7.0)
        g.replay()
        c.check()


def test_in_a_row_through_one_workspace():
    """A chain of projections, each reading what the one before it wrote, in one scratch buffer."""
    a, b = Case(512, 1024, 64, 16, 6, out="bf16", seed=1), Case(384, 512, 64, 16, 6, seed=2)
    for _ in range(3):
        a.run()
        edg.linear_int4_lora(b.desc, b.record, 6, a.y, b.dev[1], b.dev[2], b.y, a.ws)
    a.check()
    b.x = a.y.cpu()
    b.check()


