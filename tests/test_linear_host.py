"""Host side of the int4 projection: descriptor checks, record size, repacking, refusals of the call (no GPU work is reached)."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def edg():
    from paper_2609_18063_b200 import build
    build.build()
    import paper_2609_18063_b200 as m
    return m


def _canonical(rng, N, K, group):
    return (rng.integers(0, 256, (N, K // 2), dtype=np.uint8), rng.uniform(0.005, 0.02, (N, K // group)).astype(np.float16),
            rng.integers(0, 16, (N, K // group)).astype(np.float16))


@pytest.mark.parametrize("N,K,group", [(1, 32, 32), (16, 128, 64), (17, 96, 96), (33, 160, 32), (100, 384, 192), (64, 512, 512), (5, 256, 128)])
def test_pack_and_unpack_are_inverse(edg, N, K, group):
    rng = np.random.default_rng(N * 1000 + K)
    d = edg.make_linear_desc(N, K, group=group)
    t = _canonical(rng, N, K, group)
    rec = edg.pack_linear(d, *t)
    assert rec.nbytes == edg.linear_record_bytes(d)
    for a, b in zip(t, edg.unpack_linear(d, rec)):
        assert np.array_equal(a.view(np.uint8), b.view(np.uint8))


def test_record_layout(edg):
    """Word t of chunk c of a row lies at its lane's place in the block: [tile][block][half][4 g + t][chunk], low nibble first."""
    N, K = 40, 256
    d = edg.make_linear_desc(N, K, group=64)
    codes, sc, ze = _canonical(np.random.default_rng(3), N, K, 64)
    rec = edg.pack_linear(d, codes, sc, ze)
    for n, w in [(0, 0), (9, 17), (39, 31), (16, 5)]:
        b, chunk, t = w // 16, w // 4 % 4, w % 4
        at = (((n // 16) * 2 + b) * 2 + n % 16 // 8) * 512 + (n % 8 * 4 + t) * 16 + chunk * 4
        assert np.array_equal(rec[at:at + 4], codes[n, 4 * w:4 * w + 4])
    at = 3 * 2 * 1024 + ((2 * 2 + 1) * 16 + 6) * 8 + 4          # row 38, group 3: the second pair of block 1
    assert rec[at:at + 4].view(np.float16).tolist() == [sc[38, 3], ze[38, 3]]
    assert not rec[2 * 2 * 1024 + 512:2 * 2 * 1024 + 1024].any()    # rows 40.. of the last tile are zero


@pytest.mark.parametrize("kw,code", [(dict(N=0), -2), (dict(N=(1 << 24) + 1), -2), (dict(Kd=0), -2), (dict(Kd=65568), -2), (dict(group=48), -2),
                                     (dict(group=16), -2), (dict(Kd=96), -2), (dict(rank=-1), -2), (dict(rank=65), -2), (dict(out_dtype=3), -1),
                                     (dict(ldx=120), -2), (dict(ldx=132), -2), (dict(ldy=63), -2)])
def test_descriptors_that_are_refused(edg, kw, code):
    d = edg.make_linear_desc(64, 128, group=64)
    for k, v in kw.items():
        setattr(d, k, v)
    with pytest.raises(edg.EdgError) as e:
        edg.linear_record_bytes(d)
    assert e.value.code == code
    with pytest.raises(edg.EdgError):
        edg.linear_workspace_bytes(d, 1)


def test_zero_points_that_are_refused(edg):
    d = edg.make_linear_desc(16, 64, group=32)
    codes, sc, ze = _canonical(np.random.default_rng(0), 16, 64, 32)
    for bad in (0.1, 17.0, -1.0, 1 / 256, float("inf"), float("nan")):
        z = ze.copy()
        z[3, 1] = bad
        rec = np.full(edg.linear_record_bytes(d), 0xA5, np.uint8)
        with pytest.raises(edg.EdgError) as e:
            edg.pack_linear(d, codes, sc, z, rec)
        assert e.value.code == -4 and (rec == 0xA5).all()


def test_shapes_that_do_not_match(edg):
    d = edg.make_linear_desc(16, 64, group=32)
    codes, sc, ze = _canonical(np.random.default_rng(0), 16, 64, 32)
    with pytest.raises(ValueError):
        edg.pack_linear(d, codes[:8], sc, ze)
    with pytest.raises(ValueError):
        edg.pack_linear(d, codes, sc[:, :1], ze)


def test_calls_that_are_refused_before_any_launch(edg):
    d = edg.make_linear_desc(64, 128, group=64, rank=8)
    n = edg.linear_workspace_bytes(d, 4)
    ok = dict(record=4096, T=4, x=4096, A=4096, B=4096, y=4096, workspace=4096, workspace_bytes=n)

    def call(**kw):
        a = dict(ok, **kw)
        edg.linear_int4_lora(d, a["record"], a["T"], a["x"], a["A"], a["B"], a["y"], a["workspace"], a["workspace_bytes"], 0)
    for kw, code in [(dict(record=None), -1), (dict(x=None), -1), (dict(y=None), -1), (dict(A=None), -1), (dict(B=None), -1), (dict(T=0), -1),
                     (dict(T=65536), -1), (dict(record=4096 + 128), -1), (dict(x=4096 + 8), -1), (dict(y=4096 + 2), -1), (dict(A=4104), -1),
                     (dict(workspace=None), -1), (dict(workspace=4096 + 16), -7), (dict(workspace_bytes=n - 1), -7)]:
        with pytest.raises(edg.EdgError) as e:
            call(**kw)
        assert e.value.code == code, kw
    with pytest.raises(TypeError):
        edg.linear_int4_lora(edg.make_desc(None, H=1024, I=256, E=16, K=2, group=32, rank=8, n_adapters=1, n_slots=16), 4096, 1, 4096, None,
                             None, 4096, 4096, n, 0)


def test_workspace_never_falls(edg):
    for r in (0, 5, 64):
        d = edg.make_linear_desc(64, 128, group=64, rank=r)
        size = [edg.linear_workspace_bytes(d, T) for T in range(1, 300)]
        assert size[0] > 0 and all(a <= b for a, b in zip(size, size[1:]))
