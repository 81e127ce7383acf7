"""Weights in 4 bits and their products on the GPU against the 64-bit oracle.

Packing has to agree byte by byte.  A product's error: every one of the n_in products is exact or, for fp32 rows,
within 2^-24 (three terms of 8 bits), and each of the additions, cut off or rounded, is off by at most 2^-23 of
the sum of magnitudes; the result is rounded once."""
import numpy as np
import pytest
import torch

from oracle import tree_oracle as T
from paper_2505_13544_b200 import binding as M
from tests.test_operators_gpu import DT, half_step, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_in,n_out", [(8, 1), (32, 16), (128, 16), (136, 19), (264, 65), (1000, 3)])
def test_pack_and_unpack(n_in, n_out, dtype):
    rng = np.random.default_rng(n_in + n_out)
    w = torch.from_numpy(rng.standard_normal((n_in, n_out)) * np.exp(rng.uniform(-20, 14, (n_in, 1)))).to(DT[dtype])
    w[: n_in // 2, 0] = 0
    w = w.cuda()
    packed = M.mtla_qweight_pack(w)
    want = T.pack_weight(host(w))
    assert np.array_equal(packed.cpu().numpy(), want)
    back = T.unpack_weight(want, n_in, n_out)
    for t in DT.values():
        assert np.array_equal(host(M.mtla_qweight_unpack(packed, n_in, n_out, dtype=t)), back)


def test_pack_of_rows_with_a_stride_ties_and_specials():
    wide = torch.zeros(64, 40, device="cuda")
    wide[:8, 3] = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda") * 0.25
    wide[:8, 4] = -wide[:8, 3]
    wide[40, 5], wide[3, 6], wide[0, 7] = float("nan"), float("-inf"), 1e9
    w = wide[:, 3:20]
    packed = M.mtla_qweight_pack(w)
    assert np.array_equal(packed.cpu().numpy(), T.pack_weight(host(w)))
    back = M.mtla_qweight_unpack(packed, 64, 17)
    assert torch.isnan(back[32:, 2]).all() and (back[:32, 2] == 0).all() and torch.isnan(back[:32, 3]).all()
    assert back[0, 4] == 61440


def check_product(n, n_in, n_out, dtype, seed=0, x=None, size=1.0):
    rng = np.random.default_rng(seed + n)
    w = torch.from_numpy(rng.standard_normal((n_in, n_out)).astype(np.float32) / n_in ** 0.5).cuda()
    packed = M.mtla_qweight_pack(w)
    w64 = T.unpack_weight(packed.cpu().numpy(), n_in, n_out)
    if x is None:
        x = torch.from_numpy(rng.standard_normal((n, n_in)).astype(np.float32) * size).to(DT[dtype]).cuda()
    y = M.mtla_qweight_product(packed, x, n_out)
    want, mag = host(x) @ w64, np.abs(host(x)) @ np.abs(w64)
    tol = half_step(DT[dtype]) * np.abs(want) + mag * (n_in * 2.0 ** -23 + 2.0 ** -24) + 1e-38
    assert (np.abs(host(y) - want) <= tol).all(), (np.abs(host(y) - want) / tol).max()
    # The typical error is far smaller: additions err in both directions.
    rel = np.linalg.norm(host(y) - want) / np.linalg.norm(want)
    assert rel <= half_step(DT[dtype]) + 2e-6
    return packed, x, y


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,n_in,n_out", [
    (1, 8, 1), (1, 128, 16), (1, 4096, 100), (2, 136, 17), (7, 1000, 777), (8, 256, 64), (9, 512, 130), (16, 2048, 48),
    (17, 384, 31), (24, 2048, 512), (32, 64, 257), (33, 1024, 128), (64, 512, 300), (65, 640, 129), (100, 72, 1000),
    (128, 4096, 64), (200, 520, 333), (256, 128, 128), (257, 256, 16), (513, 1032, 145), (1, 8192, 7), (3, 16384, 33)])
def test_product(n, n_in, n_out, dtype):
    check_product(n, n_in, n_out, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 3, 20, 70, 300])
def test_rows_with_strides_and_none(dtype, n):
    packed, x, y = check_product(n, 264, 50, dtype)
    wide = torch.full((n, 304), float("nan"), dtype=DT[dtype], device="cuda")
    wide[:, 8:272] = x
    out = torch.full((n + 1, 61), 7.0, dtype=DT[dtype], device="cuda")
    M.mtla_qweight_product(packed, wide[:, 8:272], 50, out=out[:n, 3:53])
    assert torch.equal(out[:n, 3:53], y)
    out[:n, 3:53] = 7
    assert (out == 7).all()
    assert M.mtla_qweight_product(packed, x[:0], 50).shape == (0, 50)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [5, 40, 300])
def test_rows_do_not_reach_each_other(dtype, n):
    """A row of infinities and NaN leaves the others as they are, and an infinity stays one."""
    packed, x, y = check_product(n, 256, 48, dtype)
    bad = x.clone()
    bad[2], bad[4] = float("nan"), 0
    bad[4, 9] = float("inf")
    z = M.mtla_qweight_product(packed, bad, 48)
    keep = [i for i in range(n) if i not in (2, 4)]
    assert torch.equal(z[keep], y[keep]) and torch.isnan(z[2]).all()
    w = M.mtla_qweight_unpack(packed, 256, 48, dtype=torch.float32)[9]
    assert torch.isnan(z[4][w == 0]).all() and torch.equal(z[4].float()[w != 0], torch.inf * w[w != 0].sign())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_rows_of_any_size(dtype, size):
    for n in (2, 130):
        check_product(n, 512, 40, dtype, size=size)


def test_every_code_and_scale():
    """Rows of the unit matrix read every weight: all codes at all scales."""
    from oracle import qpool_oracle as Q
    scales = Q.SCALES[1:]
    n_out = len(scales)
    w = np.zeros((32, n_out))
    w[:16] = np.concatenate([Q.MAGNITUDES, -Q.MAGNITUDES])[:, None] * scales[None]
    w[16] = 6 * scales
    for dtype in DT.values():
        packed = M.mtla_qweight_pack(torch.from_numpy(w).float().cuda())
        for n in (8, 32):
            y = M.mtla_qweight_product(packed, torch.eye(32, dtype=dtype, device="cuda")[:n], n_out)
            assert np.array_equal(host(y), w[:n])
        y = M.mtla_qweight_product(packed, torch.eye(32, dtype=dtype, device="cuda").repeat(9, 1), n_out)
        assert np.array_equal(host(y), np.tile(w, (9, 1)))


@pytest.mark.parametrize("n", [1, 20, 150])
def test_a_captured_product_and_other_streams(n):
    packed, x, y = check_product(n, 1024, 200, "bf16")
    out = torch.empty_like(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        M.mtla_qweight_product(packed, x, 200, out=out)
    for _ in range(3):
        out.fill_(5)
        graph.replay()
        assert torch.equal(out, y)
    x.neg_()
    graph.replay()
    assert torch.equal(out, -y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [M.mtla_qweight_product(packed, x, 200, stream=s) for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    for z in got:
        assert torch.equal(z, -y)


# Over 1.5 10^8 products of weights and rows: the tensor-core kernel, with and without shares of the inputs.
MANY = [(9, 8192, 2600), (16, 4104, 5001), (17, 4104, 2200), (32, 4096, 1300), (33, 2056, 2300), (64, 2048, 1201),
        (65, 1032, 2400), (128, 1024, 1160), (129, 1000, 1250), (300, 712, 777), (513, 520, 600), (700, 136, 1700),
        (2000, 8, 9500)]


@pytest.mark.parametrize("n,n_in,n_out", MANY)
def test_product_of_many_rows(n, n_in, n_out):
    check_product(n, n_in, n_out, "bf16", size=3.0)


def test_many_rows_with_strides_and_specials():
    n, n_in, n_out = 200, 1000, 801
    packed, x, y = check_product(n, n_in, n_out, "bf16")
    wide = torch.full((n, 1040), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:1008] = x
    for width, at in ((900, 2), (901, 3), (802, 0)):       # pairs of outputs aligned or not
        out = torch.full((n + 1, width), 7.0, dtype=torch.bfloat16, device="cuda")
        got = out[:n, at:at + n_out]
        M.mtla_qweight_product(packed, wide[:, 8:1008], n_out, out=got)
        assert torch.equal(got, y)
        got.fill_(7)
        assert (out == 7).all()
    bad = x.clone()
    bad[2], bad[130], bad[130, 9] = float("nan"), 0, float("-inf")
    z = M.mtla_qweight_product(packed, bad, n_out)
    keep = [i for i in range(n) if i not in (2, 130)]
    assert torch.equal(z[keep], y[keep]) and torch.isnan(z[2]).all()
    w = M.mtla_qweight_unpack(packed, n_in, n_out, dtype=torch.float32)[9]
    assert torch.isnan(z[130][w == 0]).all() and torch.equal(z[130].float()[w != 0], -torch.inf * w[w != 0].sign())


def test_every_code_and_scale_of_many_rows():
    from oracle import qpool_oracle as Q
    w = np.zeros((32, len(Q.SCALES) - 1))
    w[:16] = np.concatenate([Q.MAGNITUDES, -Q.MAGNITUDES])[:, None] * Q.SCALES[1:][None]
    w[16] = 6 * Q.SCALES[1:]
    packed = M.mtla_qweight_pack(torch.from_numpy(w).float().cuda())
    rows = 32 * 800
    y = M.mtla_qweight_product(packed, torch.eye(32, dtype=torch.bfloat16, device="cuda").repeat(800, 1), w.shape[1])
    assert np.array_equal(host(y[:64]), np.tile(w, (2, 1))) and np.array_equal(host(y[rows - 32:]), w)


@pytest.mark.parametrize("n", [24, 256])
def test_many_rows_captured_and_on_other_streams(n):
    packed, x, y = check_product(n, 4096, 2000, "bf16")
    out = torch.empty_like(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        M.mtla_qweight_product(packed, x, 2000, out=out)
    for _ in range(3):
        out.fill_(5)
        graph.replay()
        assert torch.equal(out, y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [M.mtla_qweight_product(packed, x, 2000, stream=s) for _ in range(6) for s in streams]
    torch.cuda.synchronize()
    for z in got:
        assert torch.equal(z, y)


def test_products_that_follow_one_another():
    """Two layers' products in a row on one stream, each reading what the one before has written."""
    g = torch.Generator(device="cuda").manual_seed(5)
    w1, w2 = (torch.randn(1024, 1024, device="cuda", generator=g) / 32 for _ in range(2))
    p1, p2 = M.mtla_qweight_pack(w1), M.mtla_qweight_pack(w2)
    u1, u2 = (M.mtla_qweight_unpack(p, 1024, 1024, dtype=torch.float32).double() for p in (p1, p2))
    for n in (1, 12, 40, 400):
        x = torch.randn(n, 1024, device="cuda", generator=g).bfloat16()
        for _ in range(20):
            h = M.mtla_qweight_product(p1, x, 1024)
            y = M.mtla_qweight_product(p2, h, 1024)
        for a, u, z in ((x, u1, h), (h, u2, y)):
            want, mag = a.double() @ u, a.double().abs() @ u.abs()
            tol = 2.0 ** -8 * want.abs() + mag * (1024 * 2.0 ** -23 + 2.0 ** -24)
            assert ((z.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("n,n_out", [(1, 33), (16, 33), (40, 200), (2048, 1280)])
def test_the_most_inputs(n, n_out):
    """65536 products of one sign.  The matrix unit cuts a running sum off at every step of 16 inputs, by less than two
    units of the last of its 24 bits; the results are rounded to bf16.  2048 x 1280 is one CTA for all inputs."""
    n_in = 1 << 16
    g = torch.Generator(device="cuda").manual_seed(n)
    packed = M.mtla_qweight_pack(torch.rand(n_in, n_out, device="cuda", generator=g).add_(0.1).bfloat16())
    x = torch.rand(n, n_in, device="cuda", generator=g).add_(0.1).bfloat16()
    y = M.mtla_qweight_product(packed, x, n_out)
    w64 = M.mtla_qweight_unpack(packed, n_in, n_out, dtype=torch.float32).double()
    rows = sorted({0, n // 3, n // 2, n - 1})
    want = x[rows].double() @ w64
    off = ((y[rows].double() - want) / want).abs().max().item()
    assert off <= half_step(torch.bfloat16) + n_in / 16 * 2.0 ** -22, off
