"""GPU: products with 4-bit weights (astra_w4_linear) against the 64-bit oracle.  A product is a sum of K terms x (16 + code) and one of x per group, scaled in fp32: with
u = 2^-24, K / 8 + 40 roundings of sums that stay below 31 scale sum |x| (a 32-term MFMA counts as 32, groups are added one by one), and the result's own half step."""
import numpy as np
import pytest

from oracle import serving as sv
from paper_2505_19342_amd import binding as B
from paper_2505_19342_amd import workloads as wl

pytestmark = pytest.mark.gpu


def make(dtype, T, K, N, group, zeros, bias, seed=0):
    rng = np.random.default_rng(seed)
    rnd = wl.round_to_bf16 if dtype == "bf16" else (lambda a: np.asarray(a, np.float32))
    codes = rng.integers(0, 256, (N, K // 2)).astype(np.uint8)
    scales = rnd(((rng.random((N, K // group)) + 0.5) * 0.01).astype(np.float32))
    return (rnd(rng.standard_normal((T, K)).astype(np.float32)), codes, scales, rng.integers(0, 16, (N, K // group)).astype(np.uint8) if zeros else None,
            rnd(rng.standard_normal(N).astype(np.float32)) if bias else None)


def check(dtype, T, K, N, group, zeros=False, bias=False, y=None, stride=0, seed=0):
    import torch
    from gpu_util import empty_like_dtype, to_dev, to_host
    y = y or dtype
    x, codes, scales, z, b = make(dtype, T, K, N, group, zeros, bias, seed)
    ref = sv.w4_linear(x, codes, scales, z, b, group)
    xd = to_dev(x, dtype)
    if stride:
        wide = empty_like_dtype((T, stride), dtype).fill_(float("nan"))
        wide[:, :K] = xd
        xd = wide[:, :K]
    u8 = lambda a: None if a is None else torch.from_numpy(a).to("cuda:0")
    # a row more than there is, to see that it stays
    out = empty_like_dtype((T + 1, N), y).fill_(7.0)
    args = (B.w4_desc(dtype, K, N, group, y, stride), xd, T, u8(codes), to_dev(scales, dtype), u8(z), None if b is None else to_dev(b, dtype), out)
    B.astra_w4_linear(*args)
    torch.cuda.synchronize()
    got = to_host(out)
    assert np.all(got[T] == 7.0)
    got = got[:T]
    size = np.abs(x) @ (np.repeat(scales.astype(np.float64), group, 1) * 31).T + (0 if b is None else np.abs(b))
    bar = (K / 8 + 40) * 2.0 ** -24 * size + (2.0 ** -8 if y == "bf16" else 2.0 ** -24) * np.abs(ref)
    off = np.abs(got - ref)
    print(f"{dtype} {T}x{K}x{N} group {group}: worst {np.max(off / bar):.3f} of the bar")
    assert np.all(off <= bar)
    first = out.clone()
    B.astra_w4_linear(*args)
    torch.cuda.synchronize()
    assert torch.equal(first, out)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 64, 65, 130])
@pytest.mark.parametrize("dtype, group, zeros, bias", [("bf16", 128, False, False), ("bf16", 32, True, True), ("f32", 64, True, False), ("f32", 128, False, True)])
def test_numbers_of_tokens(T, dtype, group, zeros, bias):
    check(dtype, T, 512, 100, group, zeros, bias, seed=T)


@pytest.mark.parametrize("K, group", [(32, 32), (64, 64), (96, 32), (128, 128), (160, 32), (192, 64), (224, 32), (320, 64), (384, 128), (2080, 32), (4224, 64), (14336, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_widths(K, group, dtype):
    for T in (1, 5, 40):
        check(dtype, T, K, 50, group, zeros=T == 5, seed=K)


@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 31, 63, 65, 255, 1000, 4097])
def test_numbers_of_rows(N):
    check("bf16", 1, 256, N, 64, True, True, seed=N)
    check("bf16", 20, 256, N, 64, False, True, y="f32", seed=N)
    check("f32", 3, 256, N, 32, True, False, y="bf16", seed=N)


def test_model_sizes():
    check("bf16", 1, 4096, 6144, 128, seed=1)
    check("bf16", 8, 14336, 512, 128, y="f32", seed=2)
    check("bf16", 64, 4096, 1024, 64, True, seed=3)


def test_rows_that_lie_apart():
    check("bf16", 3, 256, 40, 64, stride=264)
    check("f32", 30, 256, 40, 64, stride=1024)


def test_infinite_and_nan_tokens_stay_in_their_rows():
    import torch
    from gpu_util import empty_like_dtype, to_dev, to_host
    x, codes, scales, _, _ = make("bf16", 20, 256, 33, 64, False, False)
    x[3, 7], x[18, 100] = np.nan, np.inf
    out = empty_like_dtype((20, 33), "f32")
    B.astra_w4_linear(B.w4_desc("bf16", 256, 33, 64, "f32"), to_dev(x, "bf16"), 20, torch.from_numpy(codes).to("cuda:0"), to_dev(scales, "bf16"), None, None, out)
    torch.cuda.synchronize()
    bad = ~np.isfinite(to_host(out))
    assert bad[[3, 18]].all() and not np.delete(bad, [3, 18], 0).any()


def test_layout_helper_and_product():
    """Weights through quantize_w4 and the product: what is lost is the weights' rounding alone."""
    import torch
    from gpu_util import to_dev, to_host
    rng = np.random.default_rng(9)
    w = (rng.standard_normal((70, 256)) * 0.02).astype(np.float32)
    x = rng.standard_normal((4, 256)).astype(np.float32)
    codes, scales, zeros = B.quantize_w4(w, 32, "f32", zeros=True)
    y = torch.empty((4, 70), device="cuda:0")
    B.astra_w4_linear(B.w4_desc("f32", 256, 70, 32), to_dev(x, "f32"), 4, torch.from_numpy(codes).to("cuda:0"), to_dev(scales, "f32"), torch.from_numpy(zeros).to("cuda:0"), None, y)
    torch.cuda.synchronize()
    step = np.repeat(scales.astype(np.float64), 32, 1)
    assert np.all(np.abs(to_host(y) - x @ w.T.astype(np.float64)) <= np.abs(x) @ (step * 1.01).T)


def test_captured_into_a_graph():
    import torch
    from gpu_util import empty_like_dtype, to_dev
    x, codes, scales, _, _ = make("bf16", 4, 1024, 300, 128, False, False)
    xd, cd, sd, out = to_dev(x, "bf16"), torch.from_numpy(codes).to("cuda:0"), to_dev(scales, "bf16"), empty_like_dtype((4, 300), "bf16")
    d = B.w4_desc("bf16", 1024, 300, 128)
    B.astra_w4_linear(d, xd, 4, cd, sd, None, None, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.astra_w4_linear(d, xd, 4, cd, sd, None, None, out)
    for _ in range(4):
        xd.copy_(torch.randn(4, 1024, device="cuda:0").to(torch.bfloat16))
        graph.replay()
        got = out.clone()
        B.astra_w4_linear(d, xd, 4, cd, sd, None, None, out)
        torch.cuda.synchronize()
        assert torch.equal(got, out)


@pytest.mark.parametrize("group, K", [(32, 32), (32, 288), (32, 1184), (64, 64), (64, 448), (64, 1088), (128, 128), (128, 384), (128, 2432)])
@pytest.mark.parametrize("T", [20, 40])
def test_wide_tiles(T, group, K):
    """Rows enough for tiles of 128 (of 32 and 64 tokens), with widths that end anywhere in a chunk, in a wavefront group's range and in a span of scales."""
    check("bf16", T, K, 24449 if T == 40 else 24577, group, zeros=K % 3 == 0, bias=K % 2 == 1 or T == 20, y="f32", seed=K + T)


@pytest.mark.parametrize("group, K", [(32, 32), (32, 1184), (64, 448), (64, 1088), (128, 384), (128, 2432)])
def test_two_workgroups_of_small_tiles_on_a_unit(group, K):
    check("bf16", 33, K, 4130, group, zeros=K % 3 != 0, bias=True, seed=K)


def test_many_tokens_of_few_rows():
    check("bf16", 1000, 128, 1, 32, True, seed=4)
    check("bf16", 12289, 96, 20, 32, y="f32", seed=5)
    check("f32", 1000, 96, 17, 32, True, seed=6)


def test_products_that_use_much_lds_captured_into_a_graph_and_on_two_streams():
    import torch
    from gpu_util import empty_like_dtype, to_dev
    K, N = 2048, 700
    graphs = []
    for dtype, T in (("bf16", 40), ("bf16", 12), ("f32", 12)):
        x, codes, scales, zeros, _ = make(dtype, T, K, N, 64, True, False, seed=T)
        a = (B.w4_desc(dtype, K, N, 64), to_dev(x, dtype), T, torch.from_numpy(codes).to("cuda:0"), to_dev(scales, dtype), torch.from_numpy(zeros).to("cuda:0"), None,
             empty_like_dtype((T, N), dtype))
        B.astra_w4_linear(*a)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.astra_w4_linear(*a)
        graphs.append((a, graph))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        wanted = []
        for a, _ in graphs:
            a[1].copy_(torch.randn(a[1].shape, device="cuda:0").to(a[1].dtype))
            B.astra_w4_linear(*a)
            wanted.append(a[7].clone())
            a[7].fill_(float("nan"))
        torch.cuda.synchronize()
        for (a, graph), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for (a, _), want in zip(graphs, wanted):
            assert torch.equal(a[7], want)
