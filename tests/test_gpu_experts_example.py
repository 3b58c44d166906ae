"""The block of examples/experts_and_adapters.py, and the grouped calls where a program leaves the plain path: captured into
a graph whose offsets change, on another stream, on weights that the ping-pong tiles start at different blocks, and on
matrices of more than 2^31 elements."""
import importlib.util
import os

import pytest
import torch

from paper_2511_13764_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "experts_and_adapters.py")
    spec = importlib.util.spec_from_file_location("experts_and_adapters", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_the_block_and_its_gradients():
    """In 32 bits against autograd in 64.  All sums are of at most 96 products of values of size 1 to 10, three products
    deep: fp32 keeps them to 1e-5 of the largest result."""
    m = example()
    width, hidden, experts, adapters, rank = 64, 96, 5, 3, 8
    blk = m.Block(width, hidden, experts, adapters, rank, dtype=torch.float32)
    gen = torch.Generator().manual_seed(2)
    at = [0, 40, 40, 77]
    segments = torch.tensor(at, device="cuda")
    d = {n: getattr(blk, n).double().cpu().requires_grad_() for n in ("W", "down", "up", "U", "D")}
    want = {n: 0.0 for n in blk.grads}
    for _ in range(2):
        x, dy = (torch.randn((at[-1], width), generator=gen) for _ in range(2))
        y, kept = blk.forward(x.cuda(), segments)
        dx = blk.backward(dy.cuda(), kept)
        order, offsets = kept[3].cpu(), kept[4].cpu()
        xd = x.double().requires_grad_()
        x1 = torch.cat([xd[a:b] @ d["W"].t() + (xd[a:b] @ d["down"][i].t()) @ d["up"][i].t()
                        for i, (a, b) in enumerate(zip(at, at[1:]))])
        ys = torch.cat([(x1[order[a:b]] @ d["U"][e].t()).relu() @ d["D"][e].t()
                        for e, (a, b) in enumerate(zip(offsets.tolist(), offsets.tolist()[1:]))])
        ref = torch.empty_like(ys)
        ref[order] = ys
        grads = torch.autograd.grad((ref * dy.double()).sum(), [xd, *(d[n] for n in want)])
        for n, g in zip(want, grads[1:]):
            want[n] = want[n] + g
        for got, w in ((y, ref.detach()), (dx, grads[0])):
            assert (got.double().cpu() - w).abs().max() <= 1e-5 * w.abs().max()
    for n, w in want.items():
        assert (blk.grads[n].double().cpu() - w).abs().max() <= 1e-5 * w.abs().max(), n
    # decode: the same rows, an adapter for each row
    ids = torch.tensor([0] * 40 + [2] * 37, device="cuda")
    assert (blk.decode(x.cuda(), ids) - y).abs().max() <= 2e-5 * y.abs().max()


def test_the_example_runs(capsys):
    example().main()
    assert "decode of 16 requests" in capsys.readouterr().out


def reference(A, W, at):
    out = torch.zeros((A.shape[0], W.shape[1]), dtype=torch.float64, device=A.device)
    for e in range(len(at) - 1):
        out[at[e]:at[e + 1]] = A[at[e]:at[e + 1]].double() @ W[e].double().t().contiguous()
    return out


def test_a_graph_finds_other_bounds_at_every_replay():
    """One capture of the three calls; each replay reads the offsets and ids that the program has written since."""
    print("[gpu-case] graph of gemm_grouped, gemm_grouped_wgrad, gemm_adapters", flush=True)
    gen = torch.Generator().manual_seed(7)
    M, N, K, G, R = 96, 264, 320, 4, 16
    X, dY = ((torch.randn((M, n), generator=gen)).bfloat16().cuda() for n in (K, N))
    W = (torch.randn((G, N, K), generator=gen) * 0.1).bfloat16().cuda()
    down, up = ((torch.randn(s, generator=gen) * 0.1).bfloat16().cuda() for s in ((G, R, K), (G, N, R)))
    off, ids = torch.zeros(G + 1, dtype=torch.int64, device="cuda"), torch.zeros(G, dtype=torch.int64, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def outputs():
        return [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((M, N), (G, N, K), (M, N), (M, R))]

    def calls(o, stream):
        B.gemm_grouped(B.DTYPE_BF16, 1, M, N, K, G, off, X, K, W, K, N * K, 0.0, o[0], N, 0, workspace=ws, stream=stream)
        B.gemm_grouped_wgrad(B.DTYPE_BF16, M, N, K, G, off, dY, N, X, K, 0.0, o[1], K, N * K, 0, workspace=ws, stream=stream)
        B.gemm_adapters(B.DTYPE_BF16, 1, M, N, K, R, G, off, ids, G, X, K, W, K, down, K, R * K, up, R, N * R, None, 0.0, o[2],
                        N, 0, None, 0, o[3], R, workspace=ws, stream=stream)
    eager, held = outputs(), outputs()
    calls(eager, None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(held, torch.cuda.current_stream().cuda_stream)
    for at, who in (([0, 10, 10, 50, 96], [3, 1, -1, 0]), ([0, 0, 96, 96, 96], [0, 2, 1, 1]), ([5, 6, 70, 71, 90], [1, 1, 9, 2]),
                    ([0, 0, 0, 0, 0], [0, 0, 0, 0]), ([0, 24, 48, 72, 96], [-1, -1, -1, 3])):
        off.copy_(torch.tensor(at))
        ids.copy_(torch.tensor(who))
        for t in eager + held:
            t.fill_(-3.0)
        graph.replay()
        calls(eager, None)
        torch.cuda.synchronize()
        for a, b in zip(held, eager):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), at
        ref = reference(X, W, at)
        rows = slice(at[0], at[-1])
        ab = reference(X.abs(), W.abs(), at)
        assert ((held[0].double() - ref).abs()[rows] <= (2.0 ** -8 * (ref.abs() + ab * K * U) + ab * (K + 4) * U)[rows]).all()


def test_calls_on_another_stream():
    side = torch.cuda.Stream()
    gen = torch.Generator().manual_seed(8)
    M, N, K, G = 300, 520, 512, 3
    at = [0, 1, 150, 300]
    with torch.cuda.stream(side):
        X, W = torch.randn((M, K), generator=gen).cuda().half(), (torch.randn((G, N, K), generator=gen) * 0.1).cuda().half()
        off, Y = torch.tensor(at, device="cuda"), torch.full((M, N), float("nan"), device="cuda")
        B.gemm_grouped(B.DTYPE_F16, 1, M, N, K, G, off, X, K, W, K, N * K, 0.0, Y, N, 1)
        ref, ab = reference(X, W, at), reference(X.abs(), W.abs(), at)
    side.synchronize()
    assert ((Y.double() - ref).abs() <= ab * (K + 4) * U).all()


@pytest.mark.parametrize("c32", [0, 1])
def test_ping_pong_tiles_that_start_at_different_blocks(c32):
    """Weights of 2^25 elements and more: every expert and column begins its reduction elsewhere.  Tiles of 256 and of 128 rows."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    sizes, N, K = [300, 0, 256, 129, 31, 128, 700, 1], 1032, 4160
    at = [0]
    for m in sizes:
        at.append(at[-1] + m)
    G, M = len(sizes), at[-1]
    X = torch.randn((M, K), device="cuda", generator=gen).bfloat16()
    W = (torch.randn((G, N, K), device="cuda", generator=gen) * 0.05).bfloat16()
    Y = torch.full((M, N), float("nan"), device="cuda", dtype=torch.float32 if c32 else torch.bfloat16)
    B.gemm_force_variant(B.variants().index("bf16_pingpong_256x256x64"), 0)
    try:
        B.gemm_grouped(B.DTYPE_BF16, 1, M, N, K, G, torch.tensor(at, device="cuda"), X, K, W, K, N * K, 0.0, Y, N, c32)
    finally:
        B.gemm_force_variant(-1, 0)
    ref, ab = reference(X, W, at), reference(X.abs(), W.abs(), at)
    err = ab * (K + 4) * U
    bound = err if c32 else err + 2.0 ** -8 * (ref.abs() + err)
    assert ((Y.double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("dtype,K", [(torch.bfloat16, 64), (torch.bfloat16, 61), (torch.float32, 64)])
def test_rows_and_weights_beyond_32_bits(dtype, K):
    """Leading dimension and stride put the last rows and the last expert's weights behind 2^31 elements."""
    print(f"[gpu-case] far rows and weights {dtype} {K}", flush=True)
    code = B.DTYPE_BF16 if dtype == torch.bfloat16 else B.DTYPE_F32
    ld, M, N, G = 1 << 25, 66, 40, 2
    flat = torch.zeros((M - 1) * ld + K, dtype=dtype, device="cuda")
    X = flat.as_strided((M, K), (ld, 1))
    gen = torch.Generator(device="cuda").manual_seed(3)
    X.copy_(torch.randn((M, K), device="cuda", generator=gen))
    stride = (1 << 31) + 8
    bank = torch.zeros(stride + N * K, dtype=dtype, device="cuda")
    W = bank.as_strided((G, N, K), (stride, K, 1))
    W.copy_(torch.randn((G, N, K), device="cuda", generator=gen))
    at = [0, 3, M]
    off = torch.tensor(at, device="cuda")
    Y = torch.full((M, N), float("nan"), device="cuda")
    B.gemm_grouped(code, 1, M, N, K, G, off, flat, ld, bank, K, stride, 0.0, Y, N, 1)
    Xc, Wc = X.contiguous(), W.contiguous()
    ref, ab = reference(Xc, Wc, at), reference(Xc.abs(), Wc.abs(), at)
    assert ((Y.double() - ref).abs() <= ab * (K + 4) * U).all()
    # the weight gradient of the same rows
    dY = torch.randn((M, N), device="cuda", generator=gen).to(dtype)
    dW = torch.full((G, N, K), float("nan"), device="cuda")
    B.gemm_grouped_wgrad(code, M, N, K, G, off, dY, N, flat, ld, 0.0, dW, K, N * K, 1)
    for e in range(G):
        y, x = dY[at[e]:at[e + 1]].double().t().contiguous(), Xc[at[e]:at[e + 1]].double()
        assert ((dW[e].double() - y @ x).abs() <= (y.abs() @ x.abs()) * (M + 4) * U).all()
