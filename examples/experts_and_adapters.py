"""A block whose rows do not share their weights: an adapted projection, then experts, forward and backward.

    x1 = x W^T + adapter of the request        gemm_adapters
    e  = the expert of every row               a router's choice
    y  = relu(x1 U_e^T + b_e) D_e^T            gemm_grouped, twice, on rows sorted by expert

The backward pass is the same calls turned over and gemm_grouped_wgrad; weight gradients are added up in
32 bits over micro-batches (beta = 1).  Nothing passes through the host: the bounds of the groups are
counted and read on the device.

    python examples/experts_and_adapters.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2511_13764_amd import binding as B  # noqa: E402

CODES = {torch.bfloat16: B.DTYPE_BF16, torch.float16: B.DTYPE_F16, torch.float32: B.DTYPE_F32}


class Block:
    def __init__(self, width, hidden, experts, adapters, rank, dtype=torch.bfloat16, device="cuda", seed=0):
        gen = torch.Generator().manual_seed(seed)

        def weights(*shape):
            return (torch.randn(shape, generator=gen) * shape[-1] ** -0.5).to(dtype).to(device)
        self.width, self.hidden, self.experts, self.adapters, self.rank = width, hidden, experts, adapters, rank
        self.dtype, self.code, self.c32 = dtype, CODES[dtype], dtype == torch.float32
        self.W = weights(width, width)
        self.down, self.up = weights(adapters, rank, width), weights(adapters, width, rank)
        self.scale = torch.ones(adapters, device=device)
        self.router = weights(experts, width).float()
        self.U, self.D = weights(experts, hidden, width), weights(experts, width, hidden)
        self.bias = torch.zeros((experts, hidden), device=device)
        # gradients, added up in 32 bits
        self.grads = {n: torch.zeros(getattr(self, n).shape, device=device) for n in ("down", "up", "U", "D")}
        self.ws = torch.empty(64 << 20, dtype=torch.uint8, device=device)

    def _project(self, transB, x, first, second, segments, offsets, ids):
        """x W^T (transB = 1) or x W beside the adapters' products: the result and the rank's sums."""
        M, w, r = x.shape[0], self.width, self.rank
        y, h = torch.empty_like(x), torch.empty((M, r), dtype=self.dtype, device=x.device)
        ld1, ld2 = (w, r) if transB else (r, w)
        B.gemm_adapters(self.code, transB, M, w, w, r, segments, offsets, ids, self.adapters, x, w, self.W, w, first, ld1,
                        r * w, second, ld2, w * r, self.scale, 0.0, y, w, self.c32, None, B.EPI_NONE, h, r, workspace=self.ws)
        return y, h

    def _experts(self, transB, x, weights, n, offsets, bias=None):
        k = x.shape[1]
        y = torch.empty((x.shape[0], n), dtype=self.dtype, device=x.device)
        B.gemm_grouped(self.code, transB, x.shape[0], n, k, self.experts, offsets, x, k, weights, k if transB else n, n * k,
                       0.0, y, n, self.c32, bias, n, B.EPI_BIAS | B.EPI_RELU if bias is not None else B.EPI_NONE,
                       workspace=self.ws)
        return y

    def _wgrad(self, name, dy, x, groups, offsets):
        g = self.grads[name]
        n, k = dy.shape[1], x.shape[1]
        B.gemm_grouped_wgrad(self.code, x.shape[0], n, k, groups, offsets, dy, n, x, k, 1.0, g, k, n * k, 1, workspace=self.ws)

    def decode(self, x, ids):
        """One token of every request: row i takes adapter ids[i] (-1: none)."""
        y, _ = self._project(1, x, self.down, self.up, x.shape[0], None, ids)
        out, _ = self._route(y)
        return out

    def _route(self, x1):
        expert = (x1.float() @ self.router.t()).argmax(1)
        order = torch.argsort(expert, stable=True)
        counts = (expert[:, None] == torch.arange(self.experts, device=x1.device)).sum(0)
        offsets = torch.zeros(self.experts + 1, dtype=torch.int64, device=x1.device)
        offsets[1:] = counts.cumsum(0)
        xs = x1[order]
        h = self._experts(1, xs, self.U, self.hidden, offsets, self.bias)
        ys = self._experts(1, h, self.D, self.width, offsets)
        y = torch.empty_like(ys)
        y[order] = ys
        return y, (order, offsets, xs, h)

    def forward(self, x, segments):
        """Rows segments[a] .. segments[a + 1] - 1 take adapter a (training: one segment for each adapter)."""
        x1, h1 = self._project(1, x, self.down, self.up, self.adapters, segments, None)
        y, kept = self._route(x1)
        return y, (x, segments, h1, *kept)

    def backward(self, dy, kept):
        """dx; the gradients of adapters and experts are added to `grads` (the router's choice has none)."""
        x, segments, h1, order, offsets, xs, h = kept
        dys = dy[order]
        self._wgrad("D", dys, h, self.experts, offsets)
        dh = self._experts(0, dys, self.D, self.hidden, offsets) * (h > 0)
        self._wgrad("U", dh, xs, self.experts, offsets)
        dxs = self._experts(0, dh, self.U, self.width, offsets)
        dx1 = torch.empty_like(dxs)
        dx1[order] = dxs
        dx, g = self._project(0, dx1, self.up, self.down, self.adapters, segments, None)
        self._wgrad("down", g, x, self.adapters, segments)
        self._wgrad("up", dx1, h1, self.adapters, segments)
        return dx


def main():
    block = Block(width=1024, hidden=2048, experts=8, adapters=4, rank=16)
    gen = torch.Generator().manual_seed(1)
    segments = torch.tensor([0, 300, 301, 301, 1000], device="cuda")
    for _ in range(2):                                              # two micro-batches
        x = torch.randn((1000, 1024), generator=gen).bfloat16().cuda()
        y, kept = block.forward(x, segments)
        dx = block.backward(torch.ones_like(y), kept)
    print("rows of every expert:", kept[4].diff().tolist())
    print("|y|", float(y.float().norm()), " |dx|", float(dx.float().norm()),
          {n: float(g.norm()) for n, g in block.grads.items()})
    tokens = block.decode(x[:16].contiguous(), torch.tensor([0, 1, 2, 3, -1] * 3 + [0], device="cuda"))
    print("decode of 16 requests:", tuple(tokens.shape), "|y|", float(tokens.float().norm()))


if __name__ == "__main__":
    main()
