"""Experts whose weights are kept in 4 bits behind a router with a balance loss: training, forward and backward, and serving.

    g, e  = the topk experts of every row and their gates      gemm_route, on logits x R^T (gemm_f32)
    y     = sum over them of g relu(x U_e^T + b_e) D_e^T       gemm_grouped_mx4, twice, on rows sorted by expert

Training: rows in bf16, the products read the images of bf16 weights, whose gradients pass through the rounding (made once
per step by `quantise`).  Serving: rows are 4-bit images too, gathered and packed in one launch.  Rows that are padding take
no expert.  Nothing passes through the host.

    python examples/routed_experts_in_4_bits.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2511_13764_amd import binding as B  # noqa: E402


def new(shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


class Experts:
    def __init__(self, width, hidden, experts, topk, seed=0):
        gen = torch.Generator().manual_seed(seed)

        def weights(*shape):
            return (torch.randn(shape, generator=gen) * shape[-1] ** -0.5).cuda()
        self.width, self.hidden, self.experts, self.topk = width, hidden, experts, topk
        self.R = weights(experts, width)
        self.U, self.D = weights(experts, hidden, width).bfloat16(), weights(experts, width, hidden).bfloat16()
        self.bias = weights(experts, hidden)
        self.grads = {n: torch.zeros(getattr(self, n).shape, device="cuda") for n in ("R", "U", "D")}
        self.ws = new(64 << 20, torch.uint8)
        self.quantise()

    def _image(self, x, rows=None, source=None):
        rows = x.shape[0] if rows is None else rows
        image = new(B.gemm_mx4_bytes(rows, x.shape[1]), torch.uint8)
        B.gemm_pack_mx4(B.DTYPE_BF16, 0, rows, x.shape[1], x, x.shape[1], x.shape[0], source, image)
        return image

    def quantise(self):
        """The images of the weights, one behind the other, and for the backward pass the numbers that they stand for."""
        for n in ("U", "D"):
            w = getattr(self, n)
            setattr(self, n + "4", torch.stack([self._image(w[e]) for e in range(self.experts)]))
            back = new(w.shape)
            for e in range(self.experts):
                B.gemm_unpack_mx4(B.DTYPE_BF16, w.shape[1], w.shape[2], getattr(self, n + "4")[e], back[e], w.shape[2])
            setattr(self, n + "q", back)

    def _route(self, x, valid):
        M, E, top = x.shape[0], self.experts, self.topk
        x32, logits = x.float(), new((M, E), torch.float32)
        B.gemm_f32(0, 1, M, E, self.width, x32, self.width, self.R, self.width, 0.0, logits, E, workspace=self.ws)
        r = dict(ids=new((M, top), torch.int64), gates=new((M, top), torch.float32), offsets=new(E + 1, torch.int64),
                 rows=new(M * top, torch.int64), place=new((M, top), torch.int64), balance=new(2 + E, torch.float32))
        B.gemm_route(B.DTYPE_F32, M, E, top, logits, E, valid, 1, *r.values(), workspace=self.ws)
        return dict(r, logits=logits, x32=x32)

    def _experts(self, code, M, a, images, n, k, offsets, bias=None):
        # (rows behind the last place are not written: zeros, so that nothing times a gate of 0 is 0)
        y = torch.zeros((M, n), dtype=torch.bfloat16, device="cuda")
        B.gemm_grouped_mx4(code, M, n, k, self.experts, offsets, a, k, images, images.stride(0), 0.0, y, n, 0, bias, n,
                           B.EPI_BIAS | B.EPI_RELU if bias is not None else B.EPI_NONE, workspace=self.ws)
        return y

    def _combine(self, ys, place, gates=None):
        each = ys[place.clamp(min=0)].float()                       # rows x topk x width
        return (each if gates is None else each * gates[:, :, None]).sum(1)

    def serve(self, x, valid=None):
        r, M = self._route(x, valid), x.shape[0] * self.topk
        h = self._experts(B.DTYPE_MX4, M, self._image(x, M, r["rows"]), self.U4, self.hidden, self.width, r["offsets"], self.bias)
        ys = self._experts(B.DTYPE_MX4, M, self._image(h), self.D4, self.width, self.hidden, r["offsets"])
        return self._combine(ys, r["place"], r["gates"]).bfloat16()

    def forward(self, x, valid=None):
        """y (fp32), the balance loss, and what `backward` takes."""
        r, M = self._route(x, valid), x.shape[0] * self.topk
        xs = x[r["rows"].clamp(min=0)]
        h = self._experts(B.DTYPE_BF16, M, xs, self.U4, self.hidden, self.width, r["offsets"], self.bias)
        ys = self._experts(B.DTYPE_BF16, M, h, self.D4, self.width, self.hidden, r["offsets"])
        return self._combine(ys, r["place"], r["gates"]), r["balance"][0], dict(r, xs=xs, h=h, ys=ys)

    def _turned(self, dy, weights, offsets):
        n, k = weights.shape[1:]
        dx = torch.zeros((dy.shape[0], k), dtype=torch.bfloat16, device="cuda")
        B.gemm_grouped(B.DTYPE_BF16, 0, dy.shape[0], k, n, self.experts, offsets, dy, n, weights, k, n * k, 0.0, dx, k, 0,
                       workspace=self.ws)
        return dx

    def _wgrad(self, name, dy, x, offsets):
        g = self.grads[name]
        n, k = g.shape[1:]
        B.gemm_grouped_wgrad(B.DTYPE_BF16, x.shape[0], n, k, self.experts, offsets, dy, n, x, k, 1.0, g, k, n * k, 1, workspace=self.ws)

    def backward(self, dy, dloss, kept):
        """dx (fp32) of dy and of the balance loss's dloss (one fp32); the weights' gradients are added to `grads`."""
        M, E, w, place, offsets = dy.shape[0], self.experts, self.width, kept["place"], kept["offsets"]
        taken = place >= 0
        # of every place: gate and row
        gate = torch.zeros(place.numel() + 1, device="cuda")
        gate[torch.where(taken, place, place.numel())] = kept["gates"] * taken
        dys = (dy[kept["rows"].clamp(min=0)] * gate[:-1, None]).bfloat16()
        self._wgrad("D", dys, kept["h"], offsets)
        dh = self._turned(dys, self.Dq, offsets) * (kept["h"] > 0)
        self._wgrad("U", dh, kept["xs"], offsets)
        dxs = self._turned(dh, self.Uq, offsets)
        # the router's: gates take dy . y_e
        dgates = (kept["ys"][place.clamp(min=0)].float() * dy[:, None, :]).sum(2)
        dlogits = new((M, E), torch.float32)
        B.gemm_route_grad(B.DTYPE_F32, M, E, self.topk, kept["logits"], E, 1, kept["ids"], offsets, kept["balance"], dgates, dloss,
                          dlogits, E)
        B.gemm_f32(1, 0, E, w, M, dlogits, E, kept["x32"], w, 1.0, self.grads["R"], w, workspace=self.ws)
        dx = self._combine(dxs, place, taken.float())
        B.gemm_f32(0, 0, M, w, E, dlogits, E, self.R, w, 1.0, dx, w, workspace=self.ws)
        return dx


def main():
    block = Experts(width=1024, hidden=2048, experts=8, topk=2)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((1000, 1024), generator=gen).bfloat16().cuda()
    valid = (torch.arange(1000, device="cuda") < 950).to(torch.uint8)
    y, loss, kept = block.forward(x, valid)
    dx = block.backward(torch.ones_like(y), torch.full((1,), 0.01, device="cuda"), kept)
    print("rows of every expert:", kept["offsets"].diff().tolist(), " balance loss", float(loss))
    print("|y|", float(y.norm()), " |dx|", float(dx.norm()), {n: float(g.norm()) for n, g in block.grads.items()})
    served = block.serve(x[:16].contiguous())
    print("16 rows served:", tuple(served.shape), "|y|", float(served.float().norm()))


if __name__ == "__main__":
    main()
