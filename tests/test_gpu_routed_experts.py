"""Router, 4-bit images and their grouped products run together, as the block of examples/routed_experts_in_4_bits.py uses them:
its gradients, its serving path step by step, both captured into a graph on another stream and replayed with other rows."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import mx4_reference as mx
import route_reference as rr
from paper_2511_13764_amd import binding as B

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -8


def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "routed_experts_in_4_bits.py")
    spec = importlib.util.spec_from_file_location("routed_experts_in_4_bits", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def d(t):
    return t.double().cpu().numpy()


class Off:
    """A number in 64 bits and how far the kernels' may be from it: every product, sum and rounding adds its own."""

    def __init__(self, v, e=0.0):
        self.v, self.e = np.asarray(v, float), np.broadcast_to(e, np.shape(v))

    def most(self):
        return np.abs(self.v) + self.e

    def __add__(self, o):
        return Off(self.v + o.v, (self.e + o.e) + U32 * (self.most() + o.most()))

    def __sub__(self, o):
        return self + Off(-o.v, o.e)

    def __mul__(self, o):
        e = np.abs(self.v) * o.e + o.most() * self.e
        return Off(self.v * o.v, e + U32 * (np.abs(self.v * o.v) + e))

    def __matmul__(self, o):                    # fp32 sums of at most K + 18 roundings
        m = self.most() @ o.most()
        return Off(self.v @ o.v, m - np.abs(self.v) @ np.abs(o.v) + (self.v.shape[-1] + 18) * U32 * m)

    def sum(self, axis, keepdims=False):
        m = self.most().sum(axis, keepdims=keepdims)
        return Off(self.v.sum(axis, keepdims=keepdims), self.e.sum(axis, keepdims=keepdims) + self.v.shape[axis] * U32 * m)

    def bf16(self):
        return Off(self.v, self.e + U16 * self.most() + 1e-38)

    def t(self):
        return Off(self.v.T, self.e.T)

    def __getitem__(self, i):
        return Off(self.v[i], self.e[i])

    def holds(self, got, what):
        got = d(got)
        assert got.shape == self.v.shape, what
        assert (np.abs(got - self.v) <= self.e).all(), (what, np.abs(got - self.v).max(), self.e.max())


def grouped(x, w, at, n):
    """Rows at[e] .. at[e + 1] - 1 of x times w[e] turned over; zeros behind the last."""
    out = Off(np.zeros((x.v.shape[0], n)), np.zeros((x.v.shape[0], n)))
    out.v, out.e = out.v.copy(), np.array(out.e)
    for e, (a, b) in enumerate(zip(at, at[1:])):
        part = x[a:b] @ Off(w[e].T)
        out.v[a:b], out.e[a:b] = part.v, part.e
    return out


@pytest.mark.parametrize("rows,padding", [(77, 10), (1, 0), (40, 40)])
def test_the_block_and_its_gradients(rows, padding):
    m = example()
    width, hidden, E, top = 64, 96, 5, 2
    blk = m.Experts(width, hidden, E, top)
    gen = torch.Generator().manual_seed(rows)
    x, dy = (torch.randn((rows, width), generator=gen) for _ in range(2))
    x = x.bfloat16()
    valid = (torch.arange(rows) < rows - padding)
    dloss = torch.tensor([0.7])
    y, loss, kept = blk.forward(x.cuda(), valid.to(torch.uint8).cuda())
    dx = blk.backward(dy.cuda(), dloss.cuda(), kept)

    # the choice, from the logits as they came out, exactly; all else with the errors that it may have
    X, R = Off(d(x)), Off(d(blk.R))
    logits = X @ R.t()
    logits.holds(kept["logits"], "logits")
    chosen = rr.route(d(kept["logits"]), top, valid.numpy(), True)
    for n in ("ids", "offsets", "rows", "place"):
        assert np.array_equal(kept[n].cpu().numpy(), chosen[n]), n
    ids, at, place = chosen["ids"], chosen["offsets"], chosen["place"]
    taken, count = ids >= 0, int(at[-1])
    exact = rr.route(logits.v, top, valid.numpy(), True)
    if count:
        assert np.array_equal(exact["ids"], ids)          # (no two logits are that close here)
    # exp(+- the logits' error) twice, and the softmax's own roundings
    p = Off(exact["p"], exact["p"] * (2.1 * logits.e.max() + (E + 40) * U32))
    gates = Off(exact["gates"], exact["gates"] * (4.2 * logits.e.max() + (2 * E + 80) * U32))
    gates.holds(kept["gates"], "gates")

    w = {n: np.stack([mx.values(mx.image(d(t)), *t.shape) for t in getattr(blk, n)]) for n in ("U", "D")}
    source = chosen["rows"][:count]
    xs = X[source]
    h = grouped(xs, w["U"], at, hidden)
    bias = np.concatenate([np.repeat(d(blk.bias)[e:e + 1], at[e + 1] - at[e], 0) for e in range(E)]) if count else np.zeros((0, hidden))
    h = h + Off(bias)
    h = Off(np.maximum(h.v, 0.0), h.e).bf16()
    h.holds(kept["h"][:count], "h")
    ys = grouped(h, w["D"], at, width).bf16()
    at_place = np.maximum(place, 0)

    def each(o):                                # places' rows, a row and choice; nothing where there is none
        if not count:
            return Off(np.zeros((rows, top, o.v.shape[1])))
        return Off(o.v[at_place] * taken[:, :, None], o.e[at_place] * taken[:, :, None])
    (each(ys) * gates[:, :, None]).sum(1).holds(y, "y")

    share = np.diff(at) / max(1, count)
    n = max(1, int(taken[:, 0].sum()))
    mean = Off(p.v[taken[:, 0]].sum(0) / n, p.e[taken[:, 0]].sum(0) / n + (rows + 4) * U32)
    total = (mean * Off(share, share * U32)).sum(0)
    Off(E * total.v, E * total.e * (1 + U32) + E * total.v * U32).holds(loss, "loss")

    # backward
    DY = Off(d(dy))
    gate = Off(np.zeros(count), np.zeros(count))
    gate = Off(gates.v[taken][np.argsort(place[taken])], gates.e[taken][np.argsort(place[taken])])
    dys = (DY[source] * gate[:, None]).bf16()
    positive = d(kept["h"][:count]) > 0
    dh = grouped(dys, w["D"].transpose(0, 2, 1), at, hidden).bf16() * Off(positive.astype(float))
    dxs = grouped(dh, w["U"].transpose(0, 2, 1), at, width).bf16()
    for name, a, b in (("D", dys, h), ("U", dh, xs)):
        for e in range(E):
            s = slice(at[e], at[e + 1])
            (a[s].t() @ b[s]).holds(blk.grads[name][e], f"gradient of {name}[{e}]")
    dgates = (each(ys) * DY[:, None, :]).sum(2)
    lead = (gates * dgates).sum(1, keepdims=True)
    chosen_part = gates * (dgates - lead)
    if count:
        f = Off(share, share * U32)
        part = p * (f - (p * f).sum(1, keepdims=True)) * Off(np.full((1, 1), float(dloss) * E / n), float(dloss) * E / n * 3 * U32)
    else:
        part = Off(np.zeros((rows, E)))
    dl = Off(part.v * taken[:, :1], part.e * taken[:, :1])
    add = np.zeros((rows, E)), np.zeros((rows, E))
    for j in range(top):
        t = np.nonzero(taken[:, j])[0]
        add[0][t, ids[t, j]] += chosen_part.v[t, j]
        add[1][t, ids[t, j]] += chosen_part.e[t, j]
    dl = dl + Off(*add)
    dl = Off(dl.v, dl.e + E * U32 * dl.most())
    (dl.t() @ X).holds(blk.grads["R"], "gradient of R")
    (each(dxs).sum(1) + dl @ R).holds(dx, "dx")


@pytest.mark.parametrize("rows", [1, 16, 300])
def test_serving_step_by_step(rows):
    m = example()
    width, hidden, E, top = 320, 520, 6, 3
    blk = m.Experts(width, hidden, E, top, seed=3)
    x = torch.randn((rows, width), generator=torch.Generator().manual_seed(rows)).bfloat16()
    valid = torch.ones(rows, dtype=torch.uint8)
    valid[5:9] = 0
    got = blk.serve(x.cuda(), valid.cuda())
    r, M = blk._route(x.cuda(), valid.cuda()), rows * top
    at, count = r["offsets"].tolist(), int(r["offsets"][-1])
    source = r["rows"].cpu().numpy()
    xs = np.where(source[:, None] < 0, 0.0, d(x)[np.maximum(source, 0)])
    image = blk._image(x.cuda(), M, r["rows"])
    assert np.array_equal(image.cpu().numpy(), mx.image(xs))
    w = {n: [mx.values(mx.image(d(t)), *t.shape) for t in getattr(blk, n)] for n in ("U", "D")}

    def product(a, name, bias):
        out, off = np.zeros((M, w[name][0].shape[0])), np.zeros((M, w[name][0].shape[0]))
        for e in range(E):
            s = slice(at[e], at[e + 1])
            out[s], off[s] = a[s] @ w[name][e].T, mx.most_off(a[s], w[name][e], True)
            if bias is not None:
                out[s] += d(bias)[e]
                off[s] += U32 * np.abs(out[s])
                out[s] = np.maximum(out[s], 0.0)
        return Off(out, off).bf16()
    h = blk._experts(B.DTYPE_MX4, M, image, blk.U4, hidden, width, r["offsets"], blk.bias)
    product(mx.values(mx.image(xs), M, width), "U", blk.bias).holds(h, "h")
    image = blk._image(h)
    assert np.array_equal(image.cpu().numpy(), mx.image(d(h)))
    ys = blk._experts(B.DTYPE_MX4, M, image, blk.D4, width, hidden, r["offsets"])
    product(mx.values(mx.image(d(h)), M, hidden), "D", None).holds(ys, "ys")
    place, gates = r["place"].cpu().numpy(), d(r["gates"])
    want = (Off(d(ys)[np.maximum(place, 0)]) * Off(gates[:, :, None])).sum(1).bf16()
    want.holds(got, "y")
    assert not got[5:9].any() and (rows < 6 or count == (rows - len(range(5, min(9, rows)))) * top)


def test_captured_on_another_stream_and_replayed_with_other_rows():
    """Forward, backward and serving in one graph; every replay gives the bits of the eager calls on what is there by then."""
    m = example()
    rows, width, hidden, E, top = 50, 256, 320, 8, 2
    blk = m.Experts(width, hidden, E, top, seed=5)
    gen = torch.Generator().manual_seed(9)
    inputs = []
    for i in range(3):
        v = torch.ones(rows, dtype=torch.uint8)
        v[[50, 20, 0][i]:] = 0                  # all rows, some, none
        inputs.append((torch.randn((rows, width), generator=gen).bfloat16().cuda(), v.cuda(), torch.randn((rows, width), generator=gen).cuda()))
    dloss = torch.full((1,), 0.3, device="cuda")

    def step(x, valid, dy):
        y, loss, kept = blk.forward(x, valid)
        dx = blk.backward(dy, dloss, kept)
        return [y, loss, dx, blk.serve(x, valid)]

    def run(step):
        for g in blk.grads.values():
            g.zero_()
        out = step()
        return [t.clone() for t in (*out, *blk.grads.values())]
    eager = [run(lambda i=i: step(*inputs[i])) for i in range(3)]
    x, valid, dy = (t.clone() for t in inputs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run(lambda: step(x, valid, dy))  # (on the other stream, not captured)
    torch.cuda.synchronize()
    for a, b in zip(other, eager[0]):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(x, valid, dy)
    for i in (1, 0, 2, 1):
        for to, t in zip((x, valid, dy), inputs[i]):
            to.copy_(t)

        def replay():
            graph.replay()
            return out
        got = run(replay)
        torch.cuda.synchronize()
        for a, b in zip(got, eager[i]):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """Two blocks, each with its workspace, on a stream each: the bits of one after the other."""
    m = example()
    gen = torch.Generator().manual_seed(11)
    blocks = [m.Experts(512, 384, E, top, seed=E) for E, top in ((8, 2), (70, 4))]
    rows = (700, 900)
    x = [torch.randn((n, 512), generator=gen).bfloat16().cuda() for n in rows]
    dy = [torch.randn((n, 512), generator=gen).cuda() for n in rows]
    dloss = torch.full((1,), 0.1, device="cuda")

    def step(i):
        y, loss, kept = blocks[i].forward(x[i])
        return [y, loss, blocks[i].backward(dy[i], dloss, kept), blocks[i].serve(x[i])]
    want = [step(0), step(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step(i))
    torch.cuda.synchronize()
    for i in (0, 1):
        for out in got[i]:
            for a, b in zip(out, want[i]):
                assert torch.equal(a, b)


def test_the_example_runs(capsys):
    example().main()
    assert "16 rows served" in capsys.readouterr().out
