"""4-bit operands, the experts that read them, and the router in front of those: what is measured, and the plain forms.

Four operators.  `gemm_pack_mx4` with `gemm_unpack_mx4`: rows of numbers quantised to 4-bit floats
that share a power of two in blocks of 32, and read back.  `gemm_mx4`: a product with such an image as
its weights and an image, or 16-bit rows, on the other side.  `gemm_grouped_mx4`: the same where rows
belong to experts with weights of their own.  `gemm_route` with `gemm_route_grad`: which experts a
row takes, how many rows every expert has and where they go, the loss that keeps experts level, and
the gradient of gates and loss.

An image of R x K numbers, with Kp = K rounded up to a multiple of 256: R rows of Kp / 2 bytes, element
2 i of a row in the low half of byte i, 2 i + 1 in the high half, zeros past K; behind them, for every 256
columns, 8 bytes a row, the powers of two (biased by 127; 255: not a number) of the 8 blocks in the order
0 4 1 5 2 6 3 7.  A 4-bit float has a sign, two bits of exponent and one of fraction: 0 .5 1 1.5 2 3 4 6.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WORKSPACE = 128 << 20
EXPERT_WEIGHTS = 8 * 11008 * 4096               # elements of the largest bank of experts
MAX_FLOPS = 2.0 * 4096 * 11008 * 4096
MAX_BYTES = 0.6e9


def _pack(name, rows, K, dtype="bf16", turned=0):
    return {"name": name, "kind": "pack", "dtype": dtype, "rows": rows, "K": K, "turned": turned}


def _mx4(name, M, N, K, left="mx4", act=False, c32=False, beta=0.0):
    return {"name": name, "kind": "mx4", "left": left, "M": M, "N": N, "K": K, "act": act, "c32": c32, "beta": beta}


def _experts(name, M, groups, N, K, left="mx4", act=False, empty=0, spread=1):
    return {"name": name, "kind": "experts", "left": left, "M": M, "groups": groups, "N": N, "K": K, "act": act,
            "empty": empty, "spread": spread}


def _route(name, M, E, top, dtype="bf16", level=1, train=False, padded=0):
    return {"name": name, "kind": "route", "dtype": dtype, "M": M, "E": E, "top": top, "level": level, "train": train,
            "padded": padded}


def listed():
    return [
        # the activations of 16 sequences in decode
        _pack("pack_16", 16, 4096),
        # ... and of a prompt in front of the down-projection
        _pack("pack_4096", 4096, 11008),
        # weights kept in 32 bits, turned over for the input gradient; a multiple of nothing
        _pack("pack_turned_odd", 2003, 1500, "f32", turned=1),
        # both sides in 4 bits: a square, and sizes that are a multiple of nothing under the fused epilogue
        _mx4("mx4_4096", 4096, 4096, 4096),
        _mx4("mx4_odd", 1000, 2003, 1500, act=True),
        # serving with 4-bit weights alone: 16 sequences, and chunks of prompts in binary16
        _mx4("weights_decode_16", 16, 11008, 4096, left="bf16"),
        _mx4("weights_chunk_512", 512, 4096, 4096, left="f16"),
        # decode of 16 sequences, two experts for each, one of eight unused
        _experts("experts_decode_32", 32, 8, 11008, 4096, left="bf16", act=True, empty=1),
        # prefill of the same layer with both sides in 4 bits
        _experts("experts_prefill_4096", 4096, 8, 11008, 4096, act=True),
        # the router of a decode step: 16 rows, two of eight experts
        _route("route_decode_16", 16, 8, 2),
        # training: 8192 rows of which some are padding, four of 64 experts, forward and backward
        _route("route_train_8192", 8192, 64, 4, train=True, padded=300),
        # many experts, logits in 32 bits, gates as they come out of the softmax over all
        _route("route_train_160", 4099, 160, 6, "f32", level=0, train=True),
    ]


# ------------------------------------------------------------------ drawn cases

def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width of the range: as it falls, or rounded to what models have (multiples of 64, of 8)."""
    x, how = _logint(rng, lo, hi), rng.random()
    return (x + 63) // 64 * 64 if how < 0.6 else (x + 7) // 8 * 8 if how < 0.8 else x


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        c.pop("name")
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return c


def _draw(rng):
    kind = rng.choices(["pack", "mx4", "weights_few", "weights", "experts_few", "experts", "route"], [3, 3, 2, 2, 2, 3, 4])[0]
    if kind == "pack":
        return _pack("", _logint(rng, 1, 8192), _width(rng, 64, 11008), rng.choice(["bf16", "bf16", "f16", "f32"]),
                     rng.choice([0, 0, 1]))
    if kind == "route":
        E = rng.choice([4, 8, 16, 64, 128, 256, rng.randrange(2, 512)])
        M = _logint(rng, 1, 16384)
        return _route("", M, E, rng.randrange(1, min(E, 8) + 1), rng.choice(["bf16", "f32", "f16"]), rng.choice([0, 1]),
                      rng.random() < 0.6, rng.choice([0, 0, M // 10]))
    N, K = _width(rng, 256, 11008), _width(rng, 256, 8192)
    half = rng.choice(["bf16", "bf16", "f16"])
    act = rng.random() < 0.4
    if kind == "mx4":
        c32 = rng.random() < 0.3
        return _mx4("", _logint(rng, 1, 4096), N, K, "mx4", act, c32, 1.0 if c32 and rng.random() < 0.5 else 0.0)
    if kind == "weights_few":
        return _mx4("", _logint(rng, 1, 64), N, K, half, act)
    if kind == "weights":
        return _mx4("", _logint(rng, 64, 4096), N, K, half, act)
    groups, spread = _logint(rng, 2, 64), rng.randrange(1, 1 << 20)
    while groups * N * K > EXPERT_WEIGHTS:
        N, K = (N + 1) // 2, (K + 1) // 2
    empty = rng.choice([0, 0, groups // 8])
    M = _logint(rng, 1, 256) if kind == "experts_few" else _logint(rng, 256, 8192)
    return _experts("", M, groups, N, K, rng.choice(["mx4", half]), act, empty, spread)


def _sizes(case):
    """Rows of every expert, from the case alone: uneven, `empty` experts without a row."""
    M, groups = case["M"], case["groups"]
    rng = random.Random(case["spread"])
    used = max(1, min(groups - case["empty"], M))
    share = [rng.expovariate(1.0) + 0.1 for _ in range(used)]
    sizes = [1 + int((M - used) * x / sum(share)) for x in share]
    for i in range(M - sum(sizes)):
        sizes[i % used] += 1
    sizes += [0] * (groups - used)
    rng.shuffle(sizes)
    return sizes


def _image_bytes(rows, K):
    """What an image cannot do without: half a byte an element, a byte for 32."""
    return rows * (K / 2 + -(-K // 32))


def work(case):
    if case["kind"] == "pack":
        n, e = case["rows"] * case["K"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": float(n * (e + 2) + 2 * _image_bytes(case["rows"], case["K"])), "flops": 0.0}
    if case["kind"] == "route":
        M, E, top, e = case["M"], case["E"], case["top"], 4 if case["dtype"] == "f32" else 2
        chosen = M * top * (8 + 4 + 8 + 8)                  # ids, gates, rows and places
        moved = M * E * e + M + chosen + 12 * E
        if case["train"]:
            moved += 2 * M * E * e + M * top * (8 + 4) + 12 * E
        return {"bytes": float(moved), "flops": 0.0}
    M, N, K = case["M"], case["N"], case["K"]
    left = _image_bytes(M, K) if case["left"] == "mx4" else 2 * M * K
    if case["kind"] == "mx4":
        c = (4 if case["c32"] else 2) * (2 if case["beta"] else 1)
        moved = left + _image_bytes(N, K) + c * M * N + (4 * N if case["act"] else 0)
    else:
        used = sum(1 for m in _sizes(case) if m)
        moved = left + used * (_image_bytes(N, K) + (4 * N if case["act"] else 0)) + 2 * M * N
    return {"bytes": float(moved), "flops": 2.0 * M * N * K}


# ------------------------------------------------------------------ images in elementary operations

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
ORDER = (0, 4, 1, 5, 2, 6, 3, 7)


def _padded_k(K):
    return (K + 255) // 256 * 256


def _blocks(x):
    """Codes (0 .. 15) and biased powers of two of rows of 32-bit numbers, K padded to a multiple of 256."""
    rows, K = x.shape
    if _padded_k(K) != K:
        x = torch.nn.functional.pad(x, (0, _padded_k(K) - K))
    x = x.reshape(rows, -1, 32)
    largest = x.abs().amax(2)
    power = (torch.frexp(largest)[1] - 3).clamp(-127, 127)          # 2^power * 4 <= largest < 2^power * 8
    power = torch.where(largest == 0, torch.full_like(power, -127), power)
    y = torch.ldexp(x, -power[:, :, None])
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = code + 8 * torch.signbit(y).to(torch.uint8)
    finite = torch.isfinite(largest)
    power = torch.where(finite, power + 127, torch.full_like(power, 255)).to(torch.uint8)
    return (code * finite[:, :, None]).reshape(rows, -1), power


def _image(x):
    """The image of rows of numbers as the library lays it out, one uint8 tensor."""
    code, power = _blocks(x.float())
    codes = code[:, 0::2] | code[:, 1::2] << 4
    powers = power.reshape(x.shape[0], -1, 8)[:, :, list(ORDER)].permute(1, 0, 2)
    return torch.cat([codes.reshape(-1), powers.reshape(-1)])


def _values(image, rows, K, dtype=torch.float32):
    """What an image stands for, rows x K."""
    Kp = _padded_k(K)
    codes = image[:rows * (Kp // 2)].reshape(rows, Kp // 2)
    powers = image[rows * (Kp // 2):rows * (Kp // 2) + rows * (Kp // 32)].reshape(Kp // 256, rows, 8)
    code = torch.stack([codes & 15, codes >> 4], 2).reshape(rows, Kp)
    grid = torch.tensor([*GRID, *(-g for g in GRID)], dtype=dtype, device=image.device)
    power = torch.empty((rows, Kp // 256, 8), dtype=torch.uint8, device=image.device)
    power[:, :, list(ORDER)] = powers.permute(1, 0, 2)
    power = power.reshape(rows, Kp // 32, 1)
    one = torch.ones((), dtype=dtype, device=image.device)
    scale = torch.where(power == 255, one * float("nan"), torch.ldexp(one, power.to(torch.int32) - 127))
    return (grid[code.long()].reshape(rows, Kp // 32, 32) * scale).reshape(rows, Kp)[:, :K]


# ------------------------------------------------------------------ inputs

def _normal(gen, sigma, *shape):
    return torch.randn(shape, device="cuda", generator=gen) * sigma


def _activations(gen, M, K):
    """Rows as a layer's input has them: a few columns far larger than the rest."""
    x = _normal(gen, 1.0, M, K)
    large = torch.rand(K, device="cuda", generator=gen) < 0.01
    return x * torch.where(large, 20.0, 1.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    if case["kind"] == "pack":
        rows, K = case["rows"], case["K"]
        x = _activations(gen, rows, K) if not case["turned"] else _normal(gen, 0.02, rows, K)
        s["X"] = (x.t().contiguous() if case["turned"] else x).to(DTYPES[case["dtype"]])
        s["image"] = torch.empty(rows * (_padded_k(K) // 2 + _padded_k(K) // 32), dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda")
        return s
    if case["kind"] == "route":
        M, E, top = case["M"], case["E"], case["top"]
        popular = _normal(gen, 0.7, E)
        s["logits"] = (_normal(gen, 1.5, M, E) + popular).to(DTYPES[case["dtype"]])
        s["valid"] = None
        if case["padded"]:
            s["valid"] = (torch.arange(M, device="cuda") < M - case["padded"]).to(torch.uint8)
        for name, shape, dt in (("ids", (M, top), torch.int64), ("gates", (M, top), torch.float32),
                                ("offsets", (E + 1,), torch.int64), ("rows", (M * top,), torch.int64),
                                ("place", (M, top), torch.int64), ("balance", (2 + E,), torch.float32),
                                ("dlogits", (M, E), DTYPES[case["dtype"]])):
            s[name] = torch.empty(shape, dtype=dt, device="cuda")
        s["dgates"] = _normal(gen, 1.0, M, top)
        s["dloss"] = torch.full((1,), 0.01 * M, device="cuda")
        s["ws"] = torch.empty(WORKSPACE // 16, dtype=torch.uint8, device="cuda")
        return s
    M, N, K = case["M"], case["N"], case["K"]
    x = _activations(gen, M, K)
    s["X"] = _image(x) if case["left"] == "mx4" else x.to(DTYPES[case["left"]])
    half = torch.float16 if case["left"] == "f16" else torch.bfloat16
    s["ws"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    if case["kind"] == "mx4":
        s["W"] = _image(_normal(gen, 0.02, N, K))
        s["bias"] = _normal(gen, 1.0, N) if case["act"] else None
        s["Y"] = _normal(gen, 1.0, M, N).to(torch.float32 if case["c32"] else half)
        return s
    G = case["groups"]
    rng = random.Random(int(seed))
    sizes = _sizes(case)
    rng.shuffle(sizes)
    starts = [0]
    for m in sizes:
        starts.append(starts[-1] + m)
    s.update(sizes=sizes, starts=starts, longest=max(sizes), offsets=torch.tensor(starts, dtype=torch.int64, device="cuda"))
    # the plan of a padded batched product: group of every row, and its place in it
    s["group"] = torch.repeat_interleave(torch.arange(G, device="cuda"), torch.tensor(sizes, device="cuda"))
    s["place"] = torch.arange(M, device="cuda") - s["offsets"][s["group"]]
    s["W"] = torch.stack([_image(_normal(gen, 0.02, N, K)) for _ in range(G)])
    s["bias"] = _normal(gen, 1.0, G, N) if case["act"] else None
    s["Y"] = torch.empty((M, N), dtype=half, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2511_13764_amd import binding as B
    c = s["case"]
    codes = {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16, "mx4": B.DTYPE_MX4}
    if c["kind"] == "pack":
        rows, K = c["rows"], c["K"]
        B.gemm_pack_mx4(codes[c["dtype"]], c["turned"], rows, K, s["X"], rows if c["turned"] else K, rows, None, s["image"])
        B.gemm_unpack_mx4(B.DTYPE_BF16, rows, K, s["image"], s["out"], K)
        return s["out"]
    if c["kind"] == "route":
        M, E, top, dt = c["M"], c["E"], c["top"], codes[c["dtype"]]
        B.gemm_route(dt, M, E, top, s["logits"], E, s["valid"], c["level"], s["ids"], s["gates"], s["offsets"], s["rows"],
                     s["place"], s["balance"], workspace=s["ws"])
        out = {n: s[n] for n in ("ids", "gates", "offsets", "rows", "place", "balance")}
        if c["train"]:
            B.gemm_route_grad(dt, M, E, top, s["logits"], E, c["level"], s["ids"], s["offsets"], s["balance"], s["dgates"],
                              s["dloss"], s["dlogits"], E)
            out["dlogits"] = s["dlogits"]
        return out
    M, N, K = c["M"], c["N"], c["K"]
    left, lda = codes[c["left"]], 0 if c["left"] == "mx4" else K
    epilogue = B.EPI_BIAS | B.EPI_RELU if c["act"] else B.EPI_NONE
    if c["kind"] == "mx4":
        B.gemm_mx4(left, M, N, K, s["X"], lda, s["W"], c["beta"], s["Y"], N, c["c32"], s["bias"], epilogue, workspace=s["ws"])
        return s["Y"]
    B.gemm_grouped_mx4(left, M, N, K, c["groups"], s["offsets"], s["X"], lda, s["W"], s["W"].stride(0), 0.0, s["Y"], N, 0,
                       s["bias"], N, epilogue, workspace=s["ws"])
    return s["Y"]


def _left(s, dtype=torch.float32):
    c = s["case"]
    return _values(s["X"], c["M"], c["K"], dtype) if c["left"] == "mx4" else s["X"].to(dtype)


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "pack":
        x = s["X"].t() if c["turned"] else s["X"]
        return _values(_image(x.float()), c["rows"], c["K"]).to(torch.bfloat16)
    if c["kind"] == "route":
        return _route_plain(s)
    M, N, K = c["M"], c["N"], c["K"]
    if c["kind"] == "mx4":
        y = _left(s) @ _values(s["W"], N, K).t()
        if c["beta"]:
            y = y + c["beta"] * s["Y"].float()
        if c["act"]:
            y = (y + s["bias"]).clamp_min(0.0)
        if c["beta"]:
            s["Y"].copy_(y)
            return s["Y"]
        return y.to(s["Y"].dtype)
    padded = torch.zeros((c["groups"], s["longest"], K), device=s["W"].device)
    padded[s["group"], s["place"]] = _left(s)
    W = torch.stack([_values(w, N, K) for w in s["W"]])
    y = torch.bmm(padded, W.transpose(1, 2))[s["group"], s["place"]]
    if c["act"]:
        y = (y + s["bias"][s["group"]]).clamp_min(0.0)
    return y.to(s["Y"].dtype)


def _route_plain(s):
    c = s["case"]
    M, E, top = c["M"], c["E"], c["top"]
    x = s["logits"].float()
    ids = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :top]
    counted = torch.ones(M, dtype=torch.bool, device=x.device) if s["valid"] is None else s["valid"] != 0
    p = torch.exp(x - x.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    gates = p.gather(1, ids)
    if c["level"]:
        gates = gates / gates.sum(1, keepdim=True)
    gates = torch.where(counted[:, None], gates, torch.zeros_like(gates))
    ids = torch.where(counted[:, None], ids, torch.full_like(ids, -1))
    flat = torch.where(ids < 0, torch.full_like(ids, E), ids).reshape(-1)
    counts = (flat[:, None] == torch.arange(E, device=x.device)).sum(0)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=x.device)
    offsets[1:] = counts.cumsum(0)
    order = torch.sort(flat, stable=True)[1]
    at = torch.arange(M * top, device=x.device)
    taken = at < offsets[E]
    rows = torch.where(taken, order // top, torch.full_like(order, -1))
    place = torch.empty_like(order)
    place[order] = torch.where(taken, at, torch.full_like(at, -1))
    n = counted.sum().float()
    share = counts.float() / counts.sum().clamp_min(1).float()
    mean = (p * counted[:, None]).sum(0) / n.clamp_min(1.0)
    balance = torch.cat([(E * (share * mean).sum()).reshape(1), n.reshape(1), mean])
    out = {"ids": ids, "gates": gates, "offsets": offsets, "rows": rows, "place": place.reshape(M, top), "balance": balance}
    if c["train"]:
        d = torch.where(counted[:, None], s["dgates"], torch.zeros_like(s["dgates"]))
        at = ids.clamp_min(0)
        if c["level"]:
            g = gates * (d - (gates * d).sum(1, keepdim=True))
            dx = torch.zeros_like(x).scatter_add_(1, at, g)
        else:
            dp = torch.zeros_like(x).scatter_add_(1, at, d)
            dx = p * (dp - (p * dp).sum(1, keepdim=True))
        even = p * (share - (p * share).sum(1, keepdim=True)) * (s["dloss"] * E / n.clamp_min(1.0))
        out["dlogits"] = (dx + even * counted[:, None]).to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------ the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "pack":
        x = (s["X"].t() if case["turned"] else s["X"]).double()
        rows, K = x.shape
        out = torch.empty_like(x)
        grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
        for k in range(0, K, 32):
            b = x[:, k:k + 32]
            largest = b.abs().amax(1, keepdim=True)
            # the power of two that leaves the largest between 4 and 8
            scale = torch.exp2(torch.floor(torch.log2(largest.clamp_min(1e-300))) - 2)
            off = (b.abs()[:, :, None] / scale[:, :, None] - grid).abs()
            near = off.amin(2, keepdim=True)
            # of two that are equally near the one whose last bit is clear
            tie = torch.where(off == near, torch.arange(8, device="cuda") % 2, torch.full_like(off, 2, dtype=torch.int64))
            out[:, k:k + 32] = torch.sign(b) * grid[tie.argmin(2)] * scale
        return out
    if case["kind"] == "route":
        M, E, top = case["M"], case["E"], case["top"]
        x = s["logits"].double()
        live = torch.arange(M, device="cuda") < M - case["padded"]
        z = torch.softmax(x, 1)
        # chosen: fewer than `top` experts have a larger logit, or an equal one and a lower number
        rank = torch.empty((M, E), dtype=torch.int64, device="cuda")
        for e in range(E):
            rank[:, e] = (x > x[:, e:e + 1]).sum(1) + (x[:, :e] == x[:, e:e + 1]).sum(1)
        chosen = (rank < top) & live[:, None]
        at = torch.zeros((M, top), dtype=torch.int64, device="cuda")
        where = chosen.nonzero()
        at[where[:, 0], rank[where[:, 0], where[:, 1]]] = where[:, 1]
        w = torch.where(chosen, z, torch.zeros_like(z))
        total = w.sum(1, keepdim=True) if case["level"] else torch.ones((M, 1), dtype=torch.float64, device="cuda")
        w = torch.where(live[:, None], w / torch.where(live[:, None], total, torch.ones_like(total)), torch.zeros_like(w))
        gates = w.gather(1, at) * live[:, None]
        n = int(live.sum())
        share, mean = chosen.double().mean(0) * M / max(1, n * top), z[live].sum(0) / max(1, n)
        balance = torch.cat([(E * (share * mean).sum()).reshape(1), torch.tensor([float(n)], dtype=torch.float64, device="cuda"), mean])
        out = {"ids": None, "gates": gates, "offsets": None, "rows": None, "place": None, "balance": balance}
        if case["train"]:
            d = torch.zeros_like(z)
            d[torch.arange(M, device="cuda")[:, None].expand(M, top), at] = s["dgates"].double()
            d = torch.where(chosen, d, torch.zeros_like(d))
            v = w if case["level"] else z
            dx = v * (d - (v * d).sum(1, keepdim=True))
            dx = dx + float(s["dloss"]) * E / max(1, n) * z * (share - (z * share).sum(1, keepdim=True))
            out["dlogits"] = dx * live[:, None]
        return out
    M, N, K = case["M"], case["N"], case["K"]
    x = _left(s, torch.float64)
    if case["kind"] == "mx4":
        y = x @ _values(s["W"], N, K, torch.float64).t().contiguous() + case["beta"] * s["Y"].double()
        return (y + s["bias"].double()).clamp_min(0.0) if case["act"] else y
    y = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    for e in range(case["groups"]):
        a, b = s["starts"][e], s["starts"][e + 1]
        if a < b:
            y[a:b] = x[a:b] @ _values(s["W"][e], N, K, torch.float64).t().contiguous()
            if case["act"]:
                y[a:b] = (y[a:b] + s["bias"][e].double()).clamp_min(0.0)
    return y
