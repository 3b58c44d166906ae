"""Products of rows that do not share their weights: what is measured of them, and their plain forms.

Three operators.  `gemm_grouped`: the rows of one call belong to experts, each with weights of
its own, in ragged groups.  `gemm_grouped_wgrad`: the weight gradient of those, a product whose
reduction is ragged.  `gemm_adapters`: one projection that all rows share, with a low-rank
adapter of each row segment's own beside it; turned over it is its input gradient, and the
gradients of its adapters are grouped weight gradients.

A case names the kind of call and its sizes; how many rows each group has follows from the case
alone, which group has how many from the seed.  Plain forms pad the groups to one length and use
batched products in 32 bits; `exact` goes group by group in 64.
"""
import math
import random

import torch

own = False

WORKSPACE = 64 << 20
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EXPERT_WEIGHTS = 8 * 11008 * 4096               # elements of the largest bank of experts
MAX_FLOPS = 2.0 * 4096 * 11008 * 4096
MAX_BYTES = 1.6e9


def _experts(name, M, groups, N, K, dtype="bf16", tB=1, act=False, empty=0, spread=1):
    return {"name": name, "kind": "experts", "dtype": dtype, "M": M, "groups": groups, "N": N, "K": K, "tB": tB,
            "act": act, "empty": empty, "spread": spread}


def _wgrad(name, M, groups, N, K, dtype="bf16", c32=False, beta=0.0, empty=0, spread=1):
    return {"name": name, "kind": "wgrad", "dtype": dtype, "M": M, "groups": groups, "N": N, "K": K, "c32": c32,
            "beta": beta, "empty": empty, "spread": spread}


def _adapters(name, M, groups, bank, R, N, K, dtype="bf16", bare=0, spread=1):
    return {"name": name, "kind": "adapters", "dtype": dtype, "M": M, "groups": groups, "bank": bank, "R": R, "N": N,
            "K": K, "bare": bare, "empty": 0, "spread": spread}


def _train(name, M, bank, R, N, K, dtype="bf16", empty=0, spread=1):
    return {"name": name, "kind": "adapters_grad", "dtype": dtype, "M": M, "groups": bank, "bank": bank, "R": R, "N": N,
            "K": K, "empty": empty, "spread": spread}


def listed():
    return [
        # decode of 16 sequences, two experts for each: 32 rows over 8 experts, one of them unused
        _experts("experts_decode_32", 32, 8, 11008, 4096, act=True, empty=1),
        # prefill of the same layer
        _experts("experts_prefill_4096", 4096, 8, 11008, 4096, act=True),
        # many small experts in binary16, two without a row
        _experts("experts_64_f16", 2048, 64, 1024, 2048, dtype="f16", empty=2),
        # widths and counts that are a multiple of nothing
        _experts("experts_odd", 1000, 5, 2003, 1500),
        # input gradient of the down-projection's experts: the weights read the other way
        _experts("experts_dinput_2048", 2048, 8, 4096, 4096, tB=0),
        # experts kept in 32 bits
        _experts("experts_f32", 777, 6, 1001, 1301, dtype="f32", empty=1),
        # weight gradients of a layer's experts, added in 32 bits over micro-batches
        _wgrad("experts_wgrad_4096", 4096, 8, 4096, 4096, c32=True, beta=1.0),
        # ... and of many small experts, rounded to the weights' type
        _wgrad("experts_wgrad_64", 4096, 64, 1024, 2048, empty=2),
        # decode: one token each of 16 requests, each request with an adapter
        _adapters("adapters_decode_16", 16, 16, 32, 16, 4096, 4096, bare=2),
        # prefill of 12 prompts through the up-projection, 8 adapters among them
        _adapters("adapters_prefill_4096", 4096, 12, 8, 16, 11008, 4096, bare=1),
        # a step that mixes chunks of prompts with single tokens, ranks of 64, odd row count
        _adapters("adapters_mixed_611", 611, 130, 64, 64, 4096, 4096, bare=9),
        # training four adapters on 2048 rows: input gradient and both adapter gradients
        _train("adapters_grad_2048", 2048, 4, 32, 4096, 4096),
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
    kind = rng.choices(["decode", "prefill", "f32", "wgrad", "adapters_decode", "adapters", "adapters_grad"],
                       [3, 4, 1, 3, 3, 3, 2])[0]
    half = rng.choice(["bf16", "bf16", "bf16", "f16"])
    spread = rng.randrange(1, 1 << 20)
    N, K = _width(rng, 512, 11008), _width(rng, 512, 8192)
    if kind.startswith("adapters"):
        R = rng.choice([8, 16, 16, 32, 64, rng.randrange(4, 64)])
        bank = _logint(rng, 2, 64)
        if kind == "adapters_grad":
            bank = min(bank, 16)
            return _train("", _logint(rng, 64, 4096), bank, R, N, K, half, rng.choice([0, 0, bank // 4]), spread)
        if kind == "adapters_decode":
            M = _logint(rng, 1, 128)
            return _adapters("", M, M, bank, R, N, K, half, rng.choice([0, 0, M // 8]), spread)
        M = _logint(rng, 64, 4096)
        groups = _logint(rng, 1, max(1, M // 8))
        return _adapters("", M, groups, bank, R, N, K, half, rng.choice([0, 0, groups // 8]), spread)
    groups = _logint(rng, 2, 64)
    while groups * N * K > EXPERT_WEIGHTS:
        N, K = (N + 1) // 2, (K + 1) // 2
    empty = rng.choice([0, 0, groups // 8])
    if kind == "f32":
        return _experts("", _logint(rng, 16, 2048), groups, min(N, 2048), min(K, 2048), "f32", rng.choice([0, 1]),
                        False, empty, spread)
    if kind == "wgrad":
        c32 = rng.random() < 0.5
        return _wgrad("", _logint(rng, 64, 8192), groups, min(N, 4096), min(K, 4096), half, c32,
                      1.0 if c32 and rng.random() < 0.5 else 0.0, empty, spread)
    M = _logint(rng, 1, 256) if kind == "decode" else _logint(rng, 256, 8192)
    return _experts("", M, groups, N, K, half, rng.choice([1, 1, 0]), rng.random() < 0.4, empty, spread)


# ------------------------------------------------------------------ who has how many rows

def _sizes(case):
    """Rows of every group, from the case alone: uneven, `empty` groups without a row."""
    M, groups = case["M"], case["groups"]
    if groups == M and not case["empty"]:
        return [1] * M
    rng = random.Random(case["spread"])
    used = max(1, min(groups - case["empty"], M))
    share = [rng.expovariate(1.0) + 0.1 for _ in range(used)]
    sizes = [1 + int((M - used) * x / sum(share)) for x in share]
    for i in range(M - sum(sizes)):
        sizes[i % used] += 1
    sizes += [0] * (groups - used)
    rng.shuffle(sizes)
    return sizes


def _bare_and_ids(case):
    """Adapter of every segment, -1 for none, from the case alone."""
    rng = random.Random(case["spread"] + 1)
    ids = [rng.randrange(case["bank"]) for _ in range(case["groups"])]
    for s in rng.sample(range(case["groups"]), min(case["bare"], case["groups"])):
        ids[s] = -1
    return ids


def work(case):
    M, N, K, G = case["M"], case["N"], case["K"], case["groups"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "experts":
        used = sum(1 for m in _sizes(case) if m)
        moved = e * (M * K + used * K * N + M * N) + (4 * used * N if case["act"] else 0)
        return {"bytes": float(moved), "flops": 2.0 * M * N * K}
    if case["kind"] == "wgrad":
        c = (4 if case["c32"] else e) * (2 if case["beta"] else 1)
        return {"bytes": float(e * M * (N + K) + c * G * N * K), "flops": 2.0 * M * N * K}
    R = case["R"]
    if case["kind"] == "adapters":
        used = len({i for i in _bare_and_ids(case) if i >= 0})
        moved = e * (M * K + K * N + M * N + used * R * (K + N) + M * R)
        return {"bytes": float(moved), "flops": 2.0 * M * N * K + 2.0 * M * R * (K + N)}
    # dY, X, H and the weights read; dX, G and the adapters' gradients written; the adapters read
    moved = e * (M * (2 * K + N + 2 * R) + K * N + 2 * G * R * (K + N))
    return {"bytes": float(moved), "flops": 2.0 * M * N * K + 4.0 * M * R * (K + N)}


# ------------------------------------------------------------------ inputs

def _normal(gen, dtype, sigma, *shape):
    return (torch.randn(shape, device="cuda", generator=gen) * sigma).to(DTYPES[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = random.Random(int(seed))
    M, N, K, G, dt = case["M"], case["N"], case["K"], case["groups"], case["dtype"]
    sizes = _sizes(case)
    rng.shuffle(sizes)
    starts = [0]
    for m in sizes:
        starts.append(starts[-1] + m)
    s = {"case": case, "sizes": sizes, "starts": starts, "longest": max(sizes),
         "offsets": torch.tensor(starts, dtype=torch.int64, device="cuda"),
         "ws": torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")}
    # the plan of a padded batched product: group of every row, and its place in it
    s["group"] = torch.repeat_interleave(torch.arange(G, device="cuda"), torch.tensor(sizes, device="cuda"))
    s["place"] = torch.arange(M, device="cuda") - s["offsets"][s["group"]]
    if case["kind"] == "experts":
        s["X"] = _normal(gen, dt, 1.0, M, K)
        s["W"] = _normal(gen, dt, 0.02, G, N, K) if case["tB"] else _normal(gen, dt, 0.02, G, K, N)
        s["bias"] = torch.randn((G, N), device="cuda", generator=gen) if case["act"] else None
        s["Y"] = torch.empty((M, N), dtype=DTYPES[dt], device="cuda")
        return s
    if case["kind"] == "wgrad":
        s["dY"], s["X"] = _normal(gen, dt, 1.0, M, N), _normal(gen, dt, 1.0, M, K)
        s["dW"] = torch.randn((G, N, K), device="cuda", generator=gen).to(torch.float32 if case["c32"] else DTYPES[dt])
        return s
    R, bank = case["R"], case["bank"]
    s["W"] = _normal(gen, dt, 0.02, N, K)
    s["down"] = _normal(gen, dt, K ** -0.5, bank, R, K)
    s["up"] = _normal(gen, dt, 0.02, bank, N, R)
    s["scale"] = torch.rand(bank, device="cuda", generator=gen) + 0.5
    s["X"] = _normal(gen, dt, 1.0, M, K)
    if case["kind"] == "adapters":
        order = list(range(bank))
        rng.shuffle(order)
        s["ids_list"] = [order[i] if i >= 0 else -1 for i in _bare_and_ids(case)]
        s["ids"] = torch.tensor(s["ids_list"], dtype=torch.int64, device="cuda")
        s["Y"] = torch.empty((M, N), dtype=DTYPES[dt], device="cuda")
        s["H"] = torch.empty((M, R), dtype=DTYPES[dt], device="cuda")
        return s
    s["dY"] = _normal(gen, dt, 1.0, M, N)
    s["H"] = _normal(gen, dt, 1.0, M, R)                    # kept from the forward pass
    s["dX"] = torch.empty((M, K), dtype=DTYPES[dt], device="cuda")
    s["G"] = torch.empty((M, R), dtype=DTYPES[dt], device="cuda")
    s["d_down"], s["d_up"] = torch.empty_like(s["down"]), torch.empty_like(s["up"])
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2511_13764_amd import binding as B
    c = s["case"]
    M, N, K, G = c["M"], c["N"], c["K"], c["groups"]
    dt = {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16}[c["dtype"]]
    c32 = c["dtype"] == "f32"
    if c["kind"] == "experts":
        epilogue = B.EPI_BIAS | B.EPI_RELU if c["act"] else B.EPI_NONE
        B.gemm_grouped(dt, c["tB"], M, N, K, G, s["offsets"], s["X"], K, s["W"], K if c["tB"] else N, N * K, 0.0,
                       s["Y"], N, c32, s["bias"], N, epilogue, workspace=s["ws"])
        return s["Y"]
    if c["kind"] == "wgrad":
        B.gemm_grouped_wgrad(dt, M, N, K, G, s["offsets"], s["dY"], N, s["X"], K, c["beta"], s["dW"], K, N * K,
                             c32 or c["c32"], workspace=s["ws"])
        return s["dW"]
    R, bank = c["R"], c["bank"]
    if c["kind"] == "adapters":
        B.gemm_adapters(dt, 1, M, N, K, R, G, None if G == M else s["offsets"], s["ids"], bank, s["X"], K, s["W"], K,
                        s["down"], K, R * K, s["up"], R, N * R, s["scale"], 0.0, s["Y"], N, c32, None, B.EPI_NONE,
                        s["H"], R, workspace=s["ws"])
        return {"Y": s["Y"], "H": s["H"]}
    B.gemm_adapters(dt, 0, M, K, N, R, G, s["offsets"], None, bank, s["dY"], N, s["W"], K,
                    s["up"], R, N * R, s["down"], K, R * K, s["scale"], 0.0, s["dX"], K, c32, None, B.EPI_NONE,
                    s["G"], R, workspace=s["ws"])
    B.gemm_grouped_wgrad(dt, M, R, K, G, s["offsets"], s["G"], R, s["X"], K, 0.0, s["d_down"], K, R * K, c32,
                         workspace=s["ws"])
    B.gemm_grouped_wgrad(dt, M, N, R, G, s["offsets"], s["dY"], N, s["H"], R, 0.0, s["d_up"], R, N * R, c32,
                         workspace=s["ws"])
    return {"dX": s["dX"], "G": s["G"], "d_down": s["d_down"], "d_up": s["d_up"]}


def _padded(s, rows):
    """Groups x longest x width in 32 bits, zeros past the end of a group."""
    out = torch.zeros((s["case"]["groups"], s["longest"], rows.shape[1]), device=rows.device)
    out[s["group"], s["place"]] = rows.float()
    return out


def _low_rank(s, rows, first, second, ids):
    """scale * (rows @ first) and that @ second, by each row's adapter; none where ids < 0."""
    at = ids.clamp_min(0)
    scale = torch.where(ids >= 0, s["scale"][at], torch.zeros_like(s["scale"][at]))
    h = torch.bmm(_padded(s, rows), first[at].float()) * scale[:, None, None]
    return h[s["group"], s["place"]], torch.bmm(h, second[at].float())[s["group"], s["place"]]


def _run_plain(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "experts":
        W = s["W"].float()
        y = torch.bmm(_padded(s, s["X"]), W.transpose(1, 2) if c["tB"] else W)[s["group"], s["place"]]
        if c["act"]:
            y = (y + s["bias"][s["group"]]).clamp_min(0.0)
        return y.to(dt)
    if c["kind"] == "wgrad":
        d = torch.bmm(_padded(s, s["dY"]).transpose(1, 2), _padded(s, s["X"]))
        if c["beta"]:
            s["dW"].copy_(c["beta"] * s["dW"].float() + d)
            return s["dW"]
        return d.to(s["dW"].dtype)
    if c["kind"] == "adapters":
        h, delta = _low_rank(s, s["X"], s["down"].transpose(1, 2), s["up"].transpose(1, 2), s["ids"])
        return {"Y": (s["X"].float() @ s["W"].float().t() + delta).to(dt), "H": h.to(dt)}
    ids = torch.arange(c["groups"], device=s["X"].device)
    g, delta = _low_rank(s, s["dY"], s["up"], s["down"], ids)
    return {"dX": (s["dY"].float() @ s["W"].float() + delta).to(dt), "G": g.to(dt),
            "d_down": torch.bmm(_padded(s, g).transpose(1, 2), _padded(s, s["X"])).to(dt),
            "d_up": torch.bmm(_padded(s, s["dY"]).transpose(1, 2), _padded(s, s["H"])).to(dt)}


# ------------------------------------------------------------------ the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    M, N, K, G = case["M"], case["N"], case["K"], case["groups"]

    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.float64, device="cuda")

    if case["kind"] == "experts":
        y = zeros(M, N)
        for e in range(G):
            a, b = s["starts"][e], s["starts"][e + 1]
            if a == b:
                continue
            w = s["W"][e].double()
            y[a:b] = s["X"][a:b].double() @ (w.t().contiguous() if case["tB"] else w)
            if case["act"]:
                y[a:b] = (y[a:b] + s["bias"][e].double()).clamp_min(0.0)
        return y
    if case["kind"] == "wgrad":
        d = case["beta"] * s["dW"].double() if case["beta"] else zeros(G, N, K)
        for e in range(G):
            a, b = s["starts"][e], s["starts"][e + 1]
            d[e] += s["dY"][a:b].double().t().contiguous() @ s["X"][a:b].double()
        return d
    R = case["R"]
    w = s["W"].double()
    if case["kind"] == "adapters":
        y, h = s["X"].double() @ w.t().contiguous(), zeros(M, R)
        for e in range(G):
            a, b, i = s["starts"][e], s["starts"][e + 1], s["ids_list"][e]
            if i < 0:
                continue
            h[a:b] = s["scale"][i].double() * (s["X"][a:b].double() @ s["down"][i].double().t().contiguous())
            y[a:b] += h[a:b] @ s["up"][i].double().t().contiguous()
        return {"Y": y, "H": h}
    dx, g, d_down, d_up = s["dY"].double() @ w, zeros(M, R), zeros(G, R, K), zeros(G, N, R)
    for i in range(G):
        a, b = s["starts"][i], s["starts"][i + 1]
        dy, x = s["dY"][a:b].double(), s["X"][a:b].double()
        g[a:b] = s["scale"][i].double() * (dy @ s["up"][i].double())
        dx[a:b] += g[a:b] @ s["down"][i].double()
        d_down[i] = g[a:b].t().contiguous() @ x
        d_up[i] = dy.t().contiguous() @ s["H"][a:b].double()
    return {"dX": dx, "G": g, "d_down": d_down, "d_up": d_up}
