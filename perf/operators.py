"""Speed and results of the microscaled 4-bit operators: quantisation, the product, and the experts of a mixture.

A block-scaled 4-bit matrix (MXFP4) holds, for each row and each 32 consecutive columns, 32 codes of one sign, two
exponent and one mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6) and a scale byte s that stands for 2^(s - 127).  Activations
are fp16 and are quantised block by block on their way into a product; products are summed in 32 bits.

Each case runs either in plain form (elementary torch operations in 32 bits) or through this framework's kernels.
"""
import math

import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32


def listed():
    return [
        # activations of a small draft tree: rows of a wider buffer, where only latency counts
        {"name": "quantise 13 rows", "kind": "quantise", "M": 13, "K": 2048, "pad": 64},
        # one matrix of a large model's feed-forward block, converted when the model is loaded
        {"name": "quantise a matrix", "kind": "quantise", "M": 28672, "K": 8192, "pad": 0},
        # one token through a small model's output projection
        {"name": "gemm 1 row", "kind": "gemm", "M": 1, "K": 2048, "N": 2048, "residual": False},
        # a draft tree through a large model's output projection, added to the residual stream
        {"name": "gemm tree", "kind": "gemm", "M": 32, "K": 8192, "N": 8192, "residual": True},
        # a prompt of no round length through a middle-sized model's feed-forward matrix
        {"name": "gemm prompt", "kind": "gemm", "M": 4001, "K": 4096, "N": 14336, "residual": False},
        # the largest draft tree routed to a model of many small experts
        {"name": "route tree", "kind": "route", "T": 64, "E": 64, "k": 8, "masked": 0.0},
        # a padded batch of prompts routed to the largest number of experts
        {"name": "route prompt", "kind": "route", "T": 16000, "E": 256, "k": 8, "masked": 0.1},
        # a single token through eight of many small experts
        {"name": "swiglu 1 token", "kind": "swiglu", "T": 1, "E": 64, "k": 8, "H": 2048, "F": 1024, "masked": 0.0},
        # a draft tree through a model of a few large experts
        {"name": "swiglu tree", "kind": "swiglu", "T": 32, "E": 8, "k": 2, "H": 4096, "F": 14336, "masked": 0.0},
        # a batch of prompts through many small experts of very unequal load
        {"name": "swiglu prompt", "kind": "swiglu", "T": 8191, "E": 64, "k": 8, "H": 2048, "F": 1024, "masked": 0.0},
        # a draft tree on its way back from a few large experts, added to the residual stream
        {"name": "down tree", "kind": "down", "T": 45, "E": 8, "k": 2, "H": 4096, "F": 14336, "masked": 0.0, "residual": True},
        # a padded batch of prompts on its way back from many experts of an odd width
        {"name": "down prompt", "kind": "down", "T": 5000, "E": 64, "k": 8, "H": 2048, "F": 1056, "masked": 0.1, "residual": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    kind = rng.choice(["quantise", "gemm", "gemm", "route", "swiglu", "swiglu", "down", "down"])
    if kind == "quantise":
        return {"kind": kind, "M": _log(rng, 1, 28672), "K": BLOCK * _log(rng, 1, 448), "pad": 8 * rng.randint(0, 9)}
    if kind == "gemm":
        return {"kind": kind, "M": _log(rng, 1, 4096), "K": BLOCK * _log(rng, 8, 448), "N": 16 * _log(rng, 8, 896),
                "residual": rng.random() < 0.5}
    E = _log(rng, 2, 256)
    k = rng.randint(1, min(8, E))
    T = _log(rng, 1, 8192)
    masked = rng.choice([0.0, 0.0, 0.2])
    if kind == "route":
        return {"kind": kind, "T": _log(rng, 1, 16384), "E": E, "k": k, "masked": masked}
    case = {"kind": kind, "T": T, "E": E, "k": k, "H": BLOCK * _log(rng, 16, 128), "F": BLOCK * _log(rng, 8, 448), "masked": masked}
    if kind == "down":
        case["residual"] = rng.random() < 0.5
    return case


def _fits(case):
    """Within the listed cases' work, their weights and their activations."""
    w = work(case)
    if max(w["bytes"], w["flops"] / 50) > 1.1e10:
        return False
    if case["kind"] in ("swiglu", "down"):
        return case["E"] * case["H"] * case["F"] <= 8 * 4096 * 14336 and case["T"] * case["k"] * max(case["H"], case["F"]) <= 65536 * 2048
    return case["kind"] != "quantise" or case["M"] * case["K"] <= 28672 * 8192


def draw(rng):
    while True:
        case = _draw(rng)
        if _fits(case):
            return case


def work(case):
    kind = case["kind"]
    bits = 0.5 + 1 / BLOCK  # bytes of an element in 4 bits
    if kind == "quantise":
        n = case["M"] * case["K"]
        return {"bytes": n * (2 + bits + 2), "flops": 0}
    if kind == "gemm":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": 2 * M * K + N * K * bits + 2 * M * N * (2 if case["residual"] else 1), "flops": 2 * M * N * K}
    T, E, k = case["T"], case["E"], case["k"]
    if kind == "route":
        return {"bytes": 2 * T * E + 16 * T * k + 4 * (E + 1), "flops": 0}
    H, F = case["H"], case["F"]
    rows = T * k * (1 - case["masked"])
    reached = E * (1 - (1 - k / E) ** T)
    if kind == "swiglu":
        return {"bytes": 2 * T * H + reached * 2 * F * H * bits + 2 * rows * F, "flops": 4 * rows * H * F}
    return {"bytes": 2 * rows * F + reached * F * H * bits + 2 * T * H * (2 if case["residual"] else 1), "flops": 2 * rows * H * F}


# ------------------------------------------------------------------ inputs


class _Inputs:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        out = torch.empty(shape, dtype=torch.float16, device="cuda")
        flat = out.view(-1)
        for i in range(0, flat.numel(), 1 << 26):
            n = min(1 << 26, flat.numel() - i)
            flat[i:i + n] = torch.randn(n, generator=self.g, device="cuda")
        return out

    def activations(self, M, K, pad=0):
        """N(0, 1) with one column in 64 twenty times as large, rows of a buffer `pad` columns wider."""
        x = self.normal(M, K + pad)
        big = torch.randperm(K, generator=self.g, device="cuda")[:max(1, K // 64)]
        x[:, big] *= 20
        return x[:, :K]

    def matrix(self, *shape):
        """Codes and scales of normal weights of deviation 0.017, as quantisation by block maxima leaves them."""
        K = shape[-1]
        v = torch.randn(1 << 17, generator=self.g, device="cuda") * 2.2
        mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
        code = torch.bucketize(v.abs(), mid) + 8 * (v < 0)
        pair = (code[0::2] + 16 * code[1::2]).to(torch.uint8)
        codes = torch.empty((*shape[:-1], K // 2), dtype=torch.uint8, device="cuda")
        flat = codes.view(-1)
        for i in range(0, flat.numel(), 1 << 27):
            n = min(1 << 27, flat.numel() - i)
            flat[i:i + n] = pair[torch.randint(1 << 16, (n,), generator=self.g, device="cuda")]
        scales = torch.randint(119, 122, (*shape[:-1], K // BLOCK), generator=self.g, device="cuda", dtype=torch.uint8)
        return codes, scales

    def logits(self, T, E, masked):
        """Router scores with unequal experts; `masked` of the tokens (padding) have no expert at all."""
        x = torch.randn(T, E, generator=self.g, device="cuda") + 0.7 * torch.randn(E, generator=self.g, device="cuda")
        if masked:
            x[torch.rand(T, generator=self.g, device="cuda") < masked] = -math.inf
        return x.to(torch.float16)


def _groups(experts, E):
    """offsets [E + 1], rows (sorted position -> token and slot) and pos (its inverse) of the experts [T, k], -1: none."""
    flat = experts.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    count = torch.bincount(key, minlength=E + 1)[:E]
    offsets = torch.cat([count.new_zeros(1), count.cumsum(0)]).to(torch.int32)
    place = torch.arange(flat.numel(), device=flat.device)
    used = place < offsets[-1]
    rows = torch.where(used, order, -1).to(torch.int32)
    pos = torch.empty_like(rows)
    pos[order] = torch.where(used, place, -1).to(torch.int32)
    return offsets, rows, pos


def prepare(case, seed):
    r = _Inputs(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "quantise":
        M, K = case["M"], case["K"]
        s["x"] = r.activations(M, K, case["pad"])
        s["codes"] = torch.empty(M, K // 2, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(M, K // BLOCK, dtype=torch.uint8, device="cuda")
        s["y"] = torch.empty(M, K, dtype=torch.float16, device="cuda")
    elif kind == "gemm":
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = r.activations(M, K)
        s["w"] = r.matrix(N, K)
        s["residual"] = r.normal(M, N) if case["residual"] else None
        s["y"] = torch.empty(M, N, dtype=torch.float16, device="cuda")
    elif kind == "route":
        s["logits"] = r.logits(case["T"], case["E"], case["masked"])
    else:
        T, E, k, H, F = (case[n] for n in ("T", "E", "k", "H", "F"))
        logits = r.logits(T, E, case["masked"]).float()
        experts = torch.topk(logits, k).indices
        s["experts"] = torch.where(torch.isinf(logits[:, :1]), -1, experts).to(torch.int32)
        s["offsets"], s["rows"], s["pos"] = _groups(s["experts"], E)
        s["most"] = int(s["offsets"].diff().max())
        if kind == "swiglu":
            s["x"] = r.activations(T, H)
            s["gate"], s["up"] = r.matrix(E, F, H), r.matrix(E, F, H)
            s["h"] = torch.zeros(T * k, F, dtype=torch.float16, device="cuda")
        else:
            s["x"] = r.activations(T * k, F)
            s["down"] = r.matrix(E, H, F)
            s["weights"] = torch.softmax(torch.randn(T, k, generator=r.g, device="cuda"), -1)
            s["residual"] = r.normal(T, H) if case["residual"] else None
            s["y"] = torch.empty(T, H, dtype=torch.float16, device="cuda")
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps beside its data: the weights in the kernels' layout, the routing's buffers, a workspace."""
    import paper_2506_11309_amd as ss
    case = s["case"]
    kind = case["kind"]
    for name in ("w", "gate", "up", "down"):
        if name in s:
            W = ss.make_mx4(*s[name])
            s[name + " handle"] = W, ss.prepack_mx4(W)
    if kind == "gemm":
        s["ws"] = ss.workspace(ss.mx4_gemm_workspace_bytes(case["M"], case["K"], case["N"]))
    elif kind == "route":
        T, E, k = case["T"], case["E"], case["k"]
        s["groups"] = ss.MoeGroups(T, k, E)
        s["experts"] = torch.empty(T, k, dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty(T, k, dtype=torch.float32, device="cuda")
        s["ws"] = ss.workspace(ss.moe_route_workspace_bytes(T, E, k))
    elif kind in ("swiglu", "down"):
        T, E, k, H, F = (case[n] for n in ("T", "E", "k", "H", "F"))
        s["groups"] = ss.MoeGroups(T, k, E, s["offsets"], s["rows"], s["pos"])
        size = ss.moe_mx4_swiglu_workspace_bytes(T, k, E, H, F) if kind == "swiglu" else ss.moe_mx4_down_workspace_bytes(T, k, E, F, H)
        s["ws"] = ss.workspace(size)


# ------------------------------------------------------------------ one pass


def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2506_11309_amd as ss
        if kind == "quantise":
            ss.mx4_quantize(s["x"], s["codes"], s["scales"])
            ss.mx4_dequantize(s["codes"], s["scales"], s["y"])
            return s["y"]
        if kind == "gemm":
            ss.mx4_gemm(s["w handle"][0], s["x"], s["y"], s["ws"], residual=s["residual"])
            return s["y"]
        if kind == "route":
            g = s["groups"]
            ss.moe_route(s["logits"], s["experts"], s["weights"], g, s["ws"])
            return {"experts": s["experts"], "weights": s["weights"], "offsets": g.offsets, "rows": g.rows, "pos": g.pos}
        if kind == "swiglu":
            ss.moe_mx4_swiglu(s["gate handle"][0], s["up handle"][0], s["x"], s["groups"], s["h"], s["ws"])
            return s["h"]
        ss.moe_mx4_down(s["down handle"][0], s["x"], s["groups"], s["weights"], s["y"], s["ws"], residual=s["residual"])
        return s["y"]
    if kind == "quantise":
        return _quantised(s["x"]).to(torch.float16)
    if kind == "gemm":
        y = _quantised(s["x"]) @ _values(*s["w"]).T
        return (y if s["residual"] is None else y + s["residual"].float()).to(torch.float16)
    if kind == "route":
        return _route(s["logits"], s["case"]["k"])
    place, valid, back = _placed(s)
    if kind == "swiglu":
        token = s["rows"].long()[place] // s["case"]["k"]
        x = _quantised(s["x"])[token].transpose(1, 2).contiguous()
        g, u = torch.bmm(_values(*s["gate"]), x), torch.bmm(_values(*s["up"]), x)
        h = (g / (1 + torch.exp(-g)) * u).transpose(1, 2)
        return _sorted(h, back)
    x = _quantised(s["x"])[place].transpose(1, 2).contiguous()
    rows = _sorted(torch.bmm(_values(*s["down"]), x).transpose(1, 2), back, torch.float32)
    pos = s["pos"].view_as(s["weights"]).long()
    part = torch.where((pos >= 0)[..., None], rows[pos.clamp(min=0)], 0) * s["weights"][..., None]
    y = part.sum(1)
    return (y if s["residual"] is None else y + s["residual"].float()).to(torch.float16)


def _quantised(x):
    """The values that x has in 4 bits, in 32 bits."""
    b = x.float().unflatten(-1, (-1, BLOCK))
    e = torch.frexp(b.abs().amax(-1, keepdim=True)).exponent - 3
    v = torch.ldexp(b, -e)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.clamp(torch.round(v / step) * step, -6, 6)
    return torch.ldexp(q, e).flatten(-2)


def _values(codes, scales):
    """A matrix in 4 bits as 32-bit values."""
    signed = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    byte = torch.arange(256, device=codes.device)
    pair = torch.stack([signed[byte % 16], signed[byte // 16]], -1)
    v = pair.index_select(0, codes.reshape(-1).int()).view(*scales.shape, BLOCK)
    return (v * torch.exp2(scales.float() - 127)[..., None]).flatten(-2)


def _route(logits, k):
    x = logits.float()
    there = x > -math.inf
    order = torch.sort(x, dim=-1, descending=True, stable=True)
    p = torch.where(there, torch.exp(x - x.amax(-1, keepdim=True)), 0)
    chosen = p.gather(1, order.indices[:, :k])
    total = chosen.sum(-1, keepdim=True)
    weights = torch.where(total > 0, chosen / total, 0)
    experts = torch.where(order.values[:, :k] > -math.inf, order.indices[:, :k], -1).to(torch.int32)
    offsets, rows, pos = _groups(experts, x.shape[1])
    return {"experts": experts, "weights": weights, "offsets": offsets, "rows": rows, "pos": pos}


def _placed(s):
    """For each expert the positions of its rows, padded to the largest group, which of them are there, and where each position stands."""
    offsets = s["offsets"].long()
    i = torch.arange(max(1, s["most"]), device=offsets.device)
    place = offsets[:-1, None] + i
    valid = place < offsets[1:, None]
    n = s["rows"].numel()
    p = torch.arange(n, device=offsets.device)
    e = torch.searchsorted(offsets[1:], p, right=True).clamp(max=offsets.numel() - 2)
    back = torch.where(p < offsets[-1], e * i.numel() + p - offsets[e], -1)
    return torch.where(valid, place, 0), valid, back


def _sorted(padded, back, dtype=torch.float16):
    """Rows of the padded groups in sorted order; zero behind the last."""
    flat = padded.reshape(-1, padded.shape[-1])
    return torch.where((back >= 0)[:, None], flat[back.clamp(min=0)], 0).to(dtype)


# ------------------------------------------------------------------ in 64 bits


def _nearest(x):
    """x quantised to 4 bits by blocks, from the definition: the block's exponent, then the nearest of eight values, ties to an even code."""
    b = x.double().reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    top = b.abs().max(-1, keepdim=True).values
    unit = torch.where(top > 0, 2.0 ** ((top.view(torch.int64) >> 52) - 1023 - 2).double(), 1.0)
    a = b.abs() / unit
    code = torch.zeros_like(a, dtype=torch.int64)
    for j in range(7):
        mid = (E2M1[j] + E2M1[j + 1]) / 2
        code += (a >= mid) if j % 2 else (a > mid)
    grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    return (grid[code] * unit * torch.sign(b)).reshape(x.shape)


def _matrix64(codes, scales):
    low, high = codes & 15, codes >> 4
    c = torch.stack([low, high], -1).reshape(*codes.shape[:-1], -1).long()
    grid = torch.tensor(E2M1, dtype=torch.float64, device=codes.device)
    v = grid[c & 7] * (1 - 2 * (c >> 3)).double()
    return v * (2.0 ** (scales.double() - 127)).repeat_interleave(BLOCK, -1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantise":
        return _nearest(s["x"])
    if kind == "gemm":
        y = _nearest(s["x"]) @ _matrix64(*s["w"]).T
        return y if s["residual"] is None else y + s["residual"].double()
    if kind == "route":
        x, k = s["logits"].double(), case["k"]
        e = torch.exp(x - x.max(-1, keepdim=True).values).nan_to_num(0.0)
        best = torch.sort(e, dim=-1, descending=True).values[:, :k]
        return {"experts": None, "weights": (best / best.sum(-1, keepdim=True)).nan_to_num(0.0), "offsets": None, "rows": None, "pos": None}
    T, E, k = case["T"], case["E"], case["k"]
    at = s["offsets"].tolist()
    if kind == "swiglu":
        out = torch.zeros(T * k, case["F"], dtype=torch.float64, device="cuda")
        x = _nearest(s["x"])
        for e in range(E):
            if at[e + 1] > at[e]:
                mine = x[(s["rows"][at[e]:at[e + 1]] // k).long()]
                g = mine @ _matrix64(s["gate"][0][e], s["gate"][1][e]).T
                out[at[e]:at[e + 1]] = g * torch.sigmoid(g) * (mine @ _matrix64(s["up"][0][e], s["up"][1][e]).T)
        return out
    out = torch.zeros(T, case["H"], dtype=torch.float64, device="cuda") if s["residual"] is None else s["residual"].double()
    flat = s["weights"].reshape(-1).double()
    for e in range(E):
        if at[e + 1] > at[e]:
            slot = s["rows"][at[e]:at[e + 1]].long()
            y = _nearest(s["x"][at[e]:at[e + 1]]) @ _matrix64(s["down"][0][e], s["down"][1][e]).T
            out.index_add_(0, slot // k, flat[slot, None] * y)
    return out
