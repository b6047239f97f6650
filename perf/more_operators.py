"""Speed and results of the 8-bit operators: quantisation, the product, the router with scores, and the experts of a mixture.

A block-scaled 8-bit matrix holds codes of one sign, four exponent and three mantissa bits (e4m3: no infinities, largest
value 448) and a 32-bit scale for each block of 128 rows and 128 columns.  Activations are fp16 and are quantised on their
way into a product, a row's 128 columns at a time, to the same codes with a power of two as scale.  The router turns its
scores into probabilities or gates in 64 bits, rounds them to 32, and compares them, with a bias added, in 32.

Each case runs either in plain form (elementary torch operations in 32 bits) or through this framework's kernels.
"""
import math

import torch

own = False

BLOCK = 128


def listed():
    return [
        # activations of a small draft tree: rows of a wider buffer, where only latency counts
        {"name": "quantise 13 rows", "kind": "quantise", "M": 13, "K": 2048, "pad": 64, "rows": 1},
        # one matrix of a large model's feed-forward block, converted when the model is loaded
        {"name": "quantise a matrix", "kind": "quantise", "M": 28672, "K": 8192, "pad": 0, "rows": 128},
        # one token through a small model's output projection
        {"name": "gemm 1 row", "kind": "gemm", "M": 1, "K": 2048, "N": 2048, "residual": False},
        # a draft tree through a large model's output projection, added to the residual stream
        {"name": "gemm tree", "kind": "gemm", "M": 32, "K": 8192, "N": 8192, "residual": True},
        # a prompt of no round length through a middle-sized model's feed-forward matrix
        {"name": "gemm prompt", "kind": "gemm", "M": 4001, "K": 4096, "N": 14336, "residual": False},
        # the largest draft tree routed by probabilities, the best groups by their best expert
        {"name": "route tree", "kind": "route", "T": 64, "E": 64, "k": 6, "score": "softmax", "bias": False, "groups": 8,
         "top_groups": 3, "best": 1, "renormalize": False, "scale": 16.0, "bits": 16, "masked": 0.0},
        # a padded batch of prompts routed by gates with a bias for balance, the best groups by their best two experts
        {"name": "route prompt", "kind": "route", "T": 16000, "E": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "best": 2, "renormalize": True, "scale": 2.5, "bits": 32, "masked": 0.1},
        # a single token through eight of many small experts
        {"name": "swiglu 1 token", "kind": "swiglu", "T": 1, "E": 64, "k": 8, "H": 2048, "F": 1024, "masked": 0.0},
        # a draft tree through a model of a few large experts
        {"name": "swiglu tree", "kind": "swiglu", "T": 32, "E": 8, "k": 2, "H": 4096, "F": 14336, "masked": 0.0},
        # a batch of prompts through many small experts of very unequal load
        {"name": "swiglu prompt", "kind": "swiglu", "T": 8191, "E": 64, "k": 8, "H": 2048, "F": 1024, "masked": 0.0},
        # a draft tree on its way back from a few large experts, added to the residual stream
        {"name": "down tree", "kind": "down", "T": 45, "E": 8, "k": 2, "H": 4096, "F": 14336, "masked": 0.0, "residual": True},
        # a padded batch of prompts on its way back from many experts of an odd width
        {"name": "down prompt", "kind": "down", "T": 5000, "E": 64, "k": 8, "H": 2048, "F": 1072, "masked": 0.1, "residual": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    kind = rng.choice(["quantise", "gemm", "gemm", "route", "route", "swiglu", "swiglu", "down", "down"])
    if kind == "quantise":
        return {"kind": kind, "M": _log(rng, 1, 28672), "K": 16 * _log(rng, 1, 896), "pad": 8 * rng.randint(0, 9),
                "rows": rng.choice([1, 128])}
    if kind == "gemm":
        return {"kind": kind, "M": _log(rng, 1, 4096), "K": 16 * _log(rng, 16, 896), "N": 16 * _log(rng, 8, 896),
                "residual": rng.random() < 0.5}
    masked = rng.choice([0.0, 0.0, 0.2])
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 8, 8, 16])
        E = groups * _log(rng, 2, 256 // groups)
        top_groups = rng.randint(1, groups)
        return {"kind": kind, "T": _log(rng, 1, 16384), "E": E, "k": rng.randint(1, min(8, E // groups * top_groups)),
                "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups,
                "best": rng.randint(1, 2), "renormalize": rng.random() < 0.5, "scale": rng.choice([1.0, 2.5, 16.0]),
                "bits": rng.choice([16, 32]), "masked": masked}
    E = _log(rng, 2, 256)
    case = {"kind": kind, "T": _log(rng, 1, 8192), "E": E, "k": rng.randint(1, min(8, E)), "H": 16 * _log(rng, 32, 256),
            "F": 16 * _log(rng, 16, 896), "masked": masked}
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


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    kind = case["kind"]
    if kind == "quantise":
        M, K = case["M"], case["K"]
        return {"bytes": 5 * M * K + 4 * -(-M // case["rows"]) * _blocks(K), "flops": 0}
    if kind == "gemm":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": 2 * M * K + N * K + 4 * _blocks(N) * _blocks(K) + 2 * M * N * (2 if case["residual"] else 1), "flops": 2 * M * N * K}
    T, E, k = case["T"], case["E"], case["k"]
    if kind == "route":
        return {"bytes": case["bits"] // 8 * T * E + (4 * E if case["bias"] else 0) + 16 * T * k + 4 * (E + 1), "flops": 0}
    H, F = case["H"], case["F"]
    rows = T * k * (1 - case["masked"])
    matrices = E * (1 - (1 - k / E) ** T) * (F * H + 4 * _blocks(F) * _blocks(H))  # of the experts that a token reaches
    if kind == "swiglu":
        return {"bytes": 2 * T * H + 2 * matrices + 2 * rows * F, "flops": 4 * rows * H * F}
    return {"bytes": 2 * rows * F + matrices + 2 * T * H * (2 if case["residual"] else 1), "flops": 2 * rows * H * F}


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
        """Codes and scales of normal weights of deviation 0.017: a block's largest, near 4.2 deviations, is at 448."""
        v = torch.randn(1 << 17, generator=self.g, device="cuda") * (448 / 4.2)
        code = _code(v.clamp(-448, 448))
        pair = code[0::2].int() + 256 * code[1::2].int()
        pair = torch.where(pair > 32767, pair - 65536, pair).to(torch.int16)
        codes = torch.empty(shape, dtype=torch.uint8, device="cuda")
        flat = codes.view(-1).view(torch.int16)
        for i in range(0, flat.numel(), 1 << 27):
            n = min(1 << 27, flat.numel() - i)
            flat[i:i + n] = pair[torch.randint(1 << 16, (n,), generator=self.g, device="cuda")]
        block = (*shape[:-2], _blocks(shape[-2]), _blocks(shape[-1]))
        largest = 0.017 * (4.2 + 0.3 * torch.randn(block, generator=self.g, device="cuda"))
        return codes, largest.clamp(min=0.03) / 448

    def logits(self, T, E, masked, dtype):
        """Router scores with unequal experts; `masked` of the tokens (padding) have no expert at all."""
        x = torch.randn(T, E, generator=self.g, device="cuda") + 0.7 * torch.randn(E, generator=self.g, device="cuda")
        if masked:
            x[torch.rand(T, generator=self.g, device="cuda") < masked] = -math.inf
        return x.to(dtype)


def _code(v):
    """e4m3 codes of values within +-448, ties to the even code."""
    a = v.abs()
    e = torch.clamp(torch.frexp(a).exponent - 1, min=-6)  # of the value, or of the subnormals
    n = torch.round(torch.ldexp(a, 3 - e)).int()          # in eighths of 2^e: 8 to 16, of subnormals 0 to 8
    c = torch.where(n < 8, n, 8 * (e + 6) + n)
    return (c + 128 * torch.signbit(v).int()).to(torch.uint8)


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
        s["codes"] = torch.empty(M, K, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(-(-M // case["rows"]), _blocks(K), device="cuda")
        s["y"] = torch.empty(M, K, dtype=torch.float16, device="cuda")
    elif kind == "gemm":
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = r.activations(M, K)
        s["w"] = r.matrix(N, K)
        s["residual"] = r.normal(M, N) if case["residual"] else None
        s["y"] = torch.empty(M, N, dtype=torch.float16, device="cuda")
    elif kind == "route":
        T, E = case["T"], case["E"]
        s["logits"] = r.logits(T, E, case["masked"], torch.float16 if case["bits"] == 16 else torch.float32)
        # what balances the load: of the spread that the experts' scores have
        spread = 0.1 if case["score"] == "sigmoid" else 0.5 / E
        s["bias"] = spread * torch.randn(E, generator=r.g, device="cuda") if case["bias"] else None
    else:
        T, E, k, H, F = (case[n] for n in ("T", "E", "k", "H", "F"))
        logits = r.logits(T, E, case["masked"], torch.float32)
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
            W = ss.make_fp8(*s[name])
            s[name + " handle"] = W, ss.prepack_fp8(W)
    if kind == "gemm":
        s["ws"] = ss.workspace(ss.fp8_gemm_workspace_bytes(case["M"], case["K"], case["N"]))
    elif kind == "route":
        T, E, k = case["T"], case["E"], case["k"]
        s["scoring"] = ss.MoeScoring(case["score"], bias=s["bias"], groups=case["groups"], top_groups=case["top_groups"],
                                     group_best=case["best"], renormalize=case["renormalize"], scale=case["scale"])
        s["groups"] = ss.MoeGroups(T, k, E)
        s["experts"] = torch.empty(T, k, dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty(T, k, dtype=torch.float32, device="cuda")
        s["ws"] = ss.workspace(ss.moe_route_workspace_bytes(T, E, k))
    elif kind in ("swiglu", "down"):
        T, E, k, H, F = (case[n] for n in ("T", "E", "k", "H", "F"))
        s["groups"] = ss.MoeGroups(T, k, E, s["offsets"], s["rows"], s["pos"])
        size = ss.moe_fp8_swiglu_workspace_bytes(T, k, E, H, F) if kind == "swiglu" else ss.moe_fp8_down_workspace_bytes(T, k, E, F, H)
        s["ws"] = ss.workspace(size)


# ------------------------------------------------------------------ one pass


def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2506_11309_amd as ss
        if kind == "quantise":
            ss.fp8_quantize(s["x"], s["codes"], s["scales"], rows=s["case"]["rows"])
            ss.fp8_dequantize(s["codes"], s["scales"], s["y"], rows=s["case"]["rows"])
            return {"y": s["y"], "scales": s["scales"]}
        if kind == "gemm":
            ss.fp8_gemm(s["w handle"][0], s["x"], s["y"], s["ws"], residual=s["residual"])
            return s["y"]
        if kind == "route":
            g = s["groups"]
            ss.moe_route_scored(s["logits"], s["scoring"], s["experts"], s["weights"], g, s["ws"])
            return {"experts": s["experts"], "weights": s["weights"], "offsets": g.offsets, "rows": g.rows, "pos": g.pos}
        if kind == "swiglu":
            ss.moe_fp8_swiglu(s["gate handle"][0], s["up handle"][0], s["x"], s["groups"], s["h"], s["ws"])
            return s["h"]
        ss.moe_fp8_down(s["down handle"][0], s["x"], s["groups"], s["weights"], s["y"], s["ws"], residual=s["residual"])
        return s["y"]
    if kind == "quantise":
        y, scales = _quantised(s["x"], s["case"]["rows"])
        return {"y": y.to(torch.float16), "scales": scales}
    if kind == "gemm":
        y = _quantised(s["x"])[0] @ _values(*s["w"]).T
        return (y if s["residual"] is None else y + s["residual"].float()).to(torch.float16)
    if kind == "route":
        return _route(s["logits"], s["bias"], s["case"])
    place, back = _placed(s)
    if kind == "swiglu":
        token = s["rows"].long()[place] // s["case"]["k"]
        x = _quantised(s["x"])[0][token].transpose(1, 2).contiguous()
        g, u = torch.bmm(_values(*s["gate"]), x), torch.bmm(_values(*s["up"]), x)
        h = (g / (1 + torch.exp(-g)) * u).transpose(1, 2)
        return _sorted(h, back, torch.float16)
    x = _quantised(s["x"])[0][place].transpose(1, 2).contiguous()
    rows = _sorted(torch.bmm(_values(*s["down"]), x).transpose(1, 2), back, torch.float32)
    pos = s["pos"].view_as(s["weights"]).long()
    part = torch.where((pos >= 0)[..., None], rows[pos.clamp(min=0)], 0) * s["weights"][..., None]
    y = part.sum(1)
    return (y if s["residual"] is None else y + s["residual"].float()).to(torch.float16)


def _quantised(x, rows=1):
    """The values that x has in 8 bits, in 32 bits, and the scales of its blocks of `rows` rows and 128 columns."""
    M, K = x.shape
    padded = torch.zeros(-(-M // rows) * rows, _blocks(K) * BLOCK, device=x.device)
    padded[:M, :K] = x
    b = padded.view(-1, rows, _blocks(K), BLOCK)
    a = b.abs().amax((1, 3), keepdim=True)
    f = torch.frexp(a)  # a / 448 = mantissa / 0.875 * 2^(exponent - 9)
    e = torch.where(a > 0, f.exponent - 9 + (f.mantissa > 0.875).int(), 0)
    v = torch.ldexp(b, -e)
    step = torch.clamp(torch.frexp(v).exponent - 1, min=-6) - 3
    q = torch.ldexp(torch.ldexp(torch.round(torch.ldexp(v, -step)), step), e)
    return q.reshape(padded.shape)[:M, :K], torch.ldexp(torch.ones_like(a), e).view(-1, _blocks(K))


def _decoded(device):
    """The values of the 256 codes."""
    byte = torch.arange(256, device=device)
    e, m = byte // 8 % 16, byte % 8
    v = torch.where(e > 0, torch.ldexp(1 + m / 8, e - 7), torch.ldexp(m / 8, torch.full_like(e, -6)))
    v[byte % 128 == 127] = math.nan
    return torch.where(byte >= 128, -v, v)


def _values(codes, scales):
    """A matrix in 8 bits as 32-bit values."""
    v = _decoded(codes.device).index_select(0, codes.reshape(-1).int()).view(codes.shape)
    rows = scales.repeat_interleave(BLOCK, -2)[..., :codes.shape[-2], :]
    v *= rows.repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]
    return v


def _route(logits, bias, case):
    x = logits.double()
    T, E = x.shape
    k, n = case["k"], case["groups"]
    there = x > -math.inf
    if case["score"] == "softmax":
        p = torch.where(there, torch.exp(x - x.amax(-1, keepdim=True)), 0)
        s = (p / p.sum(-1, keepdim=True)).float()
    else:
        s = (1 / (1 + torch.exp(-x))).float()
    c = torch.where(there, s if bias is None else s + bias, -math.inf)
    best = torch.sort(c.view(T, n, E // n), dim=-1, descending=True).values[..., :case["best"]]
    second = torch.where(best[..., -1] > -math.inf, best[..., -1], 0) if best.shape[-1] > 1 else 0
    order = torch.sort(best[..., 0] + second, dim=-1, descending=True, stable=True).indices
    chosen = torch.zeros(T, n, dtype=torch.bool, device=x.device).scatter_(1, order[:, :case["top_groups"]], True)
    c = torch.where(chosen[..., None], c.view(T, n, E // n), -math.inf).view(T, E)
    order = torch.sort(c, dim=-1, descending=True, stable=True)
    has = order.values[:, :k] > -math.inf
    w = torch.where(has, s.gather(1, order.indices[:, :k]), 0)
    if case["renormalize"]:
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, 0)
    experts = torch.where(has, order.indices[:, :k], -1).to(torch.int32)
    offsets, rows, pos = _groups(experts, E)
    return {"experts": experts, "weights": w * case["scale"], "offsets": offsets, "rows": rows, "pos": pos}


def _placed(s):
    """For each expert the positions of its rows, padded to the largest group, and where each position stands."""
    offsets = s["offsets"].long()
    i = torch.arange(max(1, s["most"]), device=offsets.device)
    place = offsets[:-1, None] + i
    valid = place < offsets[1:, None]
    p = torch.arange(s["rows"].numel(), device=offsets.device)
    e = torch.searchsorted(offsets[1:], p, right=True).clamp(max=offsets.numel() - 2)
    back = torch.where(p < offsets[-1], e * i.numel() + p - offsets[e], -1)
    return torch.where(valid, place, 0), back


def _sorted(padded, back, dtype):
    """Rows of the padded groups in sorted order; zero behind the last."""
    flat = padded.reshape(-1, padded.shape[-1])
    return torch.where((back >= 0)[:, None], flat[back.clamp(min=0)], 0).to(dtype)


# ------------------------------------------------------------------ in 64 bits


def _grid(device):
    """The 127 values of e4m3 from 0 to 448."""
    m = torch.arange(8, dtype=torch.float64, device=device)
    return torch.cat([m * 2.0 ** -9] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16)])[:127]


def _nearest(x, rows=1):
    """x quantised to 8 bits from the definition, and the scales: the least power of two that brings a block's largest to
    448 or less, then the nearest of the 127 magnitudes, ties to an even code."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    scales = torch.empty(-(-x.shape[0] // rows), _blocks(x.shape[1]), dtype=torch.float64, device=x.device)
    grid = _grid(x.device)
    mid = (grid[1:] + grid[:-1]) / 2
    step = rows * max(1, (1 << 25) // (rows * x.shape[1]))
    for i in range(0, x.shape[0], step):
        part = x[i:i + step].double()
        n = -(-part.shape[0] // rows)
        for k in range(0, x.shape[1], BLOCK):
            b = part[:, k:k + BLOCK]
            a = torch.zeros(n * rows, dtype=torch.float64, device=x.device)
            a[:b.shape[0]] = b.abs().amax(1)
            a = a.view(n, rows).amax(1)
            unit = torch.where(a > 0, 2.0 ** -40, 1.0).double()
            for _ in range(60):
                unit = torch.where(unit * 448 < a, unit * 2, unit)
            u = unit.repeat_interleave(rows)[:b.shape[0], None]
            v = b.abs() / u
            low, high = torch.bucketize(v, mid), torch.bucketize(v, mid, right=True)  # they differ at a tie
            code = torch.where(low % 2 == 0, low, high)
            out[i:i + step, k:k + BLOCK] = grid[code] * u * torch.sign(b)
            scales[i // rows:i // rows + n, k // BLOCK] = unit
    return out, scales


def _matrix64(codes, scales):
    grid = _grid(codes.device)
    c = codes.long()
    v = grid[(c & 127).clamp(max=126)] * (1 - 2 * (c >> 7)).double()
    s = scales.double().repeat_interleave(BLOCK, -2)[..., :codes.shape[-2], :]
    return v * s.repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]


def _weights64(s):
    """The router's weights, in slot order; the scores are 32-bit numbers by definition, what is made of them is not."""
    case, bias = s["case"], s["bias"]
    x = s["logits"].double()
    gate = torch.softmax(x, -1).nan_to_num(0.0) if case["score"] == "softmax" else torch.sigmoid(x)
    gate = gate.float()
    key = gate if bias is None else gate + bias
    key = key.double().masked_fill(x == -math.inf, -1e30)
    T, E = x.shape
    member = key.view(T, case["groups"], -1)
    value = member.amax(-1)
    if case["best"] == 2 and member.shape[-1] > 1:
        two = torch.topk(member, 2).values
        value = torch.where(two[..., 1] > -1e30, (two[..., 0].float() + two[..., 1].float()).double(), two[..., 0])
    # the number of groups, then of experts, that come before each: larger ones, and equal ones of lower index
    def rank(v):
        i = torch.arange(v.shape[-1], device=v.device)
        out = torch.empty(v.shape, dtype=torch.long, device=v.device)
        for t in range(0, v.shape[0], 512):
            a = v[t:t + 512]
            before = (a[:, None, :] > a[:, :, None]) | ((a[:, None, :] == a[:, :, None]) & (i[None, None, :] < i[None, :, None]))
            out[t:t + 512] = before.sum(-1)
        return out

    allowed = (rank(value) < case["top_groups"]).repeat_interleave(E // case["groups"], 1) & (key > -1e30)
    place = rank(torch.where(allowed, key, -1e30))
    taken = allowed & (place < case["k"])
    w = torch.zeros(T, case["k"], dtype=torch.float64, device=x.device)
    t, e = taken.nonzero(as_tuple=True)
    w[t, place[t, e]] = gate[t, e].double()
    if case["renormalize"]:
        w = (w / w.sum(-1, keepdim=True)).nan_to_num(0.0)
    return w * case["scale"]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantise":
        y, scales = _nearest(s["x"], case["rows"])
        return {"y": y, "scales": scales}
    if kind == "gemm":
        y = _nearest(s["x"])[0] @ _matrix64(*s["w"]).T
        return y if s["residual"] is None else y + s["residual"].double()
    if kind == "route":
        return {"experts": None, "weights": _weights64(s), "offsets": None, "rows": None, "pos": None}
    T, E, k = case["T"], case["E"], case["k"]
    at = s["offsets"].tolist()
    if kind == "swiglu":
        out = torch.zeros(T * k, case["F"], dtype=torch.float64, device="cuda")
        x = _nearest(s["x"])[0]
        for e in range(E):
            if at[e + 1] > at[e]:
                mine = x[(s["rows"][at[e]:at[e + 1]] // k).long()]
                g = mine @ _matrix64(s["gate"][0][e], s["gate"][1][e]).T
                out[at[e]:at[e + 1]] = g * torch.sigmoid(g) * (mine @ _matrix64(s["up"][0][e], s["up"][1][e]).T)
        return out
    out = torch.zeros(T, case["H"], dtype=torch.float64, device="cuda") if s["residual"] is None else s["residual"].double()
    flat = s["weights"].reshape(-1).double()
    x = _nearest(s["x"])[0]
    for e in range(E):
        if at[e + 1] > at[e]:
            slot = s["rows"][at[e]:at[e + 1]].long()
            y = x[at[e]:at[e + 1]] @ _matrix64(s["down"][0][e], s["down"][1][e]).T
            out.index_add_(0, slot // k, flat[slot, None] * y)
    return out
