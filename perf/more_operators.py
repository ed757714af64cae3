"""The timed cases of what stands around the experts' products: the norm in front of a layer, the activation between its two
products, and a whole layer for a few tokens.

A case is a dict of plain values.  `op` says what one pass does:

  norm        hm_rms_norm: s = x + residual, y = s / sqrt(mean(s^2) + eps) * weight, as values and in 8 bits
  norm_back   hm_rms_norm_backward: gradients of s and of the weight
  gated       hm_gated: a = silu(gate) * up of rows [gate | up], as values or in 8 bits
  gated_back  hm_gated_backward: gradient of [gate | up] from that of a, and a again, in the layouts that the products of the
              way back read: rows of 8 bits for the rows' gradient, columns of 8 bits for the weights'
  few         hm_layer_few: logits and rows of a few tokens -> the layer's output: choice, both products, activation, sum

`own` false computes the same with elementary torch operations in 32 bits; true makes the library's calls.  Inputs are drawn on
the GPU from the seed: rows that differ in size, as tokens do, N(0,1) logits, gradients of a few hundredths, weights of
1/sqrt(columns), norm weights near 1, balancing biases in steps of a thousandth, expert loads even or by Zipf's law.  Outputs and
workspaces are allocated once and kept, as a training loop or a server keeps them.

Values in 8 bits are e4m3 with a power of two for each block of 128, of a row, of a segment's column or of weights; both are
returned as the values they stand for.  A row of C values takes 128 ceil(C / 128) bytes, zeros behind the values, and
4 ceil(C / 512) scales, codes of 0 behind the blocks'.  The columns of segment e begin at byte 128 (offsets[e] // 128 + e) of their
row and end with zeros up to a whole block; one line of scales [C] per block.
"""
import math
import random

import torch

own = False

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _up(n, m):
    return (n + m - 1) // m * m


def _norm(name, T, H, dtype="bf16", residual="bf16", weight="f32", y="bf16", q=True):
    c = {"op": "norm", "T": T, "H": H, "dtype": dtype, "residual": residual, "weight": weight, "y": y, "q": q}
    return dict(c, name=name) if name else c


def _norm_back(name, T, H, dtype="bf16", gy="bf16", weight="f32", residual=True):
    c = {"op": "norm_back", "T": T, "H": H, "dtype": dtype, "gy": gy, "weight": weight, "residual": residual}
    return dict(c, name=name) if name else c


def _gated(name, rows, F, dtype="bf16", a="none", q=True):
    c = {"op": "gated", "rows": rows, "F": F, "dtype": dtype, "a": a, "q": q}
    return dict(c, name=name) if name else c


def _gated_back(name, rows, F, experts, load="even", dtype="bf16", gh="none", eight=True):
    c = {"op": "gated_back", "rows": rows, "F": F, "experts": experts, "load": load, "dtype": dtype, "gh": gh, "eight": eight}
    return dict(c, name=name) if name else c


def _few(name, T, E, K, H, F, score="softmax", groups=1, top_groups=1, group_best=1, bias=False, renormalise=True, scale=1.0, first=0,
         here=0, padded=0, out="bf16"):
    c = {"op": "few", "T": T, "E": E, "K": K, "H": H, "F": F, "score": score, "groups": groups, "top_groups": top_groups,
         "group_best": group_best, "bias": bias, "renormalise": renormalise, "scale": scale, "first": first, "here": here or E,
         "padded": padded, "out": out}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a served token before a layer: one row added, normed, written for the router and in 8 bits for the experts; latency
        _norm("norm 1 token", 1, 7168),
        # the same of a training layer's tokens
        _norm("norm 8192", 8192, 7168),
        # its way back, with the gradient that came past the layer
        _norm_back("norm back 8192", 8192, 7168),
        # the way back through a small fp32 norm of odd sizes without a residual
        _norm_back("norm back ragged f32", 1237, 1030, "f32", "f32", "f32", False),
        # the activation of a few served rows
        _gated("gated 64 rows", 64, 2048),
        # what a rank of a DeepSeek-V3-shaped layer has between its products
        _gated("gated 65536", 65536, 2048),
        # the way back through the activation of a Qwen3-shaped layer, all the 8-bit operands of the four products behind it
        _gated_back("gated back 32768", 32768, 768, 16),
        # the same of a small layer of skewed loads and odd sizes, fp32, with the gradient as values too
        _gated_back("gated back ragged f32", 5003, 1001, 16, "zipf", "f32", "f32"),
        # a served token through a Qwen3-shaped layer, all 128 experts here
        _few("few 1 token", 1, 128, 8, 2048, 768),
        # a served token whose eight experts of a DeepSeek-V3-shaped layer are all here
        _few("few 1 token dsv3", 1, 32, 8, 7168, 2048, "sigmoid", bias=True, scale=2.5),
        # a decoding batch at one of eight ranks of that layer: 32 of its 256 experts, about two tokens each
        _few("few 64 tokens dsv3", 64, 256, 8, 7168, 2048, "sigmoid", 8, 4, 2, bias=True, scale=2.5, first=64, here=32),
        # a small layer of odd sizes, a batch padded with tokens that have no expert, fp32 out
        _few("few ragged f32", 19, 60, 6, 1030, 1001, "softmax", renormalise=False, padded=2, out="f32"),
    ]


def _log(rng, low, high):
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return min(max(n, low), high)


def _size(rng, low, high):
    """A size of the range: a multiple of 256 or 8, or any."""
    n = _log(rng, low, high)
    return min(rng.choice((_up(n, 256), _up(n, 8), n)), high)


def draw(rng):
    op = rng.choice(("norm", "norm", "norm_back", "norm_back", "gated", "gated_back", "gated_back", "few", "few", "few"))
    kind = lambda: rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        H = _size(rng, 64, 8192)
        dtype = kind()
        y = rng.choice(("bf16", dtype, "none"))
        return _norm(None, _log(rng, 1, min(65536, 40000000 // H)), H, dtype, rng.choice(("none", dtype, "f32")), rng.choice(("bf16", "f32")), y,
                     y == "none" or rng.random() < 0.5)
    if op == "norm_back":
        H = _size(rng, 64, 8192)
        dtype = kind()
        return _norm_back(None, _log(rng, 1, min(65536, 30000000 // H)), H, dtype, rng.choice(("bf16", dtype)), rng.choice(("bf16", "f32")),
                          rng.random() < 0.6)
    if op == "gated":
        F = _size(rng, 64, 4096)
        dtype = kind()
        a = rng.choice(("none", "bf16", dtype))
        return _gated(None, _log(rng, 1, min(65536, 60000000 // F)), F, dtype, a, a == "none" or rng.random() < 0.5)
    if op == "gated_back":
        F = _size(rng, 64, 4096)
        gh = rng.choice(("none", "none", "bf16", "f32"))
        return _gated_back(None, _log(rng, 1, min(32768, 25000000 // F)), F, rng.randint(1, 32), rng.choice(("even", "zipf")), kind(), gh,
                           gh == "none" or rng.random() < 0.5)
    here, H, F = _log(rng, 4, 64), _size(rng, 64, 4096), _size(rng, 64, 2048)
    while here * H * F > 120000000:
        here = (here + 1) // 2
    E = here * rng.choice((1, 1, 2, 4))
    T, score = _log(rng, 1, 64), rng.choice(("softmax", "sigmoid"))
    groups = rng.choice([g for g in (1, 1, 2, 4) if E % g == 0 and E // g >= 2])
    top_groups = rng.randint(1, groups)
    return _few(None, T, E, rng.randint(1, min(8, E // groups * top_groups)), H, F, score, groups, top_groups,
                rng.choice((1, 2)) if groups > 1 else 1, score == "sigmoid" and rng.random() < 0.6, rng.random() < 0.7, rng.choice((1.0, 2.5)),
                rng.randrange(E // here) * here, here, rng.choice((0, 0, 0, T // 4)), rng.choice(("bf16", "bf16", "f32")))


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, sigma=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").mul_(sigma).to(dtype)


def _tokens(g, rows, cols, dtype):
    """Rows that differ in size."""
    return (_normal(g, rows, cols) * torch.exp(_normal(g, rows, 1))).to(dtype)


def _loads(case, seed):
    """Rows per expert: every row picks one, each as likely as the next or by Zipf's law over a random order of the experts."""
    rng, E = random.Random(seed), case["experts"]
    share = [1.0 / (i + 1) if case["load"] == "zipf" else 1.0 for i in range(E)]
    rng.shuffle(share)
    counts = [0] * E
    for e in rng.choices(range(E), weights=share, k=case["rows"]):
        counts[e] += 1
    return counts


def _offsets(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _rows8(rows, cols):
    return (torch.empty((rows, _up(cols, 128)), dtype=F8, device="cuda"),
            torch.empty((rows, _up(cols, 512) // 128), dtype=torch.uint8, device="cuda").view(E8))


def _columns8(blocks, cols):
    """Blocks that no segment has stay as they are."""
    return (torch.zeros((cols, 128 * blocks), dtype=torch.uint8, device="cuda").view(F8),
            torch.zeros((blocks, cols), dtype=torch.uint8, device="cuda").view(E8))


def _weights8(g, E, N, C):
    """Weights of 1/sqrt(C), an expert at a time."""
    each = [_blocks_of_weights(_normal(g, N, C, sigma=1.0 / math.sqrt(C))) for _ in range(E)]
    return torch.stack([q for q, _ in each]), torch.stack([e for _, e in each])


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    s = {"case": case}
    empty = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
    if op in ("norm", "norm_back"):
        T, H, dtype = case["T"], case["H"], DTYPES[case["dtype"]]
        s["weight"] = (1.0 + _normal(g, H, sigma=0.1)).to(DTYPES[case["weight"]])
        s["x"] = _tokens(g, T, H, dtype)
        if op == "norm":
            kind = case["residual"]
            s["residual"] = None if kind == "none" else _tokens(g, T, H, DTYPES[kind])
            s["total"] = None if kind == "none" else torch.empty_like(s["residual"])
            s["y"] = None if case["y"] == "none" else empty(T, H, dtype=DTYPES[case["y"]])
            s["rows8"] = _rows8(T, H) if case["q"] else (None, None)
        else:
            s["gy"] = _normal(g, T, H, sigma=0.03, dtype=DTYPES[case["gy"]])
            s["gtotal"] = _normal(g, T, H, sigma=0.03, dtype=dtype) if case["residual"] else None
            s["gx"], s["gweight"] = torch.empty_like(s["x"]), empty(H, dtype=torch.float32)
            if own:
                s["workspace"] = _binding().alloc_rms_norm_workspace(T, H)
    elif op in ("gated", "gated_back"):
        rows, F, dtype = case["rows"], case["F"], DTYPES[case["dtype"]]
        s["h"] = (_normal(g, rows, 2 * F) * torch.exp(_normal(g, rows, 1, sigma=0.3))).to(dtype)
        if op == "gated":
            s["a"] = None if case["a"] == "none" else empty(rows, F, dtype=DTYPES[case["a"]])
            s["rows8"] = _rows8(rows, F) if case["q"] else (None, None)
        else:
            s["ga"] = _normal(g, rows, F, sigma=0.03, dtype=dtype)
            s["offsets"] = torch.tensor(_offsets(_loads(case, seed)), dtype=torch.int32, device="cuda")
            s["gh"] = None if case["gh"] == "none" else empty(rows, 2 * F, dtype=DTYPES[case["gh"]])
            blocks = rows // 128 + case["experts"]
            s["rows8"] = s["columns8"] = s["a_columns8"] = (None, None)
            if case["eight"]:
                s["rows8"], s["columns8"], s["a_columns8"] = _rows8(rows, 2 * F), _columns8(blocks, 2 * F), _columns8(blocks, F)
    else:
        T, E, K, H, F, here = (case[k] for k in ("T", "E", "K", "H", "F", "here"))
        s["logits"] = _normal(g, T, E)
        if case["padded"]:
            s["logits"][T - case["padded"]:] = -math.inf
        s["bias"] = (torch.randint(-50, 51, (E,), generator=g, device="cuda").float() * 0.001) if case["bias"] else None
        s["x"] = _normal(g, T, H, dtype=torch.bfloat16)
        s["w13"], s["w2"] = _weights8(g, here, 2 * F, H), _weights8(g, here, H, F)
        s["ids"], s["weights"] = empty(T, K, dtype=torch.int32), empty(T, K, dtype=torch.float32)
        s["out"] = empty(T, H, dtype=DTYPES[case["out"]])
        if own:
            hm = _binding()
            s["router"] = hm.Router(E, K, case["score"], groups=case["groups"], top_groups=case["top_groups"], group_best=case["group_best"],
                                    renormalise=case["renormalise"], scale=case["scale"])
            s["workspace"] = hm.alloc_layer_few_workspace(T, s["router"], H, F)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _exponent(amax):
    """The least integer e with amax <= 448 * 2^e, at least -127."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, torch.where(m <= 0.875, e - 9, e - 8), -127).clamp_(min=-127)


def _power(code):
    """2^(code - 127), put together from its bits: pow() is not exact."""
    code = code.to(torch.int32)
    return torch.where(code > 0, code << 23, 1 << 22).view(torch.float32)


def _in_blocks(x, dim):
    """Values in 8 bits and the codes of their scales; a block is dimension `dim`."""
    code = _exponent(x.abs().amax(dim=dim, keepdim=True)) + 127
    return (x * _power(254 - code)).to(F8), code.to(torch.uint8)


def _padded(x, rows, cols):
    return torch.nn.functional.pad(x, (0, cols - x.shape[-1], 0, rows - x.shape[-2]))


def _blocks_of_rows(x):
    rows, cols = x.shape
    q, e = _in_blocks(_padded(x, rows, _up(cols, 128)).view(rows, -1, 128), 2)
    return q.view(rows, -1), _padded(e.view(rows, -1), rows, _up(cols, 512) // 128).view(E8)


def _blocks_of_columns(x, offsets):
    rows, cols = x.shape
    segments = offsets.numel() - 1
    blocks = rows // 128 + segments
    r = torch.arange(rows, device="cuda", dtype=torch.int32)
    e = torch.searchsorted(offsets[1:].contiguous(), r, right=True)
    spread = torch.zeros((128 * blocks, cols), dtype=torch.float32, device="cuda")
    spread[128 * (offsets[e] // 128 + e) + r - offsets[e]] = x
    q, code = _in_blocks(spread.view(blocks, 128, cols), 1)
    b = torch.arange(blocks, device="cuda", dtype=torch.int32)
    first = offsets[:-1] // 128 + torch.arange(segments, device="cuda", dtype=torch.int32)
    last = first + (offsets[1:] - offsets[:-1] + 127) // 128
    there = ((b[:, None] >= first) & (b[:, None] < last)).any(dim=1)
    return (q.view(128 * blocks, cols).view(torch.uint8).t().contiguous().view(F8),
            torch.where(there[:, None], code.view(blocks, cols), 0).to(torch.uint8).view(E8))


def _blocks_of_weights(w):
    """w [N, C] fp32: values [N, up(C, 128)] and codes [ceil(N / 128), up(C, 512) / 128]."""
    N, C = w.shape
    R, W = _up(N, 128), _up(C, 128)
    q, e = _in_blocks(_padded(w, R, W).view(R // 128, 128, W // 128, 128).transpose(1, 2).reshape(R // 128, W // 128, -1), 2)
    q = q.view(torch.uint8).view(R // 128, W // 128, 128, 128).transpose(1, 2).reshape(R, W)
    return q[:N].contiguous().view(F8), _padded(e.view(R // 128, W // 128), R // 128, _up(C, 512) // 128)


def _values_of_weights(q, e, C):
    """[experts, N, C] fp32."""
    return (q.float() * _power(e)[:, :, :q.shape[2] // 128].repeat_interleave(128, dim=1)[:, :q.shape[1]].repeat_interleave(128, dim=2))[:, :, :C]


def _plain_norm(s):
    case = s["case"]
    x = s["x"].float()
    out = {}
    if s["residual"] is not None:
        out["total"] = (x + s["residual"].float()).to(s["residual"].dtype)
        x = out["total"].float()
    y = x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS) * s["weight"].float()
    if case["y"] != "none":
        out["y"] = y.to(DTYPES[case["y"]])
    if case["q"]:
        out["q"], out["scale"] = _blocks_of_rows(y)
    return out


def _plain_norm_back(s):
    x, gy = s["x"].float(), s["gy"].float()
    r = 1.0 / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    u = gy * s["weight"].float()
    gx = r * (u - x * (r * r) * (u * x).mean(dim=1, keepdim=True))
    if s["gtotal"] is not None:
        gx = gx + s["gtotal"].float()
    return {"gx": gx.to(s["x"].dtype), "gweight": (gy * x * r).sum(dim=0)}


def _plain_gated(s):
    case, F = s["case"], s["case"]["F"]
    gate, up = s["h"][:, :F].float(), s["h"][:, F:].float()
    a = gate / (1.0 + torch.exp(-gate)) * up
    out = {}
    if case["a"] != "none":
        out["a"] = a.to(DTYPES[case["a"]])
    if case["q"]:
        out["q"], out["scale"] = _blocks_of_rows(a)
    return out


def _plain_gated_back(s):
    case, F = s["case"], s["case"]["F"]
    gate, up, ga = s["h"][:, :F].float(), s["h"][:, F:].float(), s["ga"].float()
    sig = 1.0 / (1.0 + torch.exp(-gate))
    gh = torch.cat([ga * up * sig * (1.0 + gate * (1.0 - sig)), ga * gate * sig], dim=1)
    out = {}
    if case["gh"] != "none":
        out["gh"] = gh.to(DTYPES[case["gh"]])
    if case["eight"]:
        out["q"], out["scale"] = _blocks_of_rows(gh)
        out["q_columns"], out["scale_columns"] = _blocks_of_columns(gh, s["offsets"])
        out["a_columns"], out["a_scale"] = _blocks_of_columns(gate * sig * up, s["offsets"])
    return out


def _first(choice, n):
    """The n largest entries of each row, descending, ties to the lowest place."""
    return torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :n]


def _plain_route(s):
    case, x = s["case"], s["logits"]
    T, E, K, groups = (case[k] for k in ("T", "E", "K", "groups"))
    best = x.max(dim=1, keepdim=True).values.clamp(min=-1e30)
    score = torch.exp(x - best) if case["score"] == "softmax" else 1.0 / (1.0 + torch.exp(-x))
    choice = x if s["bias"] is None else score + s["bias"]
    choice = torch.where(x > -math.inf, choice, -math.inf)
    if groups > 1:
        by = (score if s["bias"] is None else choice).view(T, groups, E // groups)
        top = torch.sort(by, dim=2, descending=True).values
        kept = _first(top[:, :, 0] if case["group_best"] == 1 else top[:, :, 0] + top[:, :, 1], case["top_groups"])
        keep = torch.zeros((T, groups), dtype=torch.bool, device=x.device)
        keep[torch.arange(T, device=x.device)[:, None], kept] = True
        choice = torch.where(keep[:, :, None], choice.view(T, groups, -1), -math.inf).view(T, E)
    ids = _first(choice, K)
    there = torch.gather(choice, 1, ids) > -math.inf
    w = torch.where(there, torch.gather(score, 1, ids), 0.0)
    if case["renormalise"]:
        w = w / w.sum(dim=1, keepdim=True).clamp(min=1e-30)
    elif case["score"] == "softmax":
        w = w / score.sum(dim=1, keepdim=True).clamp(min=1e-30)
    return torch.where(there, ids, -1).to(torch.int32), w * case["scale"]


def _plain_few(s):
    case = s["case"]
    H, F, here, first = (case[k] for k in ("H", "F", "here", "first"))
    ids, weights = _plain_route(s)
    # [experts here, T]: what an expert's output counts for a token
    mine = torch.arange(first, first + here, device="cuda", dtype=torch.int32)[:, None, None]
    share = torch.where(ids == mine, weights, 0.0).sum(dim=2)
    h = torch.matmul(_values_of_weights(*s["w13"], H), s["x"].float().t().contiguous())
    a = h[:, :F] / (1.0 + torch.exp(-h[:, :F])) * h[:, F:]
    y = torch.matmul(_values_of_weights(*s["w2"], F), a.contiguous())
    return {"ids": ids, "weights": weights, "out": (y * share[:, None, :]).sum(dim=0).t().to(DTYPES[case["out"]])}


# ---- the library's calls --------------------------------------------------------------------------------------------
_hm = None


def _binding():
    global _hm
    if _hm is None:
        from paper_2508_09591_amd import binding
        _hm = binding
    return _hm


def _written(**outputs):
    return {name: t for name, t in outputs.items() if t is not None}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"norm": _plain_norm, "norm_back": _plain_norm_back, "gated": _plain_gated, "gated_back": _plain_gated_back,
                "few": _plain_few}[op](s)
    hm = _binding()
    if op == "norm":
        q, scale = s["rows8"]
        hm.hm_rms_norm(s["x"], s["weight"], EPS, s["y"], q, scale, s["residual"], s["total"])
        return _written(total=s["total"], y=s["y"], q=q, scale=scale)
    if op == "norm_back":
        hm.hm_rms_norm_backward(s["gy"], s["x"], s["weight"], EPS, s["gx"], s["gweight"], s["gtotal"], s["workspace"])
        return {"gx": s["gx"], "gweight": s["gweight"]}
    if op == "gated":
        q, scale = s["rows8"]
        hm.hm_gated(s["h"], s["a"], q, scale)
        return _written(a=s["a"], q=q, scale=scale)
    if op == "gated_back":
        (q, scale), (q_columns, scale_columns), (a_columns, a_scale) = s["rows8"], s["columns8"], s["a_columns8"]
        hm.hm_gated_backward(s["h"], s["ga"], s["offsets"], s["gh"], q, scale, q_columns, scale_columns, a_columns, a_scale)
        return _written(gh=s["gh"], q=q, scale=scale, q_columns=q_columns, scale_columns=scale_columns, a_columns=a_columns, a_scale=a_scale)
    hm.hm_layer_few(s["x"], s["logits"], s["router"], *s["w13"], *s["w2"], s["ids"], s["weights"], s["out"], s["workspace"], s["bias"],
                    s["case"]["first"])
    return {"ids": s["ids"], "weights": s["weights"], "out": s["out"]}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    size = lambda d: {"bf16": 2, "f32": 4, "none": 0}[d]
    if op == "norm":
        n = case["T"] * case["H"]
        each = size(case["dtype"]) + 2 * size(case["residual"]) + size(case["y"])
        return {"bytes": n * each + (n + n // 128 if case["q"] else 0) + case["H"] * size(case["weight"]), "flops": 4 * n}
    if op == "norm_back":
        n = case["T"] * case["H"]
        return {"bytes": n * (size(case["gy"]) + size(case["dtype"]) * (3 if case["residual"] else 2)) + case["H"] * (4 + size(case["weight"])),
                "flops": 10 * n}
    if op == "gated":
        n = case["rows"] * case["F"]
        return {"bytes": n * (2 * size(case["dtype"]) + size(case["a"])) + (n + n // 128 if case["q"] else 0), "flops": 4 * n}
    if op == "gated_back":
        n = case["rows"] * case["F"]
        return {"bytes": n * (3 * size(case["dtype"]) + 2 * size(case["gh"])) + (5 * (n + n // 128) if case["eight"] else 0), "flops": 12 * n}
    T, E, K, H, F, here = (case[k] for k in ("T", "E", "K", "H", "F", "here"))
    slots = (T - case["padded"]) * K * here / E
    # experts hit: all different for one token, by chance for more
    hit = slots if T == 1 else here * (1 - (1 - K / E) ** (T - case["padded"]))
    return {"bytes": hit * 3 * H * F + T * (4 * E + 8 * K + H * (2 + size(case["out"]))), "flops": 6 * slots * H * F}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _two_to(n):
    """2^n in 64 bits, from a table of the host's."""
    return torch.tensor([2.0 ** k for k in range(-160, 161)], dtype=torch.float64, device="cuda")[n.long() + 160]


def _exact_code(amax):
    """The least code whose power of two times 448 is no less than amax, looked for among all of them."""
    return torch.searchsorted(448.0 * _two_to(torch.arange(-127, 128, device="cuda")), amax.contiguous())


def _exact_e4m3(v):
    """The nearest value of three mantissa bits and no exponent below -6, ties to even."""
    step = _two_to(torch.frexp(v.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return torch.round(v / step) * step


def _exact_rows(v):
    rows, cols = v.shape
    wide = torch.zeros((rows, _up(cols, 128)), dtype=torch.float64, device="cuda")
    wide[:, :cols] = v
    wide = wide.view(rows, -1, 128)
    code = _exact_code(wide.abs().amax(dim=2))
    codes = torch.zeros((rows, _up(cols, 512) // 128), dtype=torch.long, device="cuda")
    codes[:, :code.shape[1]] = code
    return _exact_e4m3(wide / _two_to(code - 127)[:, :, None]).view(rows, -1), _two_to(codes - 127)


def _exact_columns(v, at):
    rows, cols = v.shape
    blocks = rows // 128 + len(at) - 1
    q = torch.zeros((cols, 128 * blocks), dtype=torch.float64, device="cuda")
    p = torch.full((blocks, cols), 2.0 ** -127, dtype=torch.float64, device="cuda")
    for e in range(len(at) - 1):
        for i, r in enumerate(range(at[e], at[e + 1], 128)):
            part, b = v[r:min(r + 128, at[e + 1])], at[e] // 128 + e + i
            p[b] = _two_to(_exact_code(part.abs().amax(dim=0)) - 127)
            q[:, 128 * b:128 * b + part.shape[0]] = _exact_e4m3(part / p[b]).t()
    return q, p


def _exact_norm(s):
    case, out = s["case"], {}
    v = s["x"].double()
    if s["residual"] is not None:
        out["total"] = v + s["residual"].double()
        v = out["total"].to(s["residual"].dtype).double()   # the norm is that of the sum as it is kept
    length = torch.linalg.vector_norm(v, dim=1, keepdim=True)
    y = s["weight"].double() * v * torch.rsqrt(length * length / case["H"] + EPS)
    if case["y"] != "none":
        out["y"] = y
    if case["q"]:
        out["q"], out["scale"] = _exact_rows(y)
    return out


def _exact_norm_back(s):
    H = s["case"]["H"]
    v, gy, w = s["x"].double(), s["gy"].double(), s["weight"].double()
    m = v.square().sum(dim=1, keepdim=True) / H + EPS
    dot = (gy * w * v).sum(dim=1, keepdim=True)
    gx = gy * w * m ** -0.5 - v * dot * m ** -1.5 / H   # the derivative of v w m(v)^-1/2, term by term
    if s["gtotal"] is not None:
        gx = gx + s["gtotal"].double()
    return {"gx": gx, "gweight": (gy * v * m ** -0.5).sum(dim=0)}


def _exact_gated(s):
    case, F = s["case"], s["case"]["F"]
    gate, up = s["h"].double().split(F, dim=1)
    a, out = gate * torch.sigmoid(gate) * up, {}
    if case["a"] != "none":
        out["a"] = a
    if case["q"]:
        out["q"], out["scale"] = _exact_rows(a)
    return out


def _exact_gated_back(s):
    case, F, at = s["case"], s["case"]["F"], s["offsets"].tolist()
    gate, up = s["h"].double().split(F, dim=1)
    ga, p, not_p = s["ga"].double(), torch.sigmoid(gate), torch.sigmoid(-gate)
    gh, out = torch.cat([ga * up * (p + gate * p * not_p), ga * gate * p], dim=1), {}
    if case["gh"] != "none":
        out["gh"] = gh
    if case["eight"]:
        out["q"], out["scale"] = _exact_rows(gh)
        out["q_columns"], out["scale_columns"] = _exact_columns(gh, at)
        out["a_columns"], out["a_scale"] = _exact_columns(gate * p * up, at)
    return out


def _exact_choice(s):
    case, x = s["case"], s["logits"].double()
    T, E, K = (case[k] for k in "TEK")
    none = torch.isinf(x)
    lost = none.all(dim=1, keepdim=True)   # tokens without any expert
    s1 = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(torch.where(lost, 0.0, x), dim=1)
    c = s1 + s["bias"].double() if s["bias"] is not None else s1
    c = c.masked_fill(none, -1e30)
    if case["groups"] > 1:
        left = c.view(T, case["groups"], -1).clone()
        total = torch.zeros((T, case["groups"]), dtype=torch.float64, device="cuda")
        for _ in range(case["group_best"]):
            value, place = left.max(dim=2, keepdim=True)
            total += value[:, :, 0]
            left.scatter_(2, place, -1e30)
        group = torch.arange(case["groups"], device="cuda")
        first = group[None, :] < group[:, None]   # of two equal groups the first
        better = ((total[:, None, :] > total[:, :, None]) | ((total[:, None, :] == total[:, :, None]) & first)).sum(dim=2)
        c = c.view(T, case["groups"], -1).masked_fill((better >= case["top_groups"])[:, :, None], -1e30).view(T, E)
    place, ids = torch.arange(E, device="cuda"), []
    for _ in range(K):   # the largest, the first of equal ones
        top = c.max(dim=1, keepdim=True).values
        i = torch.where(c == top, place, E).min(dim=1).values
        ids.append(torch.where(top[:, 0] > -1e29, i, -1))
        c = c.scatter(1, i[:, None], -1e30)
    ids = torch.stack(ids, dim=1)
    w = torch.where(ids >= 0, s1.gather(1, ids.clamp(min=0)), 0.0)
    if case["renormalise"]:
        w = w / torch.where(lost, 1.0, w.sum(dim=1, keepdim=True))
    return ids, case["scale"] * w


def _exact_few(s):
    case = s["case"]
    T, H, F, first = (case[k] for k in ("T", "H", "F", "first"))
    ids, w = _exact_choice(s)
    out = torch.zeros((T, H), dtype=torch.float64, device="cuda")

    def weights(pair, e, C):
        q, code = pair[0][e], pair[1][e]
        n = torch.arange(q.shape[0], device="cuda") // 128
        k = torch.arange(C, device="cuda") // 128
        return q[:, :C].double() * _two_to(code.long() - 127)[n][:, k]

    for e in range(case["here"]):
        tokens, slots = (ids == first + e).nonzero(as_tuple=True)
        if tokens.numel():
            gate, up = (s["x"][tokens].double() @ weights(s["w13"], e, H).t().contiguous()).split(F, dim=1)
            y = (gate * torch.sigmoid(gate) * up) @ weights(s["w2"], e, F).t().contiguous()
            out[tokens] += w[tokens, slots][:, None] * y
    return {"ids": ids, "weights": w, "out": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_back": _exact_norm_back, "gated": _exact_gated, "gated_back": _exact_gated_back, "few": _exact_few}[case["op"]](s)
