"""The timed cases of the layer's own arithmetic: the router in front of the dispatch and the experts' products behind it.

A case is a dict of plain values.  `op` says what one pass does:

  route           hm_route: logits [T,E] -> expert ids and weights [T,K], as hm_plan takes them
  route_backward  hm_combine_weight_grad, hm_route_backward: the output's gradient and the rows that were merged -> gradient
                  of the router weights [T,K] -> gradient of the logits [T,E]
  quantize        values in 8 bits (e4m3) with a power of two for each block of 128: hm_quantize_rows (128 columns of a row),
                  hm_quantize_columns (128 rows of an expert's segment, stored transposed), hm_quantize_weights
                  (128 x 128, stored both ways)
  matmul          hm_expert_matmul: rows ordered by expert times their expert's weights
  matmul_dw       hm_expert_matmul_dw: the gradient of every expert's weights from the same rows

`own` false computes the same with elementary torch operations in 32 bits; true makes the library's calls.  Inputs are drawn on
the GPU from the seed: N(0,1) logits and activations, gradients of a few hundredths, weights of 1/sqrt(columns), balancing
biases in steps of a thousandth, expert loads even or by Zipf's law.  Plans and outputs are allocated once and kept,
as a training loop or a server keeps them.

Layouts.  A row of C values in 8 bits takes 128 ceil(C / 128) bytes, zeros behind the values.  Its scales are bytes, code - 127
being the exponent: [rows, 4 ceil(C / 512)] with zeros behind them.  The columns of segment e begin at byte
128 (offsets[e] // 128 + e) of their row and end with zeros up to a whole block; one line of scales [C] per block.
"""
import math
import random

import torch

own = False

F8 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
RANKS = 8   # destinations of the plan whose rows a route_backward case merges


def _up(n, m):
    return (n + m - 1) // m * m


def _route(name, T, E, K, score, groups=1, top_groups=1, group_best=1, bias=False, renormalise=True, scale=1.0, dtype="f32", masked=0):
    c = {"op": "route", "T": T, "E": E, "K": K, "score": score, "groups": groups, "top_groups": top_groups, "group_best": group_best,
         "bias": bias, "renormalise": renormalise, "scale": scale, "dtype": dtype, "masked": masked}
    return dict(c, name=name) if name else c


def _back(name, T, E, K, H, score, renormalise, scale=1.0, dtype="f32", rows="bf16"):
    c = {"op": "route_backward", "T": T, "E": E, "K": K, "H": H, "score": score, "renormalise": renormalise, "scale": scale,
         "dtype": dtype, "rows": rows}
    return dict(c, name=name) if name else c


def _quantize(name, what, rows, cols, experts=1, load="even", dtype="bf16"):
    c = {"op": "quantize", "what": what, "rows": rows, "cols": cols, "experts": experts, "load": load, "dtype": dtype}
    return dict(c, name=name) if name else c


def _matmul(name, op, rows, experts, N, H, load="even", dtype="bf16"):
    c = {"op": op, "rows": rows, "experts": experts, "N": N, "H": H, "load": load, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a served token: one row of logits, group-limited sigmoid scores with a balancing bias; nothing but latency
        _route("route 1 token", 1, 256, 8, "sigmoid", 8, 4, 2, bias=True, scale=2.5),
        # a training layer of 128 experts, bf16 logits, softmax over the chosen
        _route("route 8192 softmax", 8192, 128, 8, "softmax", dtype="bf16"),
        # the long-sequence layer: 64 Ki tokens, 256 experts in 8 groups, bias
        _route("route 65536 grouped", 65536, 256, 8, "sigmoid", 8, 4, 2, bias=True, scale=2.5),
        # the way back through a small layer of odd sizes whose softmax runs over all experts (a dense gradient), rows in fp32
        _back("route back ragged f32", 1237, 60, 6, 1030, "softmax", False, rows="f32"),
        # the way back through the DeepSeek-V3-shaped layer: 64 Ki rows of 7168
        _back("route back dsv3", 8192, 256, 8, 7168, "sigmoid", True, scale=2.5),
        # a layer's tokens before they are sent
        _quantize("quantize rows", "rows", 8192, 7168),
        # the gradient rows of one rank's experts for the weight products, segments of any length, an odd row length
        _quantize("quantize columns ragged", "columns", 6001, 2056, 16, "zipf", "bf16"),
        # an expert layer's master weights after an optimizer step, both layouts
        _quantize("quantize weights", "weights", 2048, 2048, 32, dtype="f32"),
        # one served token at eight local experts: as many products of one row
        _matmul("matmul 8 rows", "matmul", 8, 32, 4096, 7168),
        # what a rank of a DeepSeek-V3-shaped layer receives: 64 Ki rows for 32 experts, the largest product
        _matmul("matmul 65536 rows", "matmul", 65536, 32, 4096, 7168),
        # a smaller layer with skewed loads, odd row count and sizes that are no multiple of a block, fp32 out
        _matmul("matmul ragged zipf", "matmul", 5003, 16, 1000, 2056, "zipf", "f32"),
        # the weights' gradient of a Qwen3-shaped layer
        _matmul("matmul dw", "matmul_dw", 32768, 16, 1536, 2048, "even", "f32"),
    ]


def _log(rng, low, high):
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return min(max(n, low), high)


def _size(rng, low, high):
    """A size of the range: a multiple of 256 or 8, or any."""
    while True:
        n = _log(rng, low, high)
        n = rng.choice((_up(n, 256), _up(n, 8), n))
        if n != 3072:
            return n


def draw(rng):
    op = rng.choice(("route", "route", "route_backward", "route_backward", "quantize", "quantize", "matmul", "matmul", "matmul", "matmul_dw"))
    if op == "route":
        groups = rng.choice((1, 1, 1, 2, 4, 8))
        E = groups * _log(rng, max(4, 8 // groups), 512 // groups)
        top_groups = rng.randint(1, groups)
        score = rng.choice(("softmax", "sigmoid"))
        return _route(None, _log(rng, 1, 65536 if E <= 256 else 30000), E, rng.randint(1, min(10, E // groups * top_groups)), score, groups, top_groups,
                      rng.choice((1, 2)) if groups > 1 else 1, score == "sigmoid" and rng.random() < 0.6, rng.random() < 0.7,
                      rng.choice((1.0, 2.5)), rng.choice(("f32", "bf16")), rng.choice((0, 0, 1, 3)) if groups == 1 and E > 16 else 0)
    if op == "route_backward":
        E = _log(rng, 8, 512)
        return _back(None, _log(rng, 1, 8192), E, rng.randint(1, min(8, E)), _size(rng, 64, 6912), rng.choice(("softmax", "sigmoid")),
                     rng.random() < 0.6, rng.choice((1.0, 2.5)), rng.choice(("f32", "bf16")), rng.choice(("bf16", "bf16", "f32")))
    if op == "quantize":
        what = rng.choice(("rows", "columns", "weights"))
        if what == "weights":
            return _quantize(None, what, _size(rng, 64, 4096), _size(rng, 64, 4096), rng.randint(1, 12), dtype=rng.choice(("f32", "bf16")))
        return _quantize(None, what, _log(rng, 1, 16384), _size(rng, 64, 6912), rng.randint(1, 32) if what == "columns" else 1,
                         rng.choice(("even", "zipf")), rng.choice(("f32", "bf16")))
    if op == "matmul":
        return _matmul(None, op, _log(rng, 1, 32768), rng.randint(1, 32), _size(rng, 64, 4096), _size(rng, 64, 6912), rng.choice(("even", "zipf")), rng.choice(("bf16", "bf16", "f32")))
    return _matmul(None, op, _log(rng, 64, 32768), rng.randint(1, 16), _size(rng, 64, 4096), _size(rng, 64, 4096), rng.choice(("even", "zipf")), rng.choice(("bf16", "f32")))


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, sigma=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").mul_(sigma).to(dtype)


def _loads(case, seed):
    """Rows per expert: every row picks one, each as likely as the next or by Zipf's law over a random order of the experts;
    few rows pick different ones, as the slots of one token do."""
    rng, E, rows = random.Random(seed), case["experts"], case["rows"]
    if rows <= min(E, 10):
        hit = set(rng.sample(range(E), rows))
        return [int(e in hit) for e in range(E)]
    share = [1.0 / (i + 1) if case["load"] == "zipf" else 1.0 for i in range(E)]
    rng.shuffle(share)
    counts = [0] * E
    for e in rng.choices(range(E), weights=share, k=rows):
        counts[e] += 1
    return counts


def _offsets(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _logits(case, g):
    x = _normal(g, case["T"], case["E"]).to(DTYPES[case["dtype"]])
    if case.get("masked"):   # experts of a rank that is gone
        x[:, torch.randperm(case["E"], generator=g, device="cuda")[:case["masked"]]] = -math.inf
    return x


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    s = {"case": case}
    if own and "score" in case:
        s["router"] = _router(case)
    if op == "route":
        s["logits"] = _logits(case, g)
        s["bias"] = (torch.randint(-50, 51, (case["E"],), generator=g, device="cuda").float() * 0.001) if case["bias"] else None
        s["ids"] = torch.empty((case["T"], case["K"]), dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty((case["T"], case["K"]), dtype=torch.float32, device="cuda")
    elif op == "route_backward":
        T, E, K, H = (case[k] for k in "TEKH")
        s["logits"] = _logits(case, g)
        s["ids"] = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True).indices[:, :K].to(torch.int32).contiguous()
        s["gout"] = _normal(g, T, H, sigma=0.03, dtype=DTYPES[case["rows"]])
        s["y"] = _normal(g, T * K, H, dtype=DTYPES[case["rows"]])
        # one row for every slot, ordered by the rank of its expert
        rank = (torch.arange(E, device="cuda") * RANKS // E).to(torch.int32)
        order = torch.sort(rank[s["ids"].reshape(-1).long()], stable=True).indices
        s["slot_row"] = torch.empty_like(order)
        s["slot_row"][order] = torch.arange(T * K, device="cuda")
        s["grad_weights"] = torch.empty((T, K), dtype=torch.float32, device="cuda")
        s["grad_logits"] = torch.empty_like(s["logits"])
        if own:   # the plan of the forward pass, with the same rows
            hm = _binding()
            s["plan"] = hm.hm_plan(s["ids"], torch.ones((T, K), device="cuda"), rank, 1, RANKS, hm.HM_DEDUP_NONE)
    elif op == "quantize":
        rows, cols, what = case["rows"], case["cols"], case["what"]
        shape = (case["experts"], rows, cols) if what == "weights" else (rows, cols)
        # rows differ in size, as tokens do
        s["x"] = _normal(g, *shape, sigma=1.0 / math.sqrt(cols) if what == "weights" else 1.0)
        if what != "weights":
            s["x"] *= torch.exp(_normal(g, rows, 1))
        s["x"] = s["x"].to(DTYPES[case["dtype"]])
        e8 = lambda *shape: torch.empty(shape, dtype=F8, device="cuda")
        byte = lambda *shape: torch.empty(shape, dtype=torch.uint8, device="cuda")
        if what == "rows":
            s["out"] = (e8(rows, _up(cols, 128)), byte(rows, _up(cols, 512) // 128))
        elif what == "columns":
            at = _offsets(_loads(case, seed))
            s["offsets"] = torch.tensor(at, dtype=torch.int32, device="cuda")
            blocks = rows // 128 + case["experts"]
            # blocks that no segment has stay as they are
            s["out"] = (e8(cols, 128 * blocks).zero_(), byte(blocks, cols).zero_())
        else:
            E = case["experts"]
            s["out"] = (e8(E, rows, _up(cols, 128)), byte(E, _up(rows, 128) // 128, _up(cols, 512) // 128),
                        e8(E, cols, _up(rows, 128)), byte(E, _up(cols, 128) // 128, _up(rows, 512) // 128))
    else:
        rows, E, N, H = (case[k] for k in ("rows", "experts", "N", "H"))
        counts = _loads(case, seed)
        at = _offsets(counts)
        s["offsets"], s["most"] = torch.tensor(at, dtype=torch.int32, device="cuda"), max(counts)
        if op == "matmul":
            s["x"] = _blocks_of_rows(_normal(g, rows, H))
            s["w"] = [torch.cat(t) for t in zip(*(_blocks_of_weights(_normal(g, 1, N, H, sigma=1.0 / math.sqrt(H)))[:2] for _ in range(E)))]
            s["out"] = torch.empty((rows, N), dtype=DTYPES[case["dtype"]], device="cuda")
        else:
            s["gy"] = _blocks_of_columns(_normal(g, rows, N, sigma=0.03), s["offsets"])
            s["x"] = _blocks_of_columns(_normal(g, rows, H), s["offsets"])
            s["out"] = torch.empty((E, N, H), dtype=DTYPES[case["dtype"]], device="cuda")
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _scores(x, score, best):
    """Scores up to a factor of a row: exp(x - best) or the logistic function."""
    return torch.exp(x - best) if score == "softmax" else 1.0 / (1.0 + torch.exp(-x))


def _first(choice, n):
    """The n largest entries of each row, descending, ties to the lowest place."""
    return torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :n]


def _plain_route(s):
    case, x = s["case"], s["logits"].float()
    T, E, K, groups = (case[k] for k in ("T", "E", "K", "groups"))
    best = x.max(dim=1, keepdim=True).values
    score = _scores(x, case["score"], best)
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
        w = w / w.sum(dim=1, keepdim=True)
    elif case["score"] == "softmax":
        w = w / score.sum(dim=1, keepdim=True)
    return {"ids": torch.where(there, ids, -1).to(torch.int32), "weights": w * case["scale"]}


def _plain_route_backward(s):
    case, x, ids = s["case"], s["logits"].float(), s["ids"].long()
    T, K, H = (case[k] for k in "TKH")
    g = (s["gout"].float()[:, None, :] * s["y"].float()[s["slot_row"]].view(T, K, H)).sum(dim=2)
    score = _scores(x, case["score"], x.max(dim=1, keepdim=True).values)
    if case["score"] == "softmax":
        score = score / score.sum(dim=1, keepdim=True)
    chosen = torch.gather(score, 1, ids)
    if case["renormalise"]:
        total = chosen.sum(dim=1, keepdim=True)
        ds = (g - (g * chosen / total).sum(dim=1, keepdim=True)) / total
    else:
        ds = g
    ds = ds * case["scale"]
    dx = torch.zeros_like(x)
    if case["score"] == "sigmoid":
        # 1 - score = exp(-x) score
        dx.scatter_(1, ids, ds * chosen * chosen * torch.exp(-torch.gather(x, 1, ids)))
    else:
        dx.scatter_(1, ids, ds * chosen)
        if not case["renormalise"]:   # with it the sum is zero
            dx = dx - score * (ds * chosen).sum(dim=1, keepdim=True)
    return {"grad_weights": g, "grad_logits": dx.to(s["logits"].dtype)}


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
    q, e = _in_blocks(_padded(x.float(), rows, _up(cols, 128)).view(rows, -1, 128), 2)
    return q.view(rows, -1), _padded(e.view(rows, -1), rows, _up(cols, 512) // 128)


def _column_places(offsets, rows):
    """Of every row of the segments: its place among the columns of a transposed row."""
    r = torch.arange(rows, device="cuda", dtype=torch.int32)
    e = torch.searchsorted(offsets[1:].contiguous(), r, right=True)
    return 128 * (offsets[e] // 128 + e) + r - offsets[e]


def _blocks_of_columns(x, offsets):
    rows, cols = x.shape
    blocks = rows // 128 + offsets.numel() - 1
    spread = torch.zeros((128 * blocks, cols), dtype=torch.float32, device="cuda")
    spread[_column_places(offsets, rows)] = x.float()
    q, e = _in_blocks(spread.view(blocks, 128, cols), 1)
    b = torch.arange(blocks, device="cuda", dtype=torch.int32)
    first = offsets[:-1] // 128 + torch.arange(offsets.numel() - 1, device="cuda", dtype=torch.int32)
    last = first + (offsets[1:] - offsets[:-1] + 127) // 128
    there = ((b[:, None] >= first) & (b[:, None] < last)).any(dim=1)
    return q.view(128 * blocks, cols).view(torch.uint8).t().contiguous().view(F8), torch.where(there[:, None], e.view(blocks, cols), 0).to(torch.uint8)


def _blocks_of_weights(w):
    E, rows, cols = w.shape
    R, C = _up(rows, 128), _up(cols, 128)
    q, e = _in_blocks(_padded(w.float(), R, C).view(E, R // 128, 128, C // 128, 128).transpose(2, 3).reshape(E, R // 128, C // 128, -1), 3)
    q = q.view(torch.uint8).view(E, R // 128, C // 128, 128, 128).transpose(2, 3).reshape(E, R, C)
    e = e.view(E, R // 128, C // 128)
    return (q[:, :rows].contiguous().view(F8), _padded(e, R // 128, _up(cols, 512) // 128),
            q.transpose(1, 2)[:, :cols].contiguous().view(F8), _padded(e.transpose(1, 2).contiguous(), C // 128, _up(rows, 512) // 128))


def _values_of_rows(q, e):
    rows, width = q.shape
    return (q.float().view(rows, -1, 128) * _power(e)[:, :width // 128, None]).view(rows, width)


def _by_expert(offsets, rows, most):
    """[experts, most] rows of every segment, `rows` where it has ended."""
    at = offsets[:-1, None].long() + torch.arange(most, device="cuda")
    return torch.where(at < offsets[1:, None], at, rows)


def _plain_matmul(s):
    case = s["case"]
    rows, E, N, H = (case[k] for k in ("rows", "experts", "N", "H"))
    width = _up(H, 128)
    x = torch.cat([_values_of_rows(*s["x"]), torch.zeros((1, width), device="cuda")])
    q, e = s["w"]
    w = q.float() * _power(e)[:, :, :width // 128].repeat_interleave(128, dim=1)[:, :N].repeat_interleave(128, dim=2)
    at = _by_expert(s["offsets"], rows, s["most"])
    y = torch.bmm(x[at], w.transpose(1, 2).contiguous())
    out = torch.empty((rows + 1, N), device="cuda")
    out[at.view(-1)] = y.view(-1, N)
    return out[:rows].to(DTYPES[case["dtype"]])


def _values_of_columns(q, e):
    """One row per place, of the values that q [columns, places] holds, and a row of zeros behind them."""
    cols, places = q.shape
    v = (q.float().view(cols, -1, 128) * _power(e).t()[:, :, None]).view(cols, places).t()
    return torch.cat([v, torch.zeros((1, cols), device="cuda")])


def _plain_matmul_dw(s):
    case = s["case"]
    gy, x = _values_of_columns(*s["gy"]), _values_of_columns(*s["x"])
    rows, most = case["rows"], s["most"]
    places = torch.cat([_column_places(s["offsets"], rows).long(), torch.tensor([gy.shape[0] - 1], device="cuda")])
    at = places[_by_expert(s["offsets"], rows, most)]
    return torch.bmm(gy[at].transpose(1, 2).contiguous(), x[at]).to(DTYPES[case["dtype"]])


def _plain(s):
    op = s["case"]["op"]
    if op == "route":
        return _plain_route(s)
    if op == "route_backward":
        return _plain_route_backward(s)
    if op == "matmul":
        return _plain_matmul(s)
    if op == "matmul_dw":
        return _plain_matmul_dw(s)
    what = s["case"]["what"]
    if what == "rows":
        return _blocks_of_rows(s["x"])
    if what == "columns":
        return _blocks_of_columns(s["x"], s["offsets"])
    return _blocks_of_weights(s["x"])


# ---- the library's calls --------------------------------------------------------------------------------------------
_hm = None


def _binding():
    global _hm
    if _hm is None:
        from paper_2508_09591_amd import binding
        _hm = binding
    return _hm


def _router(case):
    return _binding().Router(case["E"], case["K"], case["score"], groups=case.get("groups", 1), top_groups=case.get("top_groups", 1),
                     group_best=case.get("group_best", 1), renormalise=case["renormalise"], scale=case["scale"])


def run(s):
    if not own:
        return _plain(s)
    hm, case = _binding(), s["case"]
    op = case["op"]
    if op == "route":
        hm.hm_route(s["logits"], s["router"], s["ids"], s["weights"], s["bias"])
        return {"ids": s["ids"], "weights": s["weights"]}
    if op == "route_backward":
        hm.hm_combine_weight_grad(s["gout"], s["y"], s["plan"], s["grad_weights"])
        hm.hm_route_backward(s["logits"], s["router"], s["ids"], s["grad_weights"], s["grad_logits"])
        return {"grad_weights": s["grad_weights"], "grad_logits": s["grad_logits"]}
    if op == "matmul":
        return hm.hm_expert_matmul(*s["x"], *s["w"], s["offsets"], s["out"])
    if op == "matmul_dw":
        return hm.hm_expert_matmul_dw(*s["gy"], *s["x"], s["offsets"], case["rows"], s["out"])
    if case["what"] == "rows":
        hm.hm_quantize_rows(s["x"], *s["out"])
    elif case["what"] == "columns":
        hm.hm_quantize_columns(s["x"], s["offsets"], *s["out"])
    else:
        hm.hm_quantize_weights(s["x"], *s["out"])
    return s["out"]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    size = lambda d: 2 if d == "bf16" else 4
    if op == "route":
        T, E, K = (case[k] for k in "TEK")
        return {"bytes": T * (E * size(case["dtype"]) + 8 * K) + (4 * E if case["bias"] else 0), "flops": 4 * T * E}
    if op == "route_backward":
        T, E, K, H = (case[k] for k in "TEKH")
        dense = case["score"] == "softmax" and not case["renormalise"]
        logits = T * size(case["dtype"]) * (E + (E if dense else K))
        return {"bytes": T * H * (K + 1) * size(case["rows"]) + T * K * 12 + logits, "flops": 2 * T * K * H}
    if op == "quantize":
        n = case["rows"] * case["cols"] * (case["experts"] if case["what"] == "weights" else 1)
        if case["what"] == "weights":
            return {"bytes": n * (size(case["dtype"]) + 2), "flops": 2 * n}
        return {"bytes": n * size(case["dtype"]) + n + n // 128, "flops": 2 * n}
    rows, E, N, H = (case[k] for k in ("rows", "experts", "N", "H"))
    flops = 2 * rows * N * H
    if op == "matmul":
        hit = rows if rows <= min(E, 10) else E * (1 - (1 - 1 / E) ** rows)
        return {"bytes": rows * H + hit * N * H + rows * N * size(case["dtype"]), "flops": flops}
    return {"bytes": rows * (H + N) + E * N * H * size(case["dtype"]), "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _exact_route(s):
    case, x = s["case"], s["logits"].double()
    T, E, K = (case[k] for k in "TEK")
    s1 = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, dim=1)
    c = s1 + s["bias"].double() if s["bias"] is not None else s1
    c = c.masked_fill(torch.isinf(x), -1e30)
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
    place = torch.arange(E, device="cuda")
    ids = []
    for _ in range(K):   # the largest, the first of equal ones
        top = c.max(dim=1, keepdim=True).values
        i = torch.where(c == top, place, E).min(dim=1).values
        ids.append(torch.where(top[:, 0] > -1e29, i, -1))
        c = c.scatter(1, i[:, None], -1e30)
    ids = torch.stack(ids, dim=1)
    w = torch.where(ids >= 0, s1.gather(1, ids.clamp(min=0)), 0.0)
    if case["renormalise"]:
        w = w / w.sum(dim=1, keepdim=True)
    return {"ids": ids, "weights": case["scale"] * w}


def _exact_route_backward(s):
    case, x, ids = s["case"], s["logits"].double(), s["ids"].long()
    T, E, K, H = (case[k] for k in "TEKH")
    rows = s["slot_row"].view(T, K)
    gout = s["gout"].double()
    g = torch.stack([(gout * s["y"][rows[:, k]].double()).sum(dim=1) for k in range(K)], dim=1)
    # weights = scale * p, p over the chosen: its Jacobian, term by term
    a = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, dim=1)
    p = a.gather(1, ids)
    total = p.sum(dim=1, keepdim=True) if case["renormalise"] else torch.ones((T, 1), dtype=torch.float64, device="cuda")
    mean = (g * p).sum(dim=1, keepdim=True) / total
    dp = case["scale"] * ((g - mean) / total if case["renormalise"] else g)
    dense = torch.zeros((T, E), dtype=torch.float64, device="cuda")
    if case["score"] == "sigmoid":
        dense.scatter_(1, ids, dp * p * torch.sigmoid(-x.gather(1, ids)))
    else:
        dense.scatter_(1, ids, dp * p)
        dense -= a * dense.sum(dim=1, keepdim=True)
    return {"grad_weights": g, "grad_logits": dense}


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


def _exact_quantize(s):
    case, x = s["case"], s["x"]
    what, cols = case["what"], case["cols"]
    if what == "rows":
        rows = case["rows"]
        v = torch.zeros((rows, _up(cols, 128)), dtype=torch.float64, device="cuda")
        v[:, :cols] = x.double()
        v = v.view(rows, -1, 128)
        code = _exact_code(v.abs().amax(dim=2))
        q = _exact_e4m3(v / _two_to(code.long() - 127)[:, :, None]).view(rows, -1)
        return q, None
    if what == "columns":
        at, blocks = s["offsets"].tolist(), case["rows"] // 128 + case["experts"]
        q = torch.zeros((cols, 128 * blocks), dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            for r in range(at[e], at[e + 1], 128):
                v = x[r:min(r + 128, at[e + 1])].double()
                p = _two_to(_exact_code(v.abs().amax(dim=0)) - 127)
                place = 128 * (at[e] // 128 + e) + r - at[e]
                q[:, place:place + v.shape[0]] = _exact_e4m3(v / p).t()
        return q, None
    E, rows = case["experts"], case["rows"]
    R, C = _up(rows, 128), _up(cols, 128)
    q = torch.zeros((E, rows, C), dtype=torch.float64, device="cuda")
    for i in range(0, rows, 128):
        for j in range(0, cols, 128):
            v = x[:, i:i + 128, j:j + 128].double()
            p = _two_to(_exact_code(v.abs().amax(dim=(1, 2))) - 127)
            q[:, i:i + v.shape[1], j:j + v.shape[2]] = _exact_e4m3(v / p[:, None, None])
    qt = torch.zeros((E, cols, R), dtype=torch.float64, device="cuda")
    qt[:, :, :rows] = q[:, :, :cols].transpose(1, 2)
    return q, None, qt, None


def _exact_matmul(s):
    case, at = s["case"], s["offsets"].tolist()
    (x, sx), (w, sw) = s["x"], s["w"]
    N, blocks = case["N"], x.shape[1] // 128
    power = lambda code: _two_to(code[..., :blocks].long() - 127)
    out = torch.zeros((case["rows"], N), dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        rows = slice(at[e], at[e + 1])
        if at[e] < at[e + 1]:
            a = x[rows].double().view(-1, blocks, 128) * power(sx[rows])[:, :, None]
            p = power(sw[e])
            b = w[e].double().view(N, blocks, 128) * p[torch.arange(N, device="cuda") // 128][:, :, None]
            out[rows] = a.view(-1, 128 * blocks) @ b.view(N, -1).t().contiguous()
    return out


def _exact_matmul_dw(s):
    case, at = s["case"], s["offsets"].tolist()
    dw = torch.zeros((case["experts"], case["N"], case["H"]), dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        first = at[e] // 128 + e
        n = (at[e + 1] - at[e] + 127) // 128
        v = [(q[:, 128 * first:128 * (first + n)].double().view(q.shape[0], n, 128) * _two_to(c[first:first + n].long() - 127).t()[:, :, None]).reshape(q.shape[0], -1)
             for q, c in (s["gy"], s["x"])]
        dw[e] = v[0] @ v[1].t().contiguous()
    return dw


def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "route_backward": _exact_route_backward, "quantize": _exact_quantize, "matmul": _exact_matmul,
            "matmul_dw": _exact_matmul_dw}[case["op"]](s)
