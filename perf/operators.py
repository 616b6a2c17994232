"""Operators around a layer whose experts' weights are 4-bit floats with a scale per 32 (microscaled, MXFP4), as cases
that can be timed and compared.

Four kinds of call, in the order in which one layer makes them:

  route     scores of the experts from the router's logits (softmax or sigmoid), a balance bias for the choice, groups of
            experts of which the best are kept, top-k, renormalised and scaled weights: slicemoe_route_scored
  quantize  activations to microscaled 4-bit floats and the values they stand for: slicemoe_mx4_quantize, slicemoe_mx4_dequantize
  product   rows of such activations times the matrices of the experts that the routing list names, plain or as the gated
            pair silu(gate) * up: slicemoe_mx4_product
  combine   the experts' rows of a token added up with the token's weights, on top of a residual: slicemoe_combine

`run` computes a case from the operator's formula in elementary torch operations, or, where `own` is set, through this
repository's entry points.  Widths are those of the layers that the library's benchmark is quoted on (hidden 2048, experts of
width 1408, top-6 of 64 or top-4 of 60), and generic ones.  Activations are N(0, 1), weights N(0, 0.02); routing is log(Zipf
popularity) + Gumbel noise where many tokens are routed, which gives the experts uneven shares.
"""
import numpy as np
import torch

own = False

BLOCK = 32                                            # values that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)       # what the three low bits of a 4-bit float stand for
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _b():
    from paper_2512_12990_b200 import binding
    return binding


# ---- cases ---------------------------------------------------------------------------------------------------
def _route(name, T, E, k, score="softmax", bias=False, groups=1, keep=1, best=1, renorm=True, factor=1.0, dtype="f32", rank_high=0):
    return dict(name=name, kind="route", T=T, E=E, k=k, score=score, bias=bias, groups=groups, keep=keep, best=best, renorm=renorm,
                factor=factor, dtype=dtype, rank_high=rank_high)


def _quantize(name, T, K, dtype, pad=0):
    return dict(name=name, kind="quantize", T=T, K=K, dtype=dtype, pad=pad)


def _product(name, T, k, E, N, K, gated=False, per_pair=False, dtype="bf16", zipf=0.0):
    return dict(name=name, kind="product", T=T, k=k, E=E, N=N, K=K, gated=gated, per_pair=per_pair, dtype=dtype, zipf=zipf)


def _combine(name, T, k, N, dtype, out, base):
    return dict(name=name, kind="combine", T=T, k=k, N=N, dtype=dtype, out=out, base=base)


def listed():
    return [
        # the routing of one decode token
        _route("route one token", 1, 64, 6, rank_high=3),
        # a prompt's tokens, softmax scores, renormalised
        _route("route prompt of 2048", 2048, 60, 4),
        # a long prompt through a layer of many small experts: sigmoid scores, balance bias, 4 of 8 groups kept
        _route("route 8192, 8 groups", 8192, 256, 8, score="sigmoid", bias=True, groups=8, keep=4, best=2, factor=2.5),
        # one decode token's activations
        _quantize("quantize one token", 1, 2048, "bf16"),
        # a long prompt's activations
        _quantize("quantize 8192 tokens", 8192, 2048, "bf16"),
        # a slice of a wider fp32 buffer, an odd number of rows
        _quantize("quantize fp32 slice", 1009, 1408, "f32", pad=96),
        # gate and up of the six experts of one decode token: latency and the weights' way
        _product("gated product, one token", 1, 6, 64, 1408, 2048, gated=True),
        # sixteen sequences decoded together: most experts named, each by a token or two
        _product("gated product, batch of 16", 16, 6, 64, 1408, 2048, gated=True, dtype="f32", zipf=1.1),
        # the benchmark's prompt: every expert visited, uneven numbers of tokens
        _product("gated product, prompt 2048", 2048, 4, 60, 1408, 2048, gated=True, zipf=1.0),
        # the down projection of a long prompt, every pair with a row of its own
        _product("down product, prompt 8192", 8192, 6, 64, 2048, 1408, per_pair=True, zipf=1.0),
        # the end of a decode token's layer
        _combine("combine one token", 1, 6, 2048, "bf16", "bf16", True),
        # the end of a long prompt's layer
        _combine("combine 8192 tokens", 8192, 6, 2048, "bf16", "bf16", True),
    ]


def _log_uniform(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def draw(rng):
    kind = rng.choice(["route", "quantize", "product", "product", "combine"])
    T = int(_log_uniform(rng, 1, 8193))
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        size = int(_log_uniform(rng, 4, 513 // groups + 1)) if groups > 1 else int(_log_uniform(rng, 4, 513))
        E = groups * size
        keep = rng.randint(1, groups)
        return _route("", T, E, rng.randint(1, min(12, keep * size)), score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                      groups=groups, keep=keep, best=rng.choice([1, 2]), renorm=rng.random() < 0.5, factor=rng.choice([1.0, 2.5]),
                      dtype=rng.choice(["f32", "bf16", "f16"]), rank_high=rng.randint(0, 3))
    if kind == "quantize":
        return _quantize("", T, BLOCK * int(_log_uniform(rng, 1, 65)), rng.choice(["f32", "bf16", "f16"]), pad=rng.choice([0, 0, 8, 33]))
    if kind == "combine":
        return _combine("", T, rng.randint(1, 8), int(_log_uniform(rng, 16, 2049)), rng.choice(["f32", "bf16", "f16"]),
                        rng.choice(["f32", "bf16"]), rng.random() < 0.5)
    while True:
        E = int(_log_uniform(rng, 1, 65))
        c = _product("", T, rng.randint(1, min(E, 8)), E, int(_log_uniform(rng, 16, 2049)), BLOCK * int(_log_uniform(rng, 2, 65)),
                     gated=rng.random() < 0.5, per_pair=rng.random() < 0.3, dtype=rng.choice(["f32", "bf16", "f16"]), zipf=rng.choice([0.0, 1.0]))
        if work(c)["flops"] <= 2.8e11:
            return c
        T = max(1, T // 2)


# ---- inputs ---------------------------------------------------------------------------------------------------
def _scaled(x):
    """x as [rows, blocks, 32] in fp32, the blocks' scale bytes, and the magnitudes of the 4-bit codes: the largest magnitude of a
    block has exponent 2 after scaling, values are rounded to the nearest of GRID, ties to the even code, above 6 to 6."""
    v = x.float().reshape(x.shape[0], -1, BLOCK)
    top = v.abs().amax(-1).contiguous().view(torch.int32) >> 23
    scale = (top - 2).clamp(min=0)
    a = v.abs() * ((254 - scale) << 23).view(torch.float32)[..., None]
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return v, scale, code


def _to_codes(x):
    """(codes [rows, K / 2], two to a byte, the even one low; scale bytes [rows, 4 * ceil(K / 128)], padded with zeros)."""
    v, scale, code = _scaled(x)
    n = (code + (v < 0).to(torch.uint8) * 8).reshape(x.shape[0], -1)
    s = torch.zeros((x.shape[0], (scale.shape[1] + 3) // 4 * 4), dtype=torch.uint8, device=x.device)
    s[:, :scale.shape[1]] = scale.to(torch.uint8)
    return n[:, 0::2] | (n[:, 1::2] << 4), s


def _values(codes, scale):
    """What codes and scale bytes stand for, in fp32."""
    rows, half = codes.shape
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    n = torch.stack((codes & 15, codes >> 4), -1).reshape(rows, -1, BLOCK)
    step = torch.exp2(scale[:, :half // 16].double() - 127).float()
    return (grid[n.long()] * step[..., None]).reshape(rows, -1)


def _lists(c, gen):
    """Expert ids of the tokens, k different ones each."""
    popularity = -c["zipf"] * torch.log(torch.arange(1, c["E"] + 1, device="cuda").float())
    u = torch.rand((c["T"], c["E"]), device="cuda", generator=gen).clamp(1e-7, 1 - 1e-7)
    order = torch.randperm(c["E"], device="cuda", generator=gen)
    return (popularity[order] - torch.log(-torch.log(u))).topk(c["k"], -1).indices.to(torch.int32)


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(shape, device="cuda", generator=gen) * std

    s = {}
    if c["kind"] == "route":
        s["logits"] = normal(c["T"], c["E"]).to(DTYPES[c["dtype"]])
        s["bias"] = normal(c["E"], std=0.05) if c["bias"] else None
    elif c["kind"] == "quantize":
        s["x"] = normal(c["T"], c["K"] + c["pad"]).to(DTYPES[c["dtype"]])[:, :c["K"]]
    elif c["kind"] == "combine":
        s["rows"] = normal(c["T"], c["k"], c["N"]).to(DTYPES[c["dtype"]])
        s["weights"] = torch.softmax(normal(c["T"], c["k"]), -1)
        s["base"] = normal(c["T"], c["N"]).to(DTYPES[c["out"]]) if c["base"] else None
    else:
        s["codes"], s["scale"] = _to_codes(normal(c["T"] * (c["k"] if c["per_pair"] else 1), c["K"]).bfloat16())
        s["ids"] = _lists(c, gen)
        w = [_to_codes(normal(c["N"] * (2 if c["gated"] else 1), c["K"], std=0.02)) for _ in range(c["E"])]  # gate's rows, then up's
        s["w_codes"], s["w_scale"] = torch.stack([a for a, _ in w]), torch.stack([b for _, b in w])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["c"] = case
    if own and case["kind"] == "product":
        B = _b()
        mats = []
        for codes, scale in zip(s["w_codes"], s["w_scale"]):
            w = _values(codes, scale).bfloat16()  # exact: two significant bits
            mats.append(B.slicemoe_mx4_pack(w[:case["N"]], w[case["N"]:]) if case["gated"] else B.slicemoe_mx4_pack(w))
        s["table"] = B.mx4_table(mats)
        s["ws"] = B.new_mx4_workspace(case["T"], case["k"], case["E"])
        if case["per_pair"]:
            s["codes"] = s["codes"].view(case["T"], case["k"], -1)
            s["scale"] = s["scale"].view(case["T"], case["k"], -1)
        del s["w_codes"], s["w_scale"]
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------
def _run_own(s, c):
    B = _b()
    if c["kind"] == "route":
        ids, w, prec = B.slicemoe_route_scored(s["logits"], c["k"], score=c["score"], bias=s["bias"], n_group=c["groups"], topk_group=c["keep"],
                                               group_best=c["best"], renorm=c["renorm"], scale=c["factor"], rank_high=c["rank_high"])
        return ids, w, prec
    if c["kind"] == "quantize":
        codes, scale = B.slicemoe_mx4_quantize(s["x"])
        return B.slicemoe_mx4_dequantize(codes, scale, torch.bfloat16)
    if c["kind"] == "combine":
        return B.slicemoe_combine(s["rows"], s["weights"], base=s["base"], dtype=DTYPES[c["out"]])
    return B.slicemoe_mx4_product(s["table"], s["codes"], s["scale"], s["ids"], s["ws"], dtype=DTYPES[c["dtype"]])


def _plain_route(s, c):
    x = s["logits"].double()  # keys next to each other decide which expert runs
    if c["score"] == "softmax":
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-x))
    key = p if s["bias"] is None else p + s["bias"].double()
    if c["groups"] > 1:
        best = torch.sort(key.view(c["T"], c["groups"], -1), -1, descending=True).values[..., :c["best"]].sum(-1)
        order = torch.sort(best, dim=-1, descending=True, stable=True).indices
        kept = torch.zeros_like(best, dtype=torch.bool).scatter_(1, order[:, :c["keep"]], True)
        key = torch.where(kept.repeat_interleave(c["E"] // c["groups"], -1), key, -torch.inf)
    ids = torch.sort(key, dim=-1, descending=True, stable=True).indices[:, :c["k"]]
    w = p.gather(1, ids)
    if c["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    high = (torch.arange(c["k"], device="cuda") < c["rank_high"]).to(torch.uint8).expand(c["T"], -1)
    return ids.to(torch.int32), (w * c["factor"]).float(), high


def _gated(y, c):
    if not c["gated"]:
        return y
    g, u = y[..., :c["N"]], y[..., c["N"]:]
    return g / (1 + torch.exp(-g)) * u


def _plain_product(s, c):
    pairs = c["T"] * c["k"]
    x = _values(s["codes"], s["scale"])
    out = torch.empty((pairs, c["N"]), dtype=DTYPES[c["dtype"]], device="cuda")
    expert = s["ids"].reshape(-1)
    if pairs <= BLOCK:  # a matrix for each pair
        rows = x if c["per_pair"] else x.repeat_interleave(c["k"], 0)
        used = expert.long()
        w = _values(s["w_codes"][used].flatten(0, 1), s["w_scale"][used].flatten(0, 1)).view(pairs, -1, c["K"])
        out.copy_(_gated((w @ rows[:, :, None])[..., 0], c))
    else:  # an expert's rows together
        order = torch.argsort(expert)
        first = 0
        for e, n in enumerate(torch.bincount(expert, minlength=c["E"]).tolist()):
            if n:
                at = order[first:first + n]
                rows = x[at if c["per_pair"] else at // c["k"]]
                out[at] = _gated(rows @ _values(s["w_codes"][e], s["w_scale"][e]).T, c).to(out.dtype)
            first += n
    return out.view(c["T"], c["k"], c["N"])


def run(state):
    c = state["c"]
    if own:
        return _run_own(state, c)
    if c["kind"] == "route":
        return _plain_route(state, c)
    if c["kind"] == "quantize":
        v, scale, code = _scaled(state["x"])
        grid = torch.tensor(GRID, device="cuda")
        step = torch.exp2(scale.double() - 127).float()
        return (torch.where(v < 0, -1.0, 1.0) * grid[code.long()] * step[..., None]).reshape(c["T"], c["K"]).bfloat16()
    if c["kind"] == "combine":
        y = (state["rows"].float() * state["weights"][..., None]).sum(1)
        return (y if state["base"] is None else y + state["base"].float()).to(DTYPES[c["out"]])
    return _plain_product(state, c)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def _exact_route(s, c):
    x = s["logits"].double().cpu().numpy()
    if c["score"] == "softmax":
        e = np.exp(x - x.max(1, keepdims=True))
        p = e / e.sum(1, keepdims=True)
    else:
        p = 1.0 / (1.0 + np.exp(-x))
    key = p.copy()
    if s["bias"] is not None:
        key += s["bias"].double().cpu().numpy()
    size = c["E"] // c["groups"]
    group = np.arange(c["E"]) // size
    if c["groups"] > 1:
        best = np.stack([np.sort(key[:, group == g], 1)[:, ::-1][:, :c["best"]].sum(1) for g in range(c["groups"])], 1)
        rank = np.argsort(np.argsort(-best, 1, kind="stable"), 1, kind="stable")
        key[rank[:, group] >= c["keep"]] = -np.inf
    ids = np.argsort(-key, 1, kind="stable")[:, :c["k"]]
    w = np.take_along_axis(p, ids, 1)
    if c["renorm"]:
        w = w / w.sum(1, keepdims=True)
    high = np.zeros((c["T"], c["k"]), np.uint8)
    high[:, :c["rank_high"]] = 1
    return torch.from_numpy(ids.astype(np.int32)), torch.from_numpy(w * c["factor"]), torch.from_numpy(high)


def _exact_quantize(s, c):
    v = s["x"].double().reshape(c["T"], -1, BLOCK)
    _, e = torch.frexp(v.abs().amax(-1))                # largest = m 2^e, m in [0.5, 1): its exponent is e - 1
    step = torch.exp2((e - 3).clamp(min=-127).double())[..., None]
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    y = (v / step).abs()
    far = torch.full_like(y, torch.inf)
    near = torch.zeros_like(y)
    for g in (0, 2, 4, 6, 1, 3, 5, 7):                  # the even codes first: they win a tie
        d = (y - grid[g]).abs()
        near = torch.where(d < far, grid[g], near)
        far = torch.minimum(d, far)
    return (torch.sign(v) * near * step).reshape(c["T"], c["K"])


def _exact_values(codes, scale):
    n = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device="cuda")
    for odd in (0, 1):
        nib = (codes.int() >> (4 * odd)) & 15
        m, e = (nib & 1).double(), (nib >> 1) & 3       # one mantissa bit, two exponent bits with bias 1
        n[:, odd::2] = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2(e.double() - 1)) * (1 - 2 * (nib >> 3).double())
    return n * torch.exp2(scale[:, :codes.shape[1] // 16].double() - 127).repeat_interleave(BLOCK, 1)


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "route":
        return _exact_route(s, c)
    if c["kind"] == "quantize":
        return _exact_quantize(s, c)
    if c["kind"] == "combine":
        y = torch.einsum("tkn,tk->tn", s["rows"].double(), s["weights"].double())
        return y if s["base"] is None else y + s["base"].double()
    x = _exact_values(s["codes"], s["scale"])
    ids = s["ids"].reshape(-1)
    out = torch.empty((len(ids), c["N"]), dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        at = torch.nonzero(ids == e)[:, 0]
        if not len(at):
            continue
        y = x[at if c["per_pair"] else at // c["k"]] @ _exact_values(s["w_codes"][e], s["w_scale"][e]).T
        if c["gated"]:
            y = y[:, :c["N"]] / (1 + torch.exp(-y[:, :c["N"]])) * y[:, c["N"]:]
        out[at] = y
    return out.view(c["T"], c["k"], c["N"])


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "route":
        return {"bytes": c["T"] * (c["E"] * SIZE[c["dtype"]] + 9 * c["k"]) + (4 * c["E"] if c["bias"] else 0), "flops": 4 * c["T"] * c["E"]}
    if c["kind"] == "quantize":
        n = c["T"] * c["K"]
        return {"bytes": n * SIZE[c["dtype"]] + 2 * n, "flops": 4 * n}
    if c["kind"] == "combine":
        n = c["T"] * c["N"]
        return {"bytes": n * (c["k"] * SIZE[c["dtype"]] + SIZE[c["out"]] * (2 if c["base"] else 1)) + 4 * c["T"] * c["k"], "flops": 2 * n * c["k"]}
    wide = c["N"] * (2 if c["gated"] else 1)
    rows, pairs = c["T"] * (c["k"] if c["per_pair"] else 1), c["T"] * c["k"]
    # experts that T tokens are expected to name, were all equally likely
    used = c["E"] * (1 - (1 - c["k"] / c["E"]) ** c["T"])
    code = c["K"] // 2 + c["K"] // BLOCK
    return {"bytes": int(used * wide * code + rows * code + 4 * pairs + pairs * c["N"] * SIZE[c["dtype"]]), "flops": 2 * pairs * wide * c["K"]}
