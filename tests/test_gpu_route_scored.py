"""slicemoe_route_scored on the GPU against the oracle in 64 bits: ids exact, weights to fp32 accuracy.

Weights: a score is off by at most 2^-22 relative for a sigmoid (expf 2 ulp, a sum, a quotient) and 2^-18.9 for a softmax of up to
512 (expf's 2 ulp twice, the argument's rounding times the argument, 21 additions); renormalising divides two of those, and the
factor rounds once more: 2^-17 relative, and 2^-126 where a score underflows."""
import numpy as np
import pytest

from oracle import mx4

pytestmark = pytest.mark.gpu


def _check(logits, k, dtype="f32", bias=None, **kw):
    import torch
    from paper_2512_12990_b200 import binding as B
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    x = torch.from_numpy(np.ascontiguousarray(logits)).cuda().to(dt) if not isinstance(logits, torch.Tensor) else logits
    b = None if bias is None else torch.from_numpy(bias.astype(np.float32)).cuda()
    ids, w, prec = B.slicemoe_route_scored(x, k, bias=b, rank_high=1, tau=0.3, **kw)
    ids_o, w_o, s_o = mx4.route_scored(x.double().cpu().numpy(), k, bias=None if bias is None else bias.astype(np.float32), **kw)
    assert np.array_equal(ids.cpu().numpy(), ids_o)
    w = w.double().cpu().numpy()
    assert (np.abs(w - w_o) <= 2.0 ** -17 * np.abs(w_o) + 2.0 ** -126 * abs(kw.get("scale", 1.0))).all()
    prec, sure = prec.cpu().numpy(), np.abs(s_o - 0.3) > 1e-5
    assert (prec[:, 0] == 1).all() and np.array_equal(prec[:, 1:][sure[:, 1:]], (s_o >= 0.3).astype(np.uint8)[:, 1:][sure[:, 1:]])


SHAPES = [(1, 1, 1, 1, 1, 1), (1, 64, 6, 1, 1, 1), (1, 60, 4, 1, 1, 1), (37, 64, 6, 8, 3, 2), (300, 60, 4, 4, 2, 2), (5, 7, 7, 1, 1, 1), (3, 33, 16, 3, 2, 2),
          (100, 256, 8, 8, 4, 2), (2, 512, 8, 16, 3, 1), (65, 512, 16, 32, 5, 2), (9, 129, 5, 1, 1, 1), (50, 96, 6, 6, 6, 2), (4, 30, 10, 5, 2, 2), (1030, 128, 8, 2, 1, 1)]


@pytest.mark.parametrize("T,E,k,groups,keep,best", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype,biased,renorm", [("f32", True, True), ("f32", False, False), ("bf16", True, False), ("f16", False, True)])
def test_matches_the_oracle(T, E, k, groups, keep, best, score, dtype, biased, renorm):
    rng = np.random.default_rng(T + E + k)
    _check(rng.normal(size=(T, E)).astype(np.float32), k, dtype, rng.normal(size=E) * 0.1 if biased else None, score=score, n_group=groups,
           topk_group=keep, group_best=best, renorm=renorm, scale=2.5 if renorm else 1.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_keys_that_32_bits_cannot_tell_apart(score):
    """The bias makes up for the scores' differences up to the rounding of a float32: many keys within 2^-24 of one another, whose
    order only 64 bits show."""
    rng = np.random.default_rng(3)
    for E, groups in ((64, 1), (256, 8), (40, 4)):
        x = rng.normal(size=E).astype(np.float32)
        s = mx4.route_scored(x[None], E, score)
        p = np.empty(E)
        p[s[0][0]] = s[1][0]
        bias = (0.9 - p).astype(np.float32)
        rows = np.tile(x, (50, 1))
        rows[25:] += rng.normal(size=(25, E)).astype(np.float32) * 1e-6
        for best in (1, 2):
            _check(rows, 8, bias=bias, score=score, n_group=groups, topk_group=max(1, groups // 2), group_best=best, renorm=True)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_ties_go_to_the_lower_index(score):
    rng = np.random.default_rng(4)
    x = rng.integers(-2, 3, size=(64, 96)).astype(np.float32)
    for groups, keep, best in ((1, 1, 1), (8, 3, 2), (8, 3, 1), (32, 7, 2)):
        for bias in (None, np.zeros(96), rng.integers(0, 3, size=96) * 0.125):
            _check(x, 6, bias=bias, score=score, n_group=groups, topk_group=keep, group_best=best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_infinities_nan_and_rows_with_nothing_left(score, groups):
    rng = np.random.default_rng(5)
    x = rng.normal(size=(9, 64)).astype(np.float32)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 5:] = -np.inf
    x[3, 7] = np.inf
    x[4, [7, 40]] = np.inf
    x[5] = np.finfo(np.float32).min
    x[6, ::2] = np.nan
    x[7, :60] = np.finfo(np.float32).min
    x[8] = 1e4
    bias = rng.normal(size=64) * 0.1
    bias[3] = -np.inf
    for b in (None, bias):
        _check(x, 6, bias=b, score=score, n_group=groups, topk_group=min(groups, 2), group_best=1, renorm=True)


def test_spaced_and_shifted_rows():
    import torch
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        wide = torch.randn(20, 99, device="cuda").to(dt)
        _check(wide[:, 3:63], 4, score="sigmoid", renorm=True)
        _check(wide[::2, 1:61], 4)
    _check(torch.randn(64, 20, device="cuda").t().contiguous()[:1], 4)


def test_agrees_with_route_topk():
    import torch
    from paper_2512_12990_b200 import binding as B
    x = torch.randn(200, 60, device="cuda")
    a, b = B.slicemoe_route_topk(x, 4, renorm=True, rank_high=2), B.slicemoe_route_scored(x, 4, renorm=True, rank_high=2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and torch.allclose(a[1], b[1], rtol=2e-6, atol=0)
    assert B.slicemoe_route_scored(x, 4, want_prec=False)[2] is None


def test_in_a_graph():
    import torch
    from paper_2512_12990_b200 import binding as B
    x = torch.randn(40, 256, device="cuda")
    kw = dict(score="sigmoid", n_group=8, topk_group=4, group_best=2, renorm=True, bias=torch.randn(256, device="cuda") * 0.1)
    B.slicemoe_route_scored(x, 8, **kw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ids, w, _ = B.slicemoe_route_scored(x, 8, **kw)
    x.copy_(torch.randn(40, 256, device="cuda"))
    g.replay()
    ref = B.slicemoe_route_scored(x, 8, **kw)
    assert torch.equal(ids, ref[0]) and torch.equal(w, ref[1])


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2512_12990_b200 import binding as B
    x = torch.zeros((2, 64), device="cuda")
    for kw in (dict(bias=torch.zeros(63, device="cuda")), dict(bias=torch.zeros(64)), dict(bias=torch.zeros(64, device="cuda", dtype=torch.float64))):
        with pytest.raises(ValueError):
            B.slicemoe_route_scored(x, 2, **kw)
    for bad in (x.t(), x[:, ::2], x.double(), x[0]):
        with pytest.raises(ValueError):
            B.slicemoe_route_scored(bad, 2)
    with pytest.raises(B.SliceMoEError):
        B.slicemoe_route_scored(x, 65)


def test_rows_that_overlap_are_refused():
    """A broadcast row has no spacing: read as dense rows it would be read past its end."""
    import torch
    from paper_2512_12990_b200 import binding as B
    x = torch.zeros(4 * 64, device="cuda")
    for bad in (x[:64].expand(4, 64), x.as_strided((4, 64), (32, 1))):
        with pytest.raises(B.SliceMoEError):
            B.slicemoe_route_scored(bad, 2)
        with pytest.raises(B.SliceMoEError):
            B.slicemoe_mx4_quantize(bad)
    B.slicemoe_route_scored(x[:64].expand(1, 64), 2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups", [(4, 2), (16, 8), (32, 4), (48, 6), (96, 6), (160, 5), (320, 20), (480, 15)])
def test_groups_that_32_bits_cannot_tell_apart_in_some_of_the_lanes(score, E, groups):
    """Groups of whole lanes that leave lanes without experts, worth the same down to the rounding of a float32: told apart in 64 bits, by all
    lanes of the warp together."""
    rng = np.random.default_rng(E)
    x = rng.normal(size=E).astype(np.float32)
    p = 1.0 / (1.0 + np.exp(-x.astype(np.float64))) if score == "sigmoid" else np.exp(x.astype(np.float64)) / np.exp(x.astype(np.float64)).sum()
    bias = (0.9 - p).astype(np.float32)
    rows = np.tile(x, (60, 1))
    rows[30:] += rng.normal(size=(30, E)).astype(np.float32) * 1e-6
    for best in (1, 2):
        for keep in {1, groups // 2, groups - 1}:
            _check(rows, min(6, keep * (E // groups)), bias=bias, score=score, n_group=groups, topk_group=keep, group_best=best, renorm=True)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups", [(16, 8), (64, 4), (24, 8), (320, 20)])
@pytest.mark.parametrize("size", [10.0, 300.0, 1e4, 1e6])
def test_groups_whose_keys_cancel(score, E, groups, size):
    """Biases of +size and -size in every group, in groups that share a number of lanes and in others: sums of about 1 whose error is that
    of their keys.  The logits of a token are nearly alike, so that the sums differ by less than an fp32 rounding of a key."""
    rng = np.random.default_rng(int(size) + E)
    bias = np.full(E, -2 * size)
    bias[::E // groups] = size
    bias[1::E // groups] = -size
    rows = rng.normal(size=(400, 1)) + rng.normal(size=(400, E)) * np.where(np.arange(400) % 2, 1e-5, 0.3)[:, None]
    _check(rows.astype(np.float32), min(6, E // groups), bias=bias, score=score, n_group=groups,
           topk_group=groups // 2, group_best=2, renorm=True)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups", [(16, 8), (64, 4), (24, 8)])
def test_groups_whose_sums_leave_the_range_of_fp32(score, E, groups):
    """Groups masked with the lowest float, or near it, are worth less than any other and more than one masked with -inf."""
    rng = np.random.default_rng(E)
    size, low = E // groups, float(np.finfo(np.float32).min)
    x = rng.normal(size=(20, E)).astype(np.float32)
    for worth in ([0, 0, -np.inf, low], [low, -np.inf, 0, 0], [-np.inf, low, -3e38, 0], [low, -3e38, -1.8e38, -np.inf]):
        bias = np.repeat(np.array(worth + [-np.inf] * (groups - 4)), size)
        for keep in range(1, groups):
            _check(x, min(16, keep * size), bias=bias, score=score, n_group=groups, topk_group=keep, group_best=2)
    bias = np.repeat(np.array([3e38, -low, -low, 0] + [-np.inf] * (groups - 4)), size)
    for keep in (1, 2, 3):
        _check(x, min(16, keep * size), bias=bias, score=score, n_group=groups, topk_group=keep, group_best=2)


@pytest.mark.parametrize("groups", [1, 4])
def test_scores_below_the_range_of_fp32_are_renormalised(groups):
    """The weights are ratios of scores: that the scores themselves are below what fp32 holds does not make them 0."""
    rng = np.random.default_rng(11)
    x = rng.normal(size=(12, 64)).astype(np.float32) - np.array([80, 87, 88, 89, 95, 103, 104, 150, 300, 600, 87.5, 100], np.float32)[:, None]
    x[10] -= np.arange(64, dtype=np.float32)
    x[11, ::5] = -np.inf
    kw = dict(n_group=groups, topk_group=min(groups, 2), renorm=True, scale=2.5)
    for dtype in ("f32", "bf16", "f16"):
        for bias in (None, rng.normal(size=64) * 0.1):
            _check(x, 6, dtype, bias, score="sigmoid", **kw)
    y = rng.normal(size=(12, 64)).astype(np.float32)                # experts that no token is to take, far above the others
    y[:, [3, 17, 40]] += np.array([50, 80, 87, 88, 95, 103, 104, 150, 300, 600, 87.5, 100], np.float32)[:, None]
    y[10] -= np.arange(64, dtype=np.float32)
    bias = rng.normal(size=64) * 0.1
    for mask in (-np.inf, -1e9):
        bias[[3, 17, 40]] = mask
        for dtype in ("f32", "f16"):
            _check(y, 6, dtype, bias, score="softmax", **kw)
