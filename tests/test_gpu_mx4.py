"""Microscaled 4-bit floats on the GPU - quantise, dequantise, pack, product, combine, and a layer of them - against the oracle in
64 bits.

Tolerances.  Quantisation is exact.  A product's terms are exact (two significant bits each, scales powers of two); K of them
are added in fp32 in some order, each addition off by at most 2^-23 of a partial sum (2^-24 rounded to nearest, 2^-23 if the adder cuts
off), and no partial sum is larger than the sum of magnitudes S: K 2^-23 S.  The gated form is silu(g) u with g and u off by
that: its bound is worked out by the oracle, plus 2^-20 of the value for expf, the quotient and two products (at most 8 roundings of
2^-23).  A result of 16 bits adds half a step, finfo.eps / 2 of the value, and of fp16 half the smallest subnormal."""
import numpy as np
import pytest

from oracle import mx4

pytestmark = pytest.mark.gpu


def _t(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _f64(t):
    return t.detach().double().cpu().numpy()


def _half_step(y, name):
    import torch
    if name == "f32":
        return 0.0
    i = torch.finfo(_dt(name))
    return np.abs(y) * i.eps / 2 + i.smallest_normal * i.eps / 2


# ---- quantise ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K,pad", [(1, 32, 0), (1, 2048, 0), (3, 96, 0), (5, 160, 8), (7, 416, 1), (129, 64, 33), (1000, 128, 0), (2, 4224, 24)])
def test_quantize_is_exact(dtype, rows, K, pad):
    import torch
    from paper_2512_12990_b200 import binding as B
    rng = np.random.default_rng(rows * K)
    x = _t(rng.normal(size=(rows, K + pad)) * np.exp2(rng.integers(-6, 6, size=(rows, 1)))).to(_dt(dtype))[:, pad:]
    codes, scale = B.slicemoe_mx4_quantize(x)
    c, s = mx4.quantize(_f64(x))
    assert np.array_equal(scale.cpu().numpy(), s) and np.array_equal(codes.cpu().numpy(), c)
    for out in ("f32", "bf16"):
        assert np.array_equal(_f64(B.slicemoe_mx4_dequantize(codes, scale, _dt(out))), mx4.dequantize(c, s))
    got = B.slicemoe_mx4_dequantize(codes, scale, torch.float16)
    assert torch.equal(got, _t(mx4.dequantize(c, s)).half())


def test_quantize_ties_saturation_and_extremes():
    import torch
    from paper_2512_12990_b200 import binding as B
    x = np.zeros((12, 64), np.float32)
    x[0, :8] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    x[1, :4] = [7.99, -7.0, -6.01, 6.0]
    x[2, 0] = 2.0 ** -149
    x[3, :2] = [2.0 ** -126, 2.0 ** -127]
    x[4, :2] = [3.4e38, 1e38]
    x[5, 0] = np.inf
    x[6, 40] = np.nan
    x[7, 3] = -np.inf
    x[8, :] = -0.0
    x[9, :2] = [1.0, 2.0 ** -30]
    x[10, :3] = [2.0 ** -120, 2.0 ** -123, -(2.0 ** -122)]
    x[11, :2] = [np.nextafter(np.float32(8), np.float32(0)), np.float32(1)]
    codes, scale = B.slicemoe_mx4_quantize(_t(x))
    c, s = mx4.quantize(x)
    assert np.array_equal(scale.cpu().numpy(), s) and np.array_equal(codes.cpu().numpy(), c)
    v = _f64(B.slicemoe_mx4_dequantize(codes, scale, torch.float32))
    assert np.array_equal(v, mx4.dequantize(c, s), equal_nan=True)
    assert np.isnan(v[5, :32]).all() and (v[5, 32:] == 0).all() and np.isnan(v[6, 32:]).all()


def test_dequantize_into_spaced_rows_leaves_the_rest():
    import torch
    from paper_2512_12990_b200 import binding as B
    x = torch.randn(9, 96, device="cuda")
    codes, scale = B.slicemoe_mx4_quantize(x)
    for off in (0, 1, 8):
        out = torch.full((9, 120), 7.0, device="cuda", dtype=torch.bfloat16)
        B.slicemoe_mx4_dequantize(codes, scale, out=out[:, off:off + 96])
        assert torch.equal(out[:, off:off + 96], B.slicemoe_mx4_dequantize(codes, scale, torch.bfloat16))
        assert (out[:, :off] == 7).all() and (out[:, off + 96:] == 7).all()


@pytest.mark.parametrize("N,K", [(1, 32), (16, 64), (17, 96), (100, 160), (128, 128), (129, 2048), (1408, 352)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_pack_keeps_every_code(N, K, dtype):
    import torch
    from paper_2512_12990_b200 import binding as B
    w, u = (torch.randn(N, K + 8, device="cuda").to(_dt(dtype))[:, 8:] for _ in range(2))
    m, g = B.slicemoe_mx4_pack(w), B.slicemoe_mx4_pack(w, u)
    for mat, part, src in ((m, 0, w), (g, 0, w), (g, 1, u)):
        codes, scale = B.slicemoe_mx4_quantize(src)
        c, s = B.slicemoe_mx4_unpack(mat, part)
        assert torch.equal(c, codes) and torch.equal(s, scale)
    for mat, rows in ((m, N), (g, 2 * N)):                         # what lies beyond the matrix is zeros
        assert int(torch.count_nonzero(mat.scale)) <= rows * K // 32


# ---- product -----------------------------------------------------------------------------------------------------
class Case:
    def __init__(self, T, k, E, N, K, gated=False, per_pair=False, seed=0, spread=2):
        from paper_2512_12990_b200 import binding as B
        rng = np.random.default_rng(seed + 1000 * T + K)
        rows = T * k if per_pair else T
        x = rng.normal(size=(rows, K)) * np.exp2(rng.integers(-spread, spread + 1, size=(rows, 1)))
        self.c, self.s = mx4.quantize(x)
        self.x = mx4.dequantize(self.c, self.s)
        w = [[rng.normal(size=(N, K)).astype(np.float32) * 0.1 for _ in range(2 if gated else 1)] for _ in range(E)]
        self.mats = [B.slicemoe_mx4_pack(*(_t(m) for m in ms)) for ms in w]
        values = [tuple(mx4.dequantize(*mx4.quantize(m)) for m in ms) for ms in w]
        self.values = values if gated else [v[0] for v in values]
        self.table = B.mx4_table(self.mats)
        self.ids = rng.integers(0, E, size=(T, k)).astype(np.int32)
        self.T, self.k, self.E, self.N, self.K, self.gated, self.per_pair = T, k, E, N, K, gated, per_pair
        if per_pair:
            self.x = self.x.reshape(T, k, K)
        self.ws = B.new_mx4_workspace(T, k, E, K)

    def dev(self):
        c, s = _t(self.c), _t(self.s)
        return (c.view(self.T, self.k, -1), s.view(self.T, self.k, -1)) if self.per_pair else (c, s)

    def run(self, dtype="f32", ids=None, **kw):
        from paper_2512_12990_b200 import binding as B
        ids = self.ids if ids is None else ids
        return B.slicemoe_mx4_product(self.table, *self.dev(), _t(ids), self.ws, dtype=_dt(dtype), **kw)

    def check(self, out, dtype="f32", ids=None):
        y, bound = mx4.product(self.x, self.values, self.ids if ids is None else ids)
        tol = self.K * 2.0 ** -23 * bound + (2.0 ** -20 * np.abs(y) if self.gated else 0.0) + 2.0 ** -126
        tol = tol + _half_step(np.abs(y) + tol, dtype)
        got, there = _f64(out), ~np.isnan(y)
        off = np.abs(got - y)[there] - tol[there]
        assert np.isfinite(got[there]).all() and (off <= 0).all(), f"beyond the bound by {off.max():.3e}"


@pytest.mark.parametrize("T,k,E,N,K", [
    (1, 1, 1, 1, 32), (1, 1, 1, 128, 64), (1, 6, 8, 100, 96), (1, 2, 4, 256, 2048), (3, 2, 5, 129, 160), (16, 4, 9, 64, 256), (17, 1, 1, 130, 416),
    (40, 3, 2, 200, 128), (224, 1, 1, 128, 128), (225, 1, 1, 128, 192), (300, 2, 3, 257, 288), (500, 2, 70, 48, 320), (2100, 4, 6, 32, 64), (5, 16, 40, 272, 1408),
    (20, 3, 200, 32, 96), (400, 2, 1024, 16, 64), (4, 2, 1000, 48, 64), (1, 2, 3, 40, 16384), (3, 2, 4, 24, 8192), (2, 1, 2, 20001, 64)])
@pytest.mark.parametrize("gated", [False, True])
def test_product_matches_the_oracle(T, k, E, N, K, gated):
    c = Case(T, k, E, N, K, gated)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N", [1, 33, 128, 200])
def test_product_in_16_bits_is_rounded_once(dtype, N):
    c = Case(37, 2, 4, N, 544, gated=N == 128)
    c.check(c.run(dtype), dtype)


@pytest.mark.parametrize("T,k,E", [(1, 6, 8), (33, 2, 3), (300, 3, 4), (1500, 4, 9)])
def test_product_of_a_row_per_pair(T, k, E):
    c = Case(T, k, E, 144, 224, per_pair=True)
    c.check(c.run())


def test_product_without_a_list():
    from paper_2512_12990_b200 import binding as B
    for T in (1, 64, 300):
        c = Case(T, 1, 1, 150, 256)
        c.ids[:] = 0
        out = B.slicemoe_mx4_product(c.table, *c.dev(), None, c.ws, dtype=_dt("f32"))
        assert out.shape == (T, 150)
        c.check(out[:, None])


@pytest.mark.parametrize("T", [1, 20, 700, 1200])
def test_every_pair_on_one_expert_and_the_same_expert_twice(T):
    c = Case(T, 4, 16, 64, 96)
    c.ids[:] = 11
    c.check(c.run())
    c.ids[:, 1] = 3
    c.check(c.run())


@pytest.mark.parametrize("T", [1, 20, 300, 1500])
def test_pairs_without_an_expert_are_left_as_they_were(T):
    import torch
    from paper_2512_12990_b200 import binding as B
    c = Case(T, 3, 5, 80, 64)
    ids = c.ids.copy()
    ids[:, 1] = -1
    ids[T // 2:, 0] = 5
    ids[T - 1, 2] = 2 ** 31 - 1
    out = torch.full((T, 3, 80), 77.0, device="cuda")
    c.run(ids=ids, out=out)
    c.check(out, ids=ids)
    assert (out[_t((ids < 0) | (ids >= 5))] == 77).all()
    assert B.slicemoe_get_status(c.ws) == B.STATUS_BAD_EXPERT_ID
    c.run()
    assert B.slicemoe_get_status(c.ws) == 0
    none = np.full_like(ids, -7)
    out.fill_(3.0)
    c.run(ids=none, out=out)
    assert (out == 3).all() and B.slicemoe_get_status(c.ws) == B.STATUS_BAD_EXPERT_ID


def test_a_table_entry_of_another_size_is_left_out():
    import torch
    from paper_2512_12990_b200 import binding as B
    c = Case(9, 2, 4, 96, 64)
    arr = (B.Mx4MatDesc * 4)(*[m.desc() for m in c.mats])
    arr[1].K = 128
    arr[2].codes = None
    c.table.device_array = torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8).cuda()
    out = torch.full((9, 2, 96), 5.0, device="cuda")
    c.run(out=out)
    left = (c.ids == 1) | (c.ids == 2)
    assert (out[_t(left)] == 5).all()
    c.check(out, ids=np.where(left, -1, c.ids).astype(np.int32))
    assert B.slicemoe_get_status(c.ws) == B.STATUS_BAD_EXPERT_ID


@pytest.mark.parametrize("T,k,E,K", [(1, 4, 6, 96), (50, 2, 4, 224), (700, 2, 3, 352)])
def test_a_row_depends_on_no_other_row_and_is_reproducible(T, k, E, K):
    import torch
    from paper_2512_12990_b200 import binding as B
    c = Case(T, k, E, 272, K, gated=True)
    a = c.run()
    assert torch.equal(a, c.run())
    ids, codes, scale = _t(c.ids), *c.dev()
    for t in {0, T // 2, T - 1}:
        one = B.slicemoe_mx4_product(c.table, codes[t:t + 1].contiguous(), scale[t:t + 1].contiguous(), ids[t:t + 1].contiguous(), c.ws, dtype=torch.float32)
        assert torch.equal(one[0], a[t])


@pytest.mark.parametrize("T", [2, 300])
def test_nan_blocks_and_bytes_behind_the_scales_stay_where_they_are(T):
    import torch
    from paper_2512_12990_b200 import binding as B
    c = Case(T, 2, 3, 64, 160)                       # five scales, three bytes behind them
    want = c.run()
    codes, scale = c.dev()
    scale[:, 5:] = 255
    got = B.slicemoe_mx4_product(c.table, codes, scale, _t(c.ids), c.ws, dtype=torch.float32)
    assert torch.equal(got, want)
    scale[1, 4] = 255
    got = B.slicemoe_mx4_product(c.table, codes, scale, _t(c.ids), c.ws, dtype=torch.float32)
    assert torch.isnan(got[1]).all()
    keep = [t for t in range(T) if t != 1]
    assert torch.equal(got[keep], want[keep])
    m = c.mats[int(c.ids[0, 0])]
    m.scale[16 * 3] = 255                            # row 3 of the matrix, first block
    got = B.slicemoe_mx4_product(c.table, *c.dev(), _t(c.ids), c.ws, dtype=torch.float32)
    hit = _t(c.ids == c.ids[0, 0])
    assert torch.isnan(got[hit][:, 3]).all() and torch.equal(got[~hit], want[~hit])
    rest = torch.arange(64, device="cuda") != 3
    assert torch.equal(got[hit][:, rest], want[hit][:, rest])


def test_rows_of_very_different_size():
    c = Case(24, 2, 3, 40, 256, spread=30)
    c.check(c.run())
    z = Case(4, 1, 2, 40, 128)
    z.c[:], z.s[:], z.x[:] = 0, 0, 0
    assert (_f64(z.run()) == 0).all()


@pytest.mark.parametrize("T", [1, 40, 1100])
def test_product_in_a_graph_on_another_stream(T):
    import torch
    from paper_2512_12990_b200 import binding as B
    c = Case(T, 4, 8, 160, 192, gated=True)
    (codes, scale), ids, out = c.dev(), _t(c.ids), torch.empty((T, 4, 160), device="cuda")
    ref = c.run()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        B.slicemoe_mx4_product(c.table, codes, scale, ids, c.ws, out=out)
    s.synchronize()
    assert torch.equal(out, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.slicemoe_mx4_product(c.table, codes, scale, ids, c.ws, out=out)
    ids.copy_(_t(((c.ids + 1) % 8).astype(np.int32)))
    for _ in range(3):
        out.zero_()
        g.replay()
    c.check(out, ids=((c.ids + 1) % 8).astype(np.int32))


def test_calls_on_two_streams_with_a_workspace_each():
    import torch
    from paper_2512_12990_b200 import binding as B
    c = Case(900, 3, 8, 160, 192, gated=True)
    (codes, scale), ids, ref = c.dev(), _t(c.ids), c.run()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [B.new_mx4_workspace(900, 3, 8) for _ in range(2)]
    outs = [torch.empty_like(ref) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, ws, out in zip(streams, spaces, outs):
            B.slicemoe_mx4_product(c.table, codes, scale, ids, ws, out=out, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs) and all(B.slicemoe_get_status(ws) == 0 for ws in spaces)


def test_a_call_right_behind_the_one_that_makes_its_input():
    """Kernels overlap; what one writes the next must see: quantise into the same buffers and multiply, over and over."""
    import torch
    from paper_2512_12990_b200 import binding as B
    for T in (1, 60, 700):
        c = Case(T, 2, 4, 96, 256)
        ids = _t(c.ids)
        xs = [torch.randn(T, 256, device="cuda") for _ in range(6)]
        refs = [B.slicemoe_mx4_product(c.table, *B.slicemoe_mx4_quantize(x), ids, c.ws, dtype=torch.float32) for x in xs]
        torch.cuda.synchronize()
        for _ in range(10):
            got = [B.slicemoe_mx4_product(c.table, *B.slicemoe_mx4_quantize(x), ids, c.ws, dtype=torch.float32) for x in xs]
            assert all(torch.equal(a, b) for a, b in zip(got, refs))


def test_workspace_of_a_larger_call_serves_smaller_ones():
    from paper_2512_12990_b200 import binding as B
    ws = B.new_mx4_workspace(2000, 4, 16)
    for T in (1, 900, 5, 2000):
        c = Case(T, 4, 16, 48, 96)
        c.ws = ws
        c.check(c.run())


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2512_12990_b200 import binding as B
    c = Case(4, 2, 3, 64, 96)
    (codes, scale), ids = c.dev(), _t(c.ids)
    bad = [dict(codes=codes[:, :32].contiguous()), dict(scale=scale[:2].contiguous()), dict(ids=ids.long()), dict(ids=ids[:3].contiguous()),
           dict(codes=codes.cpu()), dict(out=torch.empty((4, 2, 65), device="cuda")), dict(codes=codes.t().contiguous().t()), dict(dtype=torch.float64)]
    for kw in bad:
        a = dict(codes=codes, scale=scale, ids=ids, ws=c.ws, dtype=torch.float32) | kw
        with pytest.raises(ValueError):
            B.slicemoe_mx4_product(c.table, **a)
    with pytest.raises(B.SliceMoEError):
        B.slicemoe_mx4_product(c.table, codes, scale, ids, c.ws[:128], dtype=torch.float32)
    with pytest.raises(B.SliceMoEError):
        B.slicemoe_mx4_quantize(torch.zeros((2, 40), device="cuda"))
    with pytest.raises(ValueError):
        B.slicemoe_mx4_quantize(torch.zeros((64, 4), device="cuda").t())


# ---- combine -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (1, 6, 2048), (3, 4, 17), (50, 8, 264), (700, 2, 100), (9, 16, 8)])
@pytest.mark.parametrize("rd,od,base,listed", [("bf16", "bf16", True, False), ("f32", "f32", False, True), ("f16", "f32", True, True), ("bf16", "f16", False, False)])
def test_combine_matches_the_oracle(T, k, N, rd, od, base, listed):
    """k + 1 terms in fp32, each step off by 2^-24 of the sum of magnitudes; then half a step of the result's type."""
    import torch
    from paper_2512_12990_b200 import binding as B
    rng = np.random.default_rng(T + N)
    rows, w = _t(rng.normal(size=(T, k, N))).to(_dt(rd)), rng.normal(size=(T, k)).astype(np.float32)
    b = _t(rng.normal(size=(T, N))).to(_dt(od)) if base else None
    ids = rng.integers(-1, 5, size=(T, k)).astype(np.int32) if listed else None
    if listed:
        rows[_t((ids < 0) | (ids >= 4))] = float("nan")        # not to be read
    out = B.slicemoe_combine(rows, _t(w), None if ids is None else _t(ids), 4, b, _dt(od))
    r, keep = np.nan_to_num(_f64(rows)), w.astype(np.float64) * (1 if ids is None else (ids >= 0) & (ids < 4))
    y, mag = np.einsum("tkn,tk->tn", r, keep), np.einsum("tkn,tk->tn", np.abs(r), np.abs(keep))
    if base:
        y, mag = y + _f64(b), mag + np.abs(_f64(b))
    assert T > 100 or np.allclose(y, mx4.combine(_f64(rows), w, ids, 4, None if b is None else _f64(b)), rtol=1e-12, atol=1e-12)
    tol = (k + 1) * 2.0 ** -24 * mag
    tol = tol + _half_step(np.abs(y) + tol, od) + 2.0 ** -126
    assert (np.abs(_f64(out) - y) <= tol).all()
    if base:                                                    # in place
        same = B.slicemoe_combine(rows, _t(w), None if ids is None else _t(ids), 4, b, out=b)
        assert same is b and torch.equal(b, out)


@pytest.mark.parametrize("T,k,N,rd,od,listed", [(4100, 7, 2056, "bf16", "bf16", True), (12000, 3, 1672, "f16", "f32", False), (30001, 8, 264, "bf16", "f16", True)])
def test_combine_of_more_rows_than_l2_holds(T, k, N, rd, od, listed):
    """The same bound, in fp64 on the device; and in place."""
    import torch
    from paper_2512_12990_b200 import binding as B
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    rows = torch.randn(T, k, N, device="cuda", generator=gen).to(_dt(rd))
    w, base = torch.randn(T, k, device="cuda", generator=gen), torch.randn(T, N, device="cuda", generator=gen).to(_dt(od))
    ids = torch.randint(-1, 6, (T, k), device="cuda", generator=gen, dtype=torch.int32) if listed else None
    keep = w.double() if ids is None else w.double() * ((ids >= 0) & (ids < 5))
    y = torch.einsum("tkn,tk->tn", rows.double(), keep) + base.double()
    mag = torch.einsum("tkn,tk->tn", rows.double().abs(), keep.abs()) + base.double().abs()
    tol = (k + 1) * 2.0 ** -24 * mag + 2.0 ** -126
    if od != "f32":
        tol = tol + (y.abs() + tol) * torch.finfo(_dt(od)).eps / 2 + 2.0 ** -25
    if ids is not None:
        rows[(ids < 0) | (ids >= 5)] = float("nan")
    out = B.slicemoe_combine(rows, w, ids, 5, base, _dt(od))
    assert ((out.double() - y).abs() <= tol).all()
    none = B.slicemoe_combine(rows, w, ids, 5, None, _dt(od))
    assert ((none.double() - (y - base.double())).abs() <= tol + mag * 2.0 ** -8).all()
    B.slicemoe_combine(rows, w, ids, 5, base, out=base)
    assert torch.equal(base, out)


# ---- a layer of them ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T", [1, 5, 130, 1200])
def test_a_layer_from_logits_to_output(T):
    """Route, quantise, gated product, quantise, down product, combine.  Each step is compared with the oracle on the step before's own
    output, so that a rounding to four bits that falls either way does not carry over; then the one call that makes them all."""
    import torch
    from paper_2512_12990_b200 import binding as B
    hidden, inter, E, k = 256, 160, 12, 3
    rng = np.random.default_rng(T)
    up = Case(T, k, E, inter, hidden, gated=True, seed=1)
    down = Case(T, k, E, hidden, inter, per_pair=True, seed=2)
    x = _t(rng.normal(size=(T, hidden))).bfloat16()
    logits, bias = _t(rng.normal(size=(T, E)).astype(np.float32)), _t((rng.normal(size=E) * 0.05).astype(np.float32))
    ids, w, _ = B.slicemoe_route_scored(logits, k, score="sigmoid", bias=bias, n_group=4, topk_group=2, group_best=2, renorm=True, scale=2.5)
    ids_o, w_o, _ = mx4.route_scored(_f64(logits), k, "sigmoid", _f64(bias), 4, 2, 2, True, 2.5)
    assert np.array_equal(ids.cpu().numpy(), ids_o) and np.allclose(_f64(w), w_o, rtol=2e-6)
    up.c, up.s = (t.cpu().numpy() for t in B.slicemoe_mx4_quantize(x))
    up.x, up.ids = mx4.dequantize(up.c, up.s), ids_o
    h = up.run("bf16")
    up.check(h, "bf16")
    hc, hs = B.slicemoe_mx4_quantize(h)
    assert hc.shape == (T, k, inter // 2) and hs.shape == (T, k, 8)
    c, s = mx4.quantize(_f64(h).reshape(T * k, inter))
    assert np.array_equal(hc.cpu().numpy().reshape(T * k, -1), c) and np.array_equal(hs.cpu().numpy().reshape(T * k, -1), s)
    down.c, down.s, down.x, down.ids = c, s, mx4.dequantize(c, s).reshape(T, k, inter), ids_o
    y = down.run("bf16")
    down.check(y, "bf16")
    out = B.slicemoe_combine(y, w, ids, E, x, torch.bfloat16)
    want = mx4.combine(_f64(y), _f64(w), ids_o, E, _f64(x))
    mag = mx4.combine(np.abs(_f64(y)), np.abs(_f64(w)), ids_o, E, np.abs(_f64(x)))
    assert (np.abs(_f64(out) - want) <= 4 * 2.0 ** -24 * mag + _half_step(np.abs(want) + 4 * 2.0 ** -24 * mag, "bf16")).all()
    ws = B.new_mx4_workspace(T, k, E)
    assert torch.equal(B.mx4_expert_ffn(up.table, down.table, x, ids, w, ws, base=x), out)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    other = B.mx4_expert_ffn(up.table, down.table, x, ids, w, ws, base=x, stream=st)
    st.synchronize()
    assert torch.equal(other, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        again = B.mx4_expert_ffn(up.table, down.table, x, ids, w, ws, base=x)
    g.replay()
    g.replay()
    assert torch.equal(again, out)
    assert B.slicemoe_get_status(ws) == 0


@pytest.mark.parametrize("T,k,E,N,K,dtype", [(700, 2, 3, 1920, 1408, "f32"), (2048, 4, 60, 704, 2048, "bf16"), (3000, 6, 64, 512, 1056, "f32")])
def test_long_prompts_agree_with_single_rows(T, k, E, N, K, dtype):
    """Many items to a CTA, rings that go round often: sampled rows against calls of one token, bit for bit, and against the
    dequantised product in fp64."""
    import torch
    from paper_2512_12990_b200 import binding as B
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    w = [torch.randn(2 * N, K, device="cuda", generator=gen) * 0.1 for _ in range(E)]
    table = B.mx4_table([B.slicemoe_mx4_pack(m[:N], m[N:]) for m in w])
    codes, scale = B.slicemoe_mx4_quantize(torch.randn(T, K, device="cuda", generator=gen))
    ids = torch.rand(T, E, device="cuda", generator=gen).topk(k, -1).indices.int()
    ws = B.new_mx4_workspace(T, k, E)
    out = B.slicemoe_mx4_product(table, codes, scale, ids, ws, dtype=_dt(dtype))
    assert B.slicemoe_get_status(ws) == 0
    for t in range(0, T, T // 37):
        one = B.slicemoe_mx4_product(table, codes[t:t + 1].contiguous(), scale[t:t + 1].contiguous(), ids[t:t + 1].contiguous(), ws, dtype=_dt(dtype))
        assert torch.equal(one[0], out[t])
    x = B.slicemoe_mx4_dequantize(codes, scale, torch.float32).double()
    for e in range(0, E, max(1, E // 5)):
        at = torch.nonzero(ids == e)
        m = B.slicemoe_mx4_dequantize(*B.slicemoe_mx4_quantize(w[e]), torch.float32).double()
        g, u = (x[at[:, 0]] @ m.T).split(N, 1)
        mg, mu = (x[at[:, 0]].abs() @ m.abs().T).split(N, 1)
        y = torch.nn.functional.silu(g) * u
        tol = K * 2.0 ** -23 * (1.1 * u.abs() * mg + torch.nn.functional.silu(g).abs() * mu) + 2.0 ** -20 * y.abs()
        tol = tol + torch.from_numpy(np.asarray(_half_step((y.abs() + tol).cpu().numpy(), dtype))).cuda()
        assert ((out[at[:, 0], at[:, 1]].double() - y).abs() <= tol).all()


@pytest.mark.parametrize("T,k,E,N,K", [(1, 1, 1, 40, 16384), (3, 2, 4, 24, 16384), (16, 2, 3, 130, 8192), (300, 2, 3, 72, 4160), (230, 1, 2, 40, 16384),
                                       (3, 2, 3, 129, 2048), (700, 3, 5, 64, 992)])
def test_sums_that_fp32_holds_exactly_come_out_exact(T, k, E, N, K):
    """Every block's scale is 1: a product of two values is a whole number of quarters, 144 of them at most, and K of them stay below 2^24
    quarters.  Whatever the order, no sum is rounded: the result is that of whole numbers, and a block of K that is skipped, doubled or scaled
    wrongly anywhere shows."""
    import torch
    from paper_2512_12990_b200 import binding as B
    assert K * 144 < 2 ** 24
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + K)
    grid = torch.tensor(np.concatenate([mx4.VALUES, -mx4.VALUES]), device="cuda")

    def values(rows):                                # the first of a block 4, 6, -4 or -6: exponent 2, scale 1
        c = torch.randint(0, 16, (rows, K // 32, 32), device="cuda", generator=gen)
        c[:, :, 0] = (c[:, :, 0] & 9) | 6
        return grid[c].reshape(rows, K)

    x, w = values(T), [values(N) for _ in range(E)]
    codes, scale = B.slicemoe_mx4_quantize(x.float())
    assert (scale[:, :K // 32] == 127).all() and torch.equal(B.slicemoe_mx4_dequantize(codes, scale, torch.float32).double(), x)
    table = B.mx4_table([B.slicemoe_mx4_pack(m.float()) for m in w])
    ids = torch.randint(0, E, (T, k), device="cuda", generator=gen, dtype=torch.int32)
    out = B.slicemoe_mx4_product(table, codes, scale, ids, B.new_mx4_workspace(T, k, E, K), dtype=torch.float32)
    want = torch.empty((T, k, N), dtype=torch.float64, device="cuda")
    for e in range(E):
        at = torch.nonzero(ids == e)
        want[at[:, 0], at[:, 1]] = x[at[:, 0]] @ w[e].T
    assert torch.equal(out.double(), want)


# ---- long lists and large arrays -----------------------------------------------------------------------------------
@pytest.mark.parametrize("T,k,E,listed", [(16384, 8, 16, True), (30000, 1, 5, True), (20000, 3, 300, True), (70000, 16, 64, True), (130000, 1, 1, False)])
def test_lists_of_many_pairs(T, k, E, listed):
    """Up to a million pairs: blocks of the kernels ahead take 64, 128 and more of them, in more than one go.  Sums are whole numbers of
    quarters, so that every value is known exactly."""
    import torch
    from paper_2512_12990_b200 import binding as B
    N, K = 24, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    grid = torch.tensor(np.concatenate([mx4.VALUES, -mx4.VALUES]), device="cuda")

    def values(rows):
        c = torch.randint(0, 16, (rows, K // 32, 32), device="cuda", generator=gen)
        c[:, :, 0] = (c[:, :, 0] & 9) | 6
        return grid[c].reshape(rows, K)

    x, w = values(T), torch.stack([values(N) for _ in range(E)])
    codes, scale = B.slicemoe_mx4_quantize(x.float())
    table, ws = B.mx4_table([B.slicemoe_mx4_pack(m.float()) for m in w]), B.new_mx4_workspace(T, k, E, K)
    ids = torch.randint(0, E, (T, k), device="cuda", generator=gen, dtype=torch.int32) if listed else torch.zeros((T, 1), device="cuda", dtype=torch.int32)
    if listed:
        ids[::97, 0] = -1
    out = torch.full((T, k, N) if listed else (T, N), 77.0, device="cuda")
    B.slicemoe_mx4_product(table, codes, scale, ids if listed else None, ws, out=out)
    out = out.view(T, k, N)
    for e in range(E):
        at = torch.nonzero(ids == e)
        assert torch.equal(out[at[:, 0], at[:, 1]].double(), x[at[:, 0]] @ w[e].T)
    assert (out[ids < 0] == 77).all() and B.slicemoe_get_status(ws) == (B.STATUS_BAD_EXPERT_ID if listed else 0)


def test_arrays_of_more_than_2_31_elements():
    """Results, codes, rows and spacings whose places pass 32 bits: what lies at their ends against calls of those rows alone."""
    import torch
    from paper_2512_12990_b200 import binding as B
    # quantise and back: 4.3e9 values, 2.1e9 bytes of codes
    rows, K = 70000, 61440
    x = torch.empty((rows, K), device="cuda", dtype=torch.bfloat16).normal_()
    codes, scale = B.slicemoe_mx4_quantize(x)
    back = B.slicemoe_mx4_dequantize(codes, scale, torch.bfloat16)
    assert codes.numel() > 2 ** 31 and x.numel() > 2 ** 32
    for at in (slice(0, 3), slice(34949, 34955), slice(69899, 69906), slice(rows - 4, rows)):    # 2^31 values: row 34,952; 2^32: row 69,905
        c, s = B.slicemoe_mx4_quantize(x[at].contiguous())
        assert torch.equal(codes[at], c) and torch.equal(scale[at], s)
        assert torch.equal(back[at], B.slicemoe_mx4_dequantize(c, s, torch.bfloat16))
    del back, codes, scale
    # rows 2^31 and more elements apart
    wide = x.view(-1)[:2 ** 32].view(2, 2 ** 31)
    for off in (0, 5):
        part = wide[:, off:off + 256]
        want = part.contiguous()
        assert all(torch.equal(a, b) for a, b in zip(B.slicemoe_mx4_quantize(part), B.slicemoe_mx4_quantize(want)))
        assert all(torch.equal(a, b) for a, b in zip(B.slicemoe_route_scored(part, 8, score="sigmoid"), B.slicemoe_route_scored(want, 8, score="sigmoid")))
    # combine: 4.3e9 values in
    T, k, N = 70000, 4, 15360
    big, w = x.view(T, k, N), torch.randn(T, k, device="cuda")
    y = B.slicemoe_combine(big, w, dtype=torch.bfloat16)
    odd = B.slicemoe_combine(x.view(-1)[1:1 + (T - 1) * k * N].view(T - 1, k, N), w[1:].contiguous(), dtype=torch.float32)    # off 16 bytes
    for at in (slice(0, 3), slice(34949, 34955), slice(69899, 69906), slice(T - 4, T - 1)):
        assert torch.equal(y[at], B.slicemoe_combine(big[at].contiguous(), w[at].contiguous(), dtype=torch.bfloat16))
        rows_at = x.view(-1)[1 + at.start * k * N:1 + at.stop * k * N].clone().view(-1, k, N)
        assert torch.equal(odd[at], B.slicemoe_combine(rows_at, w[1:][at].contiguous(), dtype=torch.float32))
    del x, big, y, odd, wide, part
    # product: 2.4e9 results
    T, k, E, N, K = 18000, 8, 2, 16384 + 200, 96
    table = B.mx4_table([B.slicemoe_mx4_pack(torch.randn(N, K, device="cuda")) for _ in range(E)])
    codes, scale = B.slicemoe_mx4_quantize(torch.randn(T, K, device="cuda"))
    ids, ws = torch.randint(0, E, (T, k), device="cuda", dtype=torch.int32), B.new_mx4_workspace(T, k, E, K)
    out = B.slicemoe_mx4_product(table, codes, scale, ids, ws, dtype=torch.bfloat16)
    assert out.numel() > 2 ** 31 and B.slicemoe_get_status(ws) == 0
    for at in (slice(0, 3), slice(16184, 16190), slice(T - 3, T)):     # 2^31 values: token 16,187
        one = B.slicemoe_mx4_product(table, codes[at].contiguous(), scale[at].contiguous(), ids[at].contiguous(), ws, dtype=torch.bfloat16)
        assert torch.equal(out[at], one)
