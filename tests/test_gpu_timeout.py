"""The time-out path of the decode kernel, exercised without hanging or faulting anything: the workspace is
told to treat the intermediate vector that the CTAs exchange between the two phases as never complete,
and that no device-side wait may last longer than about a millisecond.  The kernel has to return by itself,
report SLICEMOE_STATUS_WAIT_TIMEOUT, and the same workspace has to work again once it is re-initialised."""
import time

import numpy as np
import pytest

from oracle import moe
from paper_2512_12990_b200 import synth
from tests import helpers as H

pytestmark = pytest.mark.gpu


def test_wait_timeout_is_reported_and_the_workspace_recovers():
    import torch
    from paper_2512_12990_b200 import binding as B
    sh = synth.SHAPES["tiny"]
    layer = H.Layer(sh, range(sh.n_experts))
    logits = synth.router_logits_normal(sh.seed, ("timeout-logits",), 1, sh.n_experts)
    ids, w, _ = moe.route_topk(logits, sh.top_k)
    prec = (ids >= 4).astype(np.uint8)
    xbits, x64 = H.x_inputs(sh, 1, "timeout-x")
    x = H.to_dev_bf16(xbits)
    args = (torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(prec).cuda(),
            torch.from_numpy(w.astype(np.float32)).cuda())
    y_ref = moe.expert_ffn(x64, layer.oracle_list(), ids, prec, w)

    # a normal call first
    y = B.slicemoe_expert_ffn(layer.cshape, layer.experts_tbl, x, *args, layer.ws)
    torch.cuda.synchronize()
    assert B.slicemoe_get_status(layer.ws) == 0
    H.assert_close(y.cpu().numpy(), y_ref, "before the time-out")

    # one arrival that never comes, and a limit of 2 million cycles (about a millisecond)
    B.slicemoe_workspace_set_wait(layer.ws, 2_000_000, extra_arrivals=1)
    y_bad = torch.full((1, sh.hidden), 7.0, dtype=torch.float32, device="cuda")
    t0 = time.time()
    B.slicemoe_expert_ffn(layer.cshape, layer.experts_tbl, x, *args, layer.ws, y=y_bad)
    torch.cuda.synchronize()
    assert time.time() - t0 < 5.0, "the kernel must return by itself"
    status = B.slicemoe_get_status(layer.ws)
    assert status & B.STATUS_WAIT_TIMEOUT
    assert torch.all(y_bad == 7.0), "the output is not written when h was never complete"

    # re-initialised, the workspace works again (and the limit is back to its default)
    B.lib().slicemoe_workspace_init(layer.ws.data_ptr(), layer.ws.numel(), None)
    y2 = B.slicemoe_expert_ffn(layer.cshape, layer.experts_tbl, x, *args, layer.ws)
    torch.cuda.synchronize()
    assert B.slicemoe_get_status(layer.ws) == 0
    assert torch.equal(y2, y), "same bits as before the time-out"


@pytest.mark.parametrize("T,limit", [(4, 2_000_000), (17, 200_000)])
def test_wait_timeout_of_several_tokens(T, limit):
    """The same for the kernels that take several tokens at once, in one pass and in two: their waits for the weights run
    out, y stays as it was, and the workspace works again.  (200,000 cycles: less than what the producers give copies on
    their way, which is a floor of their own.)"""
    import torch
    from paper_2512_12990_b200 import binding as B
    sh = synth.Shape("batch-timeout", 512, 384, 12, 3, 64, n_shared=1, shared_inter=256, n_layers=1, seed=7300)
    layer = H.Layer(sh, range(sh.n_experts))
    rng = np.random.default_rng(T)
    ids = np.stack([rng.permutation(sh.n_experts)[:sh.top_k] for _ in range(T)]).astype(np.int32)
    lists = [torch.from_numpy(a).cuda() for a in (ids, rng.integers(0, 2, ids.shape).astype(np.uint8), rng.random(ids.shape).astype(np.float32))]
    x = H.to_dev_bf16(H.x_inputs(sh, T, "batch-timeout-x")[0])

    def call(y=None):
        y = B.slicemoe_layer(layer.cshape, layer.experts_tbl, layer.shared_tbl, None, x, *lists, layer.ws, y=y)
        torch.cuda.synchronize()
        return y

    y = call()
    assert B.slicemoe_get_status(layer.ws) == 0
    B.slicemoe_workspace_set_wait(layer.ws, limit, extra_arrivals=1)
    y_bad = torch.full((T, sh.hidden), 7.0, device="cuda")
    t0 = time.time()
    call(y_bad)
    assert time.time() - t0 < 5.0, "the kernels must return by themselves"
    assert B.slicemoe_get_status(layer.ws) == B.STATUS_WAIT_TIMEOUT
    assert torch.all(y_bad == 7.0)
    B.lib().slicemoe_workspace_init(layer.ws.data_ptr(), layer.ws.numel(), None)
    assert torch.equal(call(), y) and B.slicemoe_get_status(layer.ws) == 0


def test_a_short_limit_is_not_spent_on_the_launch_before():
    """The down projection of several tokens starts while gate/up still runs.  Its waits are counted from the end of that
    launch: a limit of 40,000 cycles, 20 us, lets a pass through whose gate/up alone takes longer."""
    import torch
    from paper_2512_12990_b200 import binding as B
    E, k, T, h, inter = 16, 4, 16, 4096, 1408
    g = torch.Generator(device="cuda").manual_seed(5)
    pack = lambda n, c: B.slicemoe_pack(torch.randn((n, c), generator=g, device="cuda").mul_(0.02), 32)
    experts = [dict(gate=pack(inter, h), up=pack(inter, h), down=pack(h, inter)) for _ in range(E)]
    table, shape = B.expert_table(experts), B.make_shape(h, inter, E, k, 32)
    ws = B.new_workspace(shape)
    ids = torch.stack([torch.randperm(E, generator=g, device="cuda")[:k] for _ in range(T)]).to(torch.int32)
    prec = torch.randint(0, 2, (T, k), generator=g, device="cuda").to(torch.uint8)
    w, x = torch.rand((T, k), generator=g, device="cuda"), torch.randn((T, h), generator=g, device="cuda").bfloat16()
    want = B.slicemoe_layer(shape, table, None, None, x, ids, prec, w, ws)
    B.slicemoe_workspace_set_wait(ws, 40_000)
    for _ in range(20):
        assert torch.equal(B.slicemoe_layer(shape, table, None, None, x, ids, prec, w, ws), want)
    assert B.slicemoe_get_status(ws) == 0


@pytest.mark.parametrize("T", [2, 300, 3000])
def test_the_product_of_microscaled_experts_gives_up_by_itself(T):
    """The waits for weights that are never brought run out: the call returns, the status says so, and the workspace serves on once
    the switch is off again."""
    import torch
    from paper_2512_12990_b200 import binding as B
    E, k, N, K = 4, 2, 256, 1024
    mats = [B.slicemoe_mx4_pack(torch.randn(N, K, device="cuda")) for _ in range(E)]
    table, ws = B.mx4_table(mats), B.new_mx4_workspace(T, k, E)
    codes, scale = B.slicemoe_mx4_quantize(torch.randn(T, K, device="cuda"))
    ids = torch.randint(0, E, (T, k), device="cuda", dtype=torch.int32)
    ref = B.slicemoe_mx4_product(table, codes, scale, ids, ws, dtype=torch.float32)
    assert B.slicemoe_get_status(ws) == 0
    B.slicemoe_workspace_set_wait(ws, 200000, 1)
    B.slicemoe_mx4_product(table, codes, scale, ids, ws, dtype=torch.float32)
    assert B.slicemoe_get_status(ws) == B.STATUS_WAIT_TIMEOUT
    B.slicemoe_workspace_set_wait(ws, 0, 0)
    assert torch.equal(B.slicemoe_mx4_product(table, codes, scale, ids, ws, dtype=torch.float32), ref)
    assert B.slicemoe_get_status(ws) == 0


@pytest.mark.parametrize("T,k", [(2, 2), (40, 2), (260, 2), (5000, 2)])
def test_a_short_limit_of_the_product_is_not_spent_on_the_launch_before(T, k):
    """The product starts while the kernel before it still runs - here one of one block that goes through 2^20 values of K, longer
    than the limit, and lets the next start at once.  Its waits are counted from the end of that: a limit of 200,000 cycles, 100 us, lets it
    through.  (Rows resident in shared memory, planned by a warp or by all; placed by one kernel, by two.)"""
    import torch
    from paper_2512_12990_b200 import binding as B
    E, N, K, far = 4, 256, 512, 1 << 20
    long_table = B.mx4_table([B.slicemoe_mx4_pack(torch.randn(16, far, device="cuda"))])
    long_x, long_ws = B.slicemoe_mx4_quantize(torch.randn(1, far, device="cuda")), B.new_mx4_workspace(1, 1, 1, far)
    table, ws = B.mx4_table([B.slicemoe_mx4_pack(torch.randn(N, K, device="cuda")) for _ in range(E)]), B.new_mx4_workspace(T, k, E, K)
    x = B.slicemoe_mx4_quantize(torch.randn(T, K, device="cuda"))
    ids = torch.randint(0, E, (T, k), device="cuda", dtype=torch.int32)
    want = B.slicemoe_mx4_product(table, *x, ids, ws, dtype=torch.float32)
    first = B.slicemoe_mx4_product(long_table, *long_x, None, long_ws, dtype=torch.float32)
    B.slicemoe_workspace_set_wait(ws, 200_000)
    torch.cuda.synchronize()
    for _ in range(5):
        again = B.slicemoe_mx4_product(long_table, *long_x, None, long_ws, dtype=torch.float32)
        out = B.slicemoe_mx4_product(table, *x, ids, ws, dtype=torch.float32)
        assert torch.equal(out, want) and torch.equal(again, first)
    assert B.slicemoe_get_status(ws) == 0 and B.slicemoe_get_status(long_ws) == 0
