"""The context that products use which are given none."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def rows(n_rows, n, seed):
    import paper_2503_00245_b200 as P
    return P.fp4_quantize(torch.randn(n_rows, n, generator=torch.Generator().manual_seed(seed)).cuda())


def test_a_failure_is_reported_once():
    import paper_2503_00245_b200 as P
    from paper_2503_00245_b200 import binding as B
    a, w, at = rows(5, 64, 1), rows(16, 64, 2), torch.tensor([0, 5], dtype=torch.int32).cuda()
    out = P.fp4_product(a, w, at)
    assert P.fp4_check() == 0
    # (that context is one of 8 x 8 x one expert: an expert that is not there sets its status word)
    gu, down = rows(64, 8, 3), rows(8, 8, 4)
    x, y = (torch.zeros(1, 8, dtype=torch.bfloat16).cuda() for _ in range(2))
    cfg = B.make_config(8, 8, 1, 1)
    ws = torch.empty(B.moe_fp4_workspace_bytes(cfg, 1), dtype=torch.uint8).cuda()
    B.moe_fp4_experts(P.layer._shared_ctx(), x, 1, gu.c, down.c, torch.ones(1, 1, dtype=torch.int32).cuda(), torch.ones(1, 1).cuda(), y, ws)
    assert P.fp4_check() == 6
    assert P.fp4_check() == 0 and torch.equal(P.fp4_product(a, w, at), out) and P.fp4_check() == 0



def in_a_thread(call):
    """What a call returns that is the first one of a thread of its own."""
    import threading
    got = []

    def body():
        try:
            got.append(call())
        except Exception as e:
            got.append(e)
    t = threading.Thread(target=body)
    t.start()
    t.join()
    if isinstance(got[0], Exception):
        raise got[0]
    return got[0]


@pytest.mark.parametrize("n_rows", [3, 40])
def test_products_are_a_threads_first_calls(n_rows):
    """Its host side encodes tensor maps before it launches anything."""
    import paper_2503_00245_b200 as P
    a, w, at = rows(n_rows, 64, 1), rows(16, 64, 2), torch.tensor([0, n_rows], dtype=torch.int32).cuda()
    out = torch.zeros(n_rows, 16, dtype=torch.bfloat16).cuda()
    want = P.fp4_product(a, w, at)
    in_a_thread(lambda: P.fp4_product(a, w, at, out=out))
    torch.cuda.synchronize()
    assert torch.equal(out, want) and P.fp4_check() == 0


@pytest.mark.parametrize("rank,fp4", [(0, True), (0, False), (64, False)])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_layers_are_a_threads_first_calls(rank, fp4, T):
    import paper_2503_00245_b200 as P
    from synth import workloads as W
    shape = W.LayerShape("thread", 0, 256, 384, 8, 2, rank)
    t = W.make_layer(shape, T, device="cuda")
    kw = dict(d_model=256, d_ff=384, n_experts=8, top_k=2)
    if fp4:
        lay = P.MoELayer(256, 384, 8, 2, t["w_router"], t["b_router"], fp4=P.pack_fp4(t["w_gate"], t["w_up"], t["w_down"]), max_tokens=T)
    else:
        lay = P.MoELayer.from_math_layout(kw, t, x_dtype=t["x"].dtype, max_tokens=T)
    want, y = lay.forward(t["x"]).clone(), torch.zeros_like(t["x"])
    idx, wt, _ = lay.route(t["x"])
    torch.cuda.synchronize()
    in_a_thread(lambda: lay.forward(t["x"], y))
    torch.cuda.synchronize()
    assert torch.equal(y, want) and lay.check() == 0
    if fp4:
        y.zero_()
        torch.cuda.synchronize()
        in_a_thread(lambda: lay.fp4.forward(t["x"], idx, wt, y))
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_threads_on_one_context_count_every_launch():
    """Products on one context may overlap, so may their host sides (a call through ctypes runs without the interpreter's lock)."""
    import threading

    import paper_2503_00245_b200 as P
    from paper_2503_00245_b200 import binding as B
    a, w, at = rows(1, 64, 1), rows(8, 64, 2), torch.tensor([0, 1], dtype=torch.int32).cuda()
    want = P.fp4_product(a, w, at)
    ctx = B.moe_create(B.make_config(8, 8, 1, 1))
    threads, calls = 8, 2000
    outs = [torch.zeros(1, 8, dtype=torch.bfloat16).cuda() for _ in range(threads)]

    def work(i):
        for _ in range(calls):
            P.fp4_product(a, w, at, out=outs[i], ctx=ctx)
    before = B.moe_launch_count(ctx)
    pool = [threading.Thread(target=work, args=(i,)) for i in range(threads)]
    for t in pool:
        t.start()
    for t in pool:
        t.join()
    assert B.moe_launch_count(ctx) - before == threads * calls
    assert B.moe_check(ctx) == 0 and all(torch.equal(o, want) for o in outs)
    B.moe_destroy(ctx)
