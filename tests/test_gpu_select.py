"""Expert selection from logits (moe_select) against the checker: indices exactly, weights to their rounding.

Tolerance of a weight, relative: 2^-20.  It is one rounding to fp32 (2^-24) of a quotient; its numerator is formed in 64 bits, its
denominator, where it is a softmax's over all experts, may be a sum of fp32 exponentials: e^d is off by (|d| + 2) 2^-24 of itself
(rounded argument, two units in the last place), at most (1 / e + 2) 2^-24 of the largest term, and the sum rounds at most 13 times:
together below 16 * 2^-24.
"""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as Q

pytestmark = pytest.mark.gpu
RTOL = 2.0 ** -20


def run(l, bias=None, **rule):
    import paper_2503_00245_b200 as P
    kw = dict(rule)
    r = P.SelectRule(l.shape[1], kw.pop("k"), scoring=kw.pop("scoring", "softmax"), groups=kw.pop("groups", 1), groups_kept=kw.pop("kept", 1), **kw)
    idx, w = P.select_experts(l, r, bias)
    return idx.cpu().numpy(), w.cpu().numpy()


def check(l, bias=None, **rule):
    idx, w = run(l, bias, **rule)
    want, ww = Q.select(l.double().cpu().numpy(), bias=None if bias is None else bias.double().cpu().numpy(), **rule)
    assert np.array_equal(idx, want)
    assert np.all(np.abs(w - ww) <= RTOL * np.abs(ww) + 1e-45)
    return idx, w


def logits(T, E, dtype=torch.float32, seed=0, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * sigma).to(dtype).cuda()


RULES = [dict(k=2), dict(k=2, renorm=False, scale=2.5), dict(k=1, scoring="sigmoid"), dict(k=8, scoring="sigmoid", scale=0.5),
         dict(k=4, scoring="sigmoid", renorm=False)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("T,E", [(1, 8), (3, 9), (64, 8), (37, 31), (33, 32), (17, 33), (129, 64), (5, 65), (300, 256), (41, 250)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_no_groups(T, E, rule, dtype, with_bias):
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)).mul(0.2).cuda() if with_bias else None
    check(logits(T, E, dtype, T), bias, **rule)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,kept,k,top", [(256, 8, 4, 8, 2), (256, 16, 3, 7, 1), (64, 8, 8, 8, 2), (16, 4, 1, 4, 2), (96, 3, 2, 5, 2),
                                                 (75, 3, 1, 8, 1), (32, 32, 8, 8, 1), (64, 32, 2, 4, 2), (6, 2, 1, 3, 1), (250, 25, 9, 6, 2)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_groups(E, groups, kept, k, top, scoring, dtype, with_bias):
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)).mul(0.1).cuda() if with_bias else None
    check(logits(97, E, dtype, E + k), bias, k=k, scoring=scoring, groups=groups, kept=kept, group_top=top)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,kept", [(1, 1), (4, 2)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_equal_logits_go_to_the_lower_index(scoring, groups, kept, with_bias):
    g = torch.Generator().manual_seed(5)
    l = torch.randint(-2, 3, (200, 64), generator=g).float().cuda()
    bias = torch.randint(0, 2, (64,), generator=g).float().mul(0.25).cuda() if with_bias else None
    check(l, bias, k=8, scoring=scoring, groups=groups, kept=kept, group_top=2 if groups > 1 else 1)
    check(torch.zeros(3, 64, device="cuda"), None, k=8, scoring=scoring, groups=groups, kept=kept)
    check(torch.tensor([[0.0, -0.0, 0.0, -0.0]], device="cuda"), None, k=3, scoring=scoring)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_keys_next_to_each_other(scoring):
    """Logits one unit in the last place apart, and keys that only more than 32 bits tell apart."""
    one = torch.ones(50, 16)
    step = torch.arange(16).float().mul(2.0 ** -23)
    g = torch.Generator().manual_seed(8)
    for t in range(50):
        one[t] += step[torch.randperm(16, generator=g)]
    check(one.cuda(), None, k=8, scoring=scoring)
    check(one.cuda(), torch.full((16,), 0.5).cuda(), k=8, scoring=scoring)
    big = torch.full((16,), 1000.0)
    check((one * 3).cuda(), big.cuda(), k=8, scoring=scoring)
    check(logits(64, 256, seed=9), torch.full((256,), 100.0).cuda(), k=8, scoring=scoring, groups=8, kept=3, group_top=2)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
def test_switched_off_experts_and_rows_with_nothing_left(scoring, with_bias):
    inf = float("inf")
    l = logits(12, 24, seed=2)
    l[:, 3::5] = -inf
    l[1] = -inf
    l[2, 1:] = -inf
    l[3, :] = float("nan")
    l[4, ::2] = float("nan")
    bias = torch.linspace(0.3, -0.3, 24).cuda() if with_bias else None
    for kw in (dict(k=4), dict(k=4, renorm=False), dict(k=6, groups=4, kept=2, group_top=2), dict(k=6, groups=4, kept=1, group_top=1)):
        idx, w = check(l, bias, scoring=scoring, **kw)
        assert not w[1].any() and not w[3].any() and np.isfinite(w).all()
    assert run(l, bias, scoring=scoring, k=4)[0][1].tolist() == [0, 1, 2, 3]


def test_extreme_logits():
    inf = float("inf")
    l = torch.tensor([[inf, 0.0, inf, 1.0], [3e38, -3e38, 0.0, 3e38], [-1e4, -2e4, -1e4, -3e4], [80.0, 100.0, -100.0, 90.0],
                      [1e-30, 2e-30, -1e-30, 0.0]]).cuda()
    for scoring in ("softmax", "sigmoid"):
        for renorm in (True, False):
            check(l, None, k=3, scoring=scoring, renorm=renorm)
    check(l[2:3], None, k=2, scoring="sigmoid")  # scores below every fp64 number
    assert run(l[2:3], None, k=2, scoring="sigmoid")[1].tolist() == [[0.0, 0.0]]


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_infinite_and_large_biases(scoring):
    """A bias of +inf puts an expert first, of -inf behind the others; keys of a large bias differ in bits that fp32 has not got."""
    inf = float("inf")
    l = logits(60, 48, seed=6)
    bias = torch.randn(48, generator=torch.Generator().manual_seed(1)).mul(0.1)
    bias[[5, 40]] = inf
    bias[[7, 8, 30]] = -inf
    check(l, bias.cuda(), k=8, scoring=scoring)
    check(l, bias.cuda(), k=6, scoring=scoring, groups=6, kept=3, group_top=1)
    check(l, torch.full((48,), 3e7).cuda() + torch.arange(48).cuda() % 3, k=8, scoring=scoring, groups=4, kept=2, group_top=2)


def test_one_expert_and_no_tokens():
    check(logits(5, 1), None, k=1)
    check(logits(5, 1), torch.ones(1).cuda(), k=1, scoring="sigmoid", renorm=False)
    idx, w = run(torch.empty(0, 8).cuda(), k=2)
    assert idx.shape == w.shape == (0, 2)


def test_rows_may_lie_apart_and_nothing_else_is_written():
    from paper_2503_00245_b200 import binding as B
    wide = logits(40, 100, seed=4)
    check(wide[:, 10:42], None, k=3, scoring="sigmoid")
    check(wide.bfloat16()[:, 7:39], torch.zeros(32).cuda(), k=3)
    check(wide[:1, 50:82], None, k=3)

    idx, w = torch.full((44, 3), 77, dtype=torch.int32).cuda(), torch.full((44, 3), 77.0).cuda()
    B.moe_select(B.make_select_config(32, 3), wide, 40, None, idx[2:42], w[2:42], stride=100)
    assert (idx[:2] == 77).all() and (idx[42:] == 77).all() and (w[:2] == 77).all() and (w[42:] == 77).all() and (idx[2:42] < 32).all()


def test_captured_and_on_another_stream():
    import paper_2503_00245_b200 as P
    rule = P.SelectRule(64, 4, scoring="sigmoid", groups=8, groups_kept=3, group_top=2)
    l, bias = logits(70, 64, seed=1), torch.zeros(64).cuda()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        P.select_experts(l, rule, bias)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            idx, w = P.select_experts(l, rule, bias)
    for seed in (11, 12):
        l.copy_(logits(70, 64, seed=seed))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want, ww = Q.select(l.double().cpu().numpy(), 4, scoring="sigmoid", bias=np.zeros(64), groups=8, kept=3, group_top=2)
        assert np.array_equal(idx.cpu().numpy(), want) and np.allclose(w.cpu().numpy(), ww, rtol=RTOL, atol=0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d,E", [(1, 256, 8), (16, 1440, 16), (40, 1024, 8), (100, 2048, 64), (70, 136, 6), (500, 512, 40)])
def test_logits_of_the_router(T, d, E, dtype):
    """Sums of d exact products in fp32, some of them cut (2^-23 a time): at most (d + 16) 2^-23 of the sum of magnitudes."""
    from paper_2503_00245_b200 import binding as B
    g = torch.Generator().manual_seed(T + d)
    x = torch.randn(T, d, generator=g).to(dtype).cuda()
    wr = (torch.randn(d, E, generator=g) * d ** -0.5).bfloat16().cuda()
    for b in (None, torch.randn(E, generator=g).cuda()):
        ctx = B.moe_create(B.make_config(d, 64, E, 2, 0, B._dtype(x)))
        out = torch.full((T + 1, E), 7.0).cuda()
        B.moe_route_logits(ctx, x, T, B.make_weights(wr, b), out)
        torch.cuda.synchronize()
        want = x.double() @ wr.double() + (0 if b is None else b.double())
        most = x.double().abs() @ wr.double().abs() + (0 if b is None else b.double().abs())
        assert ((out[:T].double() - want).abs() <= (d + 16) * 2.0 ** -23 * most).all() and (out[T] == 7).all()
        idx, w = torch.empty(T, 2, dtype=torch.int32).cuda(), torch.empty(T, 2).cuda()
        B.moe_route(ctx, x, T, B.make_weights(wr, b), idx, w)
        import paper_2503_00245_b200 as P
        got = P.select_experts(out[:T], P.SelectRule(E, 2))
        assert torch.equal(got[0], idx)  # the same rule as the router's own, on the same logits
        assert torch.allclose(got[1], w, rtol=1e-6, atol=0)
        B.moe_destroy(ctx)
