"""Weights of chosen experts (moe_select) where logits lie far apart, and the totals of softmax weights that are not renormalised.

Tolerance, relative: 2^-20 = 16 * 2^-24.  In units of 2^-24 of the value: expf is off by 3 (2.6 measured over its arguments); a
softmax's argument, a difference of logits, loses |d| to its rounding, which the kernel has to put back (1 for that product): 4; a
sigmoid's 1 + e^-l and its reciprocal round once each: 5.  Renormalised: 5 + (5 + 3 for the sum of eight) + 1 for the quotient + 1 for the
factor `scale` = 15.  Not renormalised: 4 + (4 + 1 for the total, summed in 64 bits) + 1 + 1 = 11.
"""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as Q

pytestmark = pytest.mark.gpu
RTOL = 2.0 ** -20


def check(l, bias=None, **rule):
    import paper_2503_00245_b200 as P
    kw = dict(rule)
    r = P.SelectRule(l.shape[1], kw.pop("k"), groups=kw.pop("groups", 1), groups_kept=kw.pop("kept", 1), **kw)
    idx, w = (v.cpu().numpy() for v in P.select_experts(l, r, bias))
    want, ww = Q.select(l.double().cpu().numpy(), bias=None if bias is None else bias.double().cpu().numpy(), **rule)
    assert np.array_equal(idx, want)
    err = np.abs(w - ww)
    bad = err > RTOL * np.abs(ww) + 1e-45
    assert not bad.any(), (int(bad.sum()), float((err / np.maximum(np.abs(ww), 1e-38)).max() * 2.0 ** 20))


def logits(T, E, sigma, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * sigma).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sigma", [1.0, 4.0, 10.0, 20.0, 60.0])
@pytest.mark.parametrize("T,E,k", [(400, 8, 8), (400, 8, 2), (100, 40, 8), (60, 256, 8)])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_spread_logits(scoring, renorm, T, E, k, sigma, dtype):
    l = logits(T, E, sigma, dtype, T + E)
    check(l, None, k=k, scoring=scoring, renorm=renorm)
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)).cuda()
    check(l, bias, k=k, scoring=scoring, renorm=renorm)
    if E % 8 == 0 and E > 8:
        check(l, bias, k=k, scoring=scoring, renorm=renorm, groups=8, kept=4, group_top=2)


@pytest.mark.parametrize("renorm", [True, False])
def test_large_logits_that_lie_close(renorm):
    """A difference of large logits is exact or nearly so; one of a large and a small one is not."""
    g = torch.Generator().manual_seed(3)
    l = torch.randn(300, 16, generator=g) + 1000.0
    check(l.cuda(), None, k=8, renorm=renorm)
    l = torch.rand(300, 16, generator=g) * 1e-3
    l[:, 5] = 40.0 + torch.rand(300, generator=g)
    check(l.cuda(), None, k=8, renorm=renorm)
    check(-l.cuda() * 0.7, None, k=8, renorm=renorm)


def test_totals_of_many_equal_terms():
    """256 terms a few units below the largest: what each of them loses adds up in the total."""
    g = torch.Generator().manual_seed(4)
    l = torch.rand(200, 256, generator=g) * 0.01 - 5.3
    l[:, 17] = torch.rand(200, generator=g) + 0.1
    check(l.cuda(), None, k=4, renorm=False)
    check(l.cuda(), torch.zeros(256).cuda(), k=4, renorm=False)


def test_as_many_tokens_as_a_call_can_name():
    """2^31 - 1 of them (22 GB in all): the number of blocks comes out of a division that must not pass 32 bits before it."""
    import paper_2503_00245_b200 as P
    T = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    l = torch.zeros(T, 1, dtype=torch.bfloat16, device="cuda")
    l[T - 1] = 1.0
    idx, w = P.select_experts(l, P.SelectRule(1, 1, scoring="sigmoid", renorm=False))
    assert not idx.any()
    for part in w[: T - 1].split(1 << 28):
        assert (part == 0.5).all()
    assert abs(float(w[T - 1]) - 1 / (1 + np.exp(-1.0))) < RTOL
    del l, idx, w, part
    torch.cuda.empty_cache()


def test_logits_that_kernels_could_not_write():
    from paper_2503_00245_b200 import binding as B
    x, wr, out = torch.zeros(3, 64, dtype=torch.bfloat16).cuda(), torch.zeros(64, 8, dtype=torch.bfloat16).cuda(), torch.full((32,), 7.0).cuda()
    ctx = B.moe_create(B.make_config(64, 64, 8, 2))
    for off in (1, 2, 3):
        with pytest.raises(B.MoeError) as e:
            B.moe_route_logits(ctx, x, 3, B.make_weights(wr), out.data_ptr() + off)
        assert e.value.status == 1
    torch.cuda.synchronize()
    assert (out == 7).all()
    B.moe_route_logits(ctx, x, 3, B.make_weights(wr), out.data_ptr() + 4)
    assert not out[1:25].any() and out[0] == 7 and (out[25:] == 7).all()
    B.moe_destroy(ctx)
