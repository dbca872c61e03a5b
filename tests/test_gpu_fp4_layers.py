"""4-bit experts at the large widths, and layers whose experts a rule selects, against the oracles.

Tolerances: 4-bit experts as tests/test_gpu_fp4.py derives them.  Dense and decomposed experts (the layer's bar, tests/gpu_util.py, is a
share of the RMS of all outputs; here tokens differ in scale, where weights are not rescaled, so each is held against its own): half a
step of the output's type at each value, which for bf16 is 2^-8 |y| at most, and 1e-2 of the token's RMS for what comes before.  That
is the hidden values' rounding to bf16: relative errors that are even over half a step of 2^-8 have a standard deviation of 2^-8 / sqrt(3) =
2.3e-3 where a binade begins and half of that where it ends, 1.6e-3 on average, and y, a sum of many such values times weights, 1.6e-3 of
its own RMS: 1e-2 is six of those, and the largest of the 10^6 outputs compared here is expected at 5.  More than 16 fp32 rows are
rounded to bf16 themselves: g and u move by 1.6e-3 of their RMS each, silu(g) u by sqrt(2) of that, with h's rounding sqrt(3) 1.6e-3 = 2.8e-3
(3.0e-3 when the two roundings are done in 64-bit arithmetic on these inputs, 4.0e-3 in the worst token): 2e-2 there.
"""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as Q
from oracle import moe_oracle as O
from synth import workloads as W

from .gpu_util import experts_of, to64
from .test_gpu_fp4 import check_experts, make, routing

pytestmark = pytest.mark.gpu


def P():
    import paper_2503_00245_b200 as p
    return p


@pytest.fixture(scope="module")
def large():
    E, d, f = 4, 2048, 5632
    return E, d, f, *make(E, d, f)


@pytest.mark.parametrize("T", [2, 8, 9, 12, 16, 17, 64, 300, 2048])
def test_experts_at_the_large_widths(large, T):
    """From nine tokens to sixteen the down product's rows fit a few-token call with all of an SM's shared memory only."""
    E, d, f, gu, down = large
    k = 2
    idx, wt = routing(T, E, k)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
    ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=T)
    y = ex.forward(x, idx, wt)
    assert ex.check() == 0
    some = torch.randperm(T, generator=torch.Generator().manual_seed(1))[:40].cuda()  # (the oracle takes its time)
    # (telling: the bound, in which all errors have one sign, grows with the contractions: a fifth of the values at the paper's widths, three
    # tenths at 1.45 times those)
    check_experts(y[some], x[some], gu, down, E, d, f, idx[some], wt[some], telling=False)


def by_oracle(host, k, idx, w):
    """The experts' sum for a given routing, in 64 bits."""
    E = host["w_router"].shape[1]
    _, offsets, perm, inv = O.permute(idx, E)
    ex = experts_of(host)
    if "w_gate" in ex:
        out = O.expert_ffn_dense(host["x"], ex["w_gate"], ex["w_up"], ex["w_down"], offsets, perm, k)
    else:
        out = O.expert_ffn_wd(host["x"], *(ex[n] for n in ("gL", "gR", "uL", "uR", "dL", "dR")), offsets, perm, k)
    return O.combine(out, w, inv)


RULES = [dict(), dict(scoring="sigmoid", groups=4, groups_kept=2, group_top=2, scale=2.5), dict(renorm=False)]


@pytest.mark.parametrize("T", [1, 5, 16, 17, 80])
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("shape", [W.LayerShape("a", 1, 256, 384, 8, 2, 0), W.LayerShape("b", 1, 256, 384, 8, 2, 64),
                                   W.LayerShape("c", 1, 320, 512, 16, 3, 136, x_dtype="f32"), W.WEARABLE], ids=lambda s: s.name)
def test_layers_with_a_selection_rule(shape, rule, T):
    t = W.make_layer(shape, T, device="cuda")
    host = {n: W.to_host_bits(v) for n, v in t.items()}
    E, k = shape.n_experts, shape.top_k
    kw = dict(d_model=shape.d_model, d_ff=shape.d_ff, n_experts=E, top_k=k)
    bias = torch.linspace(0.2, -0.2, E).cuda()
    lay = P().MoELayer.from_math_layout(kw, t, x_dtype=t["x"].dtype, max_tokens=T + 5, select=P().SelectRule(E, k, **rule), select_bias=bias)
    idx, w = torch.empty(T, k, dtype=torch.int32).cuda(), torch.empty(T, k).cuda()
    y = lay.forward(t["x"], topk_idx=idx, topk_w=w)
    assert lay.check() == 0
    want = {n: rule[n] for n in ("scoring", "groups", "group_top", "renorm", "scale") if n in rule}
    i64, w64 = Q.select(to64(lay.logits(t["x"])), k, bias=bias.double().cpu().numpy(), kept=rule.get("groups_kept", 1), **want)
    assert np.array_equal(idx.cpu().numpy(), i64) and np.allclose(w.cpu().numpy(), w64, rtol=2.0 ** -20, atol=0)
    sum64 = by_oracle(host, k, i64, w64)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(sum64), 1e-300))) - 8) if y.dtype == torch.bfloat16 else 0.0
    excess = (np.abs(to64(y) - sum64) - step) / np.sqrt(np.mean(sum64 ** 2, axis=1, keepdims=True))
    assert excess.max() <= (2e-2 if y.dtype == torch.float32 and T > 16 else 1e-2), excess.max()
    out = torch.empty_like(y)
    assert lay.forward(t["x"], out) is out and torch.equal(out, y)
    assert lay.check() == 0
    lay.close()


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("rank", [0, 64])
def test_a_rule_like_the_routers_own_gives_the_layer_without_one(rank, T):
    shape = W.LayerShape("r", 1, 256, 384, 8, 2, rank)
    t = W.make_layer(shape, T, device="cuda")
    kw = dict(d_model=256, d_ff=384, n_experts=8, top_k=2)
    a = P().MoELayer.from_math_layout(kw, t, x_dtype=t["x"].dtype, max_tokens=T)
    b = P().MoELayer.from_math_layout(kw, t, x_dtype=t["x"].dtype, max_tokens=T, select=P().SelectRule(8, 2))
    ya, yb = a.forward(t["x"]), b.forward(t["x"])
    # two roundings to bf16 of sums that differ in their order, and in weights by 2^-20: within a step of one another
    assert (ya.double() - yb.double()).abs().max() <= 2.0 ** -7 * ya.double().abs().max()
    assert a.check() == 0 and b.check() == 0


@pytest.mark.parametrize("fp4", [False, True])
def test_no_tokens(fp4):
    t = W.make_layer(W.LayerShape("n", 1, 256, 384, 8, 2), 3, device="cuda")
    kw = dict(x_dtype=t["x"].dtype, max_tokens=3, select=P().SelectRule(8, 2, scoring="sigmoid"))
    kind = (dict(fp4=P().pack_fp4(t["w_gate"], t["w_up"], t["w_down"])) if fp4 else
            dict(dense=P().pack_dense(t["w_gate"], t["w_up"], t["w_down"])))
    lay = P().MoELayer(256, 384, 8, 2, t["w_router"], t["b_router"], **kind, **kw)
    assert lay.forward(t["x"][:0]).shape == (0, 256)
    assert lay.logits(t["x"][:0]).shape == (0, 8) and lay.check() == 0
    assert torch.isfinite(lay.forward(t["x"])).all() and lay.check() == 0


def test_layers_with_rules_in_a_graph_replayed_on_other_tokens():
    shape = W.LayerShape("g", 1, 256, 384, 8, 2, 64)
    lays, T = [], 6
    for i, s in enumerate((shape, shape.with_(wd_rank=0))):
        t = W.make_layer(s, T, device="cuda", layer=i)
        kw = dict(d_model=256, d_ff=384, n_experts=8, top_k=2)
        lays.append(P().MoELayer.from_math_layout(kw, t, x_dtype=t["x"].dtype, max_tokens=T, select=P().SelectRule(8, 2, scoring="sigmoid"),
                                                  select_bias=torch.zeros(8).cuda()))
    x = t["x"].clone()

    def chain():
        return lays[1].forward(lays[0].forward(x))
    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = chain()
    for i in range(4):
        x.copy_(W.make_x(shape, T, "cuda", step=i + 1))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, chain())
    assert all(lay.check() == 0 for lay in lays)
