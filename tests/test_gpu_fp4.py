"""MXFP4 rows, products and experts against the checker (oracle/fp4_oracle.py).

Quantisation and reading back are exact and compared bit by bit.

A product's sums: with `n` values of a row, S = sum |a w|.  An instruction adds 64 products to the accumulator and cuts what does
not fit: at most one unit in the last place, 2^-23 of the largest partial sum, for each of its 65 addends in the worst case a sum of
whose cuts is 2^-22 of S per step of the adder tree; n / 64 instructions: (n / 64 + 4) 2^-21 S.
A rounding to bf16 adds 2^-8 of the value (half a step, torch.finfo(bfloat16).eps / 2).

The experts' FFN rounds its hidden values to 4 bits.  With d_h the error a hidden value may have before that (from the bounds above,
|d silu(g) u| <= 1.1 |u| d_g + |silu(g)| d_u + 2^-19 |h|), a value within d_h of a border between two codes may get either; so may
all values of a block whose largest is within d_h of a power of two.  The sum over such values of (distance of the two roundings)
x |w_down| x the routing's weight is added to the bound.
"""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as Q

pytestmark = pytest.mark.gpu


def P():
    import paper_2503_00245_b200 as p
    return p


def host(t):
    return t.double().cpu().numpy()


def parts(q):
    return q.codes.cpu().numpy(), q.scales.cpu().numpy()


def assert_same(q, x64):
    """q holds exactly the codes and scales of x64; -0 and 0 are one value."""
    codes, s = Q.quantize(x64)
    packed, sc = Q.store(codes, s)
    got_c, got_s = parts(q)
    rows = x64.shape[0]
    assert np.array_equal(got_s[:, :rows], sc[:, :rows])
    n = x64.shape[1]
    a, b = Q.load(got_c, got_s, n), Q.load(packed, sc, n)
    assert np.array_equal(a, b, equal_nan=True)
    # behind n there are zeros
    tail = np.stack([got_c & 15, got_c >> 4], -1).reshape(rows, -1)[:, n:]
    assert not (tail & 7).any()


def rows_of(rows, n, dtype, seed=0):
    """Values over many binades, exact borders between codes, whole blocks of zeros."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, n, generator=g) * torch.exp(torch.randn(rows, n, generator=g))
    x *= torch.exp2(torch.randint(-20, 21, (rows, (n + 31) // 32), generator=g).float()).repeat_interleave(32, 1)[:, :n]
    ties = torch.randint(-32, 33, (rows, n), generator=g).float() / 4
    pick = torch.rand(rows, n, generator=g) < 0.5
    if rows > 1:
        x[1::3] = torch.where(pick[1::3], ties[1::3], torch.zeros(()))
        x[2::5, : min(n, 64)] = 0.0
    return x.to(dtype).cuda()


# ------------------------------------------------------------------ quantisation
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n", [(1, 8), (1, 32), (3, 40), (5, 1440), (7, 128), (4, 256), (130, 264), (33, 2048), (1, 16384), (9, 104)])
def test_rows_become_the_checkers_codes(rows, n, dtype):
    x = rows_of(rows, n, dtype, rows + n)
    q = P().fp4_quantize(x)
    assert_same(q, host(x))
    for back in (torch.float32, torch.bfloat16):
        assert np.array_equal(host(q.dequantize(back)), Q.load(*parts(q), n))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_any_strides(dtype):
    big = rows_of(70, 300, dtype, 3)
    for x in (big[:, 1:33], big[:, 8:200], big[::2, :40], big.T[:100], big.T[3:67:2, 1:], big[5:6].expand(6, 300), big[:, ::3], big[:9, :21],
              big[:, 4:5].expand(70, 64)):
        assert_same(P().fp4_quantize(x), host(x))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [72, 250])
def test_rows_gathered(n, dtype):
    x = rows_of(20, n, dtype, 5)
    g = torch.Generator().manual_seed(1)
    order = torch.randint(0, 60, (77,), generator=g).to(torch.int32)
    order[5] = order[6]
    q = P().fp4_quantize(x, order.cuda(), 3)
    assert_same(q, host(x)[order.numpy() // 3])
    order[7], order[8], order[9] = 60, -1, -3000000  # rows that are not there
    want = host(x)[np.clip(order.numpy() // 3, 0, 19)]
    want[7:10] = 0
    assert_same(P().fp4_quantize(x, order.cuda(), 3), want)
    assert P().fp4_quantize(x, torch.empty(0, dtype=torch.int32).cuda()).dequantize().shape == (0, n) if n % 8 == 0 else True


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_blocks_at_the_ends_of_the_range(dtype):
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(12, 64)
    x[0, 3], x[0, 40] = inf, 1.0
    x[1, 3], x[1, 4] = nan, 5.0
    x[2, 3], x[2, 4] = -inf, nan
    x[3] = 2.0 ** -130
    x[4] = torch.linspace(-2.0 ** -126, 2.0 ** -126, 64)
    x[5] = torch.linspace(-3.3e38, 3.3e38, 64)
    x[6] = -0.0
    x[7, 0], x[7, 1] = 2.0 ** 127, 2.0 ** 125 * 1.25
    x[8] = torch.linspace(0, 8, 64)
    x[9] = torch.linspace(-7.96875, 0, 64)
    x[10, 31], x[10, 32] = 1.0, 2.0 ** -149
    x[11] = 2.0 ** -125 * 1.5
    x = x.to(dtype).cuda()
    q = P().fp4_quantize(x)
    assert_same(q, host(x))
    assert np.array_equal(host(q.dequantize(torch.float32)), Q.load(*parts(q), 64), equal_nan=True)
    assert_same(P().fp4_quantize(x.T.contiguous().T), host(x))


def test_read_back_into_rows_that_lie_apart_and_nothing_else():
    from paper_2503_00245_b200 import binding as B
    x = rows_of(6, 40, torch.float32, 2)
    q = P().fp4_quantize(x)
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.full((7, 64), 9.0, dtype=dtype).cuda()
        B.moe_fp4_dequantize_rows(q.c, wide, 64)
        assert (wide[:, 40:] == 9).all() and (wide[6] == 9).all() and np.array_equal(host(wide)[:6, :40], Q.load(*parts(q), 40))
    # codes and scales of six rows, with guards around them
    codes, scales = torch.full((8, 32), 0x5a, dtype=torch.uint8).cuda(), torch.full((3, 8, 4), 0x5a, dtype=torch.uint8).cuda()
    B.moe_fp4_quantize_rows(x, None, 1, 6, codes[1:7], scales[1:2])
    assert (codes[0] == 0x5a).all() and (codes[7] == 0x5a).all() and (scales[0] == 0x5a).all() and (scales[2] == 0x5a).all()
    assert (scales[1, 6:] == 0x5a).all()


@pytest.mark.parametrize("E,d,f", [(2, 64, 96), (3, 136, 72), (1, 256, 40), (2, 40, 200)])
def test_packed_experts(E, d, f):
    g = torch.Generator().manual_seed(d + f)
    wg, wu, wd = (torch.randn(*s, generator=g).bfloat16().cuda() for s in ((E, d, f), (E, d, f), (E, f, d)))
    gu, down = P().pack_fp4(wg, wu, wd)
    fb = -(-f // 32)
    want = np.zeros((E, fb, 2, 32, d))
    for i, w in enumerate((wg, wu)):
        for c in range(f):
            want[:, c // 32, i, c % 32] = host(w)[:, :, c]
    assert_same(gu, want.reshape(-1, d))
    assert_same(down, host(wd).transpose(0, 2, 1).reshape(-1, f))


# ------------------------------------------------------------------ product
def random_rows(rows, n, seed, sigma=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, n, generator=g, device="cuda") * sigma
    return P().fp4_quantize(x.bfloat16())


def values(q):
    return Q.load(*parts(q), q.n)


def check_product(a, w, offsets, E, out):
    av, wv = values(a), values(w)
    want, most = Q.product(av, wv, offsets, E), Q.product(np.abs(av), np.abs(wv), offsets, E)
    got = host(out)
    tol = (a.n / 64 + 4) * 2.0 ** -21 * most
    if out.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    inside = ~np.isnan(want)
    assert np.array_equal(np.isnan(got[inside]), np.zeros(inside.sum(), bool))
    err = np.abs(got - want)[inside]
    assert (err <= tol[inside] + 1e-44).all(), float((err / np.maximum(tol[inside], 1e-300)).max())


GROUPS = {
    "one row": [0, 1], "one expert": [0, 5], "two": [0, 1, 2], "empty ones": [0, 0, 3, 3, 3, 9, 9], "all in the last": [0, 0, 0, 20],
    "at the border": [0, 9, 32], "uneven": [0, 1, 17, 19, 32], "just over": [0, 11, 33], "many": [0, 40, 40, 300, 301, 513],
    "one tile and a row": [0, 257], "whole tiles": [0, 256, 768], "65 experts' worth": list(range(0, 65)),
}


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", list(GROUPS))
@pytest.mark.parametrize("n,N", [(256, 64), (1440, 200), (40, 8), (64, 384), (136, 16), (2048, 192)])
def test_product(name, n, N, out_dtype):
    offsets = GROUPS[name]
    E, rows = len(offsets) - 1, offsets[-1]
    a, w = random_rows(rows, n, 1), random_rows(E * N, n, 2, n ** -0.5)
    out = P().fp4_product(a, w, torch.tensor(offsets, dtype=torch.int32).cuda(), out_dtype=out_dtype)
    check_product(a, w, offsets, E, out)
    from paper_2503_00245_b200 import layer as L
    assert P().binding.moe_check(L._shared_ctx()) == 0


@pytest.mark.parametrize("rows", [20, 300])
def test_product_of_values_that_are_exact(rows):
    """Small whole numbers: every sum is exact in fp32 on either path, and scales differ from block to block."""
    g = torch.Generator().manual_seed(rows)
    n, N, E = 416, 72, 3
    a = torch.randint(-2, 3, (rows, n), generator=g).float() * torch.exp2(torch.randint(0, 3, (rows, n // 32), generator=g).float()).repeat_interleave(32, 1)
    w = torch.randint(-1, 2, (E * N, n), generator=g).float() * torch.exp2(torch.randint(-1, 2, (E * N, n // 32), generator=g).float()).repeat_interleave(32, 1)
    qa, qw = P().fp4_quantize(a.cuda()), P().fp4_quantize(w.cuda())
    offsets = [0, rows // 3, rows // 2, rows]
    out = P().fp4_product(qa, qw, torch.tensor(offsets, dtype=torch.int32).cuda(), out_dtype=torch.float32)
    assert np.array_equal(host(out), Q.product(values(qa), values(qw), offsets, E))


@pytest.mark.parametrize("rows", [24, 320])
def test_rows_of_no_expert_are_left_alone(rows):
    n, N, E = 128, 40, 2
    a, w = random_rows(rows, n, 3), random_rows(E * N, n, 4)
    offsets = [3, 10, rows - 5]
    out = torch.full((rows, 64), 7.0).cuda()
    P().fp4_product(a, w, torch.tensor(offsets, dtype=torch.int32).cuda(), out=out[:, :N])
    assert (out[:3] == 7).all() and (out[rows - 5:] == 7).all() and (out[:, N:] == 7).all()
    check_product(a, w, offsets, E, out[:, :N])
    # offsets that claim more rows than there are
    out.fill_(7.0)
    P().fp4_product(a, w, torch.tensor([-4, 10, rows + 900], dtype=torch.int32).cuda(), out=out[:, :N])
    check_product(a, w, [0, 10, rows], E, out[:, :N])


@pytest.mark.parametrize("rows", [6, 200])
def test_nan_blocks_stay_in_their_row_and_column(rows):
    n, N = 256, 64
    a, w = random_rows(rows, n, 5), random_rows(N, n, 6)
    clean = P().fp4_product(a, w, torch.tensor([0, rows], dtype=torch.int32).cuda(), out_dtype=torch.float32)
    a.scales[0, 3, 2] = 255
    w.scales[1, 50, 3] = 255
    out = P().fp4_product(a, w, torch.tensor([0, rows], dtype=torch.int32).cuda(), out_dtype=torch.float32)
    bad = torch.zeros(rows, N, dtype=torch.bool).cuda()
    bad[3], bad[:, 50] = True, True
    assert out[bad].isnan().all() and torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("rows", [16, 64])
def test_scales_at_the_ends_of_the_range(rows):
    n, N = 96, 16
    a, w = random_rows(rows, n, 7), random_rows(N, n, 8)
    at = torch.tensor([0, rows], dtype=torch.int32).cuda()
    for sa, sw in ((0, 127), (0, 250), (250, 1), (127, 0), (60, 60), (254, 0)):
        a.scales.fill_(sa), w.scales.fill_(sw)
        a.scales[:, :, 3], w.scales[:, :, 3] = 0, 0
        out = P().fp4_product(a, w, at, out_dtype=torch.float32)
        check_product(a, w, [0, rows], 1, out)


def test_products_are_the_same_again_and_wherever_a_row_stands():
    a, w = random_rows(300, 512, 9), random_rows(4 * 104, 512, 10)
    at = torch.tensor([0, 100, 100, 290, 300], dtype=torch.int32).cuda()
    first = P().fp4_product(a, w, at, out_dtype=torch.float32)
    for _ in range(20):
        assert torch.equal(first, P().fp4_product(a, w, at, out_dtype=torch.float32))
    few = random_rows(30, 512, 9)
    at = torch.tensor([0, 11, 11, 19, 30], dtype=torch.int32).cuda()
    one = P().fp4_product(few, w, at, out_dtype=torch.float32)
    alone = P().Fp4Rows(few.codes[19:20].contiguous(), few.scales[:, 19:20].repeat(1, 4, 1).contiguous(), 512)
    got = P().fp4_product(alone, w, torch.tensor([0, 0, 0, 0, 1], dtype=torch.int32).cuda(), out_dtype=torch.float32)
    assert torch.equal(one[19], got[0])


def test_product_captured_and_on_two_streams():
    a, w = random_rows(200, 256, 11), random_rows(3 * 64, 256, 12)
    few = random_rows(9, 256, 13)
    at, at_few = torch.tensor([0, 50, 120, 200], dtype=torch.int32).cuda(), torch.tensor([0, 4, 4, 9], dtype=torch.int32).cuda()
    want, want_few = P().fp4_product(a, w, at), P().fp4_product(few, w, at_few)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        x, y = P().fp4_product(a, w, at), P().fp4_product(few, w, at_few)
    for _ in range(3):
        x.zero_(), y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want) and torch.equal(y, want_few)
    a.codes.copy_(random_rows(200, 256, 14).codes)
    g.replay()
    torch.cuda.synchronize()
    check_product(a, w, [0, 50, 120, 200], 3, x)
    want = P().fp4_product(a, w, at)
    torch.cuda.synchronize()
    outs = []
    for i in range(10):
        with torch.cuda.stream(s if i % 2 else torch.cuda.current_stream()):
            outs.append((P().fp4_product(a, w, at), P().fp4_product(few, w, at_few)))
    torch.cuda.synchronize()
    assert all(torch.equal(p, want) and torch.equal(q, want_few) for p, q in outs)


# ------------------------------------------------------------------ the experts' FFN
def make(E, d, f, seed=0):
    g = torch.Generator().manual_seed(seed + d + f)
    wg, wu = ((torch.randn(E, d, f, generator=g) * d ** -0.5).bfloat16().cuda() for _ in range(2))
    wd = (torch.randn(E, f, d, generator=g) * f ** -0.5).bfloat16().cuda()
    return P().pack_fp4(wg, wu, wd)


def matrices(gu, down, E, d, f):
    v = values(gu).reshape(E, -1, 2, 32, d)
    return v[:, :, 0].reshape(E, -1, d)[:, :f], v[:, :, 1].reshape(E, -1, d)[:, :f], values(down).reshape(E, d, f)


def round4(h, s):
    """h on the codes of scale bytes s (per block), as values."""
    f = h.shape[1]
    v = np.zeros((h.shape[0], s.shape[1] * 32))
    v[:, :f] = h
    v = v.reshape(h.shape[0], -1, 32)
    step = np.ldexp(1.0, s.astype(np.int64) - 127)[..., None]
    return (np.sign(v) * Q.VALUES[Q.nearest_code(np.abs(v) / step)] * step).reshape(h.shape[0], -1)[:, :f]


def expected(x, gate, up, down, idx, wt):
    """(y, bound of its error before the last rounding); see the head of this file."""
    T, d = x.shape
    f = gate.shape[1]
    xq = Q.values(*Q.quantize(x), d)
    y, tol = np.zeros_like(x), np.zeros_like(x)
    c_in, c_out = ((n / 64 + 4) * 2.0 ** -21 for n in (d, f))
    for e in range(gate.shape[0]):
        t, j = np.nonzero(idx == e)
        if not len(t):
            continue
        g, u = xq[t] @ gate[e].T, xq[t] @ up[e].T
        ax = np.abs(xq[t])
        dg, du = c_in * (ax @ np.abs(gate[e]).T), c_in * (ax @ np.abs(up[e]).T)
        silu = g / (1 + np.exp(-g))
        h = silu * u
        dh = 1.1 * (np.abs(u) + du) * dg + np.abs(silu) * du + 2.0 ** -19 * np.abs(h)
        s = Q.quantize(h)[1]
        hq = round4(h, s)
        lo, hi = round4(h - dh, s), round4(h + dh, s)
        slack = np.maximum(np.abs(hi - hq), np.abs(hq - lo))
        pad = np.zeros((len(t), s.shape[1] * 32))
        top = []
        for sign in (-1, 1):  # blocks whose scale could be another one
            pad[:, :f] = np.maximum(np.abs(h) + sign * dh, 0)
            top.append(np.frexp(pad.reshape(len(t), -1, 32).max(2))[1])
        move = (top[0] != top[1]).repeat(32, 1)[:, :f]
        slack = np.where(move, np.ldexp(1.0, s.astype(np.int64) - 127).repeat(32, 1)[:, :f] * 2.0, slack)
        o = hq @ down[e].T
        do = slack @ np.abs(down[e]).T + c_out * ((np.abs(hq) + slack) @ np.abs(down[e]).T)
        np.add.at(y, t, wt[t, j][:, None] * o)
        np.add.at(tol, t, np.abs(wt[t, j])[:, None] * (do + (idx.shape[1] + 2) * 2.0 ** -23 * np.abs(o)))
    return y, tol


def check_experts(y, x, gu, down, E, d, f, idx, wt, telling=True):
    want, tol = expected(host(x), *matrices(gu, down, E, d, f), idx.cpu().numpy(), host(wt))
    if y.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    err = np.abs(host(y) - want)
    assert (err <= tol + 1e-30).all(), float((err / np.maximum(tol, 1e-300)).max())
    # the bound says something: most of it is below the values (1440 and 3840 summands, all errors of one sign: a tenth)
    assert not telling or np.median(tol) < 0.2 * np.sqrt(np.mean(want ** 2))


def routing(T, E, k, seed=0):
    g = torch.Generator().manual_seed(seed + T)
    l = torch.randn(T, E, generator=g)
    top, idx = torch.topk(l, k, 1)
    return idx.to(torch.int32).cuda(), torch.softmax(top, 1).cuda()


SHAPES = [(8, 2, 256, 512), (6, 3, 136, 200), (8, 8, 64, 96), (1, 1, 512, 264), (16, 4, 320, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 2, 3, 8, 16, 17, 40, 300])
@pytest.mark.parametrize("E,k,d,f", SHAPES)
def test_experts(E, k, d, f, T, dtype):
    gu, down = make(E, d, f)
    idx, wt = routing(T, E, k)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(dtype).cuda()
    ex = P().Fp4Experts(d, f, E, k, gu, down, x_dtype=dtype, max_tokens=T + 3)
    y = ex.forward(x, idx, wt)
    assert ex.check() == 0
    check_experts(y, x, gu, down, E, d, f, idx, wt)
    ex.ws.fill_(255)  # (nothing is kept there from one call to the next)
    assert torch.equal(y, ex.forward(x, idx, wt))
    ex.close()


@pytest.mark.parametrize("T", [1, 3, 20])
@pytest.mark.parametrize("d,f", [(64, 65536), (16384, 64), (5632, 32)])
def test_experts_of_extreme_widths(d, f, T):
    """Rows too long for a few-token call's shared memory go the way of many tokens."""
    E, k = 2, 1
    gu, down = make(E, d, f)
    idx, wt = routing(T, E, k)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
    ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=T)
    y = ex.forward(x, idx, wt)
    assert ex.check() == 0
    check_experts(y, x, gu, down, E, d, f, idx, wt, telling=False)


@pytest.mark.parametrize("rows", [5, 40])
@pytest.mark.parametrize("n,N", [(21, 16), (65536, 24), (8, 8), (1000, 1000)])
def test_product_of_odd_and_long_rows(rows, n, N):
    g = torch.Generator().manual_seed(rows + n)
    a, w = (P().fp4_quantize(torch.randn(r, n, generator=g).cuda()) for r in (rows, 2 * N))
    offsets = [0, rows // 2, rows]
    out = P().fp4_product(a, w, torch.tensor(offsets, dtype=torch.int32).cuda(), out_dtype=torch.float32)
    check_product(a, w, offsets, 2, out)


def test_a_token_with_an_infinity_spoils_itself_alone():
    E, k, d, f = 4, 2, 128, 96
    gu, down = make(E, d, f)
    for T in (3, 40):
        idx, wt = routing(T, E, k)
        x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
        ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=T)
        y = ex.forward(x, idx, wt)
        for bad in (float("inf"), float("nan")):
            z = x.clone()
            z[1, 70] = bad
            got = ex.forward(z, idx, wt)
            keep = torch.arange(T) != 1
            assert got[1].isnan().all() and torch.equal(got[keep], y[keep])


@pytest.mark.parametrize("T", [1, 5, 600])
def test_experts_at_the_paper_widths(T):
    E, k, d, f = 8, 2, 1440, 3840
    gu, down = make(E, d, f)
    idx, wt = routing(T, E, k)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
    ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=T)
    check_experts(ex.forward(x, idx, wt), x, gu, down, E, d, f, idx, wt)
    assert ex.check() == 0


@pytest.mark.parametrize("T", [1, 9, 16, 33])
def test_uneven_routing_and_an_expert_named_twice(T):
    E, k, d, f = 8, 8, 96, 160
    gu, down = make(E, d, f)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
    ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=T)
    idx, wt = routing(T, E, k)
    for same in (idx * 0 + 5, idx * 0, idx // 2, torch.where(idx > 3, 7, 0).to(torch.int32)):
        y = ex.forward(x, same, wt)
        check_experts(y, x, gu, down, E, d, f, same, wt)
    y = ex.forward(x, idx, wt * 0)
    assert not y.any()
    assert ex.check() == 0


@pytest.mark.parametrize("T", [2, 30])
def test_experts_out_of_range_are_reported_and_spoil_their_token_alone(T):
    E, k, d, f = 4, 2, 64, 64
    gu, down = make(E, d, f)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
    ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=T)
    idx, wt = routing(T, E, k)
    y = ex.forward(x, idx, wt)
    for bad in (-1, E, 1 << 30):
        wrong = idx.clone()
        wrong[0, 1] = bad
        ex.ws.fill_(255)  # (whatever the workspace holds)
        z = ex.forward(x, wrong, wt)
        assert ex.check() == 6
        assert torch.equal(z[1:], y[1:])
    assert torch.equal(ex.forward(x, idx, wt), y) and ex.check() == 0


def test_experts_refuse():
    from paper_2503_00245_b200 import binding as B
    E, k, d, f = 4, 2, 64, 96
    gu, down = make(E, d, f)
    idx, wt = routing(8, E, k)
    x = torch.randn(8, d).bfloat16().cuda()
    ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=8)
    y = torch.full_like(x, 3.0)

    def call(ctx=None, T=8, gu=gu.c, down=down.c, ws=ex.ws):
        with pytest.raises(B.MoeError) as e:
            B.moe_fp4_experts(ex.ctx if ctx is None else ctx, x, T, gu, down, idx, wt, y, ws)
        return e.value.status
    assert call(T=-1) == 1
    assert call(gu=down.c) == 1 and call(down=gu.c) == 1
    assert call(ws=ex.ws[:256]) == 3
    assert call(ws=ex.ws[8:]) == 1
    wd = B.moe_create(B.make_config(d, f, E, k, 32))
    assert call(ctx=wd) == 2
    B.moe_destroy(wd)
    B.moe_fp4_experts(ex.ctx, x, 0, gu.c, down.c, idx, wt, y, ex.ws)
    torch.cuda.synchronize()
    assert (y == 3).all()
    for bad in (lambda: ex.forward(x.float(), idx, wt), lambda: ex.forward(x, idx.long(), wt), lambda: ex.forward(x, idx[:4], wt),
                lambda: ex.forward(torch.cat([x, x]), idx, wt), lambda: ex.forward(x, idx, wt, y.float())):
        with pytest.raises(ValueError):
            bad()


def test_experts_captured_with_changing_inputs():
    E, k, d, f = 8, 2, 256, 512
    gu, down = make(E, d, f)
    for T in (1, 6, 64):
        ex = P().Fp4Experts(d, f, E, k, gu, down, max_tokens=T)
        x = torch.randn(T, d).bfloat16().cuda()
        idx, wt = routing(T, E, k)
        y = ex.forward(x, idx, wt)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ex.forward(x, idx, wt, y)
        for seed in (1, 2, 3):
            new = torch.randn(T, d, generator=torch.Generator().manual_seed(seed)).bfloat16()
            i, w = routing(T, E, k, seed)
            x.copy_(new), idx.copy_(i), wt.copy_(w)
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            got = y.clone()
            assert torch.equal(got, ex.forward(x, idx, wt))
            check_experts(got, x, gu, down, E, d, f, idx, wt)
        assert ex.check() == 0


def test_two_layers_on_two_streams_and_calls_of_every_size_on_one():
    E, k, d, f = 8, 2, 256, 512
    gu, down = make(E, d, f)
    a, b = (P().Fp4Experts(d, f, E, k, gu, down, max_tokens=100) for _ in range(2))
    cases = [(torch.randn(T, d, generator=torch.Generator().manual_seed(T)).bfloat16().cuda(), *routing(T, E, k)) for T in (1, 100, 16, 17, 2, 90)]
    want = [a.forward(*c) for c in cases]
    fresh = [P().Fp4Experts(d, f, E, k, gu, down, max_tokens=100).forward(*c) for c in cases]
    assert all(torch.equal(p, q) for p, q in zip(want, fresh))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for c in cases:
            got.append(a.forward(*c))
            with torch.cuda.stream(s):
                got.append(b.forward(*c))
    torch.cuda.synchronize()
    assert all(torch.equal(v, want[i // 2 % len(cases)]) for i, v in enumerate(got))
    assert a.check() == 0 and b.check() == 0


# ------------------------------------------------------------------ a layer that uses all of them
@pytest.mark.parametrize("T", [1, 4, 16, 50])
@pytest.mark.parametrize("rule", [None, dict(scoring="sigmoid", groups=4, groups_kept=2, group_top=2, scale=2.5)])
def test_layer_with_4_bit_experts(T, rule):
    E, k, d, f = 16, 4, 256, 192
    gu, down = make(E, d, f)
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, d, generator=g).bfloat16().cuda()
    wr = (torch.randn(d, E, generator=g) * d ** -0.5).bfloat16().cuda()
    bias = torch.randn(E, generator=g).mul(0.1).cuda() if rule else None
    lay = P().MoELayer(d, f, E, k, wr, fp4=(gu, down), select=P().SelectRule(E, k, **rule) if rule else None, select_bias=bias, max_tokens=T)
    idx, w = torch.empty(T, k, dtype=torch.int32).cuda(), torch.empty(T, k).cuda()
    y = lay.forward(x, topk_idx=idx, topk_w=w)
    assert lay.check() == 0
    kw = dict(scoring="sigmoid", groups=4, kept=2, group_top=2, scale=2.5) if rule else {}
    want, ww = Q.select(host(lay.logits(x)), k, bias=None if bias is None else host(bias), **kw)
    assert np.array_equal(idx.cpu().numpy(), want) and np.allclose(w.cpu().numpy(), ww, rtol=1e-5)
    check_experts(y, x, gu, down, E, d, f, idx, w)
    r = lay.route(x)
    assert torch.equal(r[0], idx) and torch.equal(r[1], w) and torch.equal(lay.fp4.forward(x, idx, w), y)
    out = torch.empty_like(y)
    assert lay.forward(x, out) is out and torch.equal(out, y)
    # the steps, through the public calls: grouped rows, their 4-bit product, the same hidden rows
    offsets, perm, inv = lay.permute(idx)
    xq = P().fp4_quantize(x, perm, k)
    prod = P().fp4_product(xq, gu, offsets, out_dtype=torch.float32)
    v = prod.view(T * k, -1, 2, 32)
    h = (torch.nn.functional.silu(v[:, :, 0]) * v[:, :, 1]).flatten(1)[:, :f].contiguous()
    o = P().fp4_product(P().fp4_quantize(h), down, offsets, out_dtype=torch.float32)
    by_steps = lay.combine(o, w, inv)
    assert float((by_steps.float() - y.float()).norm() / y.float().norm()) < 0.02  # (hidden values at a border between codes)
    lay.close()


@pytest.mark.parametrize("T", [1, 7, 16, 24])
def test_layers_one_after_the_other_in_a_graph(T):
    """Kernels that start while the one ahead of them runs: a chain of layers, logits to sums, replayed on other inputs."""
    E, k, d, f = 8, 2, 512, 384
    g = torch.Generator().manual_seed(T)
    lays = []
    for i in range(3):
        wr = (torch.randn(d, E, generator=g) * d ** -0.5).bfloat16().cuda()
        rule = P().SelectRule(E, k, scoring="sigmoid", groups=4, groups_kept=2, group_top=2)
        lays.append(P().MoELayer(d, f, E, k, wr, fp4=make(E, d, f, i), select=rule, select_bias=torch.zeros(E).cuda(), max_tokens=T))

    def chain(x):
        for lay in lays:
            x = x + lay.forward(x)
        return x
    x = torch.randn(T, d, generator=g).bfloat16().cuda()
    chain(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = chain(x)
    for i in range(6):
        x.copy_(torch.randn(T, d, generator=g).bfloat16())
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(y).all() and torch.equal(y, chain(x))
    assert all(lay.check() == 0 for lay in lays)


@pytest.mark.parametrize("T", [1, 30])
def test_dense_layer_with_a_selection_rule(T):
    from oracle import moe_oracle as O
    from synth import workloads as W
    t = W.make_layer(W.TINY, T, device="cuda")
    E, k = W.TINY.n_experts, W.TINY.top_k
    kw = dict(d_model=W.TINY.d_model, d_ff=W.TINY.d_ff, n_experts=E, top_k=k)
    lay = P().MoELayer.from_math_layout(kw, t, x_dtype=t["x"].dtype, max_tokens=T, select=P().SelectRule(E, k, scoring="sigmoid"),
                                        select_bias=torch.linspace(0.2, -0.2, E).cuda())
    idx, w, _ = lay.route(t["x"])
    y = lay.forward(t["x"])
    assert lay.check() == 0
    h = {n: W.to_host_bits(v) for n, v in t.items()}
    x, out = O.widen(h["x"]), np.zeros((T, W.TINY.d_model))
    wg, wu, wd = (O.widen(h[n]) for n in ("w_gate", "w_up", "w_down"))
    for i in range(T):
        for j in range(k):
            e = int(idx[i, j])
            g = x[i] @ wg[e]
            out[i] += float(w[i, j]) * ((g / (1 + np.exp(-g)) * (x[i] @ wu[e])) @ wd[e])
    assert np.abs(host(y) - out).max() <= 2e-2 * np.sqrt((out ** 2).mean())  # the layer's own tolerance (tests/gpu_util.py)
    with pytest.raises(ValueError):
        lay.route(t["x"], want_probs=True)
    lay.close()
