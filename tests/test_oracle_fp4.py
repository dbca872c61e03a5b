"""Pins of the MXFP4 and selection checkers (oracle/fp4_oracle.py), and refusals of the library calls, without a GPU."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import fp4_oracle as Q


def test_codes_of_the_values_and_of_the_borders_between_them():
    assert Q.nearest_code(Q.VALUES).tolist() == list(range(8))
    borders = (Q.VALUES[1:] + Q.VALUES[:-1]) / 2
    assert Q.VALUES[Q.nearest_code(borders)].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    for b, lo, hi in zip(borders, Q.VALUES, Q.VALUES[1:]):
        got = Q.VALUES[Q.nearest_code(np.array([b - 1e-9, b + 1e-9]))]
        assert got.tolist() == [lo, hi]
    assert Q.VALUES[Q.nearest_code(np.array([5.01, 7.99]))].tolist() == [6.0, 6.0]


def test_a_block_worked_by_hand():
    x = np.zeros((1, 32))
    x[0, :6] = [12.0, -3.0, 1.0, 0.5, -0.49, 15.9]  # largest 15.9: 8 stands for 4, the step is 2
    codes, s = Q.quantize(x)
    assert s.tolist() == [[128]]
    assert Q.values(codes, s, 32)[0, :6].tolist() == [12.0, -3.0, 1.0, 0.0, 0.0, 12.0]  # 0.25 and 0.245 steps round to 0
    packed, sc = Q.store(codes, s)
    assert packed[0, :3].tolist() == [7 | (8 + 3) << 4, 1 | 0 << 4, 8 | 7 << 4] and sc.shape == (1, 4, 4) and sc[0, 0].tolist() == [128, 0, 0, 0]


@pytest.mark.parametrize("top,byte", [(0.0, 0), (4.0, 127), (3.999, 126), (2.0 ** -140, 0), (2.0 ** -126, 0), (2.0 ** -124, 1),
                                      (3.0e38, 252), (math.inf, 255), (math.nan, 255)])
def test_scale_bytes(top, byte):
    x = np.zeros((1, 32))
    x[0, 7] = top
    codes, s = Q.quantize(x)
    assert s[0, 0] == byte
    if byte != 255:
        assert abs(Q.values(codes, s, 32)[0, 7] - top) <= 0.25 * top + 2.0 ** -129


def test_stored_matrices_read_back():
    g = np.random.default_rng(1)
    for rows, n in ((1, 8), (3, 40), (6, 136), (5, 256)):
        codes, s = Q.quantize(g.normal(size=(rows, n)) * np.exp(g.normal(size=(rows, n))))
        assert np.array_equal(Q.load(*Q.store(codes, s), n), Q.values(codes, s, n))


def test_selection_worked_by_hand():
    l = np.log(np.array([[1.0, 2.0, 3.0, 4.0]]))
    idx, w = Q.select(l, 2)
    assert idx.tolist() == [[3, 2]] and np.allclose(w, [[4 / 7, 3 / 7]], rtol=1e-15)
    idx, w = Q.select(l, 2, bias=[0.5, 0.0, 0.0, 0.0], renorm=False, scale=2.0)  # 0.1 + 0.5 is the largest; the weight has no bias
    assert idx.tolist() == [[0, 3]] and np.allclose(w, [[0.2, 0.8]], rtol=1e-15)
    idx, _ = Q.select(l, 1, groups=2, kept=1, group_top=2)
    assert idx.tolist() == [[3]]
    idx, w = Q.select(np.array([[0.0, 0.0, -np.inf, 0.0]]), 3, scoring="sigmoid")
    assert idx.tolist() == [[0, 1, 3]] and np.allclose(w, 1 / 3)
    idx, w = Q.select(np.full((1, 4), -np.inf), 2)
    assert idx.tolist() == [[0, 1]] and not w.any()


# ---- refusals: nothing is launched, so no device is needed (the addresses are never followed)
A = 1 << 20  # an aligned address that is not null


def _fp4(rows, n, codes=A, scales=A):
    from paper_2503_00245_b200 import binding as B
    return B.moe_fp4(codes, scales, rows, n)


SELECT_BAD = [
    (dict(n_experts=0), 1), (dict(top_k=0), 1), (dict(scoring=2), 1), (dict(n_groups=3), 1), (dict(groups_kept=5), 1),
    (dict(groups_kept=0), 1), (dict(group_top=0), 1), (dict(group_top=3), 2), (dict(renorm=2), 1), (dict(scale=math.nan), 1),
    (dict(n_experts=260, n_groups=1, groups_kept=1), 2), (dict(top_k=9), 2), (dict(groups_kept=1, top_k=5), 1),
    (dict(n_experts=64, n_groups=64, groups_kept=64, group_top=1), 2), (dict(n_groups=16, groups_kept=16, group_top=2), 1),
]


@pytest.mark.parametrize("bad,status", SELECT_BAD)
def test_select_refuses(bad, status):
    from paper_2503_00245_b200 import binding as B
    good = dict(n_experts=16, top_k=2, scoring=1, n_groups=4, groups_kept=2, group_top=2, renorm=1, scale=1.0)
    call = B._lib().moe_select
    c = B.make_select_config(**good)
    assert call(C.addressof(c), None, 0, 16, 0, None, None, None, None) == 0  # no tokens: nothing to do
    c = B.make_select_config(**{**good, **bad})
    assert call(C.addressof(c), A, 0, 512, 4, None, A, A, None) == status


def test_select_refuses_arguments():
    from paper_2503_00245_b200 import binding as B
    cfg = B.make_select_config(16, 2)
    c = C.addressof(cfg)
    call = B._lib().moe_select
    assert call(None, A, 0, 16, 4, None, A, A, None) == 1
    assert call(c, A, 2, 16, 4, None, A, A, None) == 2       # type
    assert call(c, A, 0, 15, 4, None, A, A, None) == 1       # rows overlap
    assert call(c, A, 0, 16, -1, None, A, A, None) == 1
    assert call(c, None, 0, 16, 4, None, A, A, None) == 1
    assert call(c, A, 0, 16, 4, None, None, A, None) == 1
    assert call(c, A, 0, 16, 4, None, A, None, None) == 1
    assert call(c, A + 2, 0, 16, 4, None, A, A, None) == 1   # fp32 at an address that is not a multiple of 4
    assert call(c, A, 0, 16, 4, A + 1, A, A, None) == 1


def test_fp4_sizes():
    from paper_2503_00245_b200 import binding as B
    assert B.moe_fp4_bytes(5, 1440) == (5 * 720, 12 * 8 * 4)
    assert B.moe_fp4_bytes(0, 8) == (0, 0)
    assert B.moe_fp4_bytes(1 << 30, 32) == (1 << 34, 1 << 32)
    for rows, n, status in ((-1, 8, 1), (1, 0, 1), (1, 65537, 2), ((1 << 30) + 1, 8, 2)):
        with pytest.raises(B.MoeError) as e:
            B.moe_fp4_bytes(rows, n)
        assert e.value.status == status


def test_quantize_and_dequantize_refuse():
    from paper_2503_00245_b200 import binding as B
    q = B._lib().moe_fp4_quantize_rows
    good = dict(src=A, dtype=1, src_rows=4, rs=64, cs=1, row_of=None, div=1, rows=4, n=64, codes=A, scales=A, stream=None)

    def call(**k):
        return q(*{**good, **k}.values())
    assert call(rows=0, src=None, codes=None, scales=None) == 0
    for bad, status in ((dict(dtype=2), 2), (dict(n=0), 1), (dict(n=65544), 2), (dict(rows=-1), 1), (dict(rows=5), 1), (dict(div=0), 1),
                        (dict(rs=-64), 1), (dict(cs=-1), 1), (dict(src=None), 1), (dict(codes=None), 1), (dict(scales=None), 1),
                        (dict(codes=A + 8), 1), (dict(scales=A + 4), 1), (dict(src=A + 1), 1), (dict(src_rows=-1), 1)):
        assert call(**bad) == status, bad
    d = B._lib().moe_fp4_dequantize_rows

    def back(m=_fp4(4, 64), dst=A, dtype=1, stride=64):
        return d(None if m is None else C.addressof(m), dst, dtype, stride, None)
    assert back(_fp4(0, 64, None, None), None) == 0
    for got, status in ((back(None), 1), (back(_fp4(4, 60)), 2), (back(_fp4(4, 0)), 1), (back(_fp4(-1, 64)), 1), (back(dtype=3), 2),
                        (back(dst=None), 1), (back(dst=A + 8), 1), (back(stride=56), 1), (back(stride=68), 1), (back(_fp4(4, 64, A + 8)), 1),
                        (back(_fp4(4, 64, A, None)), 1)):
        assert got == status


def test_product_refuses():
    from paper_2503_00245_b200 import binding as B
    p = B._lib().moe_fp4_product

    def call(ctx=A, a=_fp4(40, 64), w=_fp4(64, 64), off=A, E=2, out=A, dtype=1, stride=32):
        return p(ctx, None if a is None else C.addressof(a), None if w is None else C.addressof(w), off, E, out, dtype, stride, None)
    assert call(a=_fp4(0, 64, None, None), off=None, out=None) == 0
    for got, status in ((call(ctx=None), 1), (call(a=None), 1), (call(w=None), 1), (call(E=0), 1), (call(E=65, w=_fp4(65 * 32, 64)), 2),
                        (call(E=3), 1), (call(w=_fp4(64, 72)), 1), (call(w=_fp4(0, 64)), 1), (call(w=_fp4(24, 64)), 2), (call(dtype=2), 2),
                        (call(stride=24), 1), (call(stride=36), 1), (call(off=None), 1), (call(out=None), 1), (call(out=A + 8), 1),
                        (call(off=A + 2), 1), (call(a=_fp4(40, 64, A + 8)), 1), (call(w=_fp4(64, 64, A, A + 8)), 1)):
        assert got == status


def test_pack_and_experts_refuse():
    from paper_2503_00245_b200 import binding as B
    f = B._lib().moe_fp4_pack_dense

    def pack(d=64, ff=40, E=2, g=A, u=A, dn=A, gu=_fp4(256, 64), down=_fp4(128, 40)):
        return f(d, ff, E, g, u, dn, C.addressof(gu), C.addressof(down), None)
    for got, status in ((pack(d=0), 1), (pack(d=60), 2), (pack(ff=44), 2), (pack(E=65), 2), (pack(g=None), 1), (pack(u=None), 1),
                        (pack(dn=None), 1), (pack(gu=_fp4(255, 64)), 1), (pack(gu=_fp4(256, 72)), 1), (pack(down=_fp4(120, 40)), 1),
                        (pack(down=_fp4(128, 48)), 1), (pack(gu=_fp4(256, 64, A + 8)), 1), (pack(down=_fp4(128, 40, A, None)), 1)):
        assert got == status
    gu, down = _fp4(256, 64), _fp4(128, 40)
    assert B._lib().moe_fp4_experts(None, A, 1, C.addressof(gu), C.addressof(down), A, A, A, A, 1 << 20, None) == 1
    sizes = [B.moe_fp4_workspace_bytes(B.make_config(1440, 3840, 8, 2), T) for T in range(0, 3000, 7)]
    assert sizes == sorted(sizes)
    for cfg, T, status in ((B.make_config(64, 44, 2, 1), 1, 2), (B.make_config(64, 40, 2, 1), -1, 1), (B.make_config(64, 40, 8, 8), 1 << 28, 2)):
        with pytest.raises(B.MoeError) as e:
            B.moe_fp4_workspace_bytes(cfg, T)
        assert e.value.status == status


def test_python_calls_refuse_what_does_not_fit():
    import torch

    import paper_2503_00245_b200 as P
    with pytest.raises(ValueError):
        P.Fp4Rows(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(1, 4, 4, dtype=torch.uint8), 96)
    with pytest.raises(TypeError):
        P.Fp4Rows(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(1, 4, 4, dtype=torch.uint8), 64)
    with pytest.raises(ValueError):
        P.select_experts(torch.zeros(3, 9), P.SelectRule(8, 2))
    with pytest.raises(ValueError):
        P.select_experts(torch.zeros(3, 8), P.SelectRule(8, 2), torch.zeros(7))
    with pytest.raises(KeyError):
        P.SelectRule(8, 2, scoring="tanh")
    with pytest.raises(ValueError):
        P.fp4_quantize(torch.zeros(8))
