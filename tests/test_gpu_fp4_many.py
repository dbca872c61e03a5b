"""Experts in 4 bits over very many tokens."""
import statistics

import pytest
import torch

pytestmark = pytest.mark.gpu


def P():
    import paper_2503_00245_b200 as p
    return p


def experts(E, k, d, f, T, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(d + f)
    wg, wu = ((torch.randn(E, d, f, generator=g) * d ** -0.5).bfloat16().cuda() for _ in range(2))
    wd = (torch.randn(E, f, d, generator=g) * f ** -0.5).bfloat16().cuda()
    return P().Fp4Experts(d, f, E, k, *P().pack_fp4(wg, wu, wd), x_dtype=dtype, max_tokens=T)


def inputs(T, d, E, k, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, d, generator=g, device="cuda").to(dtype)
    top, idx = torch.topk(torch.randn(T, E, generator=g, device="cuda"), k, dim=1)
    return x, idx.to(torch.int32), torch.softmax(top, 1)


@pytest.mark.parametrize("T,E,k,d,f,dtype", [(310000, 8, 2, 64, 32, torch.bfloat16), (700001, 64, 8, 16, 8, torch.float32),
                                             (303104, 5, 1, 1096, 8, torch.bfloat16)])
def test_more_tokens_than_a_block_holds_at_a_time(T, E, k, d, f, dtype):
    """A row's output does not depend on which rows are beside it: the whole call gives what calls of a part each give."""
    ex = experts(E, k, d, f, T, dtype)
    x, idx, wt = inputs(T, d, E, k, dtype)
    y = ex.forward(x, idx, wt)
    assert ex.check() == 0
    at = 0
    for n in (1000, 30011, 100000, T):
        part = ex.forward(x[at:at + n], idx[at:at + n], wt[at:at + n])
        assert torch.equal(part, y[at:at + n])
        at = min(T, at + n)
    bad = idx.clone()
    bad[T - 3, k - 1] = E
    z = ex.forward(x, bad, wt)
    assert ex.check() == 6
    keep = torch.arange(T, device="cuda") != T - 3
    assert torch.equal(z[keep], y[keep])


def test_time_grows_with_the_tokens_and_not_with_their_square():
    """Four times the tokens: four times the work, sixteen times if every block of a few tokens walked all of them."""
    E, k, d, f, T = 8, 8, 8, 8, 1 << 22
    ex = experts(E, k, d, f, T)
    x, idx, wt = inputs(T, d, E, k)
    took = []
    for n in (T // 4, T):
        ms = []
        for _ in range(4):
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            a.record()
            ex.forward(x[:n], idx[:n], wt[:n])
            b.record()
            torch.cuda.synchronize()
            ms.append(a.elapsed_time(b))
        took.append(statistics.median(ms[1:]))
    print("ms", took)
    assert took[1] < 8 * took[0], took
