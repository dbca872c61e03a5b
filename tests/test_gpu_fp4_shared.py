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
