"""What the Python calls of selection and 4-bit rows refuse before anything reaches the library (no GPU needed)."""
import pytest
import torch


class Unreached:
    """Stands in for the library: a call that gets there has not been refused."""

    def __getattr__(self, name):
        def call(*args):
            raise RuntimeError(f"{name} was called")
        return call


@pytest.fixture
def B(monkeypatch):
    from paper_2503_00245_b200 import binding
    monkeypatch.setattr(binding, "_LIB", Unreached())
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_current_raw_stream", lambda device: 0)
    return binding


def test_tensors_in_pageable_host_memory(B):
    """Strided ones among them: the binding passes their address to kernels."""
    rows, out = torch.zeros(4, 64), torch.zeros(4, 8)
    m = B.moe_fp4(1 << 20, 1 << 20, 4, 64)
    for call in (lambda: B.moe_select(B.make_select_config(64, 2), rows, 4, None, 1 << 20, 1 << 20),
                 lambda: B.moe_fp4_quantize_rows(rows, None, 1, 4, 1 << 20, 1 << 20),
                 lambda: B.moe_fp4_quantize_rows(rows[:, ::2], None, 1, 4, 1 << 20, 1 << 20),
                 lambda: B.moe_fp4_dequantize_rows(m, rows),
                 lambda: B.moe_fp4_product(1 << 20, m, B.moe_fp4(1 << 20, 1 << 20, 8, 64), 1 << 20, 1, out)):
        with pytest.raises(AssertionError):
            call()


def test_failures_of_products_without_a_context_can_be_asked_for(B, monkeypatch):
    import paper_2503_00245_b200 as P
    monkeypatch.setattr(P.layer, "_shared", {0: 41, 1: 42})
    asked = []
    monkeypatch.setattr(B, "moe_check", lambda ctx: asked.append(ctx) or 5)
    assert P.fp4_check() == 5 and asked == [41]
    monkeypatch.setattr(B, "_current_device", lambda: 2)  # no call yet on this one
    assert P.fp4_check() == 0 and asked == [41]


def test_threads_share_one_context(B, monkeypatch):
    import threading
    import time

    from paper_2503_00245_b200 import layer as L
    monkeypatch.setattr(L, "_shared", {})
    made, got = [], []

    def create(cfg):
        time.sleep(0.05)  # (the other threads come while the first one's is being made)
        made.append(len(made) + 1)
        return made[-1]
    monkeypatch.setattr(B, "moe_create", create)
    threads = [threading.Thread(target=lambda: got.append(L._shared_ctx())) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert made == [1] and got == [1] * 8


@pytest.mark.parametrize("layers,rules,fits", [(None, True, True), (None, False, True), (True, True, True), (False, False, True),
                                               (False, True, False), (True, False, False)])
def test_a_layers_renorm_agrees_with_its_rule(B, monkeypatch, layers, rules, fits):
    import paper_2503_00245_b200 as P
    monkeypatch.setattr(B, "make_weights", lambda *a, **k: None)
    monkeypatch.setattr(B, "moe_create", lambda cfg: 41)
    monkeypatch.setattr(B, "moe_destroy", lambda ctx: None)
    monkeypatch.setattr(B, "moe_workspace_bytes", lambda cfg, T: 16)
    kw = dict(dense=torch.zeros(1), select=P.SelectRule(8, 2, renorm=rules))
    if layers is not None:
        kw["renorm"] = layers
    if not fits:
        with pytest.raises(ValueError):
            P.MoELayer(64, 64, 8, 2, torch.zeros(64, 8), **kw)
        return
    assert P.MoELayer(64, 64, 8, 2, torch.zeros(64, 8), **kw).cfg.renorm == rules  # (closed at once, by the stand-in)
    del kw["select"]  # without a rule: as asked, True where nothing is
    assert P.MoELayer(64, 64, 8, 2, torch.zeros(64, 8), **kw).cfg.renorm == (layers is not False)


def test_experts_to_be_packed_have_fitting_shapes_and_types(B, monkeypatch):
    """The library is given three addresses and one set of sizes: a smaller matrix would be read behind its end."""
    import paper_2503_00245_b200 as P
    monkeypatch.setattr(P.layer, "_here", lambda *t: None)
    packed = []
    monkeypatch.setattr(B, "moe_fp4_pack_dense", lambda *a: packed.append(a[:3]))
    w = [torch.zeros(2, 64, 40, dtype=torch.bfloat16), torch.zeros(2, 64, 40, dtype=torch.bfloat16), torch.zeros(2, 40, 64, dtype=torch.bfloat16)]
    P.pack_fp4(*w)
    assert packed == [(64, 40, 2)]
    for i, bad in ((1, w[1][:1]), (1, w[1][:, :32]), (1, w[2]), (2, w[2][:, :32]), (2, w[1]), (2, w[2][0])):
        with pytest.raises(ValueError):
            P.pack_fp4(*w[:i], bad, *w[i + 1:])
    for i in range(3):
        with pytest.raises(TypeError):
            P.pack_fp4(*w[:i], w[i].float(), *w[i + 1:])
        with pytest.raises(TypeError):
            P.pack_fp4(*w[:i], w[i].half(), *w[i + 1:])
    assert len(packed) == 1


@pytest.fixture
def layer(B, monkeypatch):
    """A layer with a selection rule whose library calls are noted and not made."""
    import paper_2503_00245_b200 as P
    monkeypatch.setattr(P.layer, "_here", lambda *t: None)
    monkeypatch.setattr(B, "make_weights", lambda *a, **k: None)
    monkeypatch.setattr(B, "moe_create", lambda cfg: 41)
    monkeypatch.setattr(B, "moe_destroy", lambda ctx: None)
    monkeypatch.setattr(B, "moe_workspace_bytes", lambda cfg, T: 16)
    lay = P.MoELayer(64, 64, 8, 2, torch.zeros(64, 8), dense=torch.zeros(1), select=P.SelectRule(8, 2), max_tokens=4)
    lay.asked = []
    monkeypatch.setattr(B, "moe_route_logits", lambda ctx, x, T, w, out: lay.asked.append((T, tuple(out.shape))))
    yield lay
    lay.close()  # (while its context is one that nobody made)


def test_rows_whose_logits_are_asked_for_have_the_layers_width_and_type(layer):
    x = torch.zeros(3, 64, dtype=torch.bfloat16)
    layer.logits(x)
    for bad in (x[:, :56], torch.zeros(3, 72, dtype=torch.bfloat16), x.float(), x.half(), x[0], x[None]):
        for call in (layer.logits, layer.route, layer.forward):
            with pytest.raises(ValueError):
                call(bad)
    assert layer.asked == [(3, (3, 8))]


def test_experts_outputs_lie_on_the_current_device(B, monkeypatch):
    import paper_2503_00245_b200 as P

    class Tensor(torch.Tensor):
        index = 0

        def get_device(self):
            return self.index

    def made(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype).as_subclass(Tensor)
    ex = object.__new__(P.Fp4Experts)
    ex.d, ex.k, ex.x_dtype, ex.max_tokens, ex.device, ex.ctx, ex.lent = 64, 2, torch.bfloat16, 4, torch.device("cpu"), 41, True
    ex.ws, ex.gu, ex.down = made(16), P.Fp4Rows.empty(0, 64, "cpu"), P.Fp4Rows.empty(0, 64, "cpu")
    ran = []
    monkeypatch.setattr(B, "moe_fp4_experts", lambda *a: ran.append(a))
    x, idx, wt, y = made(3, 64), made(3, 2, dtype=torch.int32), made(3, 2, dtype=torch.float32), made(3, 64)
    assert ex.forward(x, idx, wt, y) is y and len(ran) == 1
    for t in (x, idx, wt, y):
        t.index = 1
        with pytest.raises(ValueError):
            ex.forward(x, idx, wt, y)
        t.index = 0
    assert len(ran) == 1


def test_addresses_that_kernels_could_not_read():
    """Nothing is launched, so no device is needed (the addresses are never followed)."""
    import ctypes as C

    from paper_2503_00245_b200 import binding as B
    A = 1 << 20
    quantize, pack = B._lib().moe_fp4_quantize_rows, B._lib().moe_fp4_pack_dense
    for off in (1, 2, 3):
        assert quantize(A, 1, 4, 64, 1, A + off, 1, 4, 64, A, A, None) == 1
    gu, down = B.moe_fp4(A, A, 256, 64), B.moe_fp4(A, A, 128, 40)
    for g, u, d in ((A + 1, A, A), (A, A + 1, A), (A, A, A + 1)):
        assert pack(64, 40, 2, g, u, d, C.addressof(gu), C.addressof(down), None) == 1


def test_numbers_longer_than_32_bits(B):
    """Of 2^32 + 5 tokens the library would be told 5."""
    import paper_2503_00245_b200 as P

    class Rows:  # stands in for a matrix on the device
        is_cuda, dtype, shape = True, torch.bfloat16, (1, (1 << 32) + 64)

        def data_ptr(self):
            return 1 << 20

        def stride(self, i):
            return 1

    A, long, rows = 1 << 20, (1 << 32) + 8, Rows()
    m, cfg = B.moe_fp4(A, A, 8, 64), B.make_config(64, 64, 8, 2)
    for v in (long, 1 << 31, -(1 << 31) - 1):
        for call in (lambda: B.moe_select(B.make_select_config(8, 2), rows, v, None, A, A), lambda: B.moe_route_logits(A, A, v, B.moe_weights(), A),
                     lambda: B.moe_fp4_bytes(8, v), lambda: B.moe_fp4_quantize_rows(rows, None, 1, 1, A, A),
                     lambda: B.moe_fp4_quantize_rows(rows, None, v, 1, A, A), lambda: B.moe_fp4_product(A, m, m, A, v, rows, 8),
                     lambda: B.moe_fp4_workspace_bytes(cfg, v), lambda: B.moe_fp4_experts(A, A, v, m, m, A, A, A, torch.zeros(8)),
                     lambda: B.moe_fp4_pack_dense(v, 8, 1, A, A, A, m, m), lambda: B.moe_fp4_pack_dense(8, v, 1, A, A, A, m, m),
                     lambda: B.make_fp4(A, A, 8, v), lambda: P.Fp4Rows.empty(0, v, "cpu")):
            with pytest.raises(OverflowError):
                call()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int16])
def test_rows_are_of_a_type_that_the_kernels_read(B, monkeypatch, dtype):
    """(Everything but float32 was read as bfloat16.)"""
    import paper_2503_00245_b200 as P
    monkeypatch.setattr(P.layer, "_here", lambda *t: None)
    monkeypatch.setattr(B, "make_weights", lambda *a, **k: None)
    monkeypatch.setattr(B, "moe_create", lambda cfg: None)
    monkeypatch.setattr(B, "moe_workspace_bytes", lambda cfg, T: 16)
    monkeypatch.setattr(B, "moe_fp4_workspace_bytes", lambda cfg, T: 16)
    q = P.Fp4Rows.empty(8, 64, "cpu")
    for ok in (torch.float32, torch.bfloat16):
        assert P.Fp4Experts(64, 64, 8, 2, q, q, x_dtype=ok).cfg.x_dtype == B.dtype_of(ok)
        assert P.MoELayer(64, 64, 8, 2, torch.zeros(64, 8), fp4=(q, q), x_dtype=ok).cfg.x_dtype == B.dtype_of(ok)
    with pytest.raises(TypeError):
        P.Fp4Experts(64, 64, 8, 2, q, q, x_dtype=dtype)
    for kind in (dict(dense=torch.zeros(1)), dict(fp4=(q, q))):
        with pytest.raises(TypeError):
            P.MoELayer(64, 64, 8, 2, torch.zeros(64, 8), **kind, x_dtype=dtype)
