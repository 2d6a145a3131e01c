"""Host-side checks of the mx4 and norm entry points: sizes, defaults, refusals before anything is enqueued.  CPU only."""
import ctypes as C

import pytest

import paper_2506_01352_amd as tahq
from oracle import mx4
from paper_2506_01352_amd import binding

P = 4096                                     # an aligned address that is never read: every call here is refused


def _status(name, *arguments):
    return getattr(binding._load(), name)(*[C.byref(a) if isinstance(a, C.Structure) else a for a in arguments])


def test_sizes_and_defaults():
    for rows, cols in ((1, 1), (32, 64), (33, 65), (777, 1600), (4096, 8192)):
        assert tahq.tahq_mx4_packed_size(rows, cols) == mx4.packed_size(rows, cols)
    assert tahq.tahq_mx4_packed_size(0, 5) == tahq.tahq_mx4_packed_size(5, 0) == tahq.tahq_mx4_packed_size(1 << 31, 1) == 0
    c, m, n = tahq.tahq_mx4_config_default(), tahq.tahq_mx4_matmul_config_default(), tahq.tahq_norm_config_default()
    assert (c.struct_size, c.dtype, c.transform, c.scale_rule, c.rows) == (C.sizeof(tahq.tahq_mx4_config), tahq.BF16, 0, tahq.MX4_FLOOR, 0)
    assert (m.struct_size, m.out_dtype, m.accumulate, m.ldc) == (C.sizeof(tahq.tahq_mx4_matmul_config), tahq.BF16, 0, 0)
    assert (n.struct_size, n.dtype, n.gate_rows, n.residual_scale, n.accumulate) == (C.sizeof(tahq.tahq_norm_config), tahq.BF16, 0, 1.0, 0)
    assert abs(n.eps - 1e-6) < 1e-12


@pytest.mark.parametrize("field, value", [("rows", 0), ("cols", 0), ("rows", 1 << 31), ("ld", 63), ("dtype", 2), ("transform", 2),
                                          ("scale_rule", 2), ("struct_size", 8)])
def test_quantizer_refuses_configurations(field, value):
    cfg = tahq.make_mx4_config(32, 64, tahq.BF16)
    setattr(cfg, field, value)
    big = 1 << 20
    assert _status("tahq_mx4_quantize", cfg, P, P, big, None, 0, None) == 2
    assert _status("tahq_mx4_dequantize", cfg, P, big, P, None) == 2
    assert tahq.tahq_mx4_linear_workspace_size(cfg, tahq.make_mx4_matmul_config(32, 5, 64, tahq.BF16)) == 0


def test_quantizer_refuses_arguments():
    cfg, need, need_t = tahq.make_mx4_config(40, 100, tahq.F32), tahq.tahq_mx4_packed_size(40, 100), tahq.tahq_mx4_packed_size(100, 40)
    q = lambda *a: _status("tahq_mx4_quantize", cfg, *a, None)      # noqa: E731
    assert q(None, P, need, None, 0) == 1 and q(P, None, 0, None, 0) == 1 and _status("tahq_mx4_quantize", None, P, P, need, None, 0, None) == 1
    assert q(P, P, need - 1, None, 0) == 4 and q(P, P, need, P, need_t - 1) == 4
    assert q(P + 4, P, need, None, 0) == 6 and q(P, P + 8, need, None, 0) == 6 and q(P, None, 0, P + 1, need_t) == 6
    d = lambda *a: _status("tahq_mx4_dequantize", cfg, *a, None)    # noqa: E731
    assert d(None, need, P) == 1 and d(P, need, None) == 1 and d(P, need - 1, P) == 4 and d(P + 2, need, P) == 6 and d(P, need, P + 2) == 6


def test_product_refuses_arguments():
    cfg = tahq.make_mx4_matmul_config(40, 50, 100, tahq.BF16)
    a, b = tahq.tahq_mx4_packed_size(40, 100), tahq.tahq_mx4_packed_size(50, 100)
    ws = tahq.tahq_mx4_matmul_workspace_size(cfg)
    call = lambda *x: _status("tahq_mx4_matmul", *x, None)          # noqa: E731
    assert call(cfg, None, a, P, b, P, P, ws) == 1 and call(cfg, P, a, None, b, P, P, ws) == 1 and call(cfg, P, a, P, b, None, P, ws) == 1
    assert call(cfg, P, a - 1, P, b, P, P, ws) == 4 and call(cfg, P, a, P, b - 1, P, P, ws) == 4
    assert call(cfg, P + 8, a, P, b, P, P, ws) == 6 and call(cfg, P, a, P, b, P + 2, P, ws) == 6
    for field, value in (("m", 0), ("n", 0), ("k", 0), ("k", 1 << 31), ("ldc", 49), ("out_dtype", 2), ("accumulate", 2), ("struct_size", 0)):
        bad = tahq.make_mx4_matmul_config(40, 50, 100, tahq.BF16)
        setattr(bad, field, value)
        assert call(bad, P, 1 << 30, P, 1 << 30, P, P, 1 << 30) == 2 and tahq.tahq_mx4_matmul_workspace_size(bad) == 0
    # a product with few tiles and a long sum keeps parts of it
    long = tahq.make_mx4_matmul_config(256, 256, 32768, tahq.F32)
    need = tahq.tahq_mx4_matmul_workspace_size(long)
    if need:
        assert call(long, P, 1 << 30, P, 1 << 30, P, P, need - 1) == 5 and call(long, P, 1 << 30, P, 1 << 30, P, None, need) == 1


def test_layer_refuses_arguments():
    x, cfg = tahq.make_mx4_config(4, 100, tahq.BF16), tahq.make_mx4_matmul_config(4, 50, 100, tahq.BF16)
    need, b = tahq.tahq_mx4_linear_workspace_size(x, cfg), tahq.tahq_mx4_packed_size(50, 100)
    assert need >= tahq.tahq_mx4_packed_size(4, 100)
    call = lambda *a: _status("tahq_mx4_linear", *a, None)          # noqa: E731
    assert call(x, cfg, None, P, b, P, P, need) == 1 and call(x, cfg, P, P, b, P, None, need) == 1
    assert call(x, cfg, P, P, b - 1, P, P, need) == 4 and call(x, cfg, P, P, b, P, P, need - 1) == 5 and call(x, cfg, P, P, b, P + 2, P, need) == 6
    for other in (tahq.make_mx4_matmul_config(5, 50, 100, tahq.BF16), tahq.make_mx4_matmul_config(4, 50, 101, tahq.BF16)):
        assert call(x, other, P, P, 1 << 30, P, P, 1 << 30) == 2 and tahq.tahq_mx4_linear_workspace_size(x, other) == 0


def _norm(**changed):
    cfg = tahq.make_norm_config(40, 100, tahq.BF16, changed.pop("gate_rows", 0))
    for k, v in changed.items():
        setattr(cfg, k, v)
    return cfg


@pytest.mark.parametrize("field, value, status", [
    ("rows", 0, 2), ("rows", 1 << 31, 2), ("cols", 0, 2), ("cols", tahq.NORM_MAX_COLS + 1, 3), ("dtype", 2, 2), ("eps", 0.0, 2), ("eps", -1.0, 2),
    ("eps", float("nan"), 2), ("eps", float("inf"), 2), ("residual_scale", float("inf"), 2), ("residual_scale", float("nan"), 2),
    ("accumulate", 2, 2), ("transform", 2, 2), ("scale_rule", 2, 2), ("struct_size", 4, 2)])
def test_norms_refuse_configurations(field, value, status):
    cfg = _norm(**{field: value})
    assert tahq.tahq_norm_workspace_size(cfg) == 0
    assert _status("tahq_norm_forward", cfg, P, P, P, None, P, P, P, None, 0, None, None) == status
    assert _status("tahq_norm_backward", cfg, P, P, P, P, None, P, P, P, P, P, P, None, P, P, 1 << 30, None) == status


def test_norms_refuse_arguments_that_do_not_belong_together():
    f = lambda cfg, *a: _status("tahq_norm_forward", cfg, *a, None)     # noqa: E731
    c, g, N = _norm(), _norm(gate_rows=8), None
    need = tahq.tahq_mx4_packed_size(40, 100)
    #        residual block w_post gate w_pre out h mx4 cap stats
    assert f(c, N, P, P, N, P, P, P, N, 0, N) == 1                      # no residual
    assert f(c, P, P, N, N, P, P, P, N, 0, N) == 1                      # a block without its weight
    assert f(c, P, P, P, N, P, N, P, N, 0, N) == 1                      # a block, and nowhere for r'
    assert f(c, P, P, P, P, P, P, P, N, 0, N) == 2                      # a gate that the configuration has not
    assert f(g, P, P, P, N, P, P, P, N, 0, N) == 1                      # none that it has
    assert f(c, P, N, P, N, P, P, P, N, 0, N) == 2                      # a weight without a block
    assert f(c, P, P, P, N, P, P, N, N, 0, N) == 1                      # a pre half, and nowhere for h
    assert f(c, P, P, P, N, N, P, P, N, 0, N) == 2                      # h without a pre half
    assert f(c, P, N, N, N, N, N, N, N, 0, N) == 1                      # nothing to do
    assert f(c, P, P, P, N, P, P, N, P, need - 1, N) == 4
    assert f(c, P + 2, P, P, N, P, P, P, N, 0, N) == 6 and f(c, P, P, P, N, P, P, P, N, 0, P + 4) == 6
    b = lambda cfg, *a: _status("tahq_norm_backward", cfg, *a, None)    # noqa: E731
    ws = tahq.tahq_norm_workspace_size(c)
    assert tahq.tahq_norm_workspace_size(g) > ws > 0
    #        gout gh block w_post gate rout w_pre stats | gres gblock gwpost ggate gwpre ws cap
    assert b(c, N, N, P, P, N, N, N, P, P, P, P, N, N, P, ws) == 1      # nothing comes back
    assert b(c, P, P, P, P, N, P, P, N, P, P, P, N, P, P, ws) == 1      # no statistics
    assert b(c, P, P, P, P, N, N, P, P, P, P, P, N, P, P, ws) == 1      # no r'
    assert b(c, P, N, P, P, N, N, P, P, P, P, P, N, N, P, ws) == 2      # a weight without its half
    assert b(c, P, P, P, P, P, P, P, P, P, P, P, P, P, P, ws) == 2      # a gate that the configuration has not
    assert b(g, P, P, P, P, N, P, P, P, P, P, P, N, P, P, 1 << 30) == 1
    assert b(c, P, P, N, N, N, P, P, P, P, P, N, N, P, P, ws) == 2      # a block's gradient without a block
    assert b(c, P, P, P, P, N, P, P, P, P, P, P, N, P, P, ws - 1) == 5
    assert b(c, P, P, P, P, N, P, P, P, P, P, P, N, P, P + 8, ws) == 6


def test_binding_refuses_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    x = torch.zeros(40, 99, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        tahq.tahq_mx4_quantize(tahq.make_mx4_config(40, 100, tahq.BF16), x, P)
    with pytest.raises(ValueError):
        tahq.tahq_mx4_quantize(tahq.make_mx4_config(40, 99, tahq.F32), x, P)
    with pytest.raises(ValueError):
        tahq.tahq_mx4_quantize(tahq.make_mx4_config(40, 60, tahq.BF16, 99), x[:, :50], P)
    with pytest.raises(ValueError):
        tahq.tahq_norm_forward(tahq.make_norm_config(40, 100, tahq.BF16), x, None, None, None, x, x, x)
    with pytest.raises(tahq.TahqError):
        tahq.Mx4Tensor(tahq.make_mx4_config(0, 100, tahq.BF16))
    with pytest.raises(tahq.TahqError):
        tahq.BlockNorm(tahq.make_norm_config(4, tahq.NORM_MAX_COLS + 1, tahq.BF16))
