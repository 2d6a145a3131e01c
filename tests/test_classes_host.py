"""What the binding and its classes hand to the library, on the CPU: tensors stand in for device memory, and calls that would enqueue
work are written down instead."""
import pytest
import torch

import paper_2506_01352_amd as tahq
from paper_2506_01352_amd import binding


class Recorder:
    """The library, with calls that take a stream recorded: (name, arguments)."""

    def __init__(self, lib):
        self.lib, self.calls = lib, []

    def __getattr__(self, name):
        if name.endswith(("_default", "_size", "_string")):
            return getattr(self.lib, name)

        def call(*arguments):
            self.calls.append((name, arguments))
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    recorder = Recorder(binding._load())
    monkeypatch.setattr(binding, "_lib", recorder)
    monkeypatch.setattr(binding, "_load", lambda: recorder)
    monkeypatch.setattr(binding, "_stream_handle", lambda stream: stream)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    return recorder


@pytest.mark.parametrize("ld", (0, 64))
def test_a_row_that_stands_for_many_is_no_matrix(library, ld):
    """A broadcast view has the rows' shape and none of their memory, whether the configuration names its row stride or leaves it at 0 = cols."""
    wide = torch.zeros(1, 64, dtype=torch.bfloat16).expand(40, 64)
    out = torch.zeros(40, 64, dtype=torch.bfloat16)
    packed, ws = (torch.zeros(1 << 16, dtype=torch.uint8) for _ in range(2))
    cfg, product = tahq.make_mx4_config(40, 64, tahq.BF16, ld), tahq.make_mx4_matmul_config(40, 64, 64, tahq.BF16, ld)
    for call in (lambda: tahq.tahq_mx4_quantize(cfg, wide, packed), lambda: tahq.tahq_mx4_dequantize(cfg, packed, wide),
                 lambda: tahq.tahq_mx4_matmul(product, packed, packed, wide, ws),
                 lambda: tahq.tahq_mx4_linear(cfg, product, wide, packed, out, ws),
                 lambda: tahq.tahq_mx4_linear(cfg, product, out, packed, wide, ws)):
        with pytest.raises((AssertionError, ValueError)):
            call()
    assert not library.calls
    tahq.tahq_mx4_quantize(cfg, out, packed)
    tahq.tahq_mx4_quantize(tahq.make_mx4_config(40, 32, tahq.BF16, 64), out[:, :32], packed)
    assert [name for name, _ in library.calls] == ["tahq_mx4_quantize"] * 2


def _norm(mx4=False, accumulate=0, **more):
    return tahq.BlockNorm(tahq.make_norm_config(6, 64, tahq.BF16, 2, accumulate=accumulate), mx4, device="cpu", **more)


def _norm_inputs():
    t = {n: torch.zeros(6, 64, dtype=torch.bfloat16) for n in ("grad_residual_out", "grad_h", "block", "residual_out")}
    t.update({n: torch.zeros(64, dtype=torch.bfloat16) for n in ("w_post", "w_pre")})
    return {**t, "gate": torch.zeros(3, 64, dtype=torch.bfloat16), "stats": torch.zeros(2, 6)}


@pytest.mark.parametrize("accumulate", (0, 1))
def test_gradients_of_norms_start_at_zero_before_any_call(library, monkeypatch, accumulate):
    """The buffers are made and cleared on torch's current stream, which a call's own stream does not wait for: not within the call."""
    norm = _norm(accumulate=accumulate)
    inputs = _norm_inputs()

    def none(*a, **k):
        raise AssertionError("memory is allocated or filled within the call")

    with monkeypatch.context() as m:
        for name in ("empty", "zeros", "empty_like", "zeros_like", "full"):
            m.setattr(torch, name, none)
        got = norm.backward(**inputs, stream=77)
    assert [(name, a[-1]) for name, a in library.calls] == [("tahq_norm_backward", 77)]
    assert all(got[n].dtype is torch.float32 and (not accumulate or (got[n] == 0).all()) for n in ("grad_w_post", "grad_w_pre", "grad_gate"))


def test_norms_without_a_backward_pass_keep_no_buffers_for_it(library):
    norm = _norm(training=False)
    with pytest.raises(ValueError, match="training"):
        norm.backward(**_norm_inputs())
    assert not library.calls and not hasattr(norm, "grad_block")


def _layer(tokens=40, n=96, k=64, dtype=torch.bfloat16, **more):
    return tahq.Mx4Linear(torch.zeros(n, k, dtype=dtype), tokens, **more)


def _x_of_weight_gradient(library):
    """Address of the matrix that the last product, the weight's gradient, took for x."""
    name, a = library.calls[-1]
    assert name == "tahq_mx4_matmul"
    return a[3]


def test_the_weights_gradient_is_of_the_x_that_the_layer_was_last_given(library):
    layer = _layer(training=True)
    x, dy = torch.zeros(40, 64, dtype=torch.bfloat16), torch.zeros(40, 96, dtype=torch.bfloat16)
    h, h_t = (torch.zeros(tahq.tahq_mx4_packed_size(*s), dtype=torch.uint8) for s in ((40, 64), (64, 40)))
    before = len(library.calls)
    with pytest.raises(ValueError, match="no x"):
        layer.backward(dy)                                           # nothing went forward
    layer.forward(x)
    for _ in range(2):
        layer.backward(dy)
        assert _x_of_weight_gradient(library) == layer.x_t.data_ptr()
    layer.product(h)                                                 # of this x the layer has nothing along tokens
    enqueued = len(library.calls)
    with pytest.raises(ValueError, match="no x"):
        layer.backward(dy)
    assert len(library.calls) == enqueued > before
    layer.product(h, x_packed_t=h_t)
    layer.backward(dy)
    assert _x_of_weight_gradient(library) == h_t.data_ptr()
    layer.forward(x)
    layer.backward(dy)
    assert _x_of_weight_gradient(library) == layer.x_t.data_ptr()


@pytest.mark.parametrize("dtype", (torch.float16, torch.float64, torch.int16, torch.uint8))
def test_layers_take_no_types_but_fp32_and_bf16(library, dtype):
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        tahq.Mx4Linear(torch.zeros(96, 64, dtype=dtype), 40)
    for training in (False, True):
        layer = _layer(training=training)
        enqueued = len(library.calls)
        with pytest.raises(ValueError, match="bfloat16"):
            layer.update(torch.zeros(96, 64, dtype=dtype))
        with pytest.raises(ValueError, match="bfloat16"):
            layer.forward(torch.zeros(40, 64, dtype=dtype))
        assert len(library.calls) == enqueued
    layer.forward(torch.zeros(40, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="bfloat16"):
        layer.backward(torch.zeros(40, 96, dtype=dtype))


@pytest.mark.parametrize("shape", [(41, 64), (80, 64), (39, 64), (64, 40), (20, 128), (40, 32), (2, 40, 64), (41 * 64,), (0, 64)])
def test_layers_take_as_many_tokens_as_they_were_made_for(library, shape):
    bad = torch.zeros(shape, dtype=torch.bfloat16)
    for training in (False, True):
        layer = _layer(training=training)
        enqueued = len(library.calls)
        with pytest.raises(ValueError, match="x is a"):
            layer.forward(bad)
        with pytest.raises(ValueError, match="weight is a"):
            layer.update(bad)
        assert len(library.calls) == enqueued
        layer.forward(torch.zeros(2, 20, 64, dtype=torch.bfloat16))          # tokens in two dimensions, or one row of them
        layer.forward(torch.zeros(40 * 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="grad_y is a"):
        layer.backward(bad)
    layer.backward(torch.zeros(4, 10, 96, dtype=torch.bfloat16))


def test_norms_take_tensors_of_their_shape(library):
    norm, t = _norm(), _norm_inputs()
    forward = {**{n: t[n] for n in ("block", "w_post", "gate", "w_pre")}, "residual": t["residual_out"]}
    norm.forward(**forward)
    norm.backward(**t)
    assert [name for name, _ in library.calls] == ["tahq_norm_forward", "tahq_norm_backward"]
    for call, inputs in ((norm.forward, forward), (norm.backward, t)):
        for name, good in inputs.items():
            for shape in ({6: [(7, 64), (12, 64), (64, 6), (5, 64)], 3: [(6, 64), (2, 64), (64, 3)], 64: [(65,), (64, 2), (6, 64)],
                           2: [(2, 7), (3, 6), (6, 2)]}[good.shape[0]]):
                with pytest.raises(ValueError, match=f" {name} is a"):
                    call(**{**inputs, name: torch.zeros(shape, dtype=good.dtype)})
    assert len(library.calls) == 2


def test_products_of_packed_matrices_that_do_not_fit_the_layer_are_refused(library):
    """What the classes pack carries its rows, columns and rotation; other bytes are taken as they are, other types are not."""
    layer = _layer(transform=1, training=True)
    size = tahq.tahq_mx4_packed_size(40, 64)

    def packed(rows, cols, transform):
        t = tahq.Mx4Tensor(tahq.make_mx4_config(rows, cols, tahq.BF16, 0, transform), transposed=True, device="cpu")
        return t.packed, t.packed_t

    def h(rows, cols, transform):
        cfg = tahq.make_norm_config(rows, cols, tahq.BF16, transform=transform)
        norm = tahq.BlockNorm(cfg, mx4=True, device="cpu")
        assert norm.h.numel() == tahq.tahq_mx4_packed_size(rows, cols)
        return norm.h

    x, x_t = packed(40, 64, 1)
    enqueued = len(library.calls)
    for bad in (packed(40, 64, 0)[0], packed(33, 64, 1)[0], packed(64, 40, 1)[0], packed(40, 63, 1)[0], x_t, h(40, 64, 0), h(64, 64, 1)):
        with pytest.raises(ValueError, match="x_packed is"):
            layer.product(bad)
    for bad in (packed(40, 64, 0)[1], packed(40, 33, 1)[1], x):
        with pytest.raises(ValueError, match="x_packed_t is"):
            layer.product(x, x_packed_t=bad)
    for bad in (torch.zeros(40, 64, dtype=torch.bfloat16), torch.zeros(40, 64), torch.zeros(size - 1, dtype=torch.uint8),
                torch.zeros(2 * size, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="x_packed is"):
            layer.product(bad)
        with pytest.raises(ValueError, match="x_packed_t is"):
            layer.product(x, x_packed_t=bad)
    assert len(library.calls) == enqueued
    for good, good_t in ((x, x_t), (h(40, 64, 1), None), (torch.zeros(size, dtype=torch.uint8), torch.zeros(size + 64, dtype=torch.uint8))):
        layer.product(good, x_packed_t=good_t)


def test_micro_batches_in_flight_keep_what_their_backward_pass_needs(library):
    """Two forward passes in front of the first backward one, as a pipeline has them: each in a slot of its own."""
    layer = _layer(training=True, in_flight=3)
    x, dy = torch.zeros(40, 64, dtype=torch.bfloat16), torch.zeros(40, 96, dtype=torch.bfloat16)
    assert len({layer.forward(x, slot=i).data_ptr() for i in range(2)}) == 2
    with pytest.raises(ValueError, match="no x"):
        layer.backward(dy, slot=2)
    of = []
    for i in range(2):
        layer.backward(dy, slot=i)
        of.append(_x_of_weight_gradient(library))
    assert len(set(of)) == 2 and of[0] == layer.x_t.data_ptr()
    assert [a[4] for name, a in library.calls if name == "tahq_mx4_quantize" and a[2] == layer.x.data_ptr()] == of

    norm = _norm(in_flight=2)
    t = _norm_inputs()
    inputs = (t["residual_out"], t["block"], t["w_post"], t["gate"], t["w_pre"])
    first, second = norm.forward(*inputs), norm.forward(*inputs, slot=1)
    assert len({v.data_ptr() for v in (*first, *second)}) == 4 and norm.stats_of(0) is norm.stats
    assert norm.stats_of(1).data_ptr() != norm.stats.data_ptr() and norm.stats_of(1).shape == norm.stats.shape
    written = [a for name, a in library.calls if name == "tahq_norm_forward"][-1]
    assert written[6] == second[0].data_ptr() and written[7] == second[1].data_ptr() and written[10] == norm.stats_of(1).data_ptr()
    for call in (lambda: layer.forward(x, slot=3), lambda: layer.backward(dy, slot=3), lambda: norm.forward(*inputs, slot=2),
                 lambda: norm.stats_of(2), lambda: layer.forward(x, slot=-1), lambda: norm.forward(*inputs, slot=-1), lambda: _layer(in_flight=0)):
        with pytest.raises((ValueError, IndexError)):
            call()


def test_tensors_of_another_floating_point_type_of_the_same_size_are_refused(library):
    """16 bits of another type than bf16 mean something else; integers of 16 bits are taken for bf16's bits, as the codec takes them."""
    half, bits, bf = (torch.zeros(40, 64, dtype=d) for d in (torch.float16, torch.int16, torch.bfloat16))
    packed, ws = (torch.zeros(1 << 16, dtype=torch.uint8) for _ in range(2))
    row, row_bf = torch.zeros(64, dtype=torch.float16), torch.zeros(64, dtype=torch.bfloat16)
    cfg, product = tahq.make_mx4_config(40, 64, tahq.BF16), tahq.make_mx4_matmul_config(40, 64, 64, tahq.BF16)
    norm = tahq.make_norm_config(40, 64, tahq.BF16)
    strided = torch.zeros(40, 128, dtype=torch.float16)[:, :64]
    stats, column, out = torch.zeros(2, 40), torch.zeros(64), torch.zeros_like(bf)
    backward = (stats, out, out, column, None, column, ws)
    for call in (lambda: tahq.tahq_mx4_quantize(cfg, half, packed), lambda: tahq.tahq_mx4_dequantize(cfg, packed, half),
                 lambda: tahq.tahq_mx4_quantize(tahq.make_mx4_config(40, 64, tahq.BF16, 128), strided, packed),
                 lambda: tahq.tahq_mx4_matmul(product, packed, packed, half, ws),
                 lambda: tahq.tahq_mx4_linear(cfg, product, half, packed, bf, ws),
                 lambda: tahq.tahq_mx4_linear(cfg, product, bf, packed, half, ws),
                 lambda: tahq.Mx4Tensor(cfg, device="cpu").quantize(half),
                 lambda: tahq.tahq_norm_forward(norm, half, None, None, None, row_bf, out, out),
                 lambda: tahq.tahq_norm_forward(norm, bf, None, None, None, row, out, out),
                 lambda: tahq.tahq_norm_forward(norm, bf, None, None, None, row_bf, out, half),
                 lambda: tahq.tahq_norm_backward(norm, half, bf, bf, row_bf, None, bf, row_bf, *backward),
                 lambda: tahq.tahq_norm_backward(norm, bf, bf, bf, row_bf, None, bf, row, *backward)):
        with pytest.raises(ValueError, match="float16"):
            call()
    gate = tahq.make_norm_config(40, 64, tahq.BF16, 40)
    with pytest.raises(ValueError, match="float16"):
        tahq.tahq_norm_forward(gate, bf, bf, row_bf, row, row_bf, out, out)
    assert not library.calls
    tahq.tahq_mx4_quantize(cfg, bits, packed)
    tahq.tahq_norm_forward(norm, bits, None, None, None, row_bf, out, out)
    tahq.tahq_norm_backward(norm, bf, bits, bf, row_bf, None, bf, row_bf, *backward)
    assert len(library.calls) == 3


@pytest.mark.parametrize("shape", [(41, 64), (64, 40), (39, 64), (40, 128)])
def test_packed_tensors_take_tensors_of_their_shape(library, shape):
    tensor = tahq.Mx4Tensor(tahq.make_mx4_config(40, 64, tahq.BF16), device="cpu")
    with pytest.raises(ValueError, match="d_in"):
        tensor.quantize(torch.zeros(shape, dtype=torch.bfloat16))
    assert not library.calls
    for good in (torch.zeros(2, 20, 64, dtype=torch.bfloat16), torch.zeros(40 * 64, dtype=torch.int16), torch.zeros(40 * 64 * 2, dtype=torch.uint8),
                 torch.zeros(41 * 64, dtype=torch.bfloat16)):
        tensor.quantize(good)
    apart = tahq.Mx4Tensor(tahq.make_mx4_config(40, 64, tahq.BF16, 80), device="cpu")
    apart.quantize(torch.zeros(40, 80, dtype=torch.bfloat16)[:, :64])
    apart.quantize(torch.zeros(40, 80, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="d_in"):
        apart.quantize(torch.zeros(50, 80, dtype=torch.bfloat16)[:, :64])
    assert len(library.calls) == 6
