"""The mx4 format's CPU definition against what its description says, and the norms' one against differences.  CPU only."""
import numpy as np
import pytest

from oracle import mx4, norm64


def test_rounding_goes_to_the_nearest_grid_point_and_ties_to_even_codes():
    ties = {0.25: 0.0, 0.75: 1.0, 1.25: 1.0, 1.75: 2.0, 2.5: 2.0, 3.5: 4.0, 5.0: 4.0}
    for at, to in ties.items():
        for sign in (1.0, -1.0):
            for nudge, want in ((0, to), (-1, None), (1, None)):
                x = np.zeros((1, 32), np.float32)
                x[0, 0] = 6.0                                             # pins the scale at 1 under both rules
                x[0, 1] = sign * (np.nextafter(np.float32(at), np.float32(nudge * 9)) if nudge else at)
                for rule in (mx4.FLOOR, mx4.COVER):
                    codes, scales = mx4.encode(x, 0, rule)
                    v = mx4.values(codes, scales)[0]
                    assert scales[0, 0] == 127 and v[0] == 6.0
                    if want is None:
                        below, above = [g for g in mx4.GRID if g < at][-1], [g for g in mx4.GRID if g > at][0]
                        want = above if nudge > 0 else below
                    assert v[1] == sign * want


@pytest.mark.parametrize("top, floor, cover", [
    (1.0, 125, 125), (1.5, 125, 125), (np.nextafter(np.float32(1.5), np.float32(2)), 125, 126), (1.99, 125, 126), (6.0, 127, 127),
    (7.9, 127, 128), (0.0, 0, 0), (1e-45, 0, 0), (2.0 ** -126, 0, 0), (2.0 ** -124, 1, 1), (3.4e38, 252, 253),
    (np.inf, 255, 255), (np.nan, 255, 255)])
def test_scales(top, floor, cover):
    x = np.zeros((1, 32), np.float32)
    x[0, 7] = top
    assert mx4.encode(x, 0, mx4.FLOOR)[1][0, 0] == floor and mx4.encode(x, 0, mx4.COVER)[1][0, 0] == cover


def test_layout_places_blocks_as_described():
    rows, cols = 37, 300
    RB, KB, KC = 2, 5, 2
    rng = np.random.default_rng(1)
    codes, scales = mx4.encode(rng.standard_normal((rows, cols)).astype(np.float32))
    packed = mx4.pack(codes, scales, cols)
    assert packed.size == mx4.packed_size(rows, cols) == RB * (KB * 1024 + KC * 256)
    for r in range(rows):
        for b in range(-(-cols // 32)):
            at = ((r // 32) * KB + b // 2) * 1024 + (b % 2) * 512 + (r % 32) * 16
            got = packed[at:at + 16]
            assert (got & 15 == codes[r, b, 0::2]).all() and (got >> 4 == codes[r, b, 1::2]).all()
            assert packed[RB * KB * 1024 + ((r // 32) * KC + b // 8) * 256 + (b % 2) * 128 + (r % 32) * 4 + b // 2 % 4] == scales[r, b]
    back = mx4.unpack(packed, rows, cols)
    assert (back[0] == codes).all() and (back[1] == scales).all()


def test_rotation_is_orthogonal_and_products_of_rotated_matrices_are_those_of_unrotated_ones():
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((5, 100)), rng.standard_normal((7, 100))
    rx, ry = (mx4.rotate(mx4.blocks(v)).reshape(v.shape[0], -1) for v in (x, y))
    assert np.allclose(rx @ ry.T, x @ y.T, atol=1e-12)
    assert np.allclose(mx4.rotate(rx.reshape(5, -1, 32)).reshape(5, -1)[:, :100], x, atol=1e-12)
    spike = np.zeros((1, 32))
    spike[0, 5] = 1.0
    assert np.allclose(np.abs(mx4.rotate(spike.reshape(1, 1, 32))), 32 ** -0.5, atol=1e-15)


@pytest.mark.parametrize("rule", (mx4.FLOOR, mx4.COVER))
@pytest.mark.parametrize("transform", (0, 1))
def test_fp32_order_agrees_with_64_bits_but_for_neighbouring_codes(transform, rule):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((64, 256)) * np.exp(rng.standard_normal((64, 256)))).astype(np.float32)
    got = mx4.values(*mx4.encode(x, transform, rule))
    y = mx4.blocks(x.astype(np.float64))
    if transform:
        y = mx4.rotate(y)
    scale = np.exp2(mx4.encode(x, transform, rule)[1].astype(np.float64) - 127)[..., None]
    a = np.abs(y) / scale
    nearest = np.abs(a[..., None] - mx4.GRID).min(-1)                      # distance to the nearest grid point, in units
    off = np.abs(np.abs(got).reshape(y.shape) / scale - np.minimum(a, 6))
    assert (off <= np.minimum(nearest, np.maximum(6 - a, nearest)) + 1e-5).all()


@pytest.mark.parametrize("halves", ("both", "post", "pre"))
@pytest.mark.parametrize("gate_rows", (0, 1, 2, 5))
def test_gradients_of_the_norms_are_those_of_differences(halves, gate_rows):
    if halves == "pre" and gate_rows:
        return
    rng = np.random.default_rng(4)
    rows, cols, eps, alpha, h = 5, 12, 1e-2, 0.75, 1e-6
    t = {n: rng.standard_normal((rows, cols)) for n in ("residual", "block", "grad_out", "grad_h")}
    t["w_post"], t["w_pre"] = rng.standard_normal(cols), rng.standard_normal(cols)
    t["gate"] = rng.standard_normal((-(-rows // gate_rows), cols)) if gate_rows else None
    if halves == "pre":
        t["block"] = t["w_post"] = None
    if halves == "post":
        t["w_pre"] = t["grad_h"] = None

    def run(**changed):
        v = {**t, **changed}
        return norm64.forward(v["residual"], v["block"], v["w_post"], v["gate"], v["w_pre"], gate_rows, eps, alpha)

    def loss(**changed):
        out, hh, _, _ = run(**changed)
        return (out * t["grad_out"]).sum() + (0 if hh is None else (hh * t["grad_h"]).sum())

    out, _, rstd_b, rstd_r = run()
    got = norm64.backward(t["grad_out"], t["grad_h"], t["block"], t["w_post"], t["gate"], out, t["w_pre"], rstd_b, rstd_r, gate_rows, alpha)
    for name in ("residual", "block", "w_post", "gate", "w_pre"):
        if t[name] is None:
            assert f"grad_{name}" not in got
            continue
        for at in np.ndindex(t[name].shape):
            up, down = t[name].copy(), t[name].copy()
            up[at] += h
            down[at] -= h
            assert abs((loss(**{name: up}) - loss(**{name: down})) / (2 * h) - got[f"grad_{name}"][at]) < 1e-6
