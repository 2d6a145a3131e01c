"""The norms around a block in 64 bits (include/tahq_norm.h), forward and backward, on the CPU: NumPy only."""
import numpy as np


def forward(residual, block, w_post, gate, w_pre, gate_rows, eps, alpha):
    """(r', h, 1/RMS(block), 1/RMS(r')); what is missing is None, its statistics zeros."""
    rows, _ = residual.shape
    out = alpha * residual.astype(np.float64)
    rstd_b, rstd_r, h = np.zeros(rows), np.zeros(rows), None
    if block is not None:
        b = block.astype(np.float64)
        rstd_b = (np.square(b).mean(1) + eps) ** -0.5
        p = b * rstd_b[:, None] * w_post
        if gate is not None:
            p = p * gate[np.arange(rows) // gate_rows]
        out = out + p
    if w_pre is not None:
        rstd_r = (np.square(out).mean(1) + eps) ** -0.5
        h = out * rstd_r[:, None] * w_pre
    return out, h, rstd_b, rstd_r


def backward(grad_out, grad_h, block, w_post, gate, residual_out, w_pre, rstd_b, rstd_r, gate_rows, alpha):
    """Gradients by name, from the statistics of the forward pass.  Under each name's "_size" the sum of its terms' magnitudes."""
    rows, cols = (grad_out if grad_out is not None else grad_h).shape
    g = np.zeros((rows, cols)) if grad_out is None else grad_out.astype(np.float64)
    size = np.abs(g)
    got = {}

    def through(u, unit, rstd):
        """The norm's Jacobian, symmetric: rstd (I - unit unit^T / cols), applied to u; and the magnitudes of its terms."""
        mean = (u * unit).sum(1, keepdims=True) / cols
        mean_size = np.abs(u * unit).sum(1, keepdims=True) / cols
        return rstd[:, None] * (u - unit * mean), rstd[:, None] * (np.abs(u) + np.abs(unit) * mean_size)

    if grad_h is not None:
        unit = residual_out.astype(np.float64) * rstd_r[:, None]
        got["grad_w_pre"], got["grad_w_pre_size"] = (grad_h * unit).sum(0), np.abs(grad_h * unit).sum(0)
        more, more_size = through(grad_h * w_pre.astype(np.float64), unit, rstd_r)
        g, size = g + more, size + more_size
    got["grad_residual"], got["grad_residual_size"] = alpha * g, abs(alpha) * size
    if block is not None:
        unit = block.astype(np.float64) * rstd_b[:, None]
        if gate is not None:
            groups = np.arange(rows) // gate_rows
            each, each_size = np.zeros((groups[-1] + 1, cols)), np.zeros((groups[-1] + 1, cols))
            np.add.at(each, groups, g * unit * w_post)
            np.add.at(each_size, groups, size * np.abs(unit * w_post))
            got["grad_gate"], got["grad_gate_size"] = each, each_size
            g, size = g * gate[groups], size * np.abs(gate[groups])
        got["grad_w_post"], got["grad_w_post_size"] = (g * unit).sum(0), (size * np.abs(unit)).sum(0)
        got["grad_block"], _ = through(g * w_post, unit, rstd_b)
        _, got["grad_block_size"] = through(size * np.abs(w_post), np.abs(unit), rstd_b)
    return got
