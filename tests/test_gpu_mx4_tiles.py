"""Products of every kind of tile against 64-bit products of what the packed matrices hold: ragged edges, rows of NaN, sums that are added to
(GPU)."""
import numpy as np
import pytest
import torch

import paper_2506_01352_amd as tahq
from mx4_products import PRODUCTS
from oracle import mx4
from test_gpu_mx4 import KINDS, _product_bound

pytestmark = pytest.mark.gpu


def _operand(rows, k, seed, spread, bad):
    """(packed bytes, values in 64 bits) of a random matrix with a block of NaN in the rows `bad`, at its first and last columns."""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((rows, k)) * np.exp(spread * rng.standard_normal((rows, 1)))).astype(np.float32)
    for i, row in enumerate(bad):
        x[row, (0, k - 1)[i % 2]] = (np.nan, np.inf)[i % 2]
    codes, scales = mx4.encode(x)
    return torch.from_numpy(mx4.pack(codes, scales, k)).cuda(), torch.from_numpy(mx4.values(codes, scales)).cuda()


@pytest.mark.parametrize("kind, parts, c, m, n, k", PRODUCTS)
def test_products_of_every_kind(kind, parts, c, m, n, k):
    a, va = _operand(m, k, 1, 1.0, (m // 2, m - 1) if m > 1 else ())
    b, vb = _operand(n, k, 2, 0.0, (n - 1, n // 3))
    # in 64 bits: the products, and those of magnitudes, which roundings go by; rows of NaN apart
    clean = [v.nan_to_num(nan=0.0) for v in (va, vb)]
    want = torch.mm(clean[0], clean[1].t().contiguous()).cpu().numpy()
    size = torch.mm(clean[0].abs(), clean[1].abs().t().contiguous()).cpu().numpy()
    nan = (va.isnan().any(1)[:, None] | vb.isnan().any(1)[None]).cpu().numpy()
    assert nan.any()
    del va, vb, clean
    for accumulate, ldc in ((0, n), (1, n + 5)):
        start = torch.randn(m + 1, ldc, generator=torch.Generator().manual_seed(4)).to(KINDS[c][1])
        out = start.cuda()
        cfg = tahq.make_mx4_matmul_config(m, n, k, KINDS[c][0], ldc, accumulate)
        need = tahq.tahq_mx4_matmul_workspace_size(cfg)
        assert (need > 0) == parts
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")        # NaN in what is not written
        tahq.tahq_mx4_matmul(cfg, a, b, out[:m, :n], ws)
        torch.cuda.synchronize()
        got, before = out.cpu().double().numpy(), start.double().numpy()
        w, s = (want + before[:m, :n], size + np.abs(before[:m, :n])) if accumulate else (want, size)
        assert (np.isnan(got[:m, :n]) == nan).all()
        fine = ~nan
        assert (np.abs(got[:m, :n] - w)[fine] <= _product_bound(s, k, w, c)[fine]).all()
        assert (got[m:] == before[m:]).all() and (got[:m, n:] == before[:m, n:]).all(), "written outside the result"
        assert (ws[need:] == 0xFF).all(), "written past the workspace"
