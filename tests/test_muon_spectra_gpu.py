"""Accuracy of the orthogonalising entry points on matrices of every kind of spectrum, as the header promises it: the 2-norm of the difference
from the oracle in 64 bits is at most 2^-9 of the result's, before any rounding of the result to bf16; 2^-13
where the products' operands have 22 bits or 64.

The five steps amplify what has the smallest singular values by up to 3.4445^5 = 485, so that a matrix of low rank shows every rounding of X
that is not along its few directions.  The result is read where it is not rounded: a Muon step with lr = 1, no momentum and no decay takes
parameters of zeros to 0 - 1 X, exact in fp32."""
import numpy as np
import pytest
import torch

from oracle import muon_oracle as M

pytestmark = pytest.mark.gpu
ABC = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
# by the way a matrix takes: up to 16 rows, to 32, to 64 and to 128 in one workgroup, thin ones, tiles
SHAPES = {"16": [(5, 7), (16, 500)], "32": [(17, 17), (20, 30), (40, 17), (32, 64), (31, 767)], "64": [(33, 33), (40, 48), (200, 33), (64, 256), (63, 1001)],
          "128": [(65, 65), (65, 200), (128, 128), (448, 127)], "thin": [(24, 3000), (64, 2000)],
          "tiles": [(130, 130), (192, 192), (300, 1000), (512, 512), (100, 2100), (512, 1280), (1400, 520)]}
# directions of a common size and noise beside them
KINDS = [(1, 0.0), (2, 0.0), (3, 0.0), (5, 0.0), (16, 0.0), (32, 0.0), (64, 0.0), (1, 1e-3), (2, 1e-3), (8, 1e-3), (1, 1e-2), (4, 5e-2), (0, 1.0)]


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


def _matrices(shape, seeds):
    out = {}
    m, n = shape
    r = min(m, n)
    for seed in range(seeds):
        rng = np.random.default_rng(10000 * seed + 100 * m + n)
        for rank, noise in KINDS:
            if rank < r:
                out[rank, noise, seed] = 1e-3 * (rng.standard_normal((m, rank)) @ rng.standard_normal((rank, n)) + noise * rng.standard_normal((m, n)))
        u, v = (np.linalg.qr(rng.standard_normal((k, r)))[0] for k in (m, n))
        for low in (1e-3, 1e-4):
            out["down to", low, seed] = (u * np.logspace(0.0, np.log10(low), r)) @ v.T
        out["rows", 2.0, seed] = rng.standard_normal((m, n)) * np.exp(2.0 * rng.standard_normal((m, 1)))
    return {k: x.astype(np.float32) for k, x in out.items()}


@pytest.mark.parametrize("way,shape", [(way, s) for way, shapes in SHAPES.items() for s in shapes], ids=lambda x: x if isinstance(x, str) else f"{x[0]}x{x[1]}")
def test_result_is_within_the_promised_share(B, way, shape):
    matrices = _matrices(shape, 4 if max(shape) <= 64 else 1)
    grads = [torch.from_numpy(g).cuda() for g in matrices.values()]
    params, momentum = [torch.zeros_like(g) for g in grads], [torch.zeros_like(g) for g in grads]
    B.cce_muon_multi_step(B.MuonTensors(grads, params, momentum), lr=1.0, momentum=0.0, nesterov=False, coefficients=ABC, eps=EPS)
    off = {}
    for (kind, g), p in zip(matrices.items(), params):
        want = M.orthogonalize(g, ABC, 5, EPS)
        off[kind] = float(np.linalg.norm(-p.cpu().numpy().astype(np.float64) - want) / np.linalg.norm(want))
    worst = max(off, key=off.get)
    assert off[worst] <= (2.0 ** -13 if way in ("16", "32", "thin") else 2.0 ** -9), (worst, off[worst], len(off))
