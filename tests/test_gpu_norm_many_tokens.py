"""More tokens than 2^31 pieces of rows: the gradient counts them in 64 bits and runs, as its workspace's size says; the way there refuses them."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, HALF_STEP, stream
from test_gpu_norm_rope import U, chain, plain_grad

pytestmark = pytest.mark.gpu


def test_pieces_beyond_32_bits():
    """Rows of six channels are four lanes; x and dy are one row for all tokens, so all rows of dx are alike and the weights' gradient is the tokens' number of times one row's."""
    d, t = 6, 2 ** 29 + 3
    g = torch.Generator()
    g.manual_seed(3)
    x, dy, w = (torch.randn(n, generator=g).to(torch.bfloat16) for n in ((1, 1, d), (1, 1, d), (d,)))
    same = lambda a: a.to(DEV).expand(1, t, d)
    dx = torch.full((1, t, d), 9.0, dtype=torch.bfloat16, device=DEV)
    wd, dw = w.to(DEV), torch.empty((1, d), device=DEV)
    norm = bs.Norm.of([wd])
    ws = torch.empty(bs.bs_norm_rope_grad_workspace(1, bs.BS_BF16, t, d), dtype=torch.uint8, device=DEV)
    with pytest.raises(bs.BlindsightError):
        bs.bs_norm_rope(norm, None, [same(x)], [dx], bs.BS_BF16, t, d, stream=stream())
    bs.bs_norm_rope_grad(norm, None, [same(x)], [same(dy)], [dx], dw, bs.BS_BF16, t, d, workspace=ws, stream=stream())
    torch.cuda.synchronize()
    want, tol, sums, tol_sums, size = plain_grad(None, x.double().numpy(), dy.double().numpy(), w.double().numpy(), float(np.float32(1e-6)), None)
    first = dx[0, 0].clone()
    assert (np.abs(first.double().cpu().numpy() - want[0, 0]) <= tol[0, 0] + HALF_STEP["bf16"] * (np.abs(want[0, 0]) + tol[0, 0])).all()
    for a in range(0, t, 2 ** 27):
        assert (dx[0, a:a + 2 ** 27] == first).all(), a
    steps = chain(1, t, 4) + 9
    off = np.abs(dw[0].double().cpu().numpy() - sums * t)
    assert (off <= t * (tol_sums + steps * U * size) + U * np.abs(sums * t)).all()
