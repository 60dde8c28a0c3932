"""The cosines and sines that vectors are turned by: pairs (1, 0) come back as them.

Absolute tolerance, for values of at most 1: sincospif is within 1 ulp, 2^-24; what the angle lost to fp32 is put back by a
multiply-add, which rounds by 2^-25; second order terms and the 64-bit angle of either side, less than 2^-30."""
import numpy as np
import pytest
import torch

import paper_2509_09754_b200 as lava

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("d,base", [(128, 500000.0), (64, 10000.0)])
def test_cosines_and_sines(d, base, interleaved, backward):
    n = 20000
    g = torch.Generator().manual_seed(d)
    pos = torch.randint(0, 131072, (n,), generator=g).int()
    freqs = lava.lava_rotary_freqs(d, base)[0]
    x = torch.zeros((n, 1, d))
    first = slice(0, d, 2) if interleaved else slice(0, d // 2)
    second = slice(1, d, 2) if interleaved else slice(d // 2, d)
    x[..., first] = 1.0
    x, out = x.cuda(), torch.empty((n, 1, d), device="cuda")
    desc = lava.RotaryDesc(head_dim=d, rotary_dim=d, dtype=lava.LAVA_F32, interleaved=interleaved, backward=backward)
    lava.lava_rotary(desc, freqs.cuda(), pos.cuda(), x, None, out, None)
    angle = pos.double().numpy()[:, None] * freqs.numpy()[None, :] * (-1.0 if backward else 1.0)
    got = out[:, 0].double().cpu().numpy()
    tol = 2.0 ** -24 + 2.0 ** -25 + 2.0 ** -30
    for part, want in ((first, np.cos(angle)), (second, np.sin(angle))):
        err = np.abs(got[:, part] - want)
        assert err.max() <= tol, (err.max() * 2 ** 24, float(np.sqrt((err ** 2).mean())) * 2 ** 24)
