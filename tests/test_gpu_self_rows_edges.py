"""Head norm of rows longer than 2^31 channels.  Tolerance: one rounding to bf16 (2^-8 of the value) and fp32 sums (2^-18 of the row's size 1)."""
import numpy as np
import pytest

import gret_ref

pytestmark = pytest.mark.gpu


def test_head_norm_of_a_token_with_more_than_2_31_channels():
    import torch
    from paper_2405_05254_b200 import binding as yx
    H, d = 2 ** 21 + 5, 1024                                  # group 2^21 begins at channel 2^31
    g = torch.Generator(device="cuda").manual_seed(3)
    x, gate, gain, bias = (torch.empty(H * d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(4))
    y = torch.full((H * d + 64,), 768.0, dtype=torch.bfloat16, device="cuda")
    ng = yx.make_norm_gate(1e-5, gate=gate, gain=gain, bias=bias)
    yx.yoco_head_norm(yx.HeadNormShape(1, H, d, 0, 0), x.view(1, -1), ng, y[:H * d].view(1, -1))
    assert bool((y[H * d:] == 768.0).all())
    for h in (0, 1, 2 ** 20, 2 ** 21 - 1, 2 ** 21, 2 ** 21 + 1, H - 1):
        at = slice(h * d, (h + 1) * d)
        f = lambda t: t[at].double().cpu().numpy().reshape(1, d)  # noqa: B023, E731
        want = gret_ref.norm_gate(f(x)[None], 1e-5, False, f(gate)[None], f(gain), f(bias))[0]
        assert (np.abs(f(y) - want) <= 2.0 ** -8 * (np.abs(want) + 2.0 ** -10)).all(), h
