"""The 8-bit cache's chunk and decode attention where many keys stand far behind one that leads."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["chunk", "decode"])
@pytest.mark.parametrize("n,octaves", [(700, 10.0), (40000, 18.1), (90000, 19.5), (90000, 20.6)])
def test_8_bit_weights_of_many_keys_behind_one_that_leads_keep_their_bits(mode, n, octaves):
    """All keys are zero but one, which leads by so many octaves and whose value is zero; the others' values are 1, so O is their
    share.  Enough streams that most are one CTA's alone.  Bound: the output's half step 2^-8; P's 2^-11 (2^7 times the weight is a
    normal fp16 number; the decode kernel, whose warps keep maxima of their own, is held to the same); the row's fp32 sum, at
    least 16 keys an addition and half a step 2^-24 each, n / 16 * 2^-24, which is the log-sum-exp's error too beside 2^-14 for the
    exponentials (cubic, 7.5e-5 relative where it is used); and n / 16 * 2^-24 for the tensor core's sums of equal products, each
    step cut at 2^-23 of the sum so far, half the last one on average."""
    import torch
    from paper_2405_05254_b200 import binding as bd
    B, H = 20, 8
    K = torch.zeros(B, H, n, 128, dtype=torch.uint8, device="cuda")
    V = torch.full_like(K, 0x38)                                    # E4M3: 1.0
    K[:, :, 69, 0], V[:, :, 69] = 0x4E, 0                           # 7.0
    q = torch.tensor(octaves * np.log(2) / 7 * 128 ** 0.5).to(torch.bfloat16)
    Q = torch.zeros(B, H, 1, 128, dtype=torch.bfloat16, device="cuda")
    Q[..., 0] = q
    O, L = torch.empty_like(Q), torch.empty(B, H, 1, device="cuda")
    lens, one = np.full(B, n, np.int32), np.ones(H, np.float32)
    shape = bd.make_shape(B, H, H, 128, 1)
    if mode == "decode":
        size, fn = bd.yoco_xattn_workspace_size(shape, lens, bd.MODE_DECODE), bd.yoco_xattn_decode_fp8
    else:
        size, fn = bd.yoco_xattn_workspace_size_chunk_fp8(shape, lens), bd.yoco_xattn_chunk_fp8
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    fn(shape, Q, K, V, one, one, None, lens, O, L, ws)
    assert bd.yoco_xattn_status(ws) == 0
    lead = np.exp(float(q) * 7 * 128 ** -0.5)
    want = (n - 1) / (n - 1 + lead)
    assert np.abs(O.double().cpu().numpy() / want - 1).max() <= 2.0 ** -8 + 2.0 ** -11 + 2 * n / 16 * 2.0 ** -24 + 2.0 ** -13
    assert np.abs(L.double().cpu().numpy() - np.log(n - 1 + lead)).max() <= n / 16 * 2.0 ** -24 + 2.0 ** -13
