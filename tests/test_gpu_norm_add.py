"""The norm with the residual's addition: bit for bit the sum and moe_rmsnorm of
it, and its 8-bit form against the definition."""
import numpy as np
import pytest
import torch

import attn_reference
import paper_2607_12875_gb300 as gb

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows(seed, T, H, act, spread=3.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((T, H), device="cuda", generator=g) * torch.exp(spread * torch.randn((T, 1), device="cuda", generator=g))
    return x.to(DT[act])


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(1, 256), (77, 512), (5, 2048), (33, 4096), (3, 4352), (130, 7168), (9, 8192), (4, 8448), (2, 16640)])
def test_sum_and_norm_bit_for_bit(act, T, H):
    x, r = rows(1, T, H, act), rows(2, T, H, act)
    x[0] = -r[0]  # a row of zeros: eps keeps it finite
    gamma = rows(3, 1, H, act, 0.0)[0]
    cfg = gb.make_config(T, H, 128, 8, 2, act=act, w=act)
    s, y = torch.empty_like(x), torch.empty_like(x)
    codes = torch.empty((T, H), dtype=torch.uint8, device="cuda")
    scales = torch.empty((T, H // 128), device="cuda")
    gb.moe_rmsnorm_add(cfg, x, r, gamma, 1e-6, s, y, codes, scales)
    want_s = x + r  # (one rounding of the sum)
    want_y = torch.empty_like(x)
    gb.moe_rmsnorm(cfg, want_s, gamma, 1e-6, want_y)
    bits = torch.int32 if act == "f32" else torch.int16
    assert torch.equal(s.view(bits), want_s.view(bits)) and torch.equal(y.view(bits), want_y.view(bits))
    # each output without the others, no residual, and the sum in the place of a term
    y2, c2, s2 = torch.empty_like(x), torch.empty_like(codes), torch.empty_like(scales)
    gb.moe_rmsnorm_add(cfg, x, r, gamma, 1e-6, None, y2)
    assert torch.equal(y2.view(bits), y.view(bits))
    gb.moe_rmsnorm_add(cfg, want_s, None, gamma, 1e-6, None, None, c2, s2)
    assert torch.equal(c2, codes) and torch.equal(s2, scales)
    for a, b, into in ((x.clone(), r, 0), (x, r.clone(), 1)):
        gb.moe_rmsnorm_add(cfg, a, b, gamma, 1e-6, (a, b)[into], y2)
        assert torch.equal((a, b)[into].view(bits), s.view(bits)) and torch.equal(y2.view(bits), y.view(bits))
    a, alone = x.clone(), torch.empty_like(x)
    gb.moe_rmsnorm_add(cfg, a, None, gamma, 1e-6, a, alone)
    gb.moe_rmsnorm(cfg, x, gamma, 1e-6, want_y)
    assert torch.equal(a.view(bits), x.view(bits)) and torch.equal(alone.view(bits), want_y.view(bits))


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(40, 768), (7, 7168), (3, 8448)])
def test_codes_and_scales(act, T, H):
    """Against the definition in 64 bits: scales equal but where a block's largest value lies within fp32's error of a
    power's border, codes within half a step of the value (and that error)."""
    x, r, gamma = rows(4, T, H, act), rows(5, T, H, act), rows(6, 1, H, act, 0.0)[0]
    r[0] = -x[0]
    gamma[128:256] = 0  # a block of zeros
    gamma[256:300] *= 1e-30
    cfg = gb.make_config(T, H, 128, 8, 2, act=act, w=act)
    s = torch.empty_like(x)
    codes = torch.empty((T, H), dtype=torch.uint8, device="cuda")
    scales = torch.empty((T, H // 128), device="cuda")
    gb.moe_rmsnorm_add(cfg, x, r, gamma, 1e-5, s, None, codes, scales)
    t = s.double().cpu().numpy()
    want = (t / np.sqrt((t * t).mean(1, keepdims=True) + 1e-5) * gamma.double().cpu().numpy()).reshape(T, -1, 128)
    got_s = scales.double().cpu().numpy()
    got = attn_reference.e4m3_values()[codes.cpu().numpy()].reshape(want.shape)
    top = np.abs(want).max(-1)
    e = np.log2(got_s)
    assert np.array_equal(e, np.round(e)) and (e >= -126).all()
    near = 1 + 4e-6  # sums of up to 8448 squares in fp32 and five operations: far below it
    assert (top <= 448 * got_s * near).all()
    assert ((top >= 224 * got_s / near) | (e == -126)).all()
    v = want / got_s[..., None]
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -40))), -6) - 3)
    assert (np.abs(got - v) <= step / 2 + 4e-6 * np.abs(v)).all()


def test_values_that_are_no_numbers_in_8_bits():
    """A NaN and an infinity in gamma: their columns' codes are NaN and +-448, the block's scale comes from the others."""
    cfg = gb.make_config(2, 256, 128, 8, 2)
    x = rows(7, 2, 256, "bf16", 0.0)
    gamma = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    c1, c2 = (torch.empty((2, 256), dtype=torch.uint8, device="cuda") for _ in range(2))
    s1, s2 = (torch.empty((2, 2), device="cuda") for _ in range(2))
    plain = gamma.clone()
    plain[3] = plain[9] = 0
    gb.moe_rmsnorm_add(cfg, x, None, plain, 1e-6, None, None, c1, s1)
    gamma[3], gamma[9] = float("nan"), float("inf")
    gb.moe_rmsnorm_add(cfg, x, None, gamma, 1e-6, None, None, c2, s2)
    assert torch.equal(s1, s2)
    assert ((c2[:, 3] & 0x7f) == 0x7f).all() and ((c2[:, 9] & 0x7f) == 0x7e).all()
    keep = torch.ones(256, dtype=torch.bool, device="cuda")
    keep[3] = keep[9] = False
    assert torch.equal(c1[:, keep], c2[:, keep])
    # a row that holds one is no number throughout
    x[1, 100] = float("nan")
    y = torch.empty_like(x)
    gb.moe_rmsnorm_add(cfg, x, None, plain, 1e-6, None, y, c1, s1)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and ((c1[1] & 0x7f) == 0x7f).all()
    assert (s1[1] == 2.0 ** -126).all()


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("H", [512, 7168, 8448])
@pytest.mark.parametrize("power", [-60, 55])
def test_codes_where_the_row_times_gamma_leaves_fp32s_range(act, H, power):
    """Rows of about 2^power, whose products with gamma are no normal fp32 numbers though the norm's elements are: columns
    with gammas of about 2^-85, 1 and 2^78. Against the definition, as above."""
    x = rows(8, 3, H, act, 0.0) * 2.0 ** power
    gamma = rows(9, 1, H, act, 0.0)[0]
    gamma[:128] *= 2.0 ** -85
    gamma[128:256] *= 2.0 ** 78
    cfg = gb.make_config(3, H, 128, 8, 2, act=act, w=act)
    codes = torch.empty((3, H), dtype=torch.uint8, device="cuda")
    scales = torch.empty((3, H // 128), device="cuda")
    gb.moe_rmsnorm_add(cfg, x, None, gamma, 0.0, None, None, codes, scales)
    t = x.double().cpu().numpy()
    want = (t / np.sqrt((t * t).mean(1, keepdims=True)) * gamma.double().cpu().numpy()).reshape(3, -1, 128)
    got_s = scales.double().cpu().numpy()
    top, near = np.abs(want).max(-1), 1 + 4e-6
    assert (top <= 448 * got_s * near).all() and (top >= 224 * got_s / near).all()
    v = want / got_s[..., None]
    got = attn_reference.e4m3_values()[codes.cpu().numpy()].reshape(want.shape)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -40))), -6) - 3)
    assert (np.abs(got - v) <= step / 2 + 4e-6 * np.abs(v)).all()
