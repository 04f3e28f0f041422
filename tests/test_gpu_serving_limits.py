"""Attention over 4-bit caches where its number formats and its tables of pages end."""
import numpy as np
import pytest
import torch

from paper_2609_05228_gb300 import ace

from test_gpu_serving_ops import DT, Step, _int

pytestmark = pytest.mark.gpu

LARGEST = float(torch.finfo(torch.bfloat16).max)


@pytest.mark.parametrize("size", [2.0 ** 120, 2.0 ** 121, 1e38, LARGEST])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("scale", [128 ** -0.5, 4.0])
@pytest.mark.parametrize("nodes", [1, 2, 4, 15, 50])
def test_int4_attention_equal_scores_of_the_largest_q(nodes, scale, sign, size):
    """Rows of one key score alike for q to bf16's largest (scores of 4e9 to 5e12, all of one sign), so the output is the mean of V:
    codes of 1 to 7 and their sums are exact, a weight's rounding is at most 2^-8 of it, the output's too. lse: the score, a sum of
    128 products in fp32, four factors (2^-24 each)."""
    rng = np.random.default_rng(nodes)
    H, G, D, page, length = 1, 4, 128, 16, 333
    total = length + nodes
    v = torch.from_numpy(rng.integers(1, 8, (total, H, D)).astype(np.float32)).bfloat16()
    v[..., ::32] = 7
    kv = ace.AceKvCache(H, D, page, 24, 1, "bf16", "int4")
    key = 7 * 2.0 ** -96
    kv.write(0, torch.full((total, H, D), key, dtype=torch.bfloat16, device="cuda"), v.cuda(), torch.arange(total, device="cuda"))
    q = torch.full((nodes, H * G, D), sign * size, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(nodes, H * G, device="cuda")
    kv.attend(0, q, torch.arange(24, dtype=torch.int32, device="cuda")[None], _int([length]), _int([0, nodes]), out, None, nodes, scale, lse)
    kv.sync()
    sums = v.double().numpy().cumsum(0)
    want = np.stack([sums[length + i] / (length + i + 1) for i in range(nodes)])
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -7 * want).all()
    score = q[0, 0, 0].item() * key * D * scale
    assert (np.abs(lse.double().cpu().numpy() - score) <= 140 * 2.0 ** -24 * abs(score)).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 80), ("f32", 64)])
@pytest.mark.parametrize("p", [60, 110, 118, 121, 124])
@pytest.mark.parametrize("nodes", [1, 2, 4, 5, 20])
def test_int4_attention_large_q_and_small_keys(dtype, D, p, nodes):
    """q of 2^p and K of 2^-p score as both of 1 do. (At p = 124 the sums of products lie among fp32's subnormals: four roundings of 2^-150
    to a row whose largest is 2^(e - 127) are 2^(e - 265) scale of a score, an eighth of the bound's 136 * 2^-24 |q| |k| scale and
    less, as |k| is 2^-122 somewhere.)"""
    s = Step([333, 70], [nodes, 1], 4, 1, D, 16, dtype, seed=p, k_scale=2.0 ** -p)
    s.q = (s.q.double() * 2.0 ** p).to(DT[dtype])
    s.qd = s.q.double().cpu().numpy()
    assert np.isfinite(s.qd).all() and (p < 124 or dtype == "f32" or np.abs(s.qd).max() > 2.0 ** 125)
    s.check(*s.run())
