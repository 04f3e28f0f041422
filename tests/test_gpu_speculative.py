"""The example's speculative decoder: drafted trees give the tokens that plain decoding gives, whatever is drafted."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decode.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("speculative_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _ratio_free(decoder):
    """Skipping by ratio looks at the whole batch, so that a token's experts would depend on its company."""
    for layer in decoder.moe:
        plain = layer.forward
        layer.forward = lambda x, y, T, mode, value, plain=plain: plain(x, y, T, "threshold", 0.15)
    return decoder


@pytest.mark.parametrize("fmt", ["plain", "fp8"])
def test_greedy_speculation_is_plain_greedy_decoding(example, fmt):
    """fp32 activations: the largest logit stands clear of rounding; the cache's rows are the same either way."""
    first = torch.arange(4, device="cuda") * 7
    torch.manual_seed(1)
    plain, steps = example.generate(_ratio_free(example.Decoder("f32", fmt)), first, 40, 0.0, drafted=False)
    torch.manual_seed(2)
    fast, fewer = example.generate(_ratio_free(example.Decoder("f32", fmt)), first, 40, 0.0)
    assert steps == 40 and fewer <= steps
    assert [o[:40] for o in fast] == [o[:40] for o in plain]


@pytest.mark.parametrize("dtype,fmt", [("bf16", "fp8"), ("bf16", "plain"), ("f32", "fp8")])
def test_sampled_steps_run_and_keep_their_books(example, dtype, fmt):
    torch.manual_seed(3)
    d = example.Decoder(dtype, fmt)
    out, steps = example.generate(d, torch.arange(4, device="cuda"), 24, 0.9)
    assert all(0 <= t < example.VOCAB for o in out for t in o)
    # every produced token but each request's last has its rows in the cache, after the first one's
    assert d.lens.tolist() == [len(o) for o in out]
