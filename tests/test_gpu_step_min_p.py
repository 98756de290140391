"""min-p on the path of long rows: greatest logits whose weight is a power of two, and
ones whose code lies past a power of two's end."""
import math

import numpy as np
import pytest
import torch

from paper_2608_23805_gb300 import api
from test_gpu_step_sample import check

pytestmark = pytest.mark.gpu


def late(rng, n):
    """Random numbers near 1: a filter that drops nothing gives another token."""
    return (1 - rng.integers(1, 1 << 20, n) / (1 << 24)).astype(np.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("temperature", [1.0, 0.001, 1e-6])
def test_greatest_logit_zero(temperature, dtype):
    """Weights of min_p that are whole multiples of 2^40."""
    rng = np.random.default_rng([1, int(1 / temperature)])
    x = -np.abs(rng.standard_normal((16, 3001))) * 4 * temperature
    x = np.sort(x, 1)[:, ::-1].copy()  # the last ones are dropped first
    x[:, 0] = 0
    x = torch.from_numpy(x).to(dtype).cuda()
    share = (np.arange(1, 17) / 16).astype(np.float32)
    for kw in ({}, {"top_k": 300}, {"top_k": 2000, "top_p": 0.9}, {"top_p": 0.8}, {"top_k": 40}):
        check(x, late(rng, 16), min_p=share, temperature=temperature, **kw)


def test_small_example():
    x = torch.tensor([[0.0, -0.1, -1.0, -2.0, -5.0]], device="cuda")
    ids, lp = api.sample(x, torch.tensor([0.95], device="cuda"), min_p=0.5)
    assert ids.tolist() == [1] and abs(lp.item() - math.log(math.exp(-0.1) / (1 + math.exp(-0.1)))) <= 2.0 ** -21


@pytest.mark.parametrize("top", [1.0, 300.0, -77.0])
def test_far_from_zero_beside_the_temperature(top):
    """|top| log2(e) / T above 4,096, several logits within T of the greatest."""
    rng = np.random.default_rng(2)
    T = float(np.float32(abs(top) / 10000))
    x = (top - np.abs(rng.standard_normal((16, 2500))) * 3 * T).astype(np.float32)
    x[:, 1000] = top
    share = (np.arange(1, 17) / 16).astype(np.float32)
    for kw in ({}, {"top_k": 300}, {"top_p": 0.7}):
        check(torch.from_numpy(x).cuda(), late(rng, 16), min_p=share, temperature=T, **kw)


# (temperature, greatest logit): log2 of the weight lies a fraction below 63 / 64 of a
# whole number as one fp32 number, and above it with what that number leaves
PAST_THE_END = [("0x1.d5a582p-9", "0x1.2bc768p+1"), ("0x1.2f38cp-7", "0x1.71db36p+2"), ("0x1.59a0b6p-7", "0x1.b4109p+0"),
                ("0x1.2f8b56p-7", "0x1.62377cp+1"), ("0x1.4949d2p-9", "0x1.c809bp+0"), ("0x1.2c7876p-7", "0x1.5fa87p+4"),
                ("0x1.23185ep-10", "0x1.695eccp-1"), ("0x1.47b694p-4", "0x1.948fcap+2")]


@pytest.mark.parametrize("min_p", [1.0, 0.9375, 0.5, 0.03125])
def test_codes_past_the_end_of_an_exponent(min_p):
    rng = np.random.default_rng(3)
    T, top = (np.array([float.fromhex(p[i]) for p in PAST_THE_END]) for i in (0, 1))
    x = (top[:, None] - rng.uniform(0.05, 6, (8, 700)) * T[:, None]).astype(np.float32)
    x[:, 137] = top
    for kw in ({}, {"top_k": 400}, {"top_p": 0.6}):
        got = check(torch.from_numpy(x).cuda(), late(rng, 8), min_p=min_p, temperature=T.astype(np.float32), **kw)
        if min_p == 1.0:
            assert (got == 137).all()


def test_equal_logits_stay_together():
    """Of equal logits min_p drops all or none, wherever they are."""
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.integers(-6, 1, (16, 5003)).astype(np.float32)).cuda()
    x[:, 17] = 0
    share = np.exp(-(np.arange(16) % 7) - 0.5).astype(np.float32)
    for kw in ({}, {"top_k": 3000}, {"top_p": 0.97}):
        check(x, late(rng, 16), min_p=share, **kw)
