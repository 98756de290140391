"""Temperatures next to the ends of fp32, with logits that differ by as much."""
import numpy as np
import pytest
import torch

from test_gpu_step_sample import check, uniform

pytestmark = pytest.mark.gpu
MOST = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("temperature", [2.0 ** -149, 1e-43, 1e-38, 1e-33, 1e-30, 1e-28])
@pytest.mark.parametrize("top", [0.0, 40.0, 60000.0])
def test_least_temperatures(temperature, top):
    """Greatest logits of `top` temperatures: both forms of a weight."""
    rng = np.random.default_rng([int(-np.log2(temperature)), int(top)])
    T = np.float32(temperature)
    x = ((top - np.abs(rng.standard_normal((8, 1200))) * 3) * float(T)).astype(np.float32)
    for kw in ({}, {"top_k": 300}, {"top_k": 20}, {"top_p": 0.8}, {"min_p": 0.3}):
        check(torch.from_numpy(x).cuda(), uniform(rng, 8), temperature=float(T), **kw)
        check(torch.from_numpy(x).bfloat16().cuda(), uniform(rng, 8), temperature=float(T), **kw)


@pytest.mark.parametrize("temperature", [1e25, 1e29, 1e33, 1e36, MOST / 4, MOST])
def test_greatest_temperatures(temperature):
    rng = np.random.default_rng(int(np.log2(temperature)))
    T = np.float32(temperature)
    x = np.clip(rng.standard_normal((8, 1200)) * 3 * float(T), -MOST, MOST).astype(np.float32)
    for kw in ({}, {"top_k": 300}, {"top_k": 20}, {"top_p": 0.8}, {"min_p": 0.3}):
        check(torch.from_numpy(x).cuda(), uniform(rng, 8), temperature=float(T), **kw)


def test_ends_of_the_type_beside_each_other():
    x = torch.tensor([[MOST, -MOST, 0.0, MOST / 2]] * 8, device="cuda")
    rng = np.random.default_rng(7)
    for T in (MOST, MOST / 2, 1e38, 1e35):
        check(x, uniform(rng, 8), temperature=float(np.float32(T)))
        check(x.repeat(1, 200), uniform(rng, 8), temperature=float(np.float32(T)))


def test_temperatures_of_each_row():
    rng = np.random.default_rng(8)
    T = np.array([2.0 ** -149, 1e-40, 1e-31, 1e-10, 1.0, 1e20, 1e31, MOST], np.float32)
    x = np.clip(-np.abs(rng.standard_normal((8, 2000))) * 3 * T.astype(np.float64)[:, None], -MOST, MOST).astype(np.float32)
    for kw in ({}, {"top_k": 500, "top_p": 0.9}):
        check(torch.from_numpy(x).cuda(), uniform(rng, 8), temperature=T, **kw)


def test_borders_at_the_greatest_temperatures():
    """Two tokens and random numbers next to the first one's share p, 2^-27 away or more:
    weights off by 2^-26 move it by p (1 - p) 2^-26, under 2^-28."""
    rng = np.random.default_rng(9)
    T = (rng.uniform(0.4, 1.0, 4000) * MOST).astype(np.float32)
    p = 1 / (1 + np.exp(-2 * MOST / T.astype(np.float64)))
    u = p.astype(np.float32)
    u = np.where(rng.random(4000) < 0.5, np.nextafter(u, np.float32(0)), u).astype(np.float32)
    far = np.abs(u.astype(np.float64) - p) >= 2.0 ** -27
    assert far.sum() > 2000
    T, u = T[far], u[far]
    check(torch.tensor([[MOST, -MOST]], device="cuda").repeat(len(T), 1), u, temperature=T)
