"""The operators of a head that answers in the corners of what they accept: temperatures and logits at the ends of binary32."""
import math

import pytest
import torch

from tests.test_gpu_answer import F32, check_draws, natural

pytestmark = pytest.mark.gpu

MOST = float(torch.finfo(F32).max)


# ---- temperatures and logits at the ends of binary32 ------------------------------------------------------------------------

@pytest.mark.parametrize("temperature", [9.5e-38, 9e-38, 5e-38, float(torch.finfo(F32).tiny), 1e-38, 1e-41, 2.0 ** -149])
@pytest.mark.parametrize("words", [1000, 9000])
def test_sample_least_temperatures(words, temperature):
    """32 / T ends at the largest number of binary32 and so do the bins of a histogram; logits of zeros, of both signs, natural ones
    with 0 as their largest, and some that differ by a few T."""
    print("sample", words, temperature, flush=True)
    g = torch.Generator().manual_seed(words)
    l = torch.zeros(5, words)
    l[1] = torch.where(torch.rand(words, generator=g) < 0.5, torch.tensor(0.0), torch.tensor(-0.0))
    n = natural(words, 2, words, F32)
    l[2:4] = n - n.amax(1, keepdim=True)
    l[3] *= 1e-38
    l[4] = -torch.floor(torch.rand(words, generator=g) * 8) * torch.tensor(temperature, dtype=F32)
    u = torch.rand(5, generator=g)
    for limits in ({}, {"top_p": 0.5}, {"top_p": 0.9}, {"top_k": 7}, {"top_k": 600}, {"top_k": 2500, "top_p": 0.7}, {"top_k": 300, "top_p": 0.6, "min_p": 0.1}, {"min_p": 0.3}):
        check_draws(l, u, temperature=temperature, **limits)


@pytest.mark.parametrize("temperature", [1e36, 2.0 ** 122, 6e36, 1e37, 2e37, 1e38, MOST, math.inf])
@pytest.mark.parametrize("words", [1000, 9000])
def test_sample_differences_beyond_binary32(words, temperature):
    """Logits whose difference is no number of binary32, at temperatures where the lower ones have mass."""
    print("sample", words, temperature, flush=True)
    g = torch.Generator().manual_seed(words)
    upper = torch.rand(words, generator=g) < 0.5
    l = torch.empty(4, words)
    l[0] = torch.where(upper, 3e38, -3e38)
    l[1] = torch.where(upper, MOST, -MOST)
    l[2] = (torch.rand(words, generator=g, dtype=torch.float64) * 2 - 1).float() * 3.2e38
    l[3] = torch.where(upper, -1e38, l[2].abs())
    l[3, ::7] = -math.inf
    u = torch.rand(4, generator=g)
    half = int(upper.sum())
    for limits in ({}, {"top_p": 0.999}, {"top_p": 0.6}, {"top_k": half + 70}, {"top_k": half + 70, "top_p": 0.9}, {"top_k": 4000, "top_p": 0.99}, {"min_p": 1e-4}):
        check_draws(l, u, temperature=temperature, **limits)
