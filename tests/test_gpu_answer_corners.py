"""The operators of a head that answers in the corners of what they accept: temperatures at the ends of binary32."""
import pytest
import torch

from tests.test_gpu_answer import F32, check_draws, natural

pytestmark = pytest.mark.gpu

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
