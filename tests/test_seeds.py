"""What a test draws from torch's generators is a function of its name: a failure repeats, and a pass holds."""
import zlib

import pytest
import torch


def want(name, device="cpu"):
    gen = torch.Generator(device=device).manual_seed(zlib.crc32(("test_seeds.py::" + name).encode()))
    return torch.randn(5, device=device, generator=gen)


@pytest.mark.parametrize("case", ["a", "b"])
def test_draws_on_the_host(case):
    assert torch.equal(torch.randn(5), want("test_draws_on_the_host[%s]" % case))


@pytest.mark.gpu
@pytest.mark.parametrize("case", ["a", "b"])
def test_draws_on_the_device(case):
    assert torch.equal(torch.randn(5, device="cuda"), want("test_draws_on_the_device[%s]" % case, "cuda"))
