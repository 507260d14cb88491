"""Edges of the operators on the loaded layout: many tokens with fp32 results."""
import pytest
import torch

import paper_2607_18957_gb300 as cfa

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def cuda_device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.fixture(autouse=True)
def no_wait_ran_out(cuda_device):
    yield
    torch.cuda.synchronize()
    cfa.op_status()


def normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("t", [16256, 16257, 20000, 65536])
@pytest.mark.parametrize("n,k", [(8, 320), (200, 72)])
@pytest.mark.parametrize("gated", [False, True])
def test_fp32_results_of_many_tokens(t, n, k, gated):
    """A product's sum of K terms in fp32 is off by at most (K + 8) 2^-23 of the sum of the terms'
    magnitudes, relu by no more, a gated product by what the errors of its factors make of it, and
    the rounding to fp32 by 2^-24."""
    x, w = normal(t, (t, k), BF16), normal(n, (2 * n if gated else n, k), BF16, k ** -0.5)
    y = cfa.linear(x, w, activation="relu", gated=gated, out_dtype="f32")
    v = x.double() @ w.double().t()
    ev = (x.double().abs() @ w.double().abs().t()) * ((k + 8) * 2.0 ** -23)
    ref, bound = v.clamp(min=0), ev
    if gated:
        a, u, ea, eu = ref[:, :n], v[:, n:], ev[:, :n], ev[:, n:]
        ref, bound = a * u, ea * u.abs() + a * eu + ea * eu
    bound = bound + 2.0 ** -23 * (ref.abs() + bound)
    assert y.dtype == F32 and y.shape == (t, n)
    worst = ((y.double() - ref).abs() - bound).max().item()
    assert worst <= 0, f"off by {worst:g} more than the bound"
