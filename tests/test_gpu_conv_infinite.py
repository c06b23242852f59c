"""Reverse mode of the convolution with an infinite input or gradient at every token in turn: the parameters' sums are infinite as their terms are, and no
token that a wave only looks at on its way adds a term of its own."""
import pytest
import torch

from paper_2404_07904_amd import binding as lib

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("what", ["x", "grad"])
@pytest.mark.parametrize("N", [70, 2000])
def test_one_infinity_a_channel(dtype, K, what, N):
    D = N
    g = torch.Generator(device="cuda").manual_seed(K)
    # signs alone, so that infinite sums have one sign and finite ones are whole numbers
    sign = lambda *s: (torch.randint(0, 2, s, generator=g, device="cuda") * 2 - 1).to(dtype)  # noqa: E731
    x, gy, w = sign(1, N, D), sign(1, N, D), sign(D, K).float()
    at = torch.arange(N, device="cuda")
    (x if what == "x" else gy)[0, at, at] = float("inf")
    gx, gw, gb, _ = lib.hgrn2_conv_bwd(x, w, torch.zeros(D, device="cuda"), gy, silu=False)
    past = torch.cat([torch.zeros(K - 1, D, device="cuda", dtype=dtype), x[0]]).double()
    want_w = torch.stack([torch.nan_to_num(gy[0].double() * past[k:k + N], nan=0.0, posinf=float("inf"), neginf=-float("inf")).sum(0) for k in range(K)], 1)
    if what == "grad":
        # (an infinite gradient times the zero before a sequence is not a number: nor is its sum)
        for k in range(K):
            want_w[at[:K - 1 - k], k] = float("nan")
    number = ~torch.isnan(want_w)
    assert torch.equal(~torch.isnan(gw), number) and torch.equal(gw.double()[number], want_w[number])
    assert torch.equal(gb.double(), gy[0].double().sum(0))
