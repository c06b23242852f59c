"""The 8-bit product in every kernel that a size may take, with more steps than a tile's ring of them has places and a last group of scales that is not whole
(tests/test_proj8_plan_host.py holds which sizes those are)."""
import pytest
import torch

from paper_2404_07904_amd import binding as lib
from test_gpu_proj8 import operands, product_check
from test_gpu_proj8_fp32 import operand
from test_proj8_plan_host import SIZES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [s[:3] for s in SIZES])
def test_bf16_results(M, N, K):
    (a, sa), (b, sb), va, vb = operands(M, N, K, 1, 128) if M * K < 1 << 24 else large(M, N, K)
    c = lib.hgrn2_proj8(a, sa, b, sb)
    product_check(c, va, vb)
    assert torch.equal(c, lib.hgrn2_proj8(a, sa, b, sb))


def large(M, N, K):
    """Operands whose values are made on the GPU: the oracle's quantisation takes a while."""
    g = torch.Generator(device="cuda").manual_seed(K)
    codes = lambda r: torch.randint(0, 256, (r, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)  # noqa: E731
    blocks = -(-K // 128)
    out = []
    for r, rows in ((M, 1), (N, 128)):
        v = codes(r).view(torch.float8_e4m3fn).float()
        s = torch.randint(120, 135, (-(-r // rows), blocks), generator=g, device="cuda").to(torch.uint8)
        q, s, stand = operand(torch.nan_to_num(v, nan=1.0), s, rows)
        out.append((q, s, stand))
    return out[0][:2], out[1][:2], out[0][2], out[1][2]


@pytest.mark.parametrize("M,N,K", [s[:3] for s in SIZES])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_every_step_counts_once(M, N, K, out):
    """One value of a row of a is not zero, at a place of its own: the result is the value of b there times it, in every block and row of the contraction."""
    g = torch.Generator(device="cuda").manual_seed(M)
    blocks = -(-K // 128)
    a = torch.zeros(M, K, device="cuda")
    at = (torch.arange(M, device="cuda") * 37 + 5) % K
    a[torch.arange(M, device="cuda"), at] = 2.0
    b = torch.randint(-8, 9, (N, K), generator=g, device="cuda").float()
    qa, sa, va = operand(a, torch.randint(124, 130, (M, blocks), generator=g, device="cuda").to(torch.uint8), 1)
    qb, sb, vb = operand(b, torch.randint(124, 130, (N, blocks), generator=g, device="cuda").to(torch.uint8), 1)
    c = lib.hgrn2_proj8(qa, sa, qb, sb, out_dtype=out)
    want = vb[:, at].t() * va[torch.arange(M, device="cuda"), at][:, None]
    assert torch.equal(c.double(), want)
