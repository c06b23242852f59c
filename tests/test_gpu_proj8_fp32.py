"""fp32 results of the 8-bit product: sums of exact products in fp32, whatever kernel a size takes."""
import pytest
import torch

from paper_2404_07904_amd import binding as lib

pytestmark = pytest.mark.gpu
F64, F32 = torch.float64, torch.float32
# few rows, small and large tiles, shares of a long contraction; blocks that are no multiple of four, odd edges
SIZES = [(1, 70, 300), (16, 33, 1200), (17, 130, 2048), (33, 257, 1100), (64, 80, 4000), (65, 64, 128), (129, 65, 1200), (300, 130, 2000), (96, 80, 16384), (257, 130, 5000),
         (2000, 2050, 640), (1793, 4100, 1200), (1025, 2049, 2176),
         (4000, 3900, 1200)]


def operand(values, scale_bytes, rows):
    """e4m3 values [M, K] and the bytes of their scales [M / rows rounded up, blocks], laid out as hgrn2_quant8 leaves them."""
    M, K = values.shape
    q = torch.zeros(M, -(-K // 128) * 128, dtype=torch.float8_e4m3fn, device="cuda")
    q[:, :K] = values.to(torch.float8_e4m3fn)
    s = torch.zeros(scale_bytes.shape[0], -(-K // 512) * 4, dtype=torch.uint8, device="cuda")
    s[:, :scale_bytes.shape[1]] = scale_bytes
    e = scale_bytes.to(F64).repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K] - 127.0
    return q, s, values.to(F64) * torch.exp2(e)


@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_sums_that_fp32_holds_are_exact(M, N, K, b_rows):
    """Values are multiples of 2^-2 and scales at least 1, so all products are multiples of 2^-4; the sums of their sizes stay below 2^20: every partial
    sum in any order is a number of fp32."""
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    pick = lambda *s: torch.randint(0, 1 << 30, s, generator=g, device="cuda")  # noqa: E731
    small = torch.tensor([0.0, 0.25, -0.25, 0.5, -0.75, 1.25, -1.75, 1.0], device="cuda")
    # (a row of a has 256 in 8 places at most, at which b is 60 at most; elsewhere products are below 4 x 1.75^2)
    a = small[pick(M, K) % 8]
    at = pick(M, 8) % K
    a.scatter_(1, at, torch.where(pick(M, 8) % 2 == 0, 256.0, -224.0))
    b = torch.where(pick(N, K) % 97 == 0, torch.where(pick(N, K) % 2 == 0, 60.0, -36.0), small[pick(N, K) % 8])
    blocks = -(-K // 128)
    a, sa, va = operand(a, 127 + (pick(M, blocks) % 2).to(torch.uint8), 1)
    b, sb, vb = operand(b, 127 + (pick(-(-N // b_rows), blocks) % 2).to(torch.uint8), b_rows)
    assert float((va.abs() @ vb.abs().t()).max()) < 2.0 ** 20
    c = lib.hgrn2_proj8(a, sa, b, sb, out_dtype=F32)
    assert torch.equal(c.to(F64), va @ vb.t())
    assert torch.equal(c, lib.hgrn2_proj8(a, sa, b, sb, out_dtype=F32))


@pytest.mark.parametrize("M,N,K", SIZES)
def test_random_sums_as_fp32_adds_them(M, N, K):
    """Rows of random values of one size along the contraction.  After k terms a partial sum is sqrt(k) terms large, an addition is off by 2^-24 of it (twice that
    if cut off), in squares over K terms 2^-23 K / sqrt(2) terms, next to a result of sqrt(K) terms: 2^-23 sqrt(K / 2) of a row in the 2-norm.  Values lie
    between 2^-100 and 2^100 by rows, and the scales with them."""
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    a = n(M, K) * torch.exp2(torch.linspace(-100, 100, M, device="cuda").round())[:, None]
    b = n(N, K) * torch.exp2(torch.linspace(-20, 20, N, device="cuda").round())[:, None]
    qa, qb = lib.hgrn2_quant8(a), lib.hgrn2_quant8(b)

    def values(q, s):
        e = s[:, :q.shape[1] // 128].to(F64).repeat_interleave(128, 1) - 127.0
        return q.to(F32).to(F64) * torch.exp2(e)

    va, vb = values(*qa), values(*qb)
    ref = va @ vb.t()
    c = lib.hgrn2_proj8(*qa, *qb, out_dtype=F32).to(F64)
    # (both in the size that a row and a column of it have, which are of unlike size)
    size = va.norm(dim=1)[:, None] * vb.norm(dim=1) * K ** -0.5
    off = ((c - ref) / size).norm(dim=1) / (ref / size).norm(dim=1)
    print("    worst row %.2e of %.2e" % (off.max().item(), 2.0 ** -23 * (K / 2) ** 0.5), flush=True)
    assert torch.isfinite(c).all() and off.max().item() <= 2.0 ** -23 * (K / 2) ** 0.5


def test_the_largest_and_smallest_values():
    big, tiny = torch.finfo(F32).max, 2.0 ** -109
    for M in (3, 80):
        a, b = torch.zeros(M, 200, device="cuda"), torch.zeros(40, 200, device="cuda")
        a[:, 0], a[0, 150], b[:, 0], b[:, 150] = big, tiny, 2.0 ** -30, 1.0
        qa, qb = lib.hgrn2_quant8(a), lib.hgrn2_quant8(b)
        # the largest value of fp32 stands for 2^128 in e4m3; the smallest scale is that of 2^-100, 2^-108, whose multiples start at 2^-117
        c = lib.hgrn2_proj8(*qa, *qb, out_dtype=F32)
        assert (c == 2.0 ** 98).all()
        b[:, 0] = 0.0
        assert (lib.hgrn2_proj8(*qa, *lib.hgrn2_quant8(b), out_dtype=F32)[0] == tiny).all()
        b[:, 0] = 2.0
        assert torch.isinf(lib.hgrn2_proj8(*qa, *lib.hgrn2_quant8(b), out_dtype=F32)).all()


@pytest.mark.parametrize("act", [None, "silu", "sigmoid"])
@pytest.mark.parametrize("M,N,K", [(5, 70, 300), (100, 70, 1200), (96, 80, 16384), (1100, 2100, 600), (3900, 4000, 300)])
def test_bias_and_activation(M, N, K, act):
    g = torch.Generator(device="cuda").manual_seed(K)
    qa, qb = (lib.hgrn2_quant8(torch.randn(r, K, generator=g, device="cuda") * K ** -0.25) for r in (M, N))
    bias = torch.randn(N, generator=g, device="cuda")
    pre = lib.hgrn2_proj8(*qa, *qb, out_dtype=F32).to(F64) + bias.to(F64)
    ref = pre * torch.sigmoid(pre) if act == "silu" else torch.sigmoid(pre) if act == "sigmoid" else pre
    got = lib.hgrn2_proj8(*qa, *qb, bias, act=act, out_dtype=F32).to(F64)
    # an addition and an activation in fp32: slopes of 1.1 at most, 2^-20 of the result for an exponential and a quotient
    assert ((got - ref).abs() <= 1.1 * 2.0 ** -23 * (pre.abs() + bias.abs()) + 2.0 ** -20 * ref.abs()).all()


@pytest.mark.parametrize("M", [3, 30, 80])
@pytest.mark.parametrize("out", [torch.bfloat16, F32])
def test_every_byte_of_a_scale(M, out):
    """Scales as others may write them: a block of zeros with the byte 0, the smallest and largest powers of two, and the byte that stands for no number."""
    K = 4 * 128
    a, b = torch.zeros(M, K, device="cuda"), torch.ones(20, K, device="cuda")
    a[:, 256] = 1.0
    byte = torch.full((M, 4), 127, dtype=torch.uint8, device="cuda")
    byte[:, 0] = 0                                        # (zeros in a)
    for e in (1, 2, 19, 127, 250, 254):
        byte[:, 2] = e
        other = torch.full((20, 4), 254 - e if e < 254 else 1, dtype=torch.uint8, device="cuda")
        qa, sa, _ = operand(a, byte, 1)
        qb, sb, _ = operand(b, other, 1)
        want = 2.0 ** (e - 127) * 2.0 ** (float(other[0, 0]) - 127)
        assert (lib.hgrn2_proj8(qa, sa, qb, sb, out_dtype=out).double() == want).all(), e
    byte[:, 2], byte[1, 2] = 127, 255
    qa, sa, _ = operand(a, byte, 1)
    qb, sb, _ = operand(b, torch.full((20, 4), 127, dtype=torch.uint8, device="cuda"), 1)
    c = lib.hgrn2_proj8(qa, sa, qb, sb, out_dtype=out)
    assert torch.isnan(c[1]).all() and (c[0] == 1.0).all() and (c[2:] == 1.0).all()
