"""Packed batches of the scan whose sequences begin far behind the first row: gradients are those of the batch without the rows before, and nothing
is read of the states of chunks that no sequence reaches, which the forward pass leaves as they were."""
import ctypes

import pytest
import torch

import mixer_oracle as oracle
from paper_2404_07904_amd import binding as lib

pytestmark = pytest.mark.gpu
F64, BF16, F32 = torch.float64, torch.bfloat16, torch.float32


def saved_bytes(n_seq, T, D, S, G, dtype):
    s = lib.hgrn2_ssm_shape(n_seq, T, D, S, G, lib.HGRN2_BF16 if dtype == BF16 else lib.HGRN2_F32, 1)
    return int(lib.lib().hgrn2_ssm_saved_states_bytes(ctypes.byref(s), 1))


# Sizes whose runs of tokens lie differently in the two directions: a run of the reverse mode reaches from the first offset back into one of
# the forward pass that holds no token of a sequence.
@pytest.mark.parametrize("dtype,T,D,S,first", [(BF16, 1000, 4096, 16, 97), (F32, 1000, 4096, 8, 111), (BF16, 700, 4096, 8, 64), (F32, 2000, 1030, 8, 70),
                                               (BF16, 400, 64, 32, 200), (F32, 300, 20, 16, 299)])
def test_states_that_were_never_saved_are_not_read(dtype, T, D, S, first):
    g = torch.Generator().manual_seed(first)
    n = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    ends = sorted({first, min(first + 1, T), (first + T) // 2, T - (T - first) // 10})
    x, dt, z, gy, Bm, Cm = (n(T, *s).to(dtype) for s in ((D,), (D,), (D,), (D,), (1, S), (1, S)))
    A, D_, bias = -torch.rand(D, S, generator=g).cuda() * 3.0 - 0.05, n(D), n(D) - 2.0

    def run(skip, poison):
        cu = torch.tensor([e - skip for e in ends], dtype=torch.int32, device="cuda")
        t = [v[skip:] for v in (x, dt, Bm, Cm, gy, z)]
        par = dict(D=D_, dt_bias=bias, z=t[5], cu_seqlens=cu)
        held = torch.full((saved_bytes(len(ends) - 1, T - skip, D, S, 1, dtype),), 255 if poison else 0, dtype=torch.uint8, device="cuda")   # NaN, whole or in halves
        _, _, states = lib.hgrn2_ssm_fwd_saving(t[0], t[1], A, t[2], t[3], saved_states=held, **par)
        return lib.hgrn2_ssm_bwd(t[0], t[1], A, t[2], t[3], t[4], saved_states=states, **par)

    got, ref = run(first, False), run(0, True)
    for name, a, b in zip(("x", "dt", "A", "B", "C", "D", "z", "dt_bias"), ref, got):
        if a.dim() > 1 and a.shape[0] == T and name != "A":
            assert (a[:first] == 0).all(), name
            a = a[first:]
        # two results, each within what one may be off by
        oracle.check("grad_" + name, a, b.cpu().to(F64), tol32=2 * oracle.TOL32 + (2 * oracle.half_step(dtype) if a.dtype == BF16 else 0.0))
