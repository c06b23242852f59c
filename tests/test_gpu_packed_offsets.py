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


# ---- offsets that are wrong: whatever comes out, nothing outside the tensors is written (which rows are read is checked without a GPU) ----
class Guarded:
    """A tensor between two stretches of bytes that have to stay as they are."""
    EDGE = 1 << 16

    def __init__(self, shape, dtype):
        size = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
        self.all = torch.full((size + 2 * self.EDGE,), 0x5A, dtype=torch.uint8, device="cuda")
        self.t = self.all[self.EDGE:self.EDGE + size].view(dtype).view(shape)
        self.t.zero_()

    @property
    def p(self):
        return ctypes.c_void_p(self.t.data_ptr())

    def whole(self):
        return bool((self.all[:self.EDGE] == 0x5A).all() and (self.all[-self.EDGE:] == 0x5A).all())


WRONG = [[0, 90, 10, 100], [0, 90, 10, 20, 30, 100], [0, 50, 20], [100, 0], [0, 100, 64, 64, 70], [-7, 1000, 3, 40], [60, 20, 90, 30, 80], [5] * 70 + [100, 2, 99]]


@pytest.mark.parametrize("dtype,S", [(F32, 16), (BF16, 32), (BF16, 5)])
@pytest.mark.parametrize("T", [100, 16, 400])
@pytest.mark.parametrize("ends", WRONG, ids=lambda e: "-".join(map(str, e[-5:])))
def test_scan_with_wrong_offsets(ends, T, dtype, S):
    B, D, io = len(ends) - 1, 20, lib.HGRN2_BF16 if dtype == BF16 else lib.HGRN2_F32
    L, shape = lib.lib(), lib.hgrn2_ssm_shape(B, T, D, S, 1, io, 1)
    s, cu = ctypes.byref(shape), torch.tensor(ends, dtype=torch.int32, device="cuda")
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def given(*size, t=dtype):
        g = Guarded(size, t)
        g.t.normal_()
        return g

    x, dt, z, gy, Bm, Cm = given(T, D), given(T, D), given(T, D), given(T, D), given(T, S), given(T, S)
    A, D_, bias, h0, ghT = given(D, S, t=F32), given(D, t=F32), given(D, t=F32), given(B, D, S, t=F32), given(B, D, S, t=F32)
    A.t.abs_().neg_()
    raw = lambda n: Guarded((max(int(n), 256),), torch.uint8)  # noqa: E731
    y, hT, saved = Guarded((T, D), dtype), Guarded((B, D, S), F32), raw(L.hgrn2_ssm_saved_states_bytes(s, 1))
    ws = raw(L.hgrn2_ssm_fwd_workspace_bytes(s, 1))
    c = ctypes.c_void_p(cu.data_ptr())
    assert L.hgrn2_ssm_fwd_saving(s, c, x.p, dt.p, A.p, Bm.p, Cm.p, D_.p, z.p, bias.p, h0.p, y.p, hT.p, saved.p, saved.t.numel(), ws.p, ws.t.numel(), stream) == 0
    torch.cuda.synchronize()
    out = [Guarded((T, D), dtype) for _ in range(3)] + [Guarded((T, S), dtype) for _ in range(2)]
    par = [Guarded((D, S), F32), Guarded((D,), F32), Guarded((D,), F32), Guarded((B, D, S), F32)]
    for kept in (True, False):
        wb = raw(L.hgrn2_ssm_bwd_workspace_bytes(s, 1, int(kept)))
        assert L.hgrn2_ssm_bwd(s, c, x.p, dt.p, A.p, Bm.p, Cm.p, D_.p, z.p, bias.p, h0.p, saved.p if kept else None, saved.t.numel() if kept else 0, gy.p, ghT.p,
                               out[0].p, out[1].p, par[0].p, out[3].p, out[4].p, par[1].p, out[2].p, par[2].p, par[3].p, wb.p, wb.t.numel(), stream) == 0
        torch.cuda.synchronize()
        assert wb.whole()
    for t in (x, dt, z, gy, Bm, Cm, A, D_, bias, h0, ghT, y, hT, saved, ws, *out, *par):
        assert t.whole()


@pytest.mark.parametrize("dtype,K", [(F32, 4), (BF16, 3)])
@pytest.mark.parametrize("T,D", [(100, 20), (40000, 8)])
@pytest.mark.parametrize("ends", WRONG, ids=lambda e: "-".join(map(str, e[-5:])))
def test_convolution_with_wrong_offsets(ends, T, D, dtype, K):
    B, io = len(ends) - 1, lib.HGRN2_BF16 if dtype == BF16 else lib.HGRN2_F32
    L, shape = lib.lib(), lib.hgrn2_conv_shape(B, T, D, K, io, 1)
    s, cu = ctypes.byref(shape), torch.tensor([e * (T // 100) for e in ends], dtype=torch.int32, device="cuda")
    stream, c = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream), ctypes.c_void_p(cu.data_ptr())
    x, gy, y, gx = (Guarded((T, D), dtype) for _ in range(4))
    w, bias, gw, gb = Guarded((D, K), F32), Guarded((D,), F32), Guarded((D, K), F32), Guarded((D,), F32)
    state, fin, gs = (Guarded((B, K - 1, D), dtype) for _ in range(3))
    for t in (x, gy, w, bias, state):
        t.t.normal_()
    ws = Guarded((int(L.hgrn2_conv_bwd_workspace_bytes(s, 1)),), torch.uint8)
    assert L.hgrn2_conv_fwd(s, c, x.p, w.p, bias.p, state.p, y.p, fin.p, stream) == 0
    torch.cuda.synchronize()
    assert L.hgrn2_conv_bwd(s, c, x.p, w.p, bias.p, state.p, gy.p, fin.p, gx.p, gw.p, gb.p, gs.p, ws.p, ws.t.numel(), stream) == 0
    torch.cuda.synchronize()
    for t in (x, gy, y, gx, w, bias, gw, gb, state, fin, gs, ws):
        assert t.whole()
