"""Host-side checks of the operators around a language model's output that need no GPU: arguments that are refused before
anything is launched, sizes of the workspace, and how tensors become rows for the reordering of states."""
import ctypes as C

import numpy as np
import pytest
import torch

P = C.c_void_p


@pytest.fixture(scope="module")
def Bd():
    from paper_2206_07882_b200 import build
    build.build()
    from paper_2206_07882_b200 import binding
    binding.lib()
    return binding


FAKE, ODD = P(4096), P(4097)      # aligned / not; never dereferenced: checks fail first


def test_norm_refusals(Bd):
    def call(x=FAKE, ldx=64, r=None, ldr=0, dtype=0, rows=4, k=64, k_pad=64, gain=FAKE, eps=1e-5, s=None, lds=0, q=FAKE, sc=FAKE):
        return Bd.lib().q4_rmsnorm_quantize(x, C.c_int64(ldx), r, C.c_int64(ldr), C.c_int32(dtype), C.c_int64(rows), C.c_int32(k),
                                            C.c_int32(k_pad), gain, C.c_float(eps), s, C.c_int64(lds), q, sc, None)
    assert call(dtype=3) == -6
    assert call(rows=-1) == -2 and call(k=0) == -2 and call(k_pad=32) == -2 and call(ldx=63) == -2
    assert call(eps=-1e-6) == -2 and call(eps=float("nan")) == -2 and call(eps=float("inf")) == -2
    assert call(x=None) == -1 and call(gain=None) == -1 and call(q=None) == -1 and call(sc=None) == -1
    assert call(r=FAKE, ldr=64) == -1 and call(s=FAKE, lds=64) == -1
    assert call(r=FAKE, ldr=63, s=FAKE, lds=64) == -2 and call(r=FAKE, ldr=64, s=FAKE, lds=63) == -2
    assert call(r=P(8192), ldr=64, s=FAKE, lds=65) == -6        # over x, at another stride
    assert call(k=60, k_pad=60) == -3 and call(q=P(4104)) == -3 and call(x=ODD) == -3 and call(gain=P(4098)) == -3
    assert call(x=ODD, dtype=1) == -3
    assert call(rows=0) == 0


def test_linear_refusals(Bd):
    def call(xq=FAKE, sx=FAKE, M=4, w=None, b=None, out=FAKE, dtype=0, ldo=128, status=None):
        m = w if w is not None else Bd.Mat(4096, 4096, 128, 64, 64, 8)
        return Bd.lib().q4_linear_token_scales(xq, sx, C.c_int32(M), C.byref(m), b, out, C.c_int32(dtype), C.c_int64(ldo), status, None)
    assert call(dtype=5) == -6
    assert call(w=Bd.Mat(4096, 4096, 128, 64, 64, 4)) == -4 and call(w=Bd.Mat(None, 4096, 128, 64, 64, 8)) == -1
    assert call(w=Bd.Mat(4096, 4096, 128, 64, 80, 8)) == -3 and call(w=Bd.Mat(4096, 4096, 128, 131041, 131072, 8)) == -2
    assert call(M=-1) == -2 and call(ldo=127) == -2
    assert call(xq=None) == -1 and call(sx=None) == -1 and call(out=None) == -1
    assert call(xq=P(4104)) == -3 and call(out=P(4098)) == -3 and call(out=ODD, dtype=2) == -3 and call(b=P(4097)) == -3
    assert call(M=0) == 0


def test_select_refusals_and_workspace(Bd):
    def call(z=FAKE, ld=100, dtype=0, score=FAKE, done=None, B=2, W=4, V=100, eos=-1, rho=0.0, par=P(8192), tok=P(8192), so=P(8192), do=None, arr=FAKE,
             ws=FAKE, n=1 << 30):
        return Bd.lib().q4_lm_beam_select(z, C.c_int64(ld), C.c_int32(dtype), score, done, C.c_int32(B), C.c_int32(W), C.c_int32(V),
                                          C.c_int32(eos), C.c_float(rho), par, tok, so, do, arr, ws, C.c_size_t(n), None)
    assert call(dtype=-1) == -6
    assert call(B=-1) == -2 and call(W=0) == -2 and call(W=33) == -2 and call(V=0) == -2 and call(ld=99) == -2
    assert call(B=1 << 30, W=4) == -2
    assert call(eos=100) == -2 and call(eos=-2) == -2 and call(done=FAKE) == -2 and call(rho=float("nan")) == -2
    for name in ("z", "score", "par", "tok", "so", "arr", "ws"):
        assert call(**{name: None}) == -1
    assert call(so=FAKE) == -6 and call(done=FAKE, do=FAKE, eos=3) == -6
    assert call(z=P(4098)) == -3 and call(ws=P(4104)) == -3 and call(arr=P(4098)) == -3
    need = Bd.workspace_bytes(Bd.WS_LM_SELECT, (2, 4, 100))
    assert need > 0 and call(n=need - 1) == -5
    assert call(B=0) == 0
    assert Bd.workspace_bytes(Bd.WS_LM_SELECT, (64, 32, 100000)) >= need


def test_reorder_refusals(Bd):
    def item(src=1 << 20, dst=1 << 21, row=64, ss=64, ds=64, n=(1, 1), s=(0, 0), d=(0, 0)):
        t = Bd.ReorderS()
        t.src, t.dst, t.row_bytes, t.src_row_step, t.dst_row_step = src, dst, row, ss, ds
        for i in range(2):
            t.n[i], t.src_step[i], t.dst_step[i] = n[i], s[i], d[i]
        return t

    def call(*items, n=None, parent=FAKE, B=2, W=4):
        arr = (Bd.ReorderS * max(len(items), 1))(*items)
        return Bd.lib().q4_beam_reorder(arr, C.c_int32(len(items) if n is None else n), parent, C.c_int32(B), C.c_int32(W), None)
    assert call(item(), n=17) == -2 and call(item(), n=-1) == -2 and call(item(), W=0) == -2 and call(item(), B=1 << 30) == -2
    assert call(item(), parent=None) == -1 and call(item(src=None)) == -1 and call(item(dst=None)) == -1
    assert call(item(), parent=P(4098)) == -3
    assert call(item(row=-1)) == -2 and call(item(ss=-64)) == -2 and call(item(ds=63)) == -2
    assert call(item(n=(-1, 1))) == -2 and call(item(n=(2, 1), s=(512, 0), d=(63, 0))) == -2
    assert call(item(n=(1 << 40, 1), s=(1 << 40, 0), d=(1 << 40, 0))) == -2
    assert call(item(n=(1 << 32, 1 << 32), row=1, ss=1, ds=1, s=(1, 1), d=(1, 1))) == -2   # more rows than addresses
    assert call(item(dst=1 << 20)) == -6                                       # in place
    assert call(item(dst=(1 << 20) + 7 * 64 + 63)) == -6                       # the last byte of the last row
    assert call(item(), item(src=1 << 21, dst=1 << 22)) == -6                  # one tensor's new rows are another's old ones
    assert call() == 0 and call(item(), B=0) == 0


def test_rows_of_tensors_for_the_reordering(Bd):
    """Every byte of a row, as the library is told it, against torch's own indexing."""
    def bytes_of(t, which):
        base, row = ((t.src, t.src_row_step), (t.dst, t.dst_row_step))[which]
        step = (t.src_step, t.dst_step)[which]
        return {(bw, i0, i1): base + i0 * step[0] + i1 * step[1] + bw * row
                for bw in range(B * W) for i0 in range(t.n[0]) for i1 in range(t.n[1])}
    B, W = 2, 3
    full = torch.zeros(4, B, W, 5, 16, 6, dtype=torch.float16)
    cases = [(full, 1), (full[:, :, :, :, :7], 1), (full[:, :, :, 1:3, :7], 1), (full[1:3], 1), (full[0], 0), (full[0, :, :, :, :1], 0),
             (full.permute(3, 1, 2, 0, 4, 5)[:, :, :, 2], 1), (torch.zeros(B, W), 0), (torch.zeros(B, W, 1, 9), 0),
             (torch.zeros(3, 4, B, W, 8), 2)]
    for src, dim in cases:
        dst = torch.zeros_like(src, memory_format=torch.contiguous_format)
        t = Bd.ReorderS.from_buffer_copy((C.c_int64 * 11)(*Bd._reorder_item(src, dst, dim, B, W)))
        assert t.n[0] * t.n[1] * t.row_bytes * B * W == src.numel() * src.element_size()
        for which, x in ((0, src), (1, dst)):
            es = x.element_size()
            got = sorted(a + j for a in bytes_of(t, which).values() for j in range(0, t.row_bytes, es))
            idx = np.indices(x.shape).reshape(x.dim(), -1)
            want = sorted((x.data_ptr() + es * sum(idx[d] * x.stride(d) for d in range(x.dim()))).tolist())
            assert got == want
        # the same places of both in the same order: rows (bw, i0, i1) of src and dst hold the same elements
        flat = torch.arange(src.numel(), dtype=torch.int32).reshape(src.shape)
        order = {}
        for which, x in ((0, src), (1, dst)):
            idx = np.indices(x.shape).reshape(x.dim(), -1)
            at = x.data_ptr() + x.element_size() * sum(idx[d] * x.stride(d) for d in range(x.dim()))
            who = dict(zip(at.tolist(), flat.flatten().tolist()))
            order[which] = {key: who[a] for key, a in bytes_of(t, which).items()}
        assert order[0] == order[1]
    with pytest.raises(ValueError):                        # three dimensions that do not follow one another
        x = torch.zeros(B, W, 4, 4, 4, 4)[:, :, ::2, :3, ::2, :3]
        Bd._reorder_item(x, torch.zeros(x.shape), 0, B, W)
    with pytest.raises(ValueError):
        x = torch.zeros(W, B, 4).transpose(0, 1)
        Bd._reorder_item(x, torch.zeros(x.shape), 0, B, W)


def test_tensors_of_other_devices_are_refused(Bd):
    with pytest.raises(ValueError):
        Bd._on_device(torch.zeros(2))
    Bd._on_device(None)
