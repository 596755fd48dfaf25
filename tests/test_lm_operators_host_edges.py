"""Host-side checks of the operators around a language model's output where a first set of tests did not look; no GPU."""
import ctypes as C

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


def test_any_number_of_moves_is_checked_as_one_call(Bd):
    def item(src, dst, row=64, n=(1, 1), step=(0, 0)):
        t = Bd.ReorderS()
        t.src, t.dst, t.row_bytes, t.src_row_step, t.dst_row_step = src, dst, row, row, row
        for i in range(2):
            t.n[i], t.src_step[i], t.dst_step[i] = n[i], step[i], step[i]
        return t

    def check(items, n=None, B=2, W=4):
        return Bd.lib().q4_beam_reorder_check((Bd.ReorderS * max(len(items), 1))(*items), len(items) if n is None else n, B, W)

    def fresh(n):       # sources from 2^30 on, destinations from 2^31 on, 512 bytes each
        return [item((1 << 30) + 512 * i, (1 << 31) + 512 * i) for i in range(n)]
    for n in (0, 1, 16, 17, 32, 33, 100):
        assert check(fresh(n)) == 0
    # a source on the last byte of another's destination, before, beside and behind a border of 16, and itself
    for n in (2, 17, 40, 100):
        for i in {0, 1, 15, 16, 31, n - 1}:
            for j in {0, 1, 15, 16, 31, n - 1}:
                if i < n and j < n:
                    items = fresh(n)
                    items[i].src = items[j].dst + 511
                    assert check(items) == -6
                    if j + 1 == n:          # (others' destinations begin there)
                        items[i].src += 1
                        assert check(items) == 0
    # what a call refuses of one item is refused wherever it stands
    for at in (0, 15, 16, 39):
        for bad, code in ((item(1 << 20, 1 << 21, row=-1), -2), (item(None, 1 << 21), -1), (item(1 << 20, None), -1),
                          (item(1 << 20, 1 << 21, n=(2, 1), step=(63, 0)), -2), (item(1 << 20, 1 << 21, n=(-1, 1)), -2)):
            items = fresh(40)
            items[at] = bad
            assert check(items) == code
        items = fresh(40)
        items[at] = item(None, None, row=0)                   # nothing to move
        assert check(items) == 0
    assert check(fresh(2), n=-1) == -2 and check(fresh(2), W=0) == -2 and check(fresh(2), B=-1) == -2 and check(fresh(2), B=1 << 30) == -2
    assert check(fresh(2), B=0) == 0 and Bd.lib().q4_beam_reorder_check(None, 3, 2, 4) == -1


def test_a_layer_over_weights_takes_only_what_its_sizes_say(Bd):
    # (on the CPU: nothing is launched)
    def mat(q=None, scale=None, rows=8, k=60, k_pad=64, bits=8):
        return Bd.DeviceMat(torch.zeros(rows, k_pad * bits // 8, dtype=torch.uint8) if q is None else q,
                            torch.ones(rows) if scale is None else scale, rows, k, k_pad, bits)
    for bits in (2, 4, 8):
        assert Bd.DeviceLinear.from_mat(mat(bits=bits), torch.zeros(8)).w.rows == 8
    for good in (mat(q=torch.zeros(8 * 64, dtype=torch.int8)), mat(q=torch.zeros(9, 64, dtype=torch.uint8), scale=torch.ones(8, 1))):
        Bd.DeviceLinear.from_mat(good)
    for bad in (mat(q=torch.zeros(7, 64, dtype=torch.uint8)), mat(q=torch.zeros(8, 60, dtype=torch.uint8)),
                mat(q=torch.zeros(64, 8, dtype=torch.uint8).t()), mat(scale=torch.ones(7)),
                mat(scale=torch.ones(8, dtype=torch.float64)), mat(scale=torch.ones(16)[::2]), mat(scale=torch.ones(8, device="meta"))):
        with pytest.raises(ValueError):
            Bd.DeviceLinear.from_mat(bad)
    for bias in (torch.zeros(7), torch.zeros(8, dtype=torch.float16), torch.zeros(16)[::2], torch.zeros(8, device="meta")):
        with pytest.raises(ValueError):
            Bd.DeviceLinear.from_mat(mat(), bias)
