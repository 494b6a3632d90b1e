"""qnn_cache4_append doesn't read the rows of a token that has no slot (below 0,
or past the last page): k and v may end at the last token that has one, as with
slots padded to a capacity. Shown on the gfx950 assembly, since a read out of
range need not show in the results; and such a call on the GPU."""
import re

import numpy as np
import pytest

import lds_hazards as H
import test_lds_async_reads as A


def _early(lines):
    """Loads of values (two words or more) that no wait for an earlier load of one
    word, the slot, comes before."""
    slot, known, early = False, False, []
    for line in lines:
        op = line.split()[0] if line.split() else ""
        if op == "global_load_dword":
            slot, known = True, False
        elif op == "s_waitcnt" and "vmcnt(0)" in line:
            known = slot
        elif re.match(r"global_load_dwordx[234]", op) and not known:
            early.append(line.strip())
    return early


def test_the_check_itself():
    slot, value, wait = "global_load_dword v8, v[2:3], off", "global_load_dwordx4 v[4:7], v[2:3], off", "s_waitcnt vmcnt(0)"
    assert _early([slot, value, wait]) == [value]
    assert _early([value]) == [value]
    assert _early([slot, wait, "s_and_saveexec_b64 s[0:1], vcc", value]) == []


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    keep = A._SOURCES, dict(A._ASM)
    A._SOURCES = ["cache4.hip"]
    A._ASM.clear()
    try:
        ks = H.kernels(A._asm("cache4.hip", tmp_path_factory))
    finally:
        A._SOURCES = keep[0]
        A._ASM.clear()
        A._ASM.update(keep[1])
    return {k: [text for _, text in v] for k, v in ks.items() if "append_kernel" in k}


@A.needs_hipcc
def test_values_are_loaded_after_their_slot(kernels):
    assert len(kernels) == 12   # three head dimensions, four types
    for name, lines in kernels.items():
        assert any("global_load_dwordx" in v for v in lines), name
        assert _early(lines) == [], name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "i8"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_rows_end_at_the_last_token_with_a_slot(dtype, D):
    import torch

    import cache4_ref as R
    from paper_2006_10226_amd import qnn as Q
    T, rows, Hk, P = 40, 21, 2, 16
    rng = np.random.default_rng(D)
    x = rng.integers(-100, 100, (2, rows, Hk, D))
    k, v = torch.from_numpy(x).to(torch.int8 if dtype == "i8" else torch.float16).cuda().unbind(0)
    slots = np.full(T, -1)
    slots[:rows] = rng.permutation(3 * P)[:rows]
    slots[rows + 1], slots[rows + 2] = 3 * P, 2**31 - 1
    st = torch.from_numpy(slots.astype(np.int32)).cuda()
    whole, short = (Q.Cache4(3, P, Hk, D, data=torch.zeros(3, R.page_bytes(P, Hk, D), dtype=torch.uint8, device="cuda"))
                    for _ in range(2))
    Q.cache4_append(whole, k, v, st[:rows].contiguous(), 0.5, 0, 0.25, 0)
    q = [Q._one_q(s, 0) for s in (0.5, 0.25)]
    Q._check(Q.lib().qnn_cache4_append(Q._stream_handle(), short.desc, k.data_ptr(), v.data_ptr(),
                                       Q.INT8 if dtype == "i8" else Q.FLOAT16, *q, T, Hk * D, Hk * D, st.data_ptr()))
    torch.cuda.synchronize()
    assert torch.equal(whole.data, short.data)
