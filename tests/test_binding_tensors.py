"""The binding's module for lists of tensors, and that a call's host work in Python does not grow with the number of tensors."""
import ctypes
import gc
import sys

import pytest
import torch


@pytest.fixture(scope="module")
def addresses():
    from paper_2509_02447_amd import binding
    return binding._tensor_addresses()


def sizes(*n):
    return (ctypes.c_int64 * len(n))(*n)


def test_lists_without_tensors(addresses):
    assert addresses([None, None], sizes(3, 4), torch.float32) == bytes(16)
    assert addresses((None,), sizes(3), torch.bfloat16) == bytes(8)
    assert addresses([], sizes(), torch.float32) == bytes(8)      # (an array of one address, for C)


@pytest.mark.parametrize("wrong", [[None], [None] * 3, [torch.zeros(3), None], [None, 5], [None, "x"], []], ids=["short", "long", "host", "number", "text", "none"])
def test_refusals(addresses, wrong):
    with pytest.raises(AssertionError):
        addresses(wrong, sizes(3, 4), torch.float32)


def test_arguments_of_other_types(addresses):
    for args in ((5, sizes(3), torch.float32), ([None], 5, torch.float32), ([None], sizes(3), 5), ([None], sizes(3))):
        with pytest.raises(TypeError):
            addresses(*args)


@pytest.mark.gpu
def test_tensors_on_the_gpu(addresses):
    buf = torch.zeros(100, device="cuda")
    good = [buf[8:11], None, torch.nn.Parameter(buf[20:24].view(2, 2)), buf[:0]]
    got = (ctypes.c_uint64 * 4).from_buffer(addresses(good, sizes(3, 9, 4, 0), torch.float32))
    assert list(got) == [buf.data_ptr() + 32, 0, buf.data_ptr() + 80, good[3].data_ptr()]
    for i, bad in ((0, buf[:4]), (0, buf[0:6:2]), (0, buf[:3].bfloat16()), (0, buf[:3].cpu()), (2, buf[:8].view(2, 4)[:, :2]), (2, buf[:4].view(2, 2).to_sparse()), (3, None)):
        row = list(good)
        row[i] = bad
        if bad is None:
            assert (ctypes.c_uint64 * 4).from_buffer(addresses(row, sizes(3, 9, 4, 0), torch.float32))[3] == 0
            continue
        with pytest.raises(AssertionError):
            addresses(row, sizes(3, 9, 4, 0), torch.float32)


@pytest.mark.gpu
def test_the_calls_of_a_step_do_not_grow_with_its_tensors():
    """Python's and C's functions that a norm, a scaling and a step enter: as many for 300 tensors as for 3."""
    import paper_2509_02447_amd as qrm
    ctx = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    norm, scale, stream = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.cuda.current_stream()
    counts = []
    for n in (3, 300):
        zeros = [[torch.zeros(5 + i % 7, device="cuda") for i in range(n)] for _ in range(5)]
        opt = qrm.AdamW(ctx, [dict(param=p, m=m, v=v) for p, m, v in zip(*zeros[:3])], torch.float32)
        seen = []

        def call():
            opt.qrm_adamw_grad_norm(zeros[3], 1.0, norm, scale, None, stream)
            opt.qrm_adamw_scale_grads(zeros[3], scale, zeros[4], stream)
            opt.qrm_adamw_step(zeros[3], 1, 1e-3, d_grad_scale=scale, stream=stream)

        call()
        gc.disable()                                               # (what it collects has calls of its own)
        sys.setprofile(lambda frame, event, arg: seen.append(event) if event in ("call", "c_call") else None)
        try:
            call()
        finally:
            sys.setprofile(None)
            gc.enable()
        counts.append(len(seen))
        torch.cuda.synchronize()
        opt.close()
    ctx.close()
    assert counts[0] == counts[1] and counts[0] > 0, counts
