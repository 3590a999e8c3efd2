"""A TensorList whose tensors get other memory between two calls: what reaches the library is where they are now.  The first tests
need no GPU: they look at the addresses, sizes and types that the library would be given."""
import ctypes as C

import pytest
import torch

from paper_2111_04007_amd import binding as B

KINDS = {
    "data": lambda t: setattr(t, "data", torch.full_like(t, 3.0)),
    "data of another size": lambda t: setattr(t, "data", torch.full((t.numel() + 100,), 3.0, dtype=t.dtype, device=t.device)),
    "data of another type": lambda t: setattr(t, "data", torch.full(t.shape, 3.0, dtype=torch.bfloat16, device=t.device)),
    "set_": lambda t: t.set_(torch.full((t.numel() + 1,), 3.0, dtype=t.dtype, device=t.device)[1:]),
    "more": lambda t: t.resize_(100_000).fill_(3.0),
    "fewer": lambda t: t.resize_(7),
    "storage": lambda t: t.untyped_storage().resize_(1 << 22),
    "a part of a common buffer": lambda t: setattr(t, "data", torch.full((3 * t.numel(),), 3.0, dtype=t.dtype, device=t.device)[t.numel():2 * t.numel()]),
}


@pytest.fixture
def given(monkeypatch):
    """Calls reach this list in place of the library, from tensors on the CPU too."""
    got = []

    def dense(device, *tensors):
        if any(t is not None and not t.is_contiguous() for t in tensors):
            raise ValueError
    monkeypatch.setattr(B, "_dense", dense)
    monkeypatch.setattr(B, "_run", lambda device, stream, fn, *args: got.append(args))
    return got


def same(n, dtypes, ptrs, counts, tensors):
    assert n == len(tensors)
    assert list((C.c_int32 * n).from_buffer(dtypes)) == [B.dtype_code(t) for t in tensors]
    assert [p or 0 for p in (C.c_void_p * n).from_buffer(ptrs)] == [t.data_ptr() for t in tensors]
    assert list((C.c_int64 * n).from_buffer(counts)) == [t.numel() for t in tensors]


@pytest.mark.parametrize("kind", KINDS)
def test_calls_are_given_where_tensors_are_now(given, kind):
    ts = [torch.nn.Parameter(torch.ones(1000), requires_grad=False), torch.ones(50), torch.ones(64, dtype=torch.bfloat16)]
    tl = B.TensorList(ts)
    s, bad, scratch = torch.empty(1, dtype=torch.float64), torch.empty(1), torch.empty(B.grad_norm_scratch_bytes(tl), dtype=torch.uint8)
    for k in (1, 0):
        with torch.no_grad():
            KINDS[kind](ts[k])
        B.op_grad_norm(tl, s, bad, scratch)
        same(*given[-1][:4], ts)
        B.op_grad_clip(tl, tl, s, 1.0)
        n, dt, dp, st, sp, c = given[-1][:6]
        same(n, dt, dp, c, ts)
        same(n, st, sp, c, ts)
        assert tl.sizes == tuple(t.numel() for t in ts)


def test_memory_that_was_left_is_nobody_elses(given):
    """Of the same size and at the same address, another type would not be told apart."""
    t = torch.ones(1 << 20)
    tl = B.TensorList([t])
    was = t.data_ptr()
    for _ in range(4):
        t.data = torch.ones(1 << 20, dtype=torch.bfloat16)
        assert t.data_ptr() != was
        t.data = torch.ones(1 << 20)
    B.op_grad_norm(tl, torch.empty(1, dtype=torch.float64), torch.empty(1), torch.empty(B.grad_norm_scratch_bytes(tl), dtype=torch.uint8))
    same(*given[-1][:4], [t])


def test_sizes_that_no_longer_fit_and_strides_are_refused(given):
    a, b = torch.ones(6, 4), torch.ones(24)
    src, dst = B.TensorList([a]), B.TensorList([b])
    s = torch.empty(1, dtype=torch.float64)
    B.op_grad_clip(dst, src, s, 1.0)
    a.data = torch.ones(5, 4)
    with pytest.raises(ValueError):
        B.op_grad_clip(dst, src, s, 1.0)
    a.data = torch.ones(4, 6).t()
    for _ in range(2):   # and again: nothing of it is kept
        with pytest.raises(ValueError):
            B.op_grad_clip(dst, src, s, 1.0)
    a.data = torch.ones(6, 4)
    B.op_grad_clip(dst, src, s, 1.0)
    same(1, given[-1][3], given[-1][4], given[-1][5], [a])
    assert len(given) == 2


def test_a_tensor_more(given):
    src = B.TensorList([torch.ones(4)])
    src.tensors.append(torch.ones(5))
    B.op_grad_norm(src, torch.empty(1, dtype=torch.float64), torch.empty(1), torch.empty(1 << 16, dtype=torch.uint8))
    same(*given[-1][:4], src.tensors)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_norm_and_clipping_of_tensors_that_moved(kind):
    ts = [torch.ones(1000, device="cuda"), torch.ones(64, dtype=torch.bfloat16, device="cuda")]
    tl = B.TensorList(ts)
    s, bad = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    scratch = torch.empty(B.grad_norm_scratch_bytes(tl), dtype=torch.uint8, device="cuda")
    before = ts[0].detach()   # what it leaves
    KINDS[kind](ts[0])
    if kind == "storage":
        ts[0].fill_(3.0)
    here = ts[0].untyped_storage().data_ptr() == before.untyped_storage().data_ptr()
    B.op_grad_norm(tl, s, bad, scratch)
    want = sum(float(t.double().square().sum()) for t in ts)
    assert float(s) == want and float(bad) == 0.0   # whole numbers
    B.op_grad_clip(tl, tl, s, want ** 0.5 / 2, 0.0)
    value = 0.5 if kind == "fewer" else 1.5
    assert bool((ts[0] == value).all()) and bool((ts[1] == 0.5).all())
    assert here or bool((before == 1.0).all())
