"""The global gradient norm and clipping on the GPU against the fp64 oracle.  Tolerances: squares of fp32 and bf16 values are
exact in 64 bits, so a sum of n of them is off by at most n 2^-53 of itself; the factor is rounded to fp32 once, the product
once, and the result once more to its type."""
import math

import numpy as np
import pytest
import torch

from oracle import ends_oracle as E
from paper_2111_04007_amd import binding as B
from paper_2111_04007_amd.synth import to_f64

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24


def tensors(sizes, types, seed, leads=(0, 1, 3, 8)):
    """Tensors that begin at different elements of one buffer each, with 32 entries of 1e30 on either side."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        lead = 32 + leads[i % len(leads)]
        flat = torch.full((n + lead + 32,), 1e30, dtype=DT[types[i % len(types)]], device="cuda")
        out.append((flat, flat[lead:lead + n]))
        out[-1][1].copy_(torch.empty(n, device="cuda").normal_(0.0, 2.0 ** (i % 7 - 3), generator=g))
    return [f for f, _ in out], [t for _, t in out]


def norm(ts):
    tl = B.TensorList(ts)
    need = B.grad_norm_scratch_bytes(tl)
    s, bad = torch.full((1,), -1.0, dtype=torch.float64, device="cuda"), torch.full((1,), -1.0, device="cuda")
    scratch = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    B.op_grad_norm(tl, s, bad, scratch[:need])
    torch.cuda.synchronize()
    assert bool((scratch[need:] == 0xFF).all())
    return tl, s, bad


def check_norm(ts, s, bad):
    ref, n_bad = E.grad_norm([to_f64(t) for t in ts])
    n = sum(t.numel() for t in ts)
    assert float(bad) == n_bad and abs(float(s) - ref) <= 2 * n * 2.0 ** -53 * ref, (float(s), ref)
    return ref


def check_clip(before, after, s, max_norm, eps):
    c = E.clip_factor(s, max_norm, eps)
    for a, b in zip(before, after):
        ref = c * to_f64(a)
        err = np.abs(to_f64(b) - ref)
        assert (err <= np.abs(ref) * ((2 * U if c < 1 else 0.0) + HALF[b.dtype] * (b.dtype != torch.float32 or c < 1)) * 1.01 + 1e-44).all()


SIZES = [(), (0,), (1,), (5,), (0, 7, 0), (1, 2, 3, 4, 5, 6, 7, 8, 9), (4097, 33, 128), (8192,), (8193, 8191), (100000, 1, 70001, 65536), (3,) * 500,
         (1_000_003, 20_000), (300_001,) * 60]   # the last: workgroups of the norm that cross from tensor to tensor


@pytest.mark.parametrize("types", [("f32",), ("bf16",), ("f32", "bf16", "bf16")])
@pytest.mark.parametrize("sizes", SIZES, ids=[str(len(s)) + "x" + str(max(s, default=0)) for s in SIZES])
def test_norm_and_clipping(sizes, types):
    flats, ts = tensors(sizes, types, len(sizes))
    tl, s, bad = norm(ts)
    ref = check_norm(ts, s, bad)
    before = [t.clone() for t in ts]
    guards = [f.clone() for f in flats]
    for ratio in (0.25, 2.0):
        most = math.sqrt(ref) * ratio
        for to in ("f32", "bf16"):   # into one buffer, tensor behind tensor
            bucket = torch.full((sum(sizes) + 64,), 1e30, dtype=DT[to], device="cuda")
            into = [bucket[32:-32][a:a + n] for a, n in zip(np.cumsum((0,) + tuple(sizes)), sizes)]
            B.op_grad_clip(B.TensorList(into), tl, s, most)
            check_clip(before, into, float(s), most, 1e-6)
            assert bool((bucket[:32] == bucket[0]).all()) and bool((bucket[-32:] == bucket[0]).all())
    for f, g in zip(flats, guards):
        assert torch.equal(f, g)
    most = math.sqrt(ref) * 0.5
    B.op_grad_clip(tl, tl, s, most, 0.0)   # in place
    check_clip(before, ts, float(s), most, 0.0)
    for f, g, t, b in zip(flats, guards, ts, before):
        t.copy_(b)
        assert torch.equal(f, g)


def test_nothing_is_changed_below_the_limit_or_without_one():
    _, ts = tensors((1000, 37), ("f32", "bf16"), 3)
    tl, s, bad = norm(ts)
    before = [t.clone() for t in ts]
    for most in (float(s) ** 0.5 * 1.5, math.inf):
        B.op_grad_clip(tl, tl, s, most)
        assert all(torch.equal(a, b) for a, b in zip(before, ts))
    s.fill_(math.nan)
    B.op_grad_clip(tl, tl, s, 1e-9)
    assert all(torch.equal(a, b) for a, b in zip(before, ts))
    s.fill_(4.0)
    B.op_grad_clip(tl, tl, s, 0.0)
    assert all(bool((t == 0).all()) for t in ts)


@pytest.mark.parametrize("types", [("f32",), ("bf16",)])
def test_entries_that_are_not_finite_are_counted_and_left_out(types):
    _, ts = tensors((9000, 10, 8192), types, 4)
    for t, i, v in ((ts[0], 0, math.nan), (ts[0], 8999, math.inf), (ts[1], 9, -math.inf), (ts[2], 8191, math.nan), (ts[2], 4096, math.inf)):
        t[i] = v
    tl, s, bad = norm(ts)
    ref = check_norm(ts, s, bad)
    before = [t.clone() for t in ts]
    B.op_grad_clip(tl, tl, s, math.sqrt(ref) / 2, 0.0)
    for a, b in zip(before, ts):
        fine = torch.isfinite(a)
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[torch.isinf(a)], b[torch.isinf(a)])
        check_clip([a[fine]], [b[fine]], float(s), math.sqrt(ref) / 2, 0.0)


def test_squares_beyond_the_range_of_fp32():
    t = torch.tensor([3e30, -4e30, 1e-30, 2e-38], device="cuda")
    _, s, bad = norm([t])
    check_norm([t], s, bad)
    tiny = torch.full((5000,), 1e-30, device="cuda")
    tl, s, bad = norm([tiny])
    check_norm([tiny], s, bad)
    B.op_grad_clip(tl, tl, s, 1e-30, 0.0)
    assert abs(float(tiny.double().norm()) - 1e-30) < 1e-36


def test_a_tensor_counts_as_often_as_it_is_listed():
    _, ts = tensors((777,), ("f32",), 5)
    _, once, _ = norm(ts)
    _, twice, _ = norm(ts * 2)
    assert abs(float(twice) - 2 * float(once)) <= 1e-12 * float(once)


def test_repeats_its_bits_and_orders_on_its_stream():
    _, ts = tensors((300_000, 50_001, 9), ("f32", "bf16"), 6)
    _, s, bad = norm(ts)
    side = torch.cuda.Stream()
    tl = B.TensorList(ts)
    again, bad2 = torch.empty_like(s), torch.empty_like(bad)
    scratch = torch.empty(B.grad_norm_scratch_bytes(tl), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    B.op_grad_norm(tl, again, bad2, scratch, stream=side)
    side.synchronize()
    assert torch.equal(s, again) and torch.equal(bad, bad2)


def test_captured_and_replayed():
    _, ts = tensors((20_000, 50_001, 9) + (40,) * 200, ("f32", "bf16"), 7)
    tl = B.TensorList(ts)
    bucket = torch.empty(sum(t.numel() for t in ts), device="cuda")
    into = B.TensorList(bucket.split([t.numel() for t in ts]))
    s, bad = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    scratch = torch.empty(B.grad_norm_scratch_bytes(tl), dtype=torch.uint8, device="cuda")

    def step():
        B.op_grad_norm(tl, s, bad, scratch)
        B.op_grad_clip(into, tl, s, 3.0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        for t in ts:
            t.mul_(-1.25)
        if k == 2:
            ts[0][5] = math.inf
        graph.replay()
        torch.cuda.synchronize()
        got = (s.clone(), bad.clone(), bucket.clone())
        bucket.fill_(9.0)
        s.fill_(9.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], s) and torch.equal(got[1], bad) and torch.equal(got[2], bucket) and float(bad) == (k >= 2)


def test_a_tensor_beyond_32_bits_of_offset():
    n = (1 << 32) + 77
    t = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    t[-1], t[-2] = 3.0, math.nan
    tl, s, bad = norm([t])
    assert float(bad) == 1.0 and float(s) == 0.25 * (n - 2) + 9.0   # all of it is exact
    B.op_grad_clip(tl, tl, s, math.sqrt(float(s)) / 2, 0.0)
    assert float(t[-1]) == 1.5 and bool(torch.isnan(t[-2])) and bool((t[:-2] == 0.25).all())


def test_workgroups_of_the_clipping_that_cross_from_tensor_to_tensor():
    sizes = (300_000_000, 7, 250_000_001, 3)   # more chunks than workgroups
    ts = [torch.full((n,), 2.0 ** -i, dtype=torch.bfloat16, device="cuda") for i, n in enumerate(sizes)]
    tl, s, bad = norm(ts)
    assert float(bad) == 0.0 and float(s) == sum(n * 4.0 ** -i for i, n in enumerate(sizes))
    B.op_grad_clip(tl, tl, s, math.sqrt(float(s)) / 2, 0.0)
    for i, t in enumerate(ts):
        assert bool((t == 2.0 ** -i / 2).all())


def test_calls_side_by_side_on_two_streams():
    """Each with a scratch of its own."""
    made = [tensors((200_000 + 7 * k, 50_001, 9), ("f32", "bf16"), 8 + k)[1] for k in range(2)]
    want = [norm(ts)[1] for ts in made]
    streams, out = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for ts in made:
        tl = B.TensorList(ts)
        bucket = torch.empty(sum(tl.sizes), device="cuda")
        out.append((tl, B.TensorList(bucket.split(list(tl.sizes))), torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda"),
                    torch.empty(B.grad_norm_scratch_bytes(tl), dtype=torch.uint8, device="cuda"), bucket))
    torch.cuda.synchronize()
    for _ in range(5):
        for st, (tl, into, s, bad, scratch, _) in zip(streams, out):
            B.op_grad_norm(tl, s, bad, scratch, stream=st)
            B.op_grad_clip(into, tl, s, 1.0, stream=st)
    torch.cuda.synchronize()
    for ts, w, (tl, into, s, bad, _, bucket) in zip(made, want, out):
        assert torch.equal(s, w) and float(bad) == 0.0
        check_clip(ts, into.tensors, float(s), 1.0, 1e-6)
