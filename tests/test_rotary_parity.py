"""Rotary positions against the fp64 oracle, entry by entry.  Tolerance: a cosine or sine is off by half a step of fp32 (2^-24 of itself; the angle in 64
bits adds p f 2^-53, under 2^-30 here), two products and their sum by one step in all each, so 4 * 2^-24 (|a c| + |b s|) + 2^-30 (|a| + |b|), and half a
step of the type for the result."""
import math

import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2111_04007_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def table_of(n, f, magnitude=1.0):
    table = torch.empty((n, 2 * len(f)), device="cuda")
    B.op_rotary_table(table, f, magnitude)
    return table


def expect(got, x, positions, f, n, interleaved=False, transpose=False, magnitude=1.0):
    """got, x: tensors [rows, heads, d]."""
    f = np.array(f)
    x64 = x.detach().cpu().double().numpy()
    want = L.rotary(x64, positions, f, n, interleaved, transpose, magnitude)
    r = 2 * len(f)
    size = np.abs(x64)
    partner = np.zeros_like(size)
    if interleaved:
        partner[..., 0:r:2], partner[..., 1:r:2] = size[..., 1:r:2], size[..., 0:r:2]
    else:
        partner[..., :r // 2], partner[..., r // 2:r] = size[..., r // 2:r], size[..., :r // 2]
    ang = np.zeros((x64.shape[0], x64.shape[2]))
    p = np.array([k if 0 <= k < n else 0 for k in positions], dtype=np.float64)
    each = p[:, None] * f
    if interleaved:
        ang[:, 0:r:2] = ang[:, 1:r:2] = each
    else:
        ang[:, :r // 2] = ang[:, r // 2:r] = each
    c, s = np.abs(np.cos(ang))[:, None] * magnitude, np.abs(np.sin(ang))[:, None] * magnitude
    c[..., r:], s[..., r:] = 0.0, 0.0
    tol = 4 * 2.0 ** -24 * (size * c + partner * s) + 2.0 ** -30 * magnitude * (size + partner) + torch.finfo(x.dtype).eps / 2 * np.abs(want)
    still = np.array([not 0 <= k < n for k in positions])
    tol[still] = 0.0
    tol[..., r:] = 0.0
    off = np.abs(got.detach().cpu().double().numpy() - want)
    assert (off <= tol).all(), (off - tol).max()


def positions_of(r, rows, n, index):
    p = r.integers(0, n, rows)
    p[r.random(rows) < 0.15] = -1
    if rows > 3:
        p[1], p[2] = n, n + 5          # beyond the table
    return p, torch.from_numpy(p).to(index).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,d,r,interleaved,transpose", [
    (1, 1, 2, 2, False, False), (1, 1, 2, 2, True, True), (3, 2, 64, 64, False, False), (17, 5, 128, 128, False, True), (65, 3, 128, 128, True, False),
    (33, 9, 80, 32, False, False), (33, 9, 80, 32, True, True), (7, 1, 96, 96, False, True), (5, 40, 96, 48, True, False), (129, 2, 22, 22, False, False),
    (9, 7, 33, 10, True, True), (2, 3, 512, 512, False, False), (4, 17, 72, 6, False, True), (11, 4, 31, 30, True, False),
])
def test_heads_of_packed_rows(dtype, rows, heads, d, r, interleaved, transpose):
    g = np.random.default_rng(rows * 1000 + d)
    n = 300
    f = B.rotary_frequencies(r)
    p, positions = positions_of(g, rows, n, torch.int64 if rows % 2 else torch.int32)
    packed = torch.from_numpy(g.standard_normal((rows, heads + 2, d))).to(DT[dtype]).cuda()
    before = packed.clone()
    table = table_of(n, f)
    x = packed[:, 1:heads + 1]
    out = torch.full((rows, heads, d), 7.0, dtype=DT[dtype], device="cuda")
    B.op_rotary(x, table, out=out, positions=positions, interleaved=interleaved, transpose=transpose)
    assert torch.equal(packed, before)
    expect(out, x, p, f, n, interleaved, transpose)
    B.op_rotary(x, table, positions=positions, interleaved=interleaved, transpose=transpose)   # in place
    assert torch.equal(x, out)
    assert torch.equal(packed[:, 0], before[:, 0]) and torch.equal(packed[:, -1], before[:, -1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_run_and_strides(dtype):
    """Positions NULL; [heads, rows, d] and every second head of a wider tensor, beginning at an odd element."""
    g = np.random.default_rng(5)
    b, s, a, d = 3, 21, 4, 48
    f = B.rotary_frequencies(d, 500.0)
    table = table_of(64, f)
    flat = torch.from_numpy(g.standard_normal(1 + 2 * a * b * s * d)).to(DT[dtype]).cuda()
    wide = flat[1:].view(2 * a, b * s, d)
    x = wide[::2].transpose(0, 1)
    before, old = x.clone(), wide.clone()
    run = [t % s for t in range(b * s)]
    out = torch.empty((a, b * s, d), dtype=DT[dtype], device="cuda").transpose(0, 1)
    B.op_rotary(x, table, out=out, seq_len=s)
    expect(out, before, run, f, 64)
    B.op_rotary(x, table, seq_len=s)
    assert torch.equal(x, out) and torch.equal(wide[1::2], old[1::2])
    B.op_rotary(x, table, seq_len=s, transpose=True)   # and back, one more rounding each way
    off = (x.double() - before.double()).abs()
    assert float(off.max()) <= 4 * torch.finfo(DT[dtype]).eps * float(before.abs().max())
    y = before.clone()
    B.op_rotary(y, table)   # all of the table's 64 positions
    expect(y, before, list(range(63)), f, 64)


@pytest.mark.parametrize("scaling,factor,original", [("none", 1.0, 0), ("linear", 4.0, 0), ("base", 8.0, 0), ("parts", 8.0, 4096)])
def test_scaled_frequencies_and_far_positions(scaling, factor, original):
    """Frequencies from their formulas; the table at positions up to 131071 within half a step of fp32 and what the angle in 64 bits is off."""
    r, base = 64, 10000.0
    f = B.rotary_frequencies(r, base, scaling, factor, original)
    i = np.arange(r // 2)
    plain = base ** (-2.0 * i / r)
    if scaling == "none":
        want = plain
    elif scaling == "linear":
        want = plain / factor
    elif scaling == "base":
        want = (base * factor ** (r / (r - 2))) ** (-2.0 * i / r)
        assert want[0] == 1.0 and abs(want[-1] * factor / plain[-1] - 1) < 1e-12
    else:
        turns = original * plain / (2 * math.pi)
        want = np.where(turns >= 4, plain, np.where(turns <= 1, plain / factor, (turns - 1) / 3 * plain + (4 - turns) / 3 * plain / factor))
        assert (want == plain).any() and (want == plain / factor).any()
    np.testing.assert_allclose(np.array(f), want, rtol=1e-13)
    n = 131072
    table = table_of(n, f, 1.25).cpu().double().numpy()
    at = np.concatenate([np.arange(100), np.random.default_rng(1).integers(0, n, 500), [n - 1]])
    ang = at[:, None] * np.array(f)
    for got, of in ((table[at, :r // 2], np.cos(ang)), (table[at, r // 2:], np.sin(ang))):
        assert (np.abs(got - 1.25 * of) <= 2.0 ** -24 * 1.25 * np.abs(of) + 1.25 * (2.0 ** -52 * np.abs(ang) + 2.0 ** -51)).all()


def test_magnitude_and_one_frequency():
    f = [0.25]
    table = table_of(10, f, 1.5)
    x = torch.randn(4, 2, 6, device="cuda")
    y = x.clone()
    p = torch.tensor([0, 9, 3, 10], dtype=torch.int32, device="cuda")
    B.op_rotary(y, table, positions=p)
    expect(y, x, p.tolist(), f, 10, magnitude=1.5)


def test_rows_without_a_position_keep_their_bits():
    f = B.rotary_frequencies(16)
    table = table_of(8, f)
    x = torch.randn(6, 3, 20, device="cuda")
    x[1, 0, 3], x[1, 1, 8], x[4, 2, 0] = float("nan"), float("inf"), -0.0
    p = torch.tensor([0, -1, 7, 8, -1, 2 ** 40], dtype=torch.int64, device="cuda")
    out = torch.empty_like(x)
    B.op_rotary(x, table, out=out, positions=p)
    for t in (1, 3, 4, 5):
        assert torch.equal(out[t].view(torch.int32), x[t].view(torch.int32))
    y = x.clone()
    B.op_rotary(y, table, positions=p)
    assert torch.equal(y.view(torch.int32), out.view(torch.int32))


def test_nothing_to_turn():
    table = table_of(4, B.rotary_frequencies(8))
    for shape in ((0, 3, 8), (3, 0, 8)):
        B.op_rotary(torch.empty(shape, device="cuda"), table)
    with pytest.raises(B.VarunaError):   # rows, and no positions that they could have
        B.op_rotary(torch.randn(3, 2, 8, device="cuda"), torch.empty((0, 8), device="cuda"), positions=torch.zeros(3, dtype=torch.int32, device="cuda"))


def test_more_than_32_bits_of_offset():
    """Rows that lie 2^30 elements apart: the last begins 2^32 bytes and more behind the first."""
    far = 1 << 30
    flat = torch.zeros(3 * far + 256, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((4, 2, 64), (far, 128, 1))
    value = torch.randn(4, 2, 64, device="cuda").bfloat16()
    x.copy_(value)
    f = B.rotary_frequencies(64)
    B.op_rotary(x, table_of(100, f), positions=torch.tensor([5, 99, 1, 42], device="cuda"))
    expect(x, value, [5, 99, 1, 42], f, 100)
    assert not bool(flat[200:1000].any())


def test_other_stream_and_replayed_graph():
    f = B.rotary_frequencies(32)
    table = table_of(50, f)
    x = torch.randn(40, 6, 32, device="cuda").bfloat16()
    p = torch.randint(0, 50, (40,), device="cuda")
    want, out = torch.empty_like(x), torch.empty_like(x)
    B.op_rotary(x, table, out=want, positions=p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.op_rotary(x, table, out=out, positions=p)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    made = torch.empty_like(table)
    with torch.cuda.graph(graph):
        B.op_rotary_table(made, f)
        B.op_rotary(x, made, out=out, positions=p)
    for k in range(3):
        x.normal_()
        p.random_(0, 50)
        made.zero_()
        B.op_rotary(x, table, out=want, positions=p)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d,r", [("bf16", 128, 128), ("f32", 80, 32), ("bf16", 66, 22)])
def test_rows_beyond_the_caches(dtype, d, r, interleaved):
    """200 MB and more of turned entries, in place, and as much of both tensors out of place: bit for bit what calls of a few rows give."""
    size = torch.finfo(DT[dtype]).bits // 8
    heads = 40
    f = B.rotary_frequencies(r)
    table = table_of(50, f)
    x = torch.randn(100, heads, d, device="cuda").to(DT[dtype])
    want = x.clone()
    B.op_rotary(want, table, seq_len=50, interleaved=interleaved)
    expect(want[:60], x[:60], [t % 50 for t in range(60)], f, 50, interleaved)
    times = -(-(210 << 20) // (100 * heads * r * size))
    many = x.repeat(times, 1, 1)
    B.op_rotary(many, table, seq_len=50, interleaved=interleaved)
    assert torch.equal(many.view(times, -1), want.view(1, -1).expand(times, -1))
    many = x.repeat(times, 1, 1)
    out = torch.empty_like(many)
    B.op_rotary(many, table, out=out, seq_len=50, interleaved=interleaved)
    assert torch.equal(out.view(times, -1), want.view(1, -1).expand(times, -1)) and torch.equal(many[-100:], x)
