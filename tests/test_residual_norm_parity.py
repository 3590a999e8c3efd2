"""Residual norms, forward and backward, against the fp64 oracle, entry by entry.  Tolerances count roundings: with e = 2^-24, a sum of h products over
a row is a chain of at most 64 sums in a thread or over waves and 6 over a wave's lanes, counted as 72 e of the sum of the absolute values; a
product, sum or conversion is e of its result, a value stored in the type half its step.  A column's sum over rows is at worst (rows + 20) e of the sum of
the absolute values.  An error of an intermediate goes on by the formula's own derivatives (the `off_` variables)."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2111_04007_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
e = 2.0 ** -24


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def half(dtype):
    return torch.finfo(DT[dtype]).eps / 2


def close(what, got, want, tol):
    got = f64(got).reshape(want.shape)
    off = np.abs(got - want)
    assert np.isfinite(got).all() and (off <= tol).all(), (what, float((off - tol).max()), float(off.max()))


class Case:
    def __init__(self, dtype, kind, rows, h, post, gate, branch=True, pre=True, bias=True, alpha=0.9, beta=1.1, seed=0, shift=0):
        g = np.random.default_rng(seed + rows * 31 + h)
        self.kind, self.dtype, self.rows, self.h, self.alpha, self.beta, self.rpg = kind, dtype, rows, h, alpha, beta, gate
        def new(shape, std=1.0, mean=0.0):   # noqa: E306  (shift: tensors that begin at an odd element)
            n = int(np.prod(shape))
            flat = torch.zeros(n + shift, dtype=DT[dtype], device="cuda")
            flat[shift:] = torch.from_numpy(mean + std * g.standard_normal(n)).to(DT[dtype]).cuda()
            return flat[shift:].view(shape)
        self.new = new
        self.x = new((rows, h), 2.0, 0.3)
        self.branch = new((rows, h), 0.7, -0.1) if branch else None
        self.gate = new((-(-rows // gate), h), 0.3, 0.6) if gate else None
        self.weight = new((h,), 0.1, 1.0) if pre else None
        self.bias = new((h,), 0.2) if pre and bias else None
        self.post_weight = new((h,), 0.1, 0.5) if post else None
        self.post_bias = new((h,), 0.2) if post and bias else None
        like = lambda: new((rows, h))  # noqa: E731
        self.y = like() if branch else None
        self.z = like() if pre else None
        stat = lambda there: torch.full((2, rows), 9.0, device="cuda") if there else None  # noqa: E731
        self.stats, self.post_stats = stat(pre), stat(post)
        self.eps = 1e-5

    def forward(self, **kw):
        B.op_residual_norm_fwd(self.x, self.z, self.weight, self.bias, branch=self.branch, y=kw.get("y", self.y), post_weight=self.post_weight,
                               post_bias=self.post_bias, gate=self.gate, rows_per_gate=self.rpg, alpha=self.alpha, beta=self.beta, kind=self.kind,
                               eps=self.eps, stats=self.stats, post_stats=self.post_stats)

    def check_statistics(self, got, x):
        want = L.statistics(x, self.kind, self.eps)
        got = f64(got)
        mean_off = 73 * e * np.abs(x).mean(1) if self.kind == "layer" else 0.0
        # a mean that is off by m adds m^2 to the variance, which counts in rows that hardly vary (one entry, say)
        assert (np.abs(got[0] - want[0]) <= mean_off).all()
        assert (np.abs(got[1] / want[1] - 1) <= 40 * e + 0.5 * np.square(mean_off) * want[1] ** 2 + 2 * e * np.abs(x).max(1) * want[1] / x.shape[1] ** 0.5).all()

    def check_normed(self, what, got, x, weight, bias):
        """got: rounded N(x) of exact x."""
        s = L.statistics(x, self.kind, self.eps)
        w, b = f64(weight), 0.0 if bias is None else f64(bias)
        want = L.normed(x, s, w, None if bias is None else b)
        close(what, got, want, self.off_normed(x, s, w, b, want) + half(self.dtype) * np.abs(want))

    def off_normed(self, x, s, w, b, want):
        rstd = s[1][:, None]
        mean_off = 73 * e * np.abs(x).mean(1, keepdims=True) + 2 * e * np.abs(x) if self.kind == "layer" else 0.0
        return np.abs(w) * rstd * mean_off + (45 * e + 0.5 * np.square(np.max(mean_off) * rstd)) * np.abs(want - b) + 2 * e * (np.abs(want) + np.abs(b))

    def check_forward(self):
        x = f64(self.x)
        y = x
        if self.branch is not None:
            u = f64(self.branch)
            off_u = np.zeros_like(u)
            if self.post_weight is not None:
                self.check_statistics(self.post_stats, u)
                s = L.statistics(u, self.kind, self.eps)
                w, b = f64(self.post_weight), 0.0 if self.post_bias is None else f64(self.post_bias)
                n = L.normed(u, s, w) + b
                off_u = self.off_normed(u, s, w, b, n)
                u = n
            by = self.beta * L.gates(f64(self.gate), self.rows, self.rpg)
            want = self.alpha * x + by * u
            close("y", self.y, want, 3 * e * np.abs(self.alpha * x) + 5 * e * np.abs(by * u) + np.abs(by) * off_u + (half(self.dtype) + e) * np.abs(want))
            y = f64(self.y)
        if self.weight is not None:   # of y as it is stored
            self.check_statistics(self.stats, y)
            self.check_normed("z", self.z, y, self.weight, self.bias)

    def backward(self, dz, dy, accumulate, dx=None, dbranch=None, scratch=None, skip=()):
        h, rows = self.h, self.rows
        self.sums = {}
        for name, there, size in (("dweight", self.weight is not None, h), ("dbias", self.bias is not None, h), ("dpost_weight", self.post_weight is not None, h),
                                  ("dpost_bias", self.post_bias is not None, h), ("dgate", self.gate is not None, -(-rows // max(1, self.rpg)) * h)):
            if there and name not in skip:
                self.sums[name] = torch.arange(size, device="cuda", dtype=torch.float32) % 7 if accumulate else torch.full((size,), float("nan"), device="cuda")
        if self.gate is not None and "dgate" in self.sums:
            self.sums["dgate"] = self.sums["dgate"].view(self.gate.shape)
        self.dx = self.new((rows, h)) if dx is None else dx
        self.dbranch = None if self.branch is None else self.new((rows, h)) if dbranch is None else dbranch
        if scratch is None:
            scratch = torch.full((max(1, B.residual_norm_bwd_scratch_bytes(rows, h, self.rpg)),), 255, dtype=torch.uint8, device="cuda")
        reads = self.post_weight is not None or self.gate is not None
        B.op_residual_norm_bwd(dz, None if self.weight is None else (self.x if self.y is None else self.y), self.stats, self.weight, self.dx, scratch, dy=dy,
                               branch=self.branch if reads else None, dbranch=self.dbranch, post_weight=self.post_weight, post_bias=self.post_bias,
                               post_stats=self.post_stats, gate=self.gate, rows_per_gate=self.rpg, alpha=self.alpha, beta=self.beta, kind=self.kind,
                               accumulate=accumulate, **self.sums)

    def check_backward(self, dz, dy, accumulate, y=None, branch=None):
        rows, h, kind = self.rows, self.h, self.kind
        dz, y = f64(dz), f64((self.x if self.y is None else self.y) if y is None else y)
        branch = f64(self.branch if branch is None else branch)
        stats, post_stats = f64(self.stats), f64(self.post_stats)
        d, off_d = (np.zeros((rows, h)) if dy is None else f64(dy)), 0.0
        old = np.arange(h) % 7 if accumulate else np.zeros(h)

        def sums(name, values, off):   # of a column
            want, size = values.sum(0), np.abs(values).sum(0)
            if name in self.sums:
                close(name, self.sums[name], want + old, off.sum(0) + (rows + 20) * e * size + 2 * e * np.abs(want + old))

        def back(g, off_g, x, s):
            """(gradient through the statistics, what it may be off) of g, itself off by off_g."""
            hat, rstd = (x - s[0][:, None]) * s[1][:, None], s[1][:, None]
            mean = lambda v: v.mean(1, keepdims=True)  # noqa: E731
            k0, k1 = mean(g * hat), mean(g) if kind == "layer" else np.zeros((rows, 1))
            off_k0 = mean(np.abs(hat) * off_g) + 77 * e * mean(np.abs(g * hat))
            off_k1 = (mean(off_g) + 74 * e * mean(np.abs(g))) if kind == "layer" else 0.0
            size = rstd * (np.abs(g) + np.abs(k1) + np.abs(hat * k0))
            return L.norm_back(g, x, s, kind), rstd * (off_g + off_k1 + np.abs(hat) * off_k0) + 8 * e * size, hat

        if self.weight is not None:
            w = f64(self.weight)
            n, off_n, hat = back(dz * w, e * np.abs(dz * w), y, stats)
            sums("dweight", dz * hat, 4 * e * np.abs(dz * hat))
            sums("dbias", dz, np.zeros_like(dz))
            size = np.abs(d) + np.abs(n)
            d, off_d = d + n, off_n + 2 * e * size
        off_d = off_d + np.zeros_like(d)
        want = self.alpha * d
        close("dx", self.dx, want, abs(self.alpha) * off_d + (half(self.dtype) + 3 * e) * np.abs(want))
        if self.branch is None:
            return
        du, off = self.beta * d, abs(self.beta) * off_d + 2 * e * np.abs(self.beta * d)
        if self.post_weight is not None:
            pw, pb = f64(self.post_weight), 0.0 if self.post_bias is None else f64(self.post_bias)
            hat = (branch - post_stats[0][:, None]) * post_stats[1][:, None]
            u = hat * pw + pb
            off_u = 5 * e * (np.abs(hat * pw) + np.abs(pb))
        else:
            u = branch
            off_u = np.zeros_like(d)
        if self.gate is not None:
            if "dgate" in self.sums:
                at = np.arange(rows) // self.rpg
                add = lambda v: np.stack([np.bincount(at, v[:, j], len(self.gate)) for j in range(h)], 1)  # noqa: E731
                old_gate = (np.arange(len(self.gate) * h) % 7 if accumulate else np.zeros(len(self.gate) * h)).reshape(-1, h)
                size = add(np.abs(du * u))
                w = add(du * u) + old_gate
                close("dgate", self.sums["dgate"], w, add(np.abs(u) * off + np.abs(du) * off_u) + (min(rows, self.rpg) + 22) * e * size + 2 * e * np.abs(w))
            g = L.gates(f64(self.gate), rows, self.rpg)
            du, off = du * g, off * np.abs(g) + e * np.abs(du * g)
        if self.post_weight is not None:
            sums("dpost_weight", du * hat, np.abs(hat) * off + 4 * e * np.abs(du * hat))
            sums("dpost_bias", du, off)
            du, off, _ = back(du * pw, np.abs(pw) * off + e * np.abs(du * pw), branch, post_stats)
        close("dbranch", self.dbranch, du, off + (half(self.dtype) + 2 * e) * np.abs(du))


WIDTHS = [(1, 1), (3, 7), (5, 64), (9, 333), (4, 512), (3, 520), (7, 1000), (2, 1024), (33, 1030), (5, 1920), (2, 2049), (3, 4096), (2, 5001), (2, 8192), (1, 8200), (2, 16384)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,h", WIDTHS)
def test_widths(dtype, kind, rows, h):
    c = Case(dtype, kind, rows, h, True, 2 if rows > 2 else rows)
    c.forward()
    c.check_forward()
    dz, dy = c.new((rows, h)), c.new((rows, h))
    c.backward(dz, dy, True)
    c.check_backward(dz, dy, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("rows,gate", [(23, 4), (23, 20), (300, 1), (5, 0)])
@pytest.mark.parametrize("h", [4104, 8200])
def test_wide_rows_with_gates(dtype, kind, post, rows, gate, h):
    """Several pieces a thread, whose sums lie in shared memory; the last gate's rows fewer than the others', more than one gate a workgroup."""
    c = Case(dtype, kind, rows, h, post, gate, bias=kind == "layer")
    c.forward()
    c.check_forward()
    dz, dy = c.new((rows, h)), c.new((rows, h))
    c.backward(dz, dy, True)
    c.check_backward(dz, dy, True)


FORMS = [dict(post=p, gate=g, bias=b) for p in (False, True) for g in (0, 1, 5, 40) for b in (False, True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(f"{k}{int(v)}" for k, v in f.items()))
@pytest.mark.parametrize("h", [72, 1100])
def test_forms(dtype, kind, form, h):
    """Post norm or none; a gate for each row, for 5 rows, for 40 of 83 rows; biases or none; begins at an odd element."""
    c = Case(dtype, kind, 83, h, shift=1, **form)
    c.forward()
    c.check_forward()
    dz, dy = c.new((83, h)), c.new((83, h))
    for accumulate in (False, True):
        c.backward(dz, dy, accumulate)
        c.check_backward(dz, dy, accumulate)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_that_are_missing(dtype):
    """No branch; no norm behind; no gradient from behind; sums that are not wanted; y not wanted."""
    c = Case(dtype, "rms", 21, 200, False, 0, branch=False, alpha=1.0)
    c.forward()
    c.check_forward()
    dz, dy = c.new((21, 200)), c.new((21, 200))
    c.backward(dz, dy, False)
    c.check_backward(dz, dy, False)
    c = Case(dtype, "layer", 21, 200, True, 4, pre=False)
    c.forward()
    c.check_forward()
    c.backward(None, dy, True)
    c.check_backward(None, dy, True)
    c = Case(dtype, "layer", 21, 200, False, 0, pre=False)
    c.forward()
    c.check_forward()
    c.backward(None, dy, True)
    c.check_backward(None, dy, True)
    c = Case(dtype, "layer", 21, 1500, True, 7)
    c.forward()
    first = c.z.clone()
    c.z.zero_()
    c.forward(y=None)
    assert torch.equal(c.z, first)
    dz = c.new((21, 1500))
    c.backward(dz, None, False, skip=("dbias", "dpost_weight"))
    c.check_backward(dz, None, False)
    c.backward(dz, None, False, skip=("dweight", "dbias", "dpost_weight", "dpost_bias", "dgate"))
    c.check_backward(dz, None, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,h,gate", [(700, 256, 0), (3000, 40, 3000), (2500, 128, 16), (2500, 128, 17), (5000, 64, 1), (1300, 1200, 300), (4100, 16, 4), (1025, 2048, 0)])
def test_many_rows(dtype, rows, h, gate):
    c = Case(dtype, "layer", rows, h, True, gate)
    c.forward()
    c.check_forward()
    dz, dy = c.new((rows, h)), c.new((rows, h))
    c.backward(dz, dy, True)
    c.check_backward(dz, dy, True)
    kept = [t.clone() for t in (c.dx, c.dbranch, *c.sums.values())]
    c.backward(dz, dy, True)   # the same bits again
    assert all(torch.equal(a, b) for a, b in zip(kept, (c.dx, c.dbranch, *c.sums.values())))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h", [96, 1536])
def test_in_place(dtype, h):
    c = Case(dtype, "rms", 37, h, True, 10)
    c.forward()
    y, z = c.y.clone(), c.z.clone()
    for first, second in ((0, 1), (1, 0)):
        x, b = c.x.clone(), c.branch.clone()
        B.op_residual_norm_fwd(x, (x, b)[second], c.weight, c.bias, branch=b, y=(x, b)[first], post_weight=c.post_weight, post_bias=c.post_bias, gate=c.gate,
                               rows_per_gate=10, alpha=c.alpha, beta=c.beta)
        assert torch.equal((x, b)[first], y) and torch.equal((x, b)[second], z)
    dz, dy = c.new((37, h)), c.new((37, h))
    c.backward(dz, dy, False)
    kept = [t.clone() for t in (c.dx, c.dbranch, *c.sums.values())]
    for to in ("dz-dy", "dy-dz", "dy-branch"):
        a, b, branch = dz.clone(), dy.clone(), c.branch
        c.branch = branch.clone()
        dx, dbranch = {"dz-dy": (a, b), "dy-dz": (b, a), "dy-branch": (b, c.branch)}[to]
        c.backward(a, b, False, dx=dx, dbranch=dbranch)
        assert all(torch.equal(p, q) for p, q in zip(kept, (c.dx, c.dbranch, *c.sums.values()))), to
        c.branch = branch


def test_no_rows():
    c = Case("f32", "layer", 0, 24, True, 3)
    c.forward()
    dz, dy = c.new((0, 24)), c.new((0, 24))
    c.backward(dz, dy, False)
    assert all(bool((t == 0).all()) for t in c.sums.values())
    c.backward(dz, dy, True)
    assert torch.equal(c.sums["dweight"], torch.arange(24, device="cuda", dtype=torch.float32) % 7)


@pytest.mark.parametrize("h", [128, 1536])
def test_a_row_that_is_not_finite_stays_alone(h):
    c = Case("bf16", "layer", 12, h, True, 12, seed=9)
    c.forward()
    y, z, s = c.y.clone(), c.z.clone(), c.stats.clone()
    c.x[4, 3], c.branch[7, h - 1] = float("inf"), float("nan")
    c.forward()
    others = [k for k in range(12) if k not in (4, 7)]
    assert torch.equal(c.y[others], y[others]) and torch.equal(c.z[others], z[others]) and torch.equal(c.stats[:, others], s[:, others])
    assert bool(c.z[4].isnan().all()) and bool(c.z[7].isnan().all()) and bool(c.y[7].isnan().all()) and int((~c.y[4].isfinite()).sum()) == 1
    dz, dy = c.new((12, h)), c.new((12, h))
    c.backward(dz, dy, False)
    assert bool(c.dx[others].isfinite().all()) and bool(c.dbranch[others].isfinite().all())


def test_large_values_and_rows_of_zeros():
    """A row of zeros has 1 / sqrt(eps); squares of 1e17 are near fp32's end."""
    x = torch.zeros(3, 256, device="cuda")
    x[1], x[2] = 1e17 * torch.randn(256, device="cuda"), 1e-12
    w = torch.ones(256, device="cuda")
    z, stats = torch.empty_like(x), torch.empty((2, 3), device="cuda")
    B.op_residual_norm_fwd(x, z, w, kind="rms", stats=stats)
    want = L.statistics(f64(x), "rms", 1e-5)
    np.testing.assert_allclose(f64(stats), want, rtol=40 * e)
    assert not bool(z[0].any()) and bool(z.isfinite().all())


@pytest.mark.parametrize("h", [3, 333, 1000, 1920, 5001])
def test_rows_of_equal_entries(h):
    """A layer norm of them is its bias: sums of up to 13 bits more than bf16's 8 are exact, and so is their mean."""
    x = torch.tensor([1000.0, -0.3, 1e-3, 12345.0], device="cuda").bfloat16()[:, None].expand(4, h).contiguous()
    w, b = torch.full((h,), 3.0, device="cuda").bfloat16(), torch.randn(h, device="cuda").bfloat16()
    z, stats = torch.empty_like(x), torch.empty((2, 4), device="cuda")
    B.op_residual_norm_fwd(x, z, w, b, kind="layer", stats=stats)
    assert torch.equal(stats[0], x[:, 0].float()) and torch.equal(z, b.expand(4, h))


def test_the_gradient_against_differences():
    """fp32 on the GPU: a sum of the outputs by two weights, moved along the gradient; second differences in 64 bits of what the GPU gave."""
    c = Case("f32", "layer", 6, 40, True, 2, seed=3)
    dz, dy = c.new((6, 40)), c.new((6, 40))
    c.forward()
    c.backward(dz, dy, False)
    value = lambda: float((c.z.double() * dz.double()).sum() + (c.y.double() * dy.double()).sum())  # noqa: E731
    for name, grad in (("x", c.dx), ("branch", c.dbranch), ("gate", c.sums["dgate"]), ("weight", c.sums["dweight"]), ("bias", c.sums["dbias"]),
                       ("post_weight", c.sums["dpost_weight"]), ("post_bias", c.sums["dpost_bias"])):
        t, g = getattr(c, name), grad.clone()
        step = 2.0 ** -6 * g / float(g.norm())
        old = t.clone()
        t.copy_(old + step)
        moved = (t - old).double()
        c.forward()
        up = value()
        t.copy_(old - moved.float())
        c.forward()
        down = value()
        t.copy_(old)
        want = float((moved * g.double()).sum()) * 2
        # third derivatives by step^3 (values and weights near 1, 240 entries): 2^-12 of the change; roundings 480 e of sums near 300
        assert abs(up - down - want) <= 2.0 ** -9 * abs(want) + 480 * e * 300, name


def test_two_streams_and_replayed_graph():
    c = Case("bf16", "rms", 300, 640, True, 100)
    dz, dy = c.new((300, 640)), c.new((300, 640))
    scratch = [torch.empty(B.residual_norm_bwd_scratch_bytes(300, 640, 100), dtype=torch.uint8, device="cuda") for _ in range(2)]
    c.forward()
    c.backward(dz, dy, False)
    want = [t.clone() for t in (c.y, c.z, c.dx, c.dbranch, *c.sums.values())]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    torch.cuda.synchronize()
    for stream, room in zip(streams, scratch):
        with torch.cuda.stream(stream):
            c.backward(dz, dy, False, scratch=room)
            got.append([c.dx, c.dbranch, *c.sums.values()])
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want[2:]))
    names = list(c.sums)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward(dz, dy, False, dx=c.dx, dbranch=c.dbranch, scratch=scratch[0])
    out = [c.y, c.z, c.dx, c.dbranch, *(c.sums[k] for k in names)]
    x0 = c.x.clone()
    for k in range(3):
        for t in out:
            t.zero_()
        c.x.copy_(x0 if k != 1 else 2 * x0)
        graph.replay()
        torch.cuda.synchronize()
        if k == 1:
            assert not torch.equal(c.y, want[0])
        else:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_more_than_32_bits_of_offset():
    """2.2e9 entries: the rows behind 2^32 bytes and behind 2^31 entries are as those before."""
    rows, h = 270000, 8192
    x = torch.empty((rows, h), dtype=torch.bfloat16, device="cuda")
    first = torch.randn(2000, h, device="cuda").bfloat16()
    for k in range(0, rows, 2000):
        x[k:k + 2000] = first
    w = torch.ones(h, device="cuda").bfloat16()
    z, stats = torch.empty_like(x), torch.empty((2, rows), device="cuda")
    B.op_residual_norm_fwd(x, z, w, stats=stats)
    for k in (2000, 130000, 262000, 268000):
        assert torch.equal(z[k:k + 2000], z[:2000])
    dx, dw = torch.empty_like(x), torch.empty(h, device="cuda")
    room = torch.empty(B.residual_norm_bwd_scratch_bytes(rows, h), dtype=torch.uint8, device="cuda")
    B.op_residual_norm_bwd(z, x, stats, w, dx, room, dweight=dw, accumulate=False)
    for k in (2000, 130000, 262000, 268000):
        assert torch.equal(dx[k:k + 2000], dx[:2000])


@pytest.mark.parametrize("dtype,h", [("bf16", 2048), ("bf16", 2055), ("bf16", 500), ("f32", 4096)])
def test_rows_beyond_the_caches(dtype, h):
    """Calls of 200, 400 and 600 MB of rows, past the caches in part or wholly: their rows are, bit for bit, those of calls of a few; sums within what their order may change."""
    size = torch.finfo(DT[dtype]).bits // 8
    for mb, gated in ((200, False), (400, True), (600, False)):
        rows = (mb << 20) // (4 * h * size)
        c = Case(dtype, "rms", 64, h, True, 64 if gated else 0, bias=False)
        few = {k: getattr(c, k) for k in ("x", "branch")}
        dz0, dy0 = c.new((64, h)), c.new((64, h))
        c.forward()
        c.check_forward()
        c.backward(dz0, dy0, False)
        small = {k: t.clone() for k, t in (("y", c.y), ("z", c.z), ("dx", c.dx), ("dbranch", c.dbranch), ("stats", c.stats), ("post_stats", c.post_stats))}
        sums = {k: f64(t) for k, t in c.sums.items()}
        times, left = divmod(rows, 64)
        again = lambda t: torch.cat([t.repeat(times, 1), t[:left]])  # noqa: E731
        c.rows, c.rpg = rows, rows if gated else 0
        c.x, c.branch, dz, dy = again(few["x"]), again(few["branch"]), again(dz0), again(dy0)
        c.y, c.z = torch.empty_like(c.x), torch.empty_like(c.x)
        c.stats, c.post_stats = torch.empty((2, rows), device="cuda"), torch.empty((2, rows), device="cuda")
        dx, db = torch.empty_like(c.x), torch.empty_like(c.x)
        c.forward()
        c.backward(dz, dy, False, dx=dx, dbranch=db)
        for k, got in (("y", c.y), ("z", c.z), ("dx", dx), ("dbranch", db)):
            assert torch.equal(got, again(small[k])), (k, mb)
        for k, got in (("stats", c.stats), ("post_stats", c.post_stats)):
            assert torch.equal(got, again(small[k].t()).t()), (k, mb)
        # the same sum `times` times and that of the rows that are left
        part = Case(dtype, "rms", 64, h, True, left or 1 if gated else 0, bias=False)
        if left:
            part.rows, part.rpg = left, left if gated else 0
            part.x, part.branch = few["x"][:left], few["branch"][:left]
            part.weight, part.post_weight = c.weight, c.post_weight
            part.gate = c.gate
            part.y, part.z = torch.empty_like(part.x), torch.empty_like(part.x)
            part.stats, part.post_stats = torch.empty((2, left), device="cuda"), torch.empty((2, left), device="cuda")
            part.forward()
            part.backward(dz0[:left], dy0[:left], False)
        for k, got in c.sums.items():
            want = times * sums[k] + (f64(part.sums[k]) if left else 0.0)
            # a column's terms are near normal, so their absolute values sum to about rows * 2 at most; sums of sums are chains of rows / 256 + 40
            assert (np.abs(f64(got) - want) <= (rows / 256 + 60 + 84 * times / 64) * e * rows * 4).all(), (k, mb)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("h", [40, 200, 1500])
def test_a_norm_without_a_branch_takes_no_scale(dtype, kind, h):
    """z = Npre(x) reads no alpha, so neither does its gradient; a branch that is there, its gradient not wanted, leaves dx its alpha."""
    c = Case(dtype, kind, 21, h, False, 0, branch=False, alpha=0.9, beta=3.0)
    c.forward()
    c.check_forward()
    dz, dy = c.new((21, h)), c.new((21, h))
    for back in (dy, None):
        c.alpha = 0.9
        c.backward(dz, back, False)
        c.alpha = 1.0
        c.check_backward(dz, back, False)
    branch, room = c.new((21, h)), torch.empty(max(1, B.residual_norm_bwd_scratch_bytes(21, h)), dtype=torch.uint8, device="cuda")
    c.alpha = 0.9
    B.op_residual_norm_bwd(dz, c.x, c.stats, c.weight, c.dx, room, dy=dy, branch=branch, alpha=0.9, beta=3.0, kind=kind)
    c.sums = {}
    c.check_backward(dz, dy, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,gate,h", [(40, 20, 128), (83, 5, 72), (83, 40, 1100), (23, 4, 4104), (23, 4, 8200), (1001, 91, 333)])
def test_a_row_that_is_not_finite_stays_in_its_gate(dtype, kind, rows, gate, h):
    """Gates whose rows the teams do not divide, a NaN in the first row or in the last gate's first: the gradients of the other gates, and all other rows, are those of
    a call without it."""
    def results(spoilt):
        c = Case(dtype, kind, rows, h, True, gate, bias=kind == "layer", seed=4)
        if spoilt is not None:
            c.branch[spoilt, h // 2] = float("nan")
        c.forward()
        dz, dy = c.new((rows, h)), c.new((rows, h))
        c.backward(dz, dy, False)
        return c, dz, dy

    clean, dz, dy = results(None)
    clean.check_backward(dz, dy, False)
    for spoilt in (0, (rows - 1) // gate * gate):
        c, *_ = results(spoilt)
        own = spoilt // gate
        fine, gates = torch.arange(rows, device="cuda") != spoilt, torch.arange(len(c.gate), device="cuda") != own
        assert bool(c.dx[spoilt].isnan().all()) and bool(c.dbranch[spoilt].isnan().all()) and bool(c.sums["dgate"][own].isnan().all())
        assert torch.equal(c.dx[fine], clean.dx[fine]) and torch.equal(c.dbranch[fine], clean.dbranch[fine])
        assert torch.equal(c.sums["dgate"][gates], clean.sums["dgate"][gates]), spoilt


@pytest.mark.parametrize("gate", [4, 20])
def test_a_first_row_of_zeros_without_eps_stays_in_its_gate(gate):
    """Its deviation's reciprocal is infinite."""
    c = Case("f32", "rms", 41, 200, True, gate, bias=False)
    c.eps = 0.0
    c.branch[0] = 0
    c.forward()
    assert bool(c.post_stats[1, 0].isinf())
    dz, dy = c.new((41, 200)), c.new((41, 200))
    c.backward(dz, dy, False)
    assert bool(c.sums["dgate"][0].isnan().all()) and bool(c.sums["dgate"][1:].isfinite().all()) and bool(c.dbranch[1:].isfinite().all())


@pytest.mark.parametrize("gate", [0, 3])
def test_no_rows_need_no_scratch(gate):
    c = Case("bf16", "layer", 0, 24, True, gate)
    c.forward()
    dz, dy = c.new((0, 24)), c.new((0, 24))
    room = torch.empty(B.residual_norm_bwd_scratch_bytes(0, 24, gate), dtype=torch.uint8, device="cuda")
    assert room.numel() == 0
    for accumulate in (False, True):
        c.backward(dz, dy, accumulate, scratch=room)
        want = torch.arange(24, device="cuda", dtype=torch.float32) % 7 if accumulate else torch.zeros(24, device="cuda")
        assert all(torch.equal(t, want) for t in c.sums.values() if t.numel())


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", [0, 1, 4, 16, 64])
@pytest.mark.parametrize("dtype,h", [("bf16", 2048), ("bf16", 2055), ("bf16", 500), ("f32", 4096), ("f32", 1023)])
def test_forms_beyond_the_caches(dtype, h, gate, post, kind):
    """Backward calls of 200 MB, as a layer norm with biases or an RMS norm, with and without post norm, a gate for every few rows or several for many: 64 rows many times over, which
    are, bit for bit, those of a call of 64 (whose oracle they have), as is the gradient of a gate for up to 16 rows; the other sums are as many times those, within what their order may
    change."""
    size = torch.finfo(DT[dtype]).bits // 8
    times = (200 << 20) // (6 * h * size * 64)
    c = Case(dtype, kind, 64, h, post, gate, bias=kind == "layer")
    c.forward()
    c.check_forward()
    dz0, dy0 = c.new((64, h)), c.new((64, h))
    c.backward(dz0, dy0, False)
    c.check_backward(dz0, dy0, False)
    small = {k: t.clone() for k, t in (("dx", c.dx), ("dbranch", c.dbranch), *c.sums.items())}
    again = lambda t: t.repeat(times, 1)  # noqa: E731
    c.rows = 64 * times
    c.x, c.branch, c.y, dz, dy = again(c.x), again(c.branch), again(c.y), again(dz0), again(dy0)
    c.stats = c.stats.repeat(1, times)
    c.post_stats = c.post_stats.repeat(1, times) if post else None
    each = times   # repetitions under one gate
    if 0 < gate < 64:
        c.gate = again(c.gate)
    elif gate == 64:   # three gates and a shorter fourth
        each = times * 2 // 7
        c.rpg = 64 * each
        c.gate = c.gate.repeat(-(-times // each), 1)
    c.backward(dz, dy, False, dx=torch.empty_like(c.x), dbranch=torch.empty_like(c.x))
    assert torch.equal(c.dx, again(small["dx"])) and torch.equal(c.dbranch, again(small["dbranch"]))
    if 0 < gate < 64:
        assert torch.equal(c.sums.pop("dgate"), again(small.pop("dgate")))
    for k, got in c.sums.items():
        many = np.full((1, 1), times) if k != "dgate" else np.array([[min(each, times - j * each)] for j in range(len(c.gate))])
        want = many * f64(small[k]).reshape(1, h)
        # a column's terms are near normal, their absolute values sum to under 4 a row; a chain of rows / 256 and 60 joins here, 84 roundings of the sum of 64 rows there
        assert (np.abs(f64(got).reshape(want.shape) - want) <= (c.rows / 256 + 60 + 84) * e * 64 * many * 4).all(), k
