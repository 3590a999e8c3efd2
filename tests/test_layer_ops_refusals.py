"""Argument checks of rotary positions, the residual norms and AdamW: they return before any GPU work, so made-up addresses do; no GPU needed."""
import ctypes as C
import math

import pytest
import torch

from paper_2111_04007_amd import binding as B

P = [C.c_void_p(i << 36) for i in range(1, 24)]   # far apart, aligned, never read
INF, NAN = float("inf"), float("nan")


def at(p, n):
    return C.c_void_p(p.value + n)


def refused(code, fn, *args):
    lib = B.load()
    assert getattr(lib, fn)(*args) == code, (fn, args)
    assert lib.varuna_last_error()


def frequencies(r=8, base=1e4, scaling=0, factor=1.0, length=64.0, low=1.0, high=4.0, to=(C.c_double * 256)()):
    return "varuna_rotary_frequencies", r, base, scaling, factor, length, low, high, to


@pytest.mark.parametrize("kw", [
    dict(r=0), dict(r=7), dict(r=514), dict(base=0.0), dict(base=-1.0), dict(base=INF), dict(base=NAN), dict(scaling=-1), dict(scaling=4), dict(scaling=1, factor=0.5),
    dict(scaling=1, factor=INF), dict(scaling=2, factor=NAN), dict(scaling=2, factor=2.0, r=2), dict(scaling=3, factor=2.0, length=0.0), dict(scaling=3, factor=2.0, low=-1.0),
    dict(scaling=3, factor=2.0, low=4.0), dict(scaling=3, factor=2.0, high=INF), dict(scaling=3, factor=2.0, high=NAN), dict(to=None),
])
def test_frequencies_refuse(kw):
    refused(B.EINVAL, *frequencies(**kw))


def test_frequencies_on_the_host():
    assert list(B.rotary_frequencies(4, 100.0)) == [1.0, 0.1]
    assert list(B.rotary_frequencies(4, 100.0, "linear", 4.0)) == [0.25, 0.025]
    assert math.isclose(B.rotary_frequencies(4, 100.0, "base", 4.0)[1], 0.025)
    assert list(B.rotary_frequencies(2, 100.0, "parts", 4.0, 2 * math.pi, 2.0, 3.0)) == [0.25]
    assert list(B.rotary_frequencies(2, 100.0, "parts", 4.0, 8 * math.pi, 2.0, 3.0)) == [1.0]
    assert math.isclose(B.rotary_frequencies(2, 100.0, "parts", 4.0, 5 * math.pi, 2.0, 3.0)[0], 0.625)
    with pytest.raises(ValueError):
        B.rotary_frequencies(4, scaling="other")
    with pytest.raises(B.VarunaError):
        B.rotary_frequencies(5)


def test_table_refuses():
    f = (C.c_double * 4)(1, 2, 3, 4)
    def table(n=10, r=8, f=f, m=1.0, to=P[0]):
        return "varuna_op_rotary_table", n, r, f, m, to, None
    for kw in (dict(n=-1), dict(r=0), dict(r=3), dict(r=514), dict(f=None), dict(to=None), dict(to=at(P[0], 2)), dict(m=INF), dict(f=(C.c_double * 4)(1, NAN, 3, 4))):
        refused(B.EINVAL, *table(**kw))
    refused(B.EUNSUPPORTED, *table(n=(1 << 30) + 1))


def rotary(dtype=B.F32, index=B.I64, inter=0, trans=0, rows=4, heads=3, d=16, r=8, x=P[0], xr=48, xh=16, out=P[0], o_r=48, oh=16, pos=P[1], seq=0, n=10, table=P[2]):
    return "varuna_op_rotary", dtype, index, inter, trans, rows, heads, d, r, x, xr, xh, out, o_r, oh, pos, seq, n, table, None


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(index=2), dict(inter=2), dict(trans=-1), dict(rows=-1), dict(heads=-1), dict(d=0), dict(r=0), dict(r=7), dict(r=18), dict(n=-1), dict(n=0), dict(x=None), dict(out=None),
    dict(table=None), dict(pos=None), dict(pos=None, seq=11), dict(xr=-48, o_r=-48), dict(xh=-16, oh=-16), dict(x=at(P[0], 2)), dict(out=at(P[0], 2)), dict(pos=at(P[1], 4)),
    dict(table=at(P[2], 2)), dict(xh=8, oh=8, xr=8, o_r=8), dict(xr=40, o_r=40), dict(xr=0, o_r=0), dict(o_r=64), dict(out=at(P[0], 64)), dict(out=at(P[0], 16), o_r=64),
    dict(out=at(P[0], 4 * 150)), dict(pos=at(P[0], 8)), dict(table=at(P[0], -300)), dict(out=P[3], oh=15), dict(out=P[3], o_r=8, oh=16), dict(x=P[3], xr=1 << 40, out=at(P[3], 64)),
])
def test_rotary_refuses(kw):
    refused(B.EINVAL, *rotary(**kw))


def test_rotary_refuses_sizes_beyond_its_range():
    for kw in (dict(rows=1 << 31), dict(heads=1 << 20, rows=1 << 12), dict(d=65537), dict(n=(1 << 30) + 1), dict(xr=1 << 62, o_r=1 << 62)):
        refused(B.EUNSUPPORTED, *rotary(**kw))


def norm(dtype=B.F32, kind=0, rows=4, h=8, rpg=2, alpha=1.0, beta=1.0, eps=1e-5):
    return C.byref(B.CNorm(dtype, kind, rows, h, rpg, alpha, beta, eps))


def fwd(n=None, x=P[0], branch=P[1], pw=P[2], pb=P[3], gate=P[4], w=P[5], b=P[6], y=P[7], z=P[8], ps=P[9], st=P[10], **kw):
    return "varuna_op_residual_norm_fwd", norm(**kw) if n is None else n, x, branch, pw, pb, gate, w, b, y, z, ps, st, None


BAD = [dict(dtype=2), dict(kind=2), dict(rows=-1), dict(h=0), dict(rpg=0), dict(alpha=INF), dict(beta=NAN), dict(eps=-1.0), dict(eps=INF)]


@pytest.mark.parametrize("kw", BAD + [
    dict(n=C.POINTER(B.CNorm)()), dict(x=None), dict(branch=None), dict(branch=None, gate=None, y=None), dict(branch=None, pw=None, pb=None, ps=None, gate=None), dict(pw=None), dict(pw=None, pb=None),
    dict(w=None), dict(z=None), dict(w=None, z=None), dict(w=None, z=None, b=None), dict(w=None, z=None, b=None, st=None, y=None), dict(x=at(P[0], 2)), dict(y=at(P[7], 1)),
    dict(st=at(P[10], 2)), dict(y=at(P[0], 32)), dict(z=at(P[1], -4)), dict(y=P[8]), dict(z=at(P[7], 124)), dict(y=P[2]), dict(z=P[5]), dict(y=P[4]), dict(z=at(P[4], 60)),
    dict(st=P[0]), dict(ps=P[10]), dict(st=at(P[8], 120)), dict(ps=P[6]),
])
def test_norm_forward_refuses(kw):
    refused(B.EINVAL, *fwd(**kw))


def bwd(n=None, dz=P[0], dy=P[1], y=P[2], branch=P[3], pw=P[4], pb=P[5], gate=P[6], w=P[7], ps=P[8], st=P[9], dx=P[10], db=P[11], g=P[12:17], acc=1, scratch=P[17], **kw):
    return "varuna_op_residual_norm_bwd", norm(**kw) if n is None else n, dz, dy, y, branch, pw, pb, gate, w, ps, st, dx, db, *g, acc, scratch, None


def sums(**kw):
    g = list(P[12:17])
    for k, v in kw.items():
        g["w b pw pb gate".split().index(k)] = v
    return dict(g=g)


@pytest.mark.parametrize("kw", BAD + [
    dict(n=C.POINTER(B.CNorm)()), dict(dz=None), dict(y=None), dict(st=None), dict(dx=None), dict(db=None), dict(branch=None), dict(ps=None), dict(w=None), dict(pw=None), dict(gate=None),
    dict(acc=2), dict(scratch=None), dict(scratch=at(P[17], 128)), dict(w=None, dz=None, y=None, st=None), dict(w=None, dz=None, y=None, st=None, dy=None, **sums(w=None, b=None)),
    dict(dx=P[2]), dict(dx=P[3]), dict(dx=at(P[0], 4)), dict(db=P[2]), dict(db=at(P[3], 64)), dict(db=P[10]), dict(dx=P[0], db=P[0]), dict(dx=at(P[10], 2)), dict(dy=at(P[1], 2)),
    sums(w=P[0]), sums(w=P[13]), sums(gate=P[6]), sums(pb=at(P[12], 28)), sums(gate=at(P[16], 2)), sums(pw=at(P[17], 256)), dict(scratch=P[3]), dict(dx=P[17]), dict(dx=P[8]), sums(b=P[9]),
])
def test_norm_backward_refuses(kw):
    refused(B.EINVAL, *bwd(**kw))


def test_norm_refuses_sizes_beyond_its_range():
    for kw in (dict(rows=(1 << 30) + 1), dict(h=16385)):
        refused(B.EUNSUPPORTED, *fwd(**kw))
        refused(B.EUNSUPPORTED, *bwd(**kw))
    refused(B.EUNSUPPORTED, *bwd(rows=1 << 30, rpg=20, h=1))
    f = B.residual_norm_bwd_scratch_bytes
    assert f(-1, 8) == 0 and f(4, 0) == 0 and f(4, 8, -1) == 0 and f(4, 16385) == 0 and f(0, 8) == 0
    assert f(1000, 64) >= f(1000, 64, 1000) > 0
    for rows in (1, 100, 5000, 100000):
        for gate in (0, 1, 5, 16, 17, 100, rows):
            assert 0 < f(rows, 64, gate) <= 5 * 64 * 4 * max(1100 + 2 * (rows // max(17, gate) if gate else 1), 1)


def span(n, p, dtype=B.F32, count=16):
    return (C.c_int32 * n)(*[dtype] * n), (C.c_void_p * n)(*[q if q is None else q.value for q in p[:n]]), (C.c_int64 * n)(*[count] * n)


def hp(lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.1, scale=1.0, most=1.0, ceps=1e-6, step=1, bits=8):
    return C.byref(B.CAdamW(lr, b1, b2, eps, wd, scale, most, ceps, step, bits))


T, Q, N = span(2, (P[0], P[1]))
_, G, _ = span(2, (P[2], P[3]))


def adamw(h=None, n=2, pt=T, p=Q, gt=T, g=G, c=N, decays=None, master=P[4], m=P[5], v=P[6], s=P[7], sq=P[8], skip=P[9], lr_step=P[10], **kw):
    return "varuna_op_adamw", hp(**kw) if h is None else h, n, pt, p, gt, g, c, decays, master, m, v, s, sq, skip, lr_step, None


@pytest.mark.parametrize("kw", [
    dict(h=C.POINTER(B.CAdamW)()), dict(n=-1), dict(pt=None), dict(p=None), dict(gt=None), dict(g=None), dict(c=None), dict(pt=span(2, P, 2)[0]), dict(c=span(2, P, 0, -1)[2]), dict(p=span(2, (P[0], None))[1]),
    dict(g=span(2, (None, P[2]))[1]), dict(p=span(2, (P[0], at(P[1], 2)))[1]), dict(bits=16), dict(bits=32), dict(s=None), dict(b1=1.0), dict(b2=-0.1), dict(b1=NAN), dict(lr=INF), dict(eps=-1.0), dict(eps=INF),
    dict(wd=NAN), dict(scale=INF), dict(lr_step=None, step=0), dict(lr_step=None, step=(1 << 40) + 1), dict(most=-1.0), dict(most=NAN), dict(ceps=-1.0), dict(ceps=INF), dict(m=None), dict(v=None),
    dict(sq=at(P[8], 4)), dict(skip=at(P[9], 2)), dict(lr_step=at(P[10], 4)), dict(m=at(P[5], 4)), dict(v=at(P[6], 8)), dict(master=at(P[4], 4), pt=span(2, P, B.BF16)[0]), dict(s=at(P[7], 8)),
    dict(pt=span(2, P, B.BF16)[0], master=None), dict(decays=(C.c_float * 2)(1.0, INF)),
    dict(p=span(2, (P[0], P[0]))[1]), dict(p=span(2, (P[0], at(P[0], 60)))[1]), dict(g=span(2, (P[0], P[3]))[1]), dict(g=span(2, (P[2], at(P[1], 60)))[1]), dict(m=P[0]), dict(m=P[2]), dict(v=P[5]),
    dict(v=at(P[5], 496)), dict(s=at(P[6], 496)), dict(sq=P[5]), dict(skip=P[7]), dict(lr_step=at(P[1], 8)), dict(master=P[6], pt=span(2, P, B.BF16)[0]),
])
def test_adamw_refuses(kw):
    refused(B.EINVAL, *adamw(**kw))


def test_adamw_state():
    f = B.load().varuna_op_adamw_state_entries
    assert f(0, None) == 0 and f(-1, None) == -1 and f(1, None) == -1
    assert f(4, (C.c_int64 * 4)(0, 1, 256, 257)) == 256 + 256 + 512
    assert f(1, (C.c_int64 * 1)(-1)) == -1 and f(1, (C.c_int64 * 1)((1 << 33) + 1)) == -1 and f(2, (C.c_int64 * 2)(1 << 33, 1)) == -1
    refused(B.EUNSUPPORTED, *adamw(c=(C.c_int64 * 2)(1 << 33, 1)))


def test_binding_refuses_tensors_that_are_not_on_a_gpu_or_do_not_fit():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    with pytest.raises(ValueError):
        B.op_rotary_table(torch.zeros(4, 8), B.rotary_frequencies(8))
    with pytest.raises(ValueError):
        B.op_rotary(torch.zeros(4, 2, 8), torch.zeros(4, 8))
    with pytest.raises(ValueError):
        B.op_residual_norm_fwd(x, x, w)
    with pytest.raises(ValueError):
        B.op_residual_norm_bwd(x, x, torch.zeros(8), w, x, torch.zeros(1 << 16, dtype=torch.uint8))


def test_norm_backward_refuses_more_gates_than_a_launch_has_workgroups():
    """Gates of more than 16 rows have a workgroup each at least; those of fewer share them."""
    f = B.residual_norm_bwd_scratch_bytes
    for h in (1, 512, 4096):
        assert f(17 << 22, h, 17) == 0 and f(1 << 30, h, 200) == 0
        refused(B.EUNSUPPORTED, *bwd(rows=17 << 22, rpg=17, h=h))
        most = (1 << 22) - 1
        assert f(17 * most, h, 17) == most * 5 * 4 * (-(-h // 64) * 64)
        assert f(1 << 30, h, 16) > 0 and f(1 << 30, h, 0) > 0
