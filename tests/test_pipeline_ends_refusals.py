"""Argument checks of the embedding, the loss and the global gradient norm: they return before any GPU work, so made-up
addresses do; no GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2111_04007_amd import binding as B

A, D, E, S = (C.c_void_p(i << 40) for i in (1, 2, 3, 4))   # far apart, aligned, never read


def at(p, n):
    return C.c_void_p(p.value + n)


def refused(code, fn, *args):
    lib = B.load()
    assert getattr(lib, fn)(*args) == code, (fn, args)
    assert lib.varuna_last_error()


def fwd(dtype=B.F32, index=B.I64, rows=4, h=8, vocab=10, ids=A, table=D, scale=1.0, seq=0, n_pos=0, positions=None, places=None, out=E):
    return "varuna_op_embedding_fwd", dtype, index, rows, h, vocab, ids, table, scale, seq, n_pos, positions, places, out, None


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(index=2), dict(rows=-1), dict(h=0), dict(vocab=0), dict(scale=float("inf")), dict(ids=None), dict(table=None), dict(out=None),
    dict(positions=S), dict(places=S, seq=2), dict(places=S, n_pos=4), dict(places=S, seq=5, n_pos=4), dict(places=S, seq=-1, n_pos=4),
    dict(ids=at(A, 4)), dict(table=at(D, 2)), dict(out=at(E, 1)), dict(out=D), dict(out=at(D, 316)), dict(out=at(A, 16)),
    dict(places=S, seq=2, n_pos=4, out=at(S, 64)), dict(places=E, positions=S, n_pos=4, out=S),
])
def test_embedding_forward_refuses(kw):
    refused(B.EINVAL, *fwd(**kw))


def test_embedding_forward_refuses_sizes_beyond_its_range():
    refused(B.EUNSUPPORTED, *fwd(rows=1 << 31))
    refused(B.EUNSUPPORTED, *fwd(vocab=1 << 31))
    refused(B.EUNSUPPORTED, *fwd(h=(1 << 20) + 1))


def bwd(dtype=B.F32, index=B.I64, rows=4, h=8, vocab=10, ids=A, seq=0, dy=D, scale=1.0, acc=1, grad=E, scratch=S):
    return "varuna_op_embedding_bwd", dtype, index, rows, h, vocab, ids, seq, dy, scale, acc, grad, scratch, None


@pytest.mark.parametrize("kw", [
    dict(dtype=-1), dict(index=3), dict(rows=-1), dict(h=0), dict(vocab=0), dict(dy=None), dict(grad=None), dict(scratch=None), dict(acc=2), dict(scale=float("nan")),
    dict(ids=None), dict(ids=None, seq=11), dict(ids=at(A, 4)), dict(dy=at(D, 2)), dict(grad=at(E, 2)), dict(scratch=at(S, 16)),
    dict(grad=D), dict(grad=at(A, 16)), dict(scratch=E), dict(scratch=D), dict(scratch=A),
])
def test_embedding_backward_refuses(kw):
    refused(B.EINVAL, *bwd(**kw))


def test_embedding_backward_scratch():
    refused(B.EUNSUPPORTED, *bwd(rows=1 << 31))
    assert B.embedding_bwd_scratch_bytes(-1, 8, 10) == 0 and B.embedding_bwd_scratch_bytes(4, 0, 10) == 0 and B.embedding_bwd_scratch_bytes(4, 8, 0) == 0
    last = 0
    for rows in (0, 1, 5, 64, 1000, 4096, 16384, 100001):
        n = B.embedding_bwd_scratch_bytes(rows, 1024, 50257)
        assert n >= last > -1 and n < rows * 1024 * 4 + (1 << 20)   # never as much as dy in fp32 and a table of ids
        last = n


def loss(dtype=B.F32, index=B.I64, rows=4, vocab=10, ld=10, x=A, y=D, e=0.0, g=1.0, scale=None, loss=E, ldd=10, dx=S, out2=None):
    return "varuna_op_cross_entropy", dtype, index, rows, vocab, ld, x, y, e, g, scale, loss, ldd, dx, out2, None


@pytest.mark.parametrize("kw", [
    dict(dtype=5), dict(index=-1), dict(rows=-1), dict(vocab=0, ld=0), dict(ld=9), dict(ldd=9), dict(x=None), dict(y=None), dict(loss=None),
    dict(e=-0.1), dict(e=1.1), dict(e=float("nan")), dict(x=at(A, 2)), dict(dx=at(S, 2)), dict(y=at(D, 4)), dict(loss=at(E, 2)), dict(out2=at(E, 66)),
    dict(scale=at(D, 66)), dict(dx=A, ldd=12), dict(dx=at(A, 4)), dict(dx=at(A, 156)), dict(dx=D), dict(loss=A), dict(loss=at(D, 28)), dict(out2=A), dict(out2=at(E, 12)),
    dict(out2=S), dict(loss=at(S, 40)), dict(scale=E), dict(scale=S),
])
def test_cross_entropy_refuses(kw):
    refused(B.EINVAL, *loss(**kw))


def test_cross_entropy_refuses_sizes_beyond_its_range():
    refused(B.EUNSUPPORTED, *loss(rows=(1 << 24) + 1))
    refused(B.EUNSUPPORTED, *loss(vocab=(1 << 30) + 1, ld=(1 << 30) + 1, ldd=(1 << 30) + 1))


def span(n, p, dtype=B.F32, count=16):
    return (C.c_int32 * n)(*[dtype] * n), (C.c_void_p * n)(*[q if q is None else q.value for q in p]), (C.c_int64 * n)(*[count] * n)


def test_grad_norm_refuses():
    t, p, c = span(2, (A, D))
    def norm(n=2, t=t, p=p, c=c, s=E, bad=at(E, 8), scratch=S):
        return "varuna_op_grad_norm", n, t, p, c, s, bad, scratch, None
    for kw in (dict(n=-1), dict(t=None), dict(p=None), dict(c=None), dict(t=span(2, (A, D), 2)[0]), dict(c=span(2, (A, D), 0, -1)[2]), dict(p=span(2, (A, None))[1]),
               dict(p=span(2, (A, at(D, 2)))[1]), dict(s=None), dict(bad=None), dict(scratch=None), dict(s=at(E, 4)), dict(bad=at(E, 2)), dict(bad=at(E, 4)),
               dict(scratch=at(S, 8)), dict(scratch=E), dict(scratch=D), dict(s=at(A, 56)), dict(bad=at(D, 60))):
        refused(B.EINVAL, *norm(**kw))
    refused(B.EUNSUPPORTED, *norm(c=span(2, (A, D), 0, (1 << 41) + 1)[2]))
    lib = B.load()
    assert lib.varuna_op_grad_norm_scratch_bytes(-1, c) == 0 and lib.varuna_op_grad_norm_scratch_bytes(2, None) == 0
    assert 0 < lib.varuna_op_grad_norm_scratch_bytes(0, None) <= lib.varuna_op_grad_norm_scratch_bytes(2, c)


def test_grad_clip_refuses():
    t, p, c = span(2, (A, D))
    _, q, _ = span(2, (E, at(E, 64)))
    half = span(2, (A, D), B.BF16)[0]
    def clip(n=2, dt=t, d=q, t=t, p=p, c=c, s=S, most=1.0, eps=0.0):
        return "varuna_op_grad_clip", n, dt, d, t, p, c, s, most, eps, None
    for kw in (dict(n=-1), dict(dt=None), dict(d=None), dict(t=None), dict(p=None), dict(c=None), dict(s=None), dict(s=at(S, 4)), dict(most=-1.0),
               dict(most=float("nan")), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(d=span(2, (E, E))[1]),                 # two tensors into one place
               dict(d=span(2, (E, at(E, 60)))[1]),
               dict(d=span(2, (A, A))[1], p=span(2, (A, A))[1]),   # the same tensor twice, in place
               dict(d=span(2, (at(A, 4), E))[1]),          # next to its own src
               dict(d=span(2, (D, A))[1]),                 # another tensor's src
               dict(d=span(2, (D, E))[1]),
               dict(d=p, dt=half),                         # in place in another type
               dict(d=span(2, (A, S))[1]), dict(d=span(2, (A, at(S, -56)))[1])):
        refused(B.EINVAL, *clip(**kw))


def test_binding_refuses_tensors_that_are_not_on_a_gpu_or_do_not_fit():
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):
        B.op_embedding_fwd(ids, torch.zeros(10, 8), x)
    with pytest.raises(ValueError):
        B.op_embedding_bwd(ids, x, torch.zeros(10, 8), torch.zeros(1 << 16, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.op_cross_entropy(x, ids, torch.zeros(4))
    with pytest.raises(ValueError):
        B.TensorList([x])
    with pytest.raises(TypeError):
        B.index_code(torch.zeros(1, dtype=torch.int16))
