"""Forms of the embedding that its other tests do not run: outputs beyond the last-level cache (four rows to a thread) in fp32, with given
positions, with ids that are none and a scale; running positions in every type, scaled, added to, and where there are waves enough for many rows
of each; 64-bit ids whose low half alone would be a row.

Tolerances as in test_embedding_parity.py: half a step of fp32 for every product and sum on the way, half a step of the output's type at the end."""
import numpy as np
import pytest
import torch

from paper_2111_04007_amd import binding as B
from tests.test_embedding_parity import DT, HALF, U, backward, check_backward, check_forward, guarded, on_gpu, rng, untouched

pytestmark = pytest.mark.gpu

LOW = (1 << 32) + 1   # its low half is row 1


def odd_ids(r, rows, vocab):
    """Rows of the table, and all kinds of ids that are none among them."""
    ids = r.integers(0, vocab, rows)
    for i, v in enumerate((-1, vocab, LOW, -(1 << 40), -(1 << 32), (1 << 63) - 1, -(1 << 63), (1 << 40) + vocab - 1)):
        ids[i::31] = v
    return ids


@pytest.mark.parametrize("dtype,rows,h,seq", [("f32", 16500, 4096, 2048), ("f32", 65600, 1032, 1000), ("f32", 9000, 8201, 2048), ("bf16", 16500, 8192, 2048), ("bf16", 65600, 2064, 1000),
                                              ("bf16", 33001, 4104, 16384), ("bf16", 16500, 8201, 2048)])
def test_forward_larger_than_the_last_level_cache(dtype, rows, h, seq):
    r = rng(rows, h)
    ids = torch.from_numpy(odd_ids(r, rows, 50)).cuda()
    table, places = on_gpu(r.standard_normal((50, h)), DT[dtype]), on_gpu(r.standard_normal((seq, h)), DT[dtype])
    given = torch.from_numpy(r.integers(-1, seq + 1, rows)).cuda()
    given[5::97] = LOW
    out = torch.empty((rows, h), dtype=DT[dtype], device="cuda")
    running = torch.arange(rows, device="cuda") % seq
    for scale in (1.0, -0.75):
        for at, kw in ((None, {}), (running, dict(pos_table=places)), (given, dict(pos_table=places, positions=given))):
            out.fill_(float("nan"))
            B.op_embedding_fwd(ids, table, out, scale=scale, **kw)
            for a in range(0, rows, 4000):
                i, term, place = ids[a:a + 4000], None, 0.0
                term = torch.where(((i >= 0) & (i < 50))[:, None], scale * table[i.clamp(0, 49)].double(), 0.0)
                if at is not None:
                    p = at[a:a + 4000]
                    place = torch.where(((p >= 0) & (p < seq))[:, None], places[p.clamp(0, seq - 1)].double(), 0.0)
                ref = term + place
                bound = U * (term.abs() + ref.abs()) + HALF[dtype] * ref.abs() * (1 + 2 * U) + 1e-45
                assert bool(((out[a:a + 4000].double() - ref).abs() <= bound).all()), (scale, a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forward_of_ids_and_positions_beyond_32_bits(dtype):
    r = rng(21)
    ids, given = odd_ids(r, 200, 40), odd_ids(r, 200, 30)
    table, places = on_gpu(r.standard_normal((40, 72)), DT[dtype]), on_gpu(r.standard_normal((30, 72)), DT[dtype])
    out, flat, where = guarded((200, 72), DT[dtype], 0)
    B.op_embedding_fwd(torch.from_numpy(ids).cuda(), table, out, pos_table=places, positions=torch.from_numpy(given).cuda())
    check_forward(ids, table, 1.0, given, places, out, dtype)
    assert untouched(flat, where)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows,h,vocab,lead", [(200, 64, 40, 0), (200, 65, 40, 1), (1, 64, 3, 0), (256, 8, 300, 0), (257, 64, 40, 0), (3000, 72, 900, 0), (3000, 33, 900, 1), (9000, 16, 2, 0), (9000, 24, 1, 0)])
def test_backward_of_ids_beyond_32_bits(rows, h, vocab, lead, accumulate):
    r = rng(rows, h, 22)
    ids = odd_ids(r, rows, vocab)
    dy = on_gpu(r.standard_normal((rows, h)), torch.bfloat16, lead)
    grad, flat, where = guarded((vocab, h), torch.float32, lead)
    old = r.standard_normal((vocab, h)).astype(np.float32)
    grad.copy_(torch.from_numpy(old) if accumulate else torch.tensor(float("nan")))
    backward(ids, dy, grad, "i64", scale=0.5, accumulate=accumulate)
    check_backward(ids, dy, 0.5, grad, old.astype(np.float64), accumulate)
    assert untouched(flat, where)


# The last four: positions x slices of columns fill the chip, with more rows of each than are summed by themselves otherwise; and one whose
# few positions have so many rows that they are sorted.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows,seq,vocab,h,lead", [(1, 5, 9, 40, 0), (10, 10, 12, 24, 0), (1001, 91, 512, 333, 0), (1001, 91, 100, 336, 1), (700, 2, 5, 40, 0), (200, 1, 4, 40, 0), (40, 1, 4, 24, 0),
                                                   (2000, 7, 9, 65, 1), (150_000, 1100, 1101, 16, 0), (150_001, 1100, 1103, 17, 0), (20_000, 129, 130, 4104, 0), (4000, 3, 4, 48, 0)])
def test_backward_of_positions_that_run(dtype, rows, seq, vocab, h, lead, accumulate):
    r = rng(rows, seq, h)
    dy = on_gpu(r.standard_normal((rows, h)).astype(np.float32), DT[dtype], lead)
    scale = float(np.float32(-1.3))
    grad, flat, where = guarded((vocab, h), torch.float32, lead)
    old = torch.from_numpy(r.standard_normal((vocab, h)).astype(np.float32)).cuda()
    grad.copy_(old if accumulate else torch.full_like(old, float("nan")))
    backward(None, dy, grad, "i64", scale=scale, accumulate=accumulate, seq_len=seq)
    # the formula on the GPU in 64 bits, rows of one position side by side
    whole = -(-rows // seq)
    terms = torch.zeros((whole * seq, h), dtype=torch.float64, device="cuda")
    terms[:rows] = dy.double() * scale
    ref, mag = torch.zeros((vocab, h), dtype=torch.float64, device="cuda"), torch.zeros((vocab, h), dtype=torch.float64, device="cuda")
    ref[:seq], mag[:seq] = terms.view(whole, seq, h).sum(0), terms.abs().view(whole, seq, h).sum(0)
    ref += old.double() if accumulate else 0.0
    assert bool(((grad.double() - ref).abs() <= U * ((whole + 2) * mag + ref.abs()) * 1.01).all())
    assert untouched(flat, where)
    if accumulate:   # rows behind the last position keep their bits
        n = min(rows, seq)
        assert torch.equal(grad[n:], old[n:])
