"""One mini-batch of a whole small model through the library: token and position embedding, a pipeline stage, final LayerNorm,
the head's product on the token table itself (tied), the loss, everything backward, the norm over all gradients, clipping, and
the stage's update -- against the same model in fp64 with torch's autograd.  The tolerances are the stage's."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_2111_04007_amd import binding as B, synth
from tests.parity_util import TOL

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCAB, PLACES = 1003, 80


def _reference(cfg, layers, table, places, gamma, beta, tokens, targets, count):
    """(loss, gradients of the layers, of table, places, gamma and beta) in fp64."""
    leaf = lambda t: t.double().clone().requires_grad_()  # noqa: E731
    layers = [{k: leaf(v) for k, v in l.items()} for l in layers]
    table, places, gamma, beta = leaf(table), leaf(places), leaf(gamma), leaf(beta)
    h, a, s, b = cfg.hidden, cfg.n_heads, cfg.seq_len, cfg.micro_batch
    total = 0.0
    for tok, tgt in zip(tokens, targets):
        x = torch.where((tok >= 0)[:, None], table[tok.clamp(min=0)], 0.0) + places[torch.arange(b * s) % s]
        for p in layers:
            qkv = F.linear(F.layer_norm(x, (h,), p["ln1_g"], p["ln1_b"], cfg.ln_eps or 1e-5), p["wqkv"], p["bqkv"])
            q, k, v = (t.reshape(b, s, a, h // a).transpose(1, 2).contiguous() for t in qkv.split(h, dim=1))
            score = q @ k.transpose(2, 3).contiguous() / (h // a) ** 0.5
            if cfg.causal:
                score = score.masked_fill(torch.ones(s, s).triu(1).bool(), float("-inf"))
            x = x + F.linear((score.softmax(-1) @ v).transpose(1, 2).reshape(b * s, h), p["wo"], p["bo"])
            u = F.linear(F.layer_norm(x, (h,), p["ln2_g"], p["ln2_b"], cfg.ln_eps or 1e-5), p["w1"], p["b1"])
            x = x + F.linear(F.gelu(u, approximate="tanh"), p["w2"], p["b2"])
        logits = F.linear(F.layer_norm(x, (h,), gamma, beta, 1e-5), table)
        total = total + F.cross_entropy(logits, tgt, ignore_index=-1, reduction="sum", label_smoothing=0.1)
    (total / count).backward()
    return float(total.detach()), [{k: v.grad for k, v in l.items()} for l in layers], table.grad, places.grad, gamma.grad, beta.grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_mini_batch_of_a_whole_model(dtype):
    cfg = synth.StageConfig("whole", 2, 128, 2, 64, 2, 3, 512, True, dtype, 0.05, seed=5)
    T, h, M = cfg.tokens, cfg.hidden, cfg.n_micro_batches
    r = np.random.default_rng(11)
    near = lambda shape, std, mean=0.0: torch.from_numpy(mean + std * r.standard_normal(shape)).to(DT[dtype])  # noqa: E731
    table, places, gamma, beta = near((VOCAB, h), 0.3), near((PLACES, h), 0.1), near((h,), 0.1, 1.0), near((h,), 0.1)
    layers = synth.make_params(cfg, perturb=0.05)
    tokens = [torch.from_numpy((VOCAB * r.random(T) ** 3).astype(np.int64)) for _ in range(M)]
    targets = [torch.from_numpy(r.integers(0, VOCAB, T)) for _ in range(M)]
    for m in range(M):
        tokens[m][-5:], targets[m][-6:] = -1, -1   # padding, and the token before it
    count = sum(int((t >= 0).sum()) for t in targets)

    dev = lambda t: t.cuda()  # noqa: E731
    E, P, g, b = dev(table), dev(places), dev(gamma), dev(beta)
    st = B.Stage(cfg, "cuda:0")
    st.set_params(layers)
    st.grad_accum_reset()
    dE, dP, dg, db = (torch.zeros(t.shape, device="cuda") for t in (table, places, gamma, beta))
    new = lambda *shape, dtype=DT[dtype]: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    x, y, n, dn, dy, dx, none = (new(T, h) for _ in range(7))
    none.zero_()
    logits, bias = new(T, VOCAB), torch.zeros(VOCAB, dtype=DT[dtype], device="cuda")
    stats, loss, out2 = new(2 * T, dtype=torch.float32), new(T, dtype=torch.float32), new(2, dtype=torch.float32)
    partial = new(B.colreduce_scratch_bytes(T, 2 * h) // 4, dtype=torch.float32)
    scratch = new(max(B.embedding_bwd_scratch_bytes(T, h, v) for v in (VOCAB, PLACES)), dtype=torch.uint8)
    scale = torch.full((1,), 1.0 / count, device="cuda")
    total = 0.0
    for m in range(M):
        tok, tgt = dev(tokens[m]), dev(targets[m])
        B.op_embedding_fwd(tok, E, x, pos_table=P, seq_len=cfg.seq_len)
        st.forward(m, x, y)
        B.op_layernorm_fwd(y, g, b, n, stats)
        B.op_gemm(B.OP_FWD, 0, n, E, logits, bias=bias, M=T, N=VOCAB, K=h)
        B.op_cross_entropy(logits, tgt, loss, dlogits=logits, out2=out2, label_smoothing=0.1, scale=scale)   # in place
        B.op_gemm(B.OP_DGRAD, 0, logits, E, dn, M=T, N=h, K=VOCAB)
        B.op_gemm(B.OP_WGRAD, 0, logits, n, dE, M=VOCAB, N=h, K=T)
        B.op_layernorm_bwd(dn, y, stats, g, none, dy, dg, db, partial)
        st.backward_recompute(m, dy, dx)
        B.op_embedding_bwd(tok, dx, dE, scratch)
        B.op_embedding_bwd(None, dx, dP, scratch, seq_len=cfg.seq_len)
        total += float(out2[0])
        assert float(out2[1]) == T - 6
    st.grad_flush()

    ref = _reference(cfg, layers, table, places, gamma, beta, tokens, targets, count)
    tol = TOL[dtype]
    assert abs(total - ref[0]) <= tol * ref[0]
    off, num, den = {}, 0.0, 0.0

    def compare(name, got, want):
        nonlocal num, den
        got = got.detach().cpu().double().reshape(want.shape)
        off[name] = float((got - want).norm() / want.norm())
        num, den = num + float((got - want).square().sum()), den + float(want.square().sum())
    for l in range(cfg.n_layers):
        for k in B.PARAM_NAMES:
            compare(f"{l}.{k}", st.grad_view(l, k), ref[1][l][k])
    for k, got, want in (("table", dE, ref[2]), ("places", dP, ref[3]), ("gamma", dg, ref[4]), ("beta", db, ref[5])):
        compare(k, got, want)
    off["all"] = (num / den) ** 0.5
    assert all(v <= tol for v in off.values()), off
    assert bool((dP[cfg.seq_len:] == 0).all())

    # the norm over the stage's buffer and the ends' tensors, and all of them clipped to half of it
    every = B.TensorList([st.grads, dE, dP, dg, db])
    sum_sq, bad = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    room = torch.empty(B.grad_norm_scratch_bytes(every), dtype=torch.uint8, device="cuda")
    before = [t.clone() for t in every.tensors]
    B.op_grad_norm(every, sum_sq, bad, room)
    own = torch.zeros(2, device="cuda")
    st.grad_stats(own)
    assert float(bad) == 0.0 and abs(float(sum_sq) ** 0.5 - den ** 0.5) <= tol * den ** 0.5
    assert abs(float(own[0]) - float(st.grads.double().square().sum())) <= 1e-6 * float(own[0])
    most = 0.5 * den ** 0.5
    B.op_grad_clip(every, every, sum_sq, most)
    left = sum(float(t.double().square().sum()) for t in every.tensors) ** 0.5
    assert abs(left - most) <= 1e-5 * most   # fp32 products of a factor rounded to fp32, and the norm's own 1e-6
    for t, o in zip(every.tensors, before):
        torch.testing.assert_close(t.double(), o.double() * (most / (float(sum_sq) ** 0.5 + 1e-6)), rtol=3 * 2.0 ** -24, atol=0.0)
    # nonfinite counts into the update's flag
    master, m1, m2 = st.params.float(), torch.zeros_like(st.grads), torch.zeros_like(st.grads)
    kept = master.clone()
    dE[3, 3] = float("inf")
    B.op_grad_norm(every, sum_sq, bad, room)
    st.adam_step(master, m1, m2, 1, lr=1e-3, skip=bad)
    assert float(bad) == 1.0 and torch.equal(master, kept)
    dE[3, 3] = 0.0
    B.op_grad_norm(every, sum_sq, bad, room)
    st.adam_step(master, m1, m2, 1, lr=1e-3, skip=bad)
    assert float(bad) == 0.0 and not torch.equal(master, kept)
    st.close()
