"""A mini-batch of a whole small model whose layers turn queries and keys by rotary positions and have a norm before and after each block, a learned gate and a
residual scale, through the library: embedding, products, attention, loss, everything backward, the norm over all gradients, and the AdamW step that clips by
it -- against the same model in fp64 with torch's autograd, and the update against the oracle's on the gradients that the GPU made.  The tolerances are the stage's."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import layer_oracle as L
from paper_2111_04007_amd import binding as B
from tests.parity_util import TOL

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCAB, H, HEADS, S, BATCH, MLP, LAYERS, M = 501, 128, 4, 40, 2, 256, 2, 2
T, D, R = S * BATCH, H // HEADS, 24
ALPHA, BETA, COUNT = 0.9, 0.8, M * (T - 3)
SHAPES = {"table": (VOCAB, H), "first": (H,)}
for k in range(LAYERS):
    SHAPES.update({f"{k}.wqkv": (3 * H, H), f"{k}.bqkv": (3 * H,), f"{k}.wo": (H, H), f"{k}.bo": (H,), f"{k}.post1": (H,), f"{k}.gate1": (1, H), f"{k}.pre2": (H,),
                   f"{k}.w1": (MLP, H), f"{k}.b1": (MLP,), f"{k}.w2": (H, MLP), f"{k}.b2": (H,), f"{k}.post2": (H,), f"{k}.gate2": (1, H), f"{k}.next": (H,)})


def _positions(lengths):
    return torch.cat([torch.arange(S) + 100 * b for b in range(BATCH)]) + lengths


def _reference(p, freq, tokens, targets, starts):
    p = {k: v.double().clone().requires_grad_() for k, v in p.items()}
    f = torch.tensor(list(freq), dtype=torch.float64)
    norm = lambda x, w: x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w  # noqa: E731
    total = 0.0
    for tok, tgt, start in zip(tokens, targets, starts):
        ang = _positions(start)[:, None] * f

        def turn(x):   # [T, HEADS, D], the first R entries
            a, b, rest = x[..., :R // 2], x[..., R // 2:R], x[..., R:]
            c, s = ang.cos()[:, None], ang.sin()[:, None]
            return torch.cat([a * c - b * s, a * s + b * c, rest], 2)
        x = p["table"][tok]
        z = norm(x, p["first"])
        for k in range(LAYERS):
            q, ke, v = (F.linear(z, p[f"{k}.wqkv"], p[f"{k}.bqkv"])).split(H, 1)
            q, ke = turn(q.reshape(T, HEADS, D)), turn(ke.reshape(T, HEADS, D))
            q, ke, v = (t.reshape(BATCH, S, HEADS, D).transpose(1, 2).contiguous() for t in (q, ke, v))
            score = (q @ ke.transpose(2, 3).contiguous() / D ** 0.5).masked_fill(torch.ones(S, S).triu(1).bool(), float("-inf"))
            a = F.linear((score.softmax(-1) @ v).transpose(1, 2).reshape(T, H), p[f"{k}.wo"], p[f"{k}.bo"])
            x = ALPHA * x + BETA * p[f"{k}.gate1"] * norm(a, p[f"{k}.post1"])
            z = norm(x, p[f"{k}.pre2"])
            m = F.linear(F.gelu(F.linear(z, p[f"{k}.w1"], p[f"{k}.b1"]), approximate="tanh"), p[f"{k}.w2"], p[f"{k}.b2"])
            x = ALPHA * x + BETA * p[f"{k}.gate2"] * norm(m, p[f"{k}.post2"])
            z = norm(x, p[f"{k}.next"])
        total = total + F.cross_entropy(F.linear(z, p["table"]), tgt, ignore_index=-1, reduction="sum")
    (total / COUNT).backward()
    return float(total.detach()), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("dtype,bits", [("f32", 32), ("f32", 8), ("bf16", 32), ("bf16", 8)])
def test_mini_batch_and_update(dtype, bits):
    r = np.random.default_rng(17)
    near = lambda shape, std, mean=0.0: torch.from_numpy(mean + std * r.standard_normal(shape)).to(DT[dtype])  # noqa: E731
    std = {"table": 0.5}
    params = {k: near(s, std.get(k, 0.1 if len(s) == 1 or "gate" in k else 0.08), 1.0 if k.split(".")[-1] in ("first", "post1", "pre2", "post2", "next", "gate1", "gate2") else 0.0)
              for k, s in SHAPES.items()}
    tokens = [torch.from_numpy(r.integers(0, VOCAB, T)) for _ in range(M)]
    targets = [torch.from_numpy(r.integers(0, VOCAB, T)) for _ in range(M)]
    starts = [0, 333]
    for t in targets:
        t[-3:] = -1
    freq = B.rotary_frequencies(R, 10000.0, "parts", 4.0, 128.0)

    p = {k: v.cuda() for k, v in params.items()}
    g = {k: torch.zeros(s, device="cuda") for k, s in SHAPES.items()}
    new = lambda *shape, dtype=DT[dtype]: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    f32 = lambda *shape: new(*shape, dtype=torch.float32)  # noqa: E731
    table = f32(1024, R)
    B.op_rotary_table(table, freq)
    scratch = new(max(B.residual_norm_bwd_scratch_bytes(T, H, T), B.embedding_bwd_scratch_bytes(T, H, VOCAB)), dtype=torch.uint8)
    partial = f32(B.colreduce_scratch_bytes(T, 3 * H) // 4)
    zero = torch.zeros(VOCAB, dtype=DT[dtype], device="cuda")
    scale = torch.full((1,), 1.0 / COUNT, device="cuda")
    loss, out2, total = f32(T), f32(2), 0.0
    product = lambda x, w, b, out, epi=0, aux=None: B.op_gemm(B.OP_FWD, epi, x, p[w], out, bias=p[b] if isinstance(b, str) else b, aux_out=aux, M=T,  # noqa: E731
                                                               N=p[w].shape[0], K=p[w].shape[1])

    def products_back(dy, w, b, x, dx, epi=0, aux=None):
        n, k = p[w].shape
        B.op_gemm(B.OP_WGRAD, 0, dy, x, g[w], M=n, N=k, K=T)
        B.op_colsum(dy, g[b], partial)
        B.op_gemm(B.OP_DGRAD, epi, dy, p[w], dx, aux_in=aux, M=T, N=k, K=n)

    for tok, tgt, start in zip(tokens, targets, starts):
        tok, tgt, at = tok.cuda(), tgt.cuda(), _positions(start).cuda()
        x, z, first = new(T, H), new(T, H), f32(2, T)
        B.op_embedding_fwd(tok, p["table"], x)
        B.op_residual_norm_fwd(x, z, p["first"], stats=first)
        kept, stream = [], x
        for k in range(LAYERS):
            c = {"z": z, "qkv": new(T, 3 * H), "ctx": new(T, H), "lse": f32(BATCH, HEADS, S), "a": new(T, H), "y1": new(T, H), "z1": new(T, H), "u": new(T, MLP),
                 "g": new(T, MLP), "m": new(T, H), "y2": new(T, H), "z2": new(T, H), **{n: f32(2, T) for n in ("s1", "s2", "p1", "p2")}}
            product(c["z"], f"{k}.wqkv", f"{k}.bqkv", c["qkv"])
            B.op_rotary(c["qkv"].view(T, 3 * HEADS, D)[:, :2 * HEADS], table, positions=at)
            B.op_attention_fwd(c["qkv"], c["ctx"], c["lse"], BATCH, S, HEADS, D, True)
            product(c["ctx"], f"{k}.wo", f"{k}.bo", c["a"])
            B.op_residual_norm_fwd(stream, c["z1"], p[f"{k}.pre2"], branch=c["a"], y=c["y1"], post_weight=p[f"{k}.post1"], gate=p[f"{k}.gate1"], alpha=ALPHA, beta=BETA,
                                   stats=c["s1"], post_stats=c["p1"])
            product(c["z1"], f"{k}.w1", f"{k}.b1", c["g"], 1, c["u"])
            product(c["g"], f"{k}.w2", f"{k}.b2", c["m"])
            B.op_residual_norm_fwd(c["y1"], c["z2"], p[f"{k}.next"], branch=c["m"], y=c["y2"], post_weight=p[f"{k}.post2"], gate=p[f"{k}.gate2"], alpha=ALPHA, beta=BETA,
                                   stats=c["s2"], post_stats=c["p2"])
            kept.append(c)
            stream, z = c["y2"], c["z2"]
        logits, dz, dy = new(T, VOCAB), new(T, H), None
        product(z, "table", zero, logits)
        B.op_cross_entropy(logits, tgt, loss, dlogits=logits, out2=out2, scale=scale)
        total += float(out2[0])
        B.op_gemm(B.OP_DGRAD, 0, logits, p["table"], dz, M=T, N=H, K=VOCAB)
        B.op_gemm(B.OP_WGRAD, 0, logits, z, g["table"], M=VOCAB, N=H, K=T)
        for k in reversed(range(LAYERS)):
            c, dx, db = kept[k], new(T, H), new(T, H)
            B.op_residual_norm_bwd(dz, c["y2"], c["s2"], p[f"{k}.next"], dx, scratch, dy=dy, branch=c["m"], dbranch=db, post_weight=p[f"{k}.post2"], post_stats=c["p2"],
                                   gate=p[f"{k}.gate2"], alpha=ALPHA, beta=BETA, dweight=g[f"{k}.next"], dpost_weight=g[f"{k}.post2"], dgate=g[f"{k}.gate2"])
            du = new(T, MLP)
            products_back(db, f"{k}.w2", f"{k}.b2", c["g"], du, 3, c["u"])
            products_back(du, f"{k}.w1", f"{k}.b1", c["z1"], dz)
            B.op_residual_norm_bwd(dz, c["y1"], c["s1"], p[f"{k}.pre2"], dx, scratch, dy=dx, branch=c["a"], dbranch=db, post_weight=p[f"{k}.post1"], post_stats=c["p1"],
                                   gate=p[f"{k}.gate1"], alpha=ALPHA, beta=BETA, dweight=g[f"{k}.pre2"], dpost_weight=g[f"{k}.post1"], dgate=g[f"{k}.gate1"])
            dctx, dqkv = new(T, H), new(T, 3 * H)
            products_back(db, f"{k}.wo", f"{k}.bo", c["ctx"], dctx)
            B.op_attention_bwd(c["qkv"], c["ctx"], c["lse"], dctx, dqkv, f32(BATCH, HEADS, S), BATCH, S, HEADS, D, True)
            B.op_rotary(dqkv.view(T, 3 * HEADS, D)[:, :2 * HEADS], table, positions=at, transpose=True)
            products_back(dqkv, f"{k}.wqkv", f"{k}.bqkv", c["z"], dz)
            dy = dx
        B.op_residual_norm_bwd(dz, x, first, p["first"], dz, scratch, dy=dy, dweight=g["first"])
        B.op_embedding_bwd(tok, dz, g["table"], scratch)

    want_total, want = _reference(params, freq, tokens, targets, starts)
    tol = TOL[dtype]
    assert abs(total - want_total) <= tol * want_total
    off = {k: float((g[k].cpu().double() - w).norm() / w.norm()) for k, w in want.items()}
    assert all(v <= tol for v in off.values()), off

    # the update, clipped to half of the norm, on the gradients as they are
    names = list(p)
    plist, glist = B.TensorList([p[k] for k in names]), B.TensorList([g[k] for k in names])
    state = B.AdamWState(plist, bits, [float(p[k].dim() == 2 and "gate" not in k) for k in names])
    sum_sq, bad = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    B.op_grad_norm(glist, sum_sq, bad, torch.empty(B.grad_norm_scratch_bytes(glist), dtype=torch.uint8, device="cuda"))
    norm = float(sum_sq) ** 0.5
    assert abs(norm - sum(float(w.square().sum()) for w in want.values()) ** 0.5) <= tol * norm
    old = {k: v.clone() for k, v in p.items()}
    B.op_adamw(plist, glist, state, 1, 1e-2, weight_decay=0.1, sum_sq=sum_sq, max_norm=norm / 2, skip=bad)
    for i, k in enumerate(names):
        c = 0.5 * norm / (norm + 1e-6)
        w, _, _ = L.adamw(old[k].cpu().double().numpy(), c * g[k].cpu().double().numpy(), 0.0, 0.0, 1, 1e-2, 0.9, 0.999, 1e-8, 0.1 if p[k].dim() == 2 and "gate" not in k else 0.0)
        got = p[k].cpu().double().numpy()
        # a rounding of the type, fp32 roundings of w and of an update of at most 1e-2
        assert (np.abs(got - w) <= torch.finfo(DT[dtype]).eps / 2 * np.abs(w) * (1 if dtype == "bf16" else 0) + 2.0 ** -24 * (4 * np.abs(w) + 30 * 1e-2)).all(), k
    # an overflow anywhere leaves everything as it is
    kept = [t.clone() for t in p.values()]
    g["0.w1"][3, 3] = float("inf")
    B.op_grad_norm(glist, sum_sq, bad, torch.empty(B.grad_norm_scratch_bytes(glist), dtype=torch.uint8, device="cuda"))
    B.op_adamw(plist, glist, state, 2, 1e-2, weight_decay=0.1, sum_sq=sum_sq, max_norm=norm / 2, skip=bad)
    assert float(bad) == 1.0 and all(torch.equal(a, b) for a, b in zip(kept, p.values()))
