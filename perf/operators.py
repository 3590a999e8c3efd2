"""The operators at the two ends of a pipeline and the norm that joins its stages, as a program that trains a whole model
with this library calls them: the first stage's embedding and its gradient, the last stage's loss with its gradient, and
the global gradient norm with clipping.

Kinds of a case:
  embedding       scale * table[token] + positions[position], rounded once
  embedding_grad  the table's fp32 gradient, rows of one token summed: written by the first micro-batch, added to by the rest
  loss            cross entropy over the vocabulary, label smoothing and uncounted rows, with the gradient of the logits or without
  clip            sum of squares and number of non-finite entries over many tensors, then those tensors, clipped, side by
                  side in one buffer (the bucket that is exchanged)
Types: bf16 or fp32 tensors, 32- or 64-bit ids.  An id outside its table is none: padding.
"""
import math
import random

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
INDEX = {"i32": torch.int32, "i64": torch.int64}


def _embedding(dtype, index, rows, seq, hidden, vocab, positions, scale=1.0, pad=0.0):
    return {"kind": "embedding", "dtype": dtype, "index": index, "rows": rows, "seq": seq, "hidden": hidden, "vocab": vocab, "positions": positions,
            "scale": scale, "pad": pad}


def _embedding_grad(dtype, index, rows, seq, hidden, vocab, of="tokens", scale=1.0, pad=0.0, micro_batches=1):
    return {"kind": "embedding_grad", "dtype": dtype, "index": index, "rows": rows, "seq": seq, "hidden": hidden, "vocab": vocab, "of": of,
            "scale": scale, "pad": pad, "micro_batches": micro_batches}


def _loss(dtype, index, rows, vocab, pitch, smoothing=0.0, ignored=0.0, masked=0, grad=True):
    return {"kind": "loss", "dtype": dtype, "index": index, "rows": rows, "vocab": vocab, "pitch": pitch, "smoothing": smoothing, "ignored": ignored,
            "masked": masked, "grad": grad}


def _clip(dtype, to, tensors, elements, mix, ratio, broken=0):
    return {"kind": "clip", "dtype": dtype, "to": to, "tensors": tensors, "elements": elements, "mix": mix, "ratio": ratio, "broken": broken}


def listed():
    return [
        # the smallest configuration's micro-batch, 2 sequences of 64 tokens, 128 wide: a launch and its latency
        {"name": "embedding-tiny-fp32", **_embedding("f32", "i64", 128, 64, 128, 1000, "sequence")},
        # the widest configuration (8192) on eight sequences of 2048 tokens, padded at their ends
        {"name": "embedding-8192-wide", **_embedding("bf16", "i32", 16384, 2048, 8192, 50257, "sequence", 1.0, 0.1)},
        # a ragged batch of odd width whose positions' table learns: every position is the sum over the sequences
        {"name": "embedding-grad-positions-odd", **_embedding_grad("f32", "i64", 1001, 91, 333, 512, "positions", 1.0)},
        # a BERT-large-shaped mini-batch: two micro-batches of 8 sequences of 512 tokens, the second adds to the first
        {"name": "embedding-grad-1024-wide", **_embedding_grad("bf16", "i64", 4096, 512, 1024, 30522, "tokens", 32.0, 0.1, 2)},
        # the widest configuration's table, 1.6 GB of fp32 gradient, from eight sequences of 2048 tokens
        {"name": "embedding-grad-8192-wide", **_embedding_grad("bf16", "i32", 16384, 2048, 8192, 50257)},
        # the smallest micro-batch's loss, fp32
        {"name": "loss-tiny-fp32", **_loss("f32", "i64", 128, 1000, 1000)},
        # a micro-batch of four sequences of 1024 tokens, rows of the logits padded to whole tiles of the product before, a
        # part of the rows without a target (prompt and padding)
        {"name": "loss-4096-rows", **_loss("bf16", "i64", 4096, 50257, 50304, 0.0, 0.15)},
        # odd rows of an odd vocabulary side by side, so that no row begins where the one before did; label smoothing
        {"name": "loss-odd-smoothing", **_loss("bf16", "i32", 1023, 30523, 30523, 0.1)},
        # evaluation: losses alone, in fp32, some of the vocabulary masked
        {"name": "loss-evaluation-fp32", **_loss("f32", "i64", 2048, 50257, 50304, 0.0, 0.1, 47, False)},
        # a long micro-batch over a large vocabulary: 2.1 GB of logits and as much of gradient
        {"name": "loss-large-vocabulary", **_loss("bf16", "i64", 8192, 128000, 128000, 0.0, 0.05)},
        # the twelve parameter tensors of the smallest configuration's layer
        {"name": "clip-layer-128-wide", **_clip("f32", "f32", 12, 198272, 1, 2.0)},
        # a 2.5B-shaped stage of four layers with the token table at its end, 274 M entries, into a bf16 bucket
        {"name": "clip-stage-and-table", **_clip("f32", "bf16", 50, 273650304, 2, 4.0)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some(rng, lo, hi, mult):
    """A size in [lo, hi], spread over its logarithm: two in three are multiples of `mult`, the others anything."""
    v = _log(rng, lo, hi)
    return max(mult, v // mult * mult) if rng.random() < 2 / 3 else v


def draw(rng):
    kind = rng.choice(("embedding", "embedding_grad", "embedding_grad", "loss", "loss", "loss", "clip"))
    dtype, index = rng.choice(("f32", "bf16", "bf16")), rng.choice(("i32", "i64"))
    if kind in ("embedding", "embedding_grad"):
        rows, hidden, vocab = _log(rng, 1, 16384), _some(rng, 8, 8192, 64), _log(rng, 2, 130000)
        if dtype == "f32":
            rows, hidden = min(rows, 8192), min(hidden, 4096)
        vocab = max(2, min(vocab, 50257 * 8192 // hidden))
        seq = max(1, min(rows, _log(rng, 16, 2048)))
        scale, pad = rng.choice((1.0, math.sqrt(hidden))), rng.choice((0.0, 0.0, 0.2))
        if kind == "embedding":
            return _embedding(dtype, index, rows, seq, hidden, vocab, rng.choice(("none", "sequence", "given")), scale, pad)
        if rng.random() < 0.25:
            return _embedding_grad(dtype, index, rows, seq, hidden, seq + rng.choice((0, 0, 100)), "positions", 1.0)
        return _embedding_grad(dtype, index, rows, seq, hidden, vocab, "tokens", scale, pad, rng.choice((1, 1, 2)))
    if kind == "loss":
        rows, vocab = _log(rng, 1, 8192), _some(rng, 2, 130000, 16)
        rows = max(1, min(rows, 2_000_000_000 // SIZE[dtype] // vocab))
        pitch = rng.choice((vocab, -(-vocab // 64) * 64, vocab + 3))
        return _loss(dtype, index, rows, vocab, pitch, rng.choice((0.0, 0.0, 0.1)), rng.choice((0.0, 0.2)), 0, rng.random() < 0.75)
    tensors = rng.randint(1, 60)
    return _clip(dtype, rng.choice((dtype, "bf16")), tensors, max(tensors, _log(rng, 1000, 250_000_000)), rng.randint(0, 10 ** 6), rng.choice((0.5, 3.0)),
                 rng.choice((0, 0, 0, 2)))


# ---- inputs -------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, device="cuda", dtype=DT[dtype]).normal_(0.0, std, generator=g)


def _weights(vocab):
    """How often tokens occur: as one over their rank, nearly."""
    return 1.0 / (torch.arange(vocab, dtype=torch.float64) + 2.7)


def _tokens(g, c):
    """Ids by rank spread over the table; from a sequence's own length on, -1."""
    rows, vocab, seq = c["rows"], c["vocab"], c["seq"]
    cdf = _weights(vocab).cuda().cumsum(0)
    rank = torch.searchsorted(cdf, torch.rand(rows, device="cuda", dtype=torch.float64, generator=g) * cdf[-1]).clamp(max=vocab - 1)
    ids = torch.randperm(vocab, device="cuda", generator=g)[rank]
    if c["pad"]:
        at = torch.arange(rows, device="cuda")
        n = -(-rows // seq)
        length = (seq * (1 - 2 * c["pad"] * torch.rand(n, device="cuda", generator=g))).ceil().long()
        ids = torch.where(at % seq < length[at // seq], ids, -1)
    return ids.to(INDEX[c["index"]])


def _parts(c):
    """The tensors' sizes: a few large ones, many small ones, as a model's are."""
    r = random.Random(c["mix"])
    w = [math.exp(r.uniform(0.0, 9.0)) for _ in range(c["tensors"])]
    left = c["elements"] - c["tensors"]
    sizes = [1 + int(left * x / sum(w)) for x in w]
    sizes[0] += c["elements"] - sum(sizes)
    return sizes


def _inputs(c, seed):
    g = _gen(seed)
    if c["kind"] == "embedding":
        s = {"ids": _tokens(g, c), "table": _normal(g, (c["vocab"], c["hidden"]), c["dtype"], 0.02), "places": None, "given": None}
        if c["positions"] != "none":
            s["places"] = _normal(g, (c["seq"], c["hidden"]), c["dtype"], 0.02)
        if c["positions"] == "given":
            s["given"] = torch.randint(0, c["seq"], (c["rows"],), device="cuda", generator=g).to(INDEX[c["index"]])
        return s
    if c["kind"] == "embedding_grad":
        n = c["micro_batches"]
        return {"ids": [_tokens(g, c) if c["of"] == "tokens" else None for _ in range(n)], "dy": [_normal(g, (c["rows"], c["hidden"]), c["dtype"]) for _ in range(n)]}
    if c["kind"] == "loss":
        logits = _normal(g, (c["rows"], c["pitch"]), c["dtype"], 2.0)
        target = torch.randint(0, c["vocab"], (c["rows"],), device="cuda", generator=g)
        at = torch.arange(c["rows"], device="cuda")
        logits[at, target] += 4.0  # a model that has learnt something
        if c["masked"]:  # the last entries are no tokens: those that are targets move to the first
            logits[:, c["vocab"] - c["masked"]:c["vocab"]] = -math.inf
            target = torch.where(target >= c["vocab"] - c["masked"], 0, target)
        if c["ignored"]:
            target = torch.where(torch.rand(c["rows"], device="cuda", generator=g) < c["ignored"], -100, target)
        counted = (target >= 0).sum().clamp(min=1)
        return {"logits": logits[:, :c["vocab"]], "target": target.to(INDEX[c["index"]]), "scale": (1.0 / counted).float().reshape(1)}
    grads = [_normal(g, (k,), c["dtype"], 1e-3 * 2.0 ** (i % 5)) for i, k in enumerate(_parts(c))]
    for i in range(c["broken"]):
        grads[(i * 7) % len(grads)][-1] = (math.inf, math.nan)[i % 2]
    # the norm is about `ratio` times what is allowed
    most = math.sqrt(sum(k * (1e-3 * 2.0 ** (i % 5)) ** 2 for i, k in enumerate(_parts(c)))) / c["ratio"]
    return {"grads": grads, "most": most}


def prepare(case, seed):
    c = dict(case)
    s = {"case": c, **_inputs(c, seed)}
    dev = {"device": "cuda"}
    if c["kind"] == "embedding":
        s["out"] = torch.empty((c["rows"], c["hidden"]), dtype=DT[c["dtype"]], **dev)
    elif c["kind"] == "embedding_grad":
        s["grad"] = torch.empty((c["vocab"], c["hidden"]), dtype=torch.float32, **dev)
    elif c["kind"] == "loss":
        s["loss"], s["sums"] = torch.empty(c["rows"], **dev), torch.empty(2, **dev)
        s["dlogits"] = torch.empty((c["rows"], c["pitch"]), dtype=DT[c["dtype"]], **dev)[:, :c["vocab"]] if c["grad"] else None
    else:
        s["bucket"] = torch.empty(c["elements"], dtype=DT[c["to"]], **dev)
        s["sum"], s["bad"] = torch.empty(1, dtype=torch.float64, **dev), torch.empty(1, **dev)
    if own:  # the workspaces and the list of tensors that a program keeps
        from paper_2111_04007_amd import binding as B
        if c["kind"] == "embedding_grad":
            s["scratch"] = torch.empty(B.embedding_bwd_scratch_bytes(c["rows"], c["hidden"], c["vocab"]), dtype=torch.uint8, **dev)
        elif c["kind"] == "clip":
            s["from"], s["into"] = B.TensorList(s["grads"]), B.TensorList(list(s["bucket"].split(_parts(c))))
            s["scratch"] = torch.empty(B.grad_norm_scratch_bytes(s["from"]), dtype=torch.uint8, **dev)
    return s


# ---- the operators in their plain form ----------------------------------------------------------------------

def _rows_of(ids, vocab):
    """(which ids are in the table, ids with the others at 0)"""
    ok = (ids >= 0) & (ids < vocab)
    return ok, torch.where(ok, ids, 0).long()


def _plain_embedding(s, c):
    ok, at = _rows_of(s["ids"], c["vocab"])
    x = torch.where(ok[:, None], c["scale"] * s["table"][at].float(), 0.0)
    if c["positions"] != "none":
        where = s["given"].long() if c["positions"] == "given" else torch.arange(c["rows"], device=x.device) % c["seq"]
        x = x + s["places"][where].float()
    return x.to(DT[c["dtype"]])


def _plain_add(grad, ids, dy, c):
    if ids is None:
        ids = torch.arange(c["rows"], device=dy.device) % c["seq"]
    ok, at = _rows_of(ids, c["vocab"])
    return grad.index_add_(0, at, torch.where(ok[:, None], c["scale"] * dy.float(), 0.0))


def _plain_loss(s, c):
    x, e = s["logits"].float(), c["smoothing"]
    ok, y = _rows_of(s["target"], c["vocab"])
    m = x.amax(1, keepdim=True)
    p = (x - m).exp()
    total = p.sum(1, keepdim=True)
    log = total.log() + m
    loss = (total.log() + (m - x.gather(1, y[:, None])))[:, 0]
    if e:
        loss = (1 - e) * loss + e * (log[:, 0] - x.mean(1))
    loss = torch.where(ok, loss, 0.0)
    sums = torch.stack([loss.double().sum(), ok.double().sum()]).float()
    if not c["grad"]:
        return loss, sums
    p = p / total - e / c["vocab"]
    p.scatter_add_(1, y[:, None], p.new_full((c["rows"], 1), e - 1))
    return loss, sums, (torch.where(ok[:, None], p, 0.0) * s["scale"]).to(DT[c["dtype"]])


def _plain_clip(s, c):
    fine = [torch.isfinite(t) for t in s["grads"]]
    total = torch.stack([torch.where(f, t, 0).double().square().sum() for t, f in zip(s["grads"], fine)]).sum()
    bad = torch.stack([(~f).sum() for f in fine]).sum()
    by = (s["most"] / (total.sqrt() + 1e-6)).clamp(max=1.0).float()
    return torch.cat([t.float() * by for t in s["grads"]]).to(DT[c["to"]]), total.reshape(1), bad.float().reshape(1)


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["kind"] == "embedding":
            return _plain_embedding(s, c)
        if c["kind"] == "embedding_grad":
            s["grad"].zero_()
            return [_plain_add(s["grad"], ids, dy, c) for ids, dy in zip(s["ids"], s["dy"])][-1]
        return _plain_loss(s, c) if c["kind"] == "loss" else _plain_clip(s, c)
    from paper_2111_04007_amd import binding as B
    if c["kind"] == "embedding":
        B.op_embedding_fwd(s["ids"], s["table"], s["out"], scale=c["scale"], pos_table=s["places"], positions=s["given"], seq_len=c["seq"])
        return s["out"]
    if c["kind"] == "embedding_grad":
        for k, (ids, dy) in enumerate(zip(s["ids"], s["dy"])):
            B.op_embedding_bwd(ids, dy, s["grad"], s["scratch"], scale=c["scale"], accumulate=k > 0, seq_len=c["seq"])
        return s["grad"]
    if c["kind"] == "loss":
        B.op_cross_entropy(s["logits"], s["target"], s["loss"], dlogits=s["dlogits"], out2=s["sums"], label_smoothing=c["smoothing"], scale=s["scale"])
        return (s["loss"], s["sums"], s["dlogits"]) if c["grad"] else (s["loss"], s["sums"])
    B.op_grad_norm(s["from"], s["sum"], s["bad"], s["scratch"])
    B.op_grad_clip(s["into"], s["from"], s["sum"], s["most"], eps=1e-6)
    return s["bucket"], s["sum"], s["bad"]


def _distinct(c):
    """How many rows of the table the tokens are expected to meet."""
    w = _weights(c["vocab"])
    return float((1.0 - (1.0 - w / w.sum()) ** (c["rows"] * (1.0 - c["pad"]))).sum())


def work(case):
    c = case
    if c["kind"] == "clip":
        return {"bytes": c["elements"] * (SIZE[c["dtype"]] + SIZE[c["to"]]), "flops": 3 * c["elements"]}
    index, size = 4 if c["index"] == "i32" else 8, SIZE[c["dtype"]]
    if c["kind"] == "loss":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * size * (2 if c["grad"] else 1) + c["rows"] * (index + 4), "flops": n * (6 if c["grad"] else 4)}
    row = c["rows"] * c["hidden"]
    if c["kind"] == "embedding":
        places = 0 if c["positions"] == "none" else min(c["seq"], c["rows"]) * c["hidden"]
        ids = c["rows"] * index * (2 if c["positions"] == "given" else 1)
        return {"bytes": (row + _distinct(c) * c["hidden"] + places) * size + ids, "flops": 2 * row}
    n = c["micro_batches"]
    ids = c["rows"] * index if c["of"] == "tokens" else 0
    again = 8 * c["hidden"] * _distinct(c) if n > 1 else 0
    return {"bytes": n * (row * size + ids) + 4 * c["vocab"] * c["hidden"] + (n - 1) * again, "flops": 2 * n * row}


# ---- what the outputs are, in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    if c["kind"] == "embedding":
        none = s["table"].new_zeros((1, c["hidden"])).double()  # the row of an id that is none
        table = torch.cat([s["table"].double() * c["scale"], none])
        ids = s["ids"].long()
        out = torch.nn.functional.embedding(torch.where((ids < 0) | (ids >= c["vocab"]), c["vocab"], ids), table)
        if c["positions"] == "given":
            out += torch.nn.functional.embedding(s["given"].long(), s["places"].double())
        elif c["positions"] == "sequence":
            n = -(-c["rows"] // c["seq"])
            out += s["places"].double().repeat(n, 1)[:c["rows"]]
        return out
    if c["kind"] == "embedding_grad":
        grad = torch.zeros((c["vocab"] + 1, c["hidden"]), dtype=torch.float64, device="cuda")
        for ids, dy in zip(s["ids"], s["dy"]):
            if ids is None:
                ids = torch.arange(c["seq"], device="cuda").repeat(-(-c["rows"] // c["seq"]))[:c["rows"]]
            ids = ids.long()
            grad.index_put_((torch.where((ids < 0) | (ids >= c["vocab"]), c["vocab"], ids),), dy.double(), accumulate=True)
        return grad[:-1] * c["scale"]
    if c["kind"] == "loss":
        loss = torch.zeros(c["rows"], dtype=torch.float64, device="cuda")
        dx = torch.empty((c["rows"], c["vocab"]), dtype=torch.float64, device="cuda") if c["grad"] else None
        step = max(1, 100_000_000 // c["vocab"])
        for a in range(0, c["rows"], step):
            logp = torch.log_softmax(s["logits"][a:a + step].double(), 1)
            y = s["target"][a:a + step].long()
            there = (y >= 0) & (y < c["vocab"])
            n = torch.arange(y.numel(), device="cuda")[there]
            want = torch.zeros_like(logp)
            want[there] = c["smoothing"] / c["vocab"]
            want[n, y[there]] += 1 - c["smoothing"]
            loss[a:a + step] = -torch.where(want > 0, want * logp, 0.0).sum(1)
            if c["grad"]:
                dx[a:a + step] = torch.where(there[:, None], logp.exp() - want, 0.0) * s["scale"].double()
        sums = torch.stack([loss.sum(), ((s["target"] >= 0) & (s["target"] < c["vocab"])).sum().double()])
        return (loss, sums, dx) if c["grad"] else (loss, sums)
    whole = torch.cat(s["grads"]).double()
    fine = whole[torch.isfinite(whole)]
    norm = torch.linalg.vector_norm(fine)
    clipped = whole if float(norm) + 1e-6 <= s["most"] else whole * (s["most"] / (norm + 1e-6))
    return clipped, torch.dot(fine, fine).reshape(1), torch.tensor([float(whole.numel() - fine.numel())], dtype=torch.float64, device="cuda")
