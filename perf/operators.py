"""Workloads of the training operators: embedding rows, attention over sampled blocks, softmax cross entropy.

Each case is one pass of one operator, in the sizes that mini-batch training on the graphs of ``workloads/`` meets:

* ``lookup``       rows of an embedding table, scaled, by node id
* ``lookup_grad``  the table's gradient from the rows' gradients, ids repeating (dense table, or its touched rows)
* ``attend``       softmax attention of a block's destinations over their sampled neighbours (serving: forward only)
* ``attend_train`` the same, forward and backward
* ``xent``         softmax cross entropy of hidden rows against every row of a table, loss and both gradients

``run`` computes a pass in elementary tensor operations (32 bits, rounded once), or, where ``own`` is true, by the
package's kernels.  ``exact`` is the same from the definition in 64 bits.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
_TYPES = {F32: torch.float32, BF16: torch.bfloat16}
_BYTES = {F32: 4, BF16: 2}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # input nodes of one batch of 64 seeds on the small bag-of-words graph: wide odd rows, latency counts
        dict(name="lookup_small_wide", op="lookup", table=2708, dim=1433, ids=1100, type=F32, out=F32, scale=1.0),
        # the 2 M input nodes of a batch of 8,192 seeds, sqrt(d) scaling, bf16 table
        dict(name="lookup_batch_large", op="lookup", table=2449029, dim=128, ids=2031616, type=BF16, out=BF16, scale=11.313708),
        # endpoints of the positive and negative pairs of a link-prediction step: hubs repeat, dense f32 gradient
        dict(name="lookup_grad_dense", op="lookup_grad", table=169343, dim=128, ids=40961, type=F32, out=F32, scale=1.0, sparse=False),
        # input nodes of several accumulated batches on the largest graph: only the touched rows are produced
        dict(name="lookup_grad_touched", op="lookup_grad", table=1 << 26, dim=128, ids=2031616, type=BF16, out=BF16, scale=11.313708, sparse=True),
        # serving a handful of seeds: one hop of 5 neighbours
        dict(name="attend_few", op="attend", dst=64, src=384, longest=5, skew=0.2, empty=0.05, masked=0.0, heads=4, kv_heads=4, head_dim=16, type=F32),
        # input-side block of a batch of 8,192 seeds (fan-out 20)
        dict(name="attend_batch_large", op="attend", dst=262144, src=2031616, longest=20, skew=0.2, empty=0.02, masked=0.0, heads=4, kv_heads=4, head_dim=32, type=BF16),
        # the blocks of a batch of 1,024 seeds with f32 features
        dict(name="attend_train_mid", op="attend_train", dst=26011, src=97003, longest=15, skew=0.2, empty=0.02, masked=0.0, heads=8, kv_heads=8, head_dim=16, type=F32),
        # whole neighbourhoods instead of samples: hub rows of thousands, shared key/value heads, masked edges
        dict(name="attend_train_hubs", op="attend_train", dst=4097, src=60013, longest=20011, skew=60.0, empty=0.05, masked=0.1, heads=8, kv_heads=2, head_dim=24, type=BF16),
        # input-side block of a batch of 8,192 seeds, training
        dict(name="attend_train_large", op="attend_train", dst=262144, src=2031616, longest=20, skew=0.2, empty=0.02, masked=0.0, heads=4, kv_heads=4, head_dim=32, type=BF16),
        # node classification: few classes, many rows
        dict(name="xent_classes", op="xent", rows=4096, vocab=47, dim=128, scale=1.0, ignored=0.05, type=BF16),
        # predicting a context node among all nodes, odd feature width
        dict(name="xent_nodes_mid", op="xent", rows=1024, vocab=169343, dim=100, scale=1.0, ignored=0.05, type=BF16),
        # the same with the largest batch
        dict(name="xent_nodes_large", op="xent", rows=8192, vocab=169343, dim=128, scale=1.0, ignored=0.02, type=BF16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "attend", "attend_train", "xent"])
    kind = rng.choice([F32, BF16])
    if op in ("lookup", "lookup_grad"):
        dim = rng.choice([_log_int(rng, 8, 1433), 8 * _log_int(rng, 2, 64), 128])
        ids = min(_log_int(rng, 64, 2031616), 260000000 // dim)
        out = rng.choice([kind, F32, BF16])
        scale = rng.choice([1.0, math.sqrt(dim)])
        if op == "lookup":
            return dict(op=op, table=min(_log_int(rng, 64, 2449029), 313000000 // dim), dim=dim, ids=ids, type=kind, out=out, scale=scale)
        sparse = rng.random() < 0.5
        table = _log_int(rng, 64, 1 << 26) if sparse else min(_log_int(rng, 64, 736389), 200000000 // dim)
        return dict(op=op, table=table, dim=dim, ids=ids, type=kind, out=out, scale=scale, sparse=sparse)
    if op in ("attend", "attend_train"):
        head_dim = rng.choice([8, 16, 20, 24, 32, 33, 64, 128])
        kv = rng.choice([h for h in (1, 2, 4, 8) if h * head_dim <= 256])
        heads = kv * rng.choice([1, 1, 2, 4])
        full = rng.random() < 0.25          # whole neighbourhoods: few long rows among many short ones
        width = heads * head_dim
        if full:
            dst, longest, skew = _log_int(rng, 64, 8192), _log_int(rng, 64, 20011), 30.0
            dst = max(64, min(dst, 300000000 // (width * max(1, longest // 30))))
        else:
            # a single neighbour's probability is 1 whatever its score: training draws have rows of several
            dst, longest, skew = _log_int(rng, 1, 262144), rng.randint(1 if op == "attend" else 4, 32), 0.2
            dst = max(1 if op == "attend" else 8, min(dst, 500000000 // (width * longest)))
        src = dst + min(_log_int(rng, 1, 2000000), 200000000 // (kv * head_dim))
        return dict(op=op, dst=dst, src=src, longest=longest, skew=skew, empty=rng.choice([0.0, 0.05, 0.3]), masked=rng.choice([0.0, 0.1]),
                    heads=heads, kv_heads=kv, head_dim=head_dim, type=kind)
    rows, vocab, dim = _log_int(rng, 1, 8192), _log_int(rng, 2, 2449029), rng.choice([rng.randint(16, 256), 64, 128, 256])
    vocab = max(2, min(vocab, 170000000000 // (rows * dim), 1380000000 // rows))
    return dict(op="xent", rows=rows, vocab=vocab, dim=dim, scale=rng.choice([1.0, 0.5]), ignored=rng.choice([0.0, 0.05]), type=BF16)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _skewed(g, n, top):
    """n ids below `top`, low ones far more often (the endpoint distribution of a power-law graph)."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (u * u * top).long().clamp_(max=top - 1).int()


def prepare(case, seed):
    g, t = _generator(seed), _TYPES[case["type"]]
    op = case["op"]
    if op == "lookup":
        return dict(case=case, table=_normal(g, (case["table"], case["dim"]), t),
                    ids=torch.randint(0, case["table"], (case["ids"],), generator=g, device="cuda", dtype=torch.int32))
    if op == "lookup_grad":
        return dict(case=case, ids=_skewed(g, case["ids"], case["table"]), dout=_normal(g, (case["ids"], case["dim"]), t))
    if op in ("attend", "attend_train"):
        n = case["dst"]
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        length = ((case["longest"] + 1) * u ** case["skew"]).long().clamp_(max=case["longest"])
        length[torch.rand(n, generator=g, device="cuda") < case["empty"]] = 0
        indptr = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        indptr[1:] = torch.cumsum(length, 0).int()
        edges = int(indptr[-1])
        indices = _skewed(g, edges, case["src"])
        if case["masked"]:
            indices[torch.rand(edges, generator=g, device="cuda") < case["masked"]] = -1
        # a fixed permutation puts the frequent sources anywhere in the list
        perm = torch.randperm(case["src"], generator=g, device="cuda").int()
        indices = torch.where(indices >= 0, perm[indices.clamp(min=0).long()], indices) if edges else indices
        s = dict(case=case, indptr=indptr, indices=indices,
                 q=_normal(g, (n, case["heads"], case["head_dim"]), t),
                 k=_normal(g, (case["src"], case["kv_heads"], case["head_dim"]), t),
                 v=_normal(g, (case["src"], case["kv_heads"], case["head_dim"]), t))
        if op == "attend_train":
            s["dout"] = _normal(g, (n, case["heads"], case["head_dim"]), t)
        return s
    labels = _skewed(g, case["rows"], case["vocab"])
    labels[torch.rand(case["rows"], generator=g, device="cuda") < case["ignored"]] = -1
    return dict(case=case, hidden=_normal(g, (case["rows"], case["dim"]), t),
                table=_normal(g, (case["vocab"], case["dim"]), t, 2.0 / math.sqrt(case["dim"])), labels=labels,
                dloss=torch.full((case["rows"],), 1.0 / case["rows"], device="cuda"))


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_lookup(s):
    c = s["case"]
    return (s["table"][s["ids"].long()].float() * c["scale"]).to(_TYPES[c["out"]])


def _plain_lookup_grad(s):
    c = s["case"]
    rows = s["dout"].float() * c["scale"]
    if not c["sparse"]:
        return torch.zeros(c["table"], c["dim"], device="cuda").index_add_(0, s["ids"].long(), rows).to(_TYPES[c["out"]])
    unique, place = torch.unique(s["ids"], return_inverse=True)
    grad = torch.zeros(c["ids"], c["dim"], device="cuda").index_add_(0, place, rows).to(_TYPES[c["out"]])
    ids = torch.full((c["ids"],), -1, dtype=torch.int32, device="cuda")
    ids[:unique.numel()] = unique
    return dict(ids=ids, count=torch.tensor([unique.numel()], dtype=torch.int32, device="cuda"), grad=grad)


def _softmax_over_rows(score, dst, n):
    """Probabilities of the edges of each row, and log-sum-exp per row (-inf where a row has no edge)."""
    top = torch.full((n, score.shape[1]), -math.inf, dtype=score.dtype, device=score.device)
    top = top.scatter_reduce(0, dst[:, None].expand_as(score), score, "amax")
    weight = torch.exp(score - top[dst])
    total = torch.zeros_like(top).index_add_(0, dst, weight)
    return weight / total[dst], top + torch.log(total)


def _plain_attend(s, train):
    c, t = s["case"], _TYPES[s["case"]["type"]]
    n, group, scale = c["dst"], c["heads"] // c["kv_heads"], 1.0 / math.sqrt(c["head_dim"])
    keep = s["indices"] >= 0
    dst = torch.repeat_interleave(torch.arange(n, device="cuda"), (s["indptr"][1:] - s["indptr"][:-1]).long())[keep]
    src = s["indices"][keep].long()
    q = s["q"].float()[dst]
    k = s["k"][src].float().repeat_interleave(group, 1)
    v = s["v"][src].float().repeat_interleave(group, 1)
    p, lse = _softmax_over_rows((q * k).sum(-1) * scale, dst, n)
    out = torch.zeros(n, c["heads"], c["head_dim"], device="cuda").index_add_(0, dst, p[..., None] * v)
    if not train:
        return dict(out=out.to(t), lse=lse)
    dout = s["dout"].float()
    delta = (dout * out).sum(-1)
    do = dout[dst]
    ds = p * ((do * v).sum(-1) - delta[dst]) * scale
    dq = torch.zeros_like(out).index_add_(0, dst, ds[..., None] * k)
    shape = (c["src"], c["kv_heads"], c["head_dim"])
    edges = (-1, c["kv_heads"], group, c["head_dim"])
    dk = torch.zeros(shape, device="cuda").index_add_(0, src, (ds[..., None] * q).view(edges).sum(2))
    dv = torch.zeros(shape, device="cuda").index_add_(0, src, (p[..., None] * do).view(edges).sum(2))
    return dict(out=out.to(t), lse=lse, dq=dq.to(t), dk=dk.to(t), dv=dv.to(t))


def _plain_xent(s):
    c, t = s["case"], _TYPES[s["case"]["type"]]
    hidden, table, valid = s["hidden"].float(), s["table"].float(), s["labels"] >= 0
    at, label = torch.arange(c["rows"], device="cuda"), s["labels"].clamp(min=0).long()
    logits = (hidden @ table.t()).mul_(c["scale"])
    top = logits.amax(1, keepdim=True)
    picked = logits[at, label]
    p = logits.sub_(top).exp_()
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    loss = torch.where(valid, lse - picked, torch.zeros_like(lse))
    p.div_(total)
    p[at, label] -= 1.0
    p.mul_(torch.where(valid, s["dloss"], torch.zeros_like(lse))[:, None] * c["scale"])
    return dict(loss=loss, lse=lse, dhidden=(p @ table).to(t), dtable=(p.t() @ hidden).to(t))


# ------------------------------------------------------------------------------------------------ the package's operators
def _workspace(s, size):
    """The state's workspace, made at the first pass as a training program does before its loop."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(size(), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_run(s):
    import paper_2406_17918_b200 as gs

    c = s["case"]
    op = c["op"]
    if op == "lookup":
        return gs.gs_embedding_lookup(s["table"], s["ids"], scale=c["scale"], out_dtype=_TYPES[c["out"]])
    if op == "lookup_grad":
        ws = _workspace(s, lambda: gs.gs_embedding_workspace_bytes(c["ids"], c["table"], c["dim"]))
        if not c["sparse"]:
            return gs.gs_embedding_backward(s["dout"], s["ids"], c["table"], ws, scale=c["scale"], out_dtype=_TYPES[c["out"]])
        ids, count, grad = gs.gs_embedding_backward_sparse(s["dout"], s["ids"], c["table"], ws, scale=c["scale"], out_dtype=_TYPES[c["out"]])
        return dict(ids=ids, count=count, grad=grad)
    if op in ("attend", "attend_train"):
        ws = _workspace(s, lambda: gs.gs_block_attention_workspace_bytes(c["dst"], c["src"], s["indices"].numel(), c["heads"], c["kv_heads"], c["head_dim"]))
        out, lse = gs.gs_block_attention_forward(s["indptr"], s["indices"], s["q"], s["k"], s["v"], ws, max_row=c["longest"])
        if op == "attend":
            return dict(out=out, lse=lse)
        reverse = gs.gs_block_reverse(s["indptr"], s["indices"], c["src"], ws)
        dq, dk, dv = gs.gs_block_attention_backward(s["indptr"], s["indices"], reverse, s["q"], s["k"], s["v"], out, lse, s["dout"], ws, max_row=c["longest"])
        return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)
    ws = _workspace(s, lambda: gs.gs_xent_workspace_bytes(c["rows"], c["vocab"], c["dim"]))
    loss, lse = gs.gs_xent_forward(s["hidden"], s["table"], s["labels"], ws, scale=c["scale"])
    dhidden, dtable = gs.gs_xent_backward(s["hidden"], s["table"], s["labels"], lse, s["dloss"], ws, scale=c["scale"])
    return dict(loss=loss, lse=lse, dhidden=dhidden, dtable=dtable)


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "lookup":
        return _plain_lookup(state)
    if op == "lookup_grad":
        return _plain_lookup_grad(state)
    if op in ("attend", "attend_train"):
        return _plain_attend(state, op == "attend_train")
    return _plain_xent(state)


# ------------------------------------------------------------------------------------------------ work
def _edges(case):
    """Expected edges of a block (row lengths are floor((longest + 1) u^skew), some rows empty, some edges masked)."""
    f, s = case["longest"], case["skew"]
    mean = sum(1.0 - (k / (f + 1.0)) ** (1.0 / s) for k in range(1, f + 1))
    return case["dst"] * (1.0 - case["empty"]) * mean


def _distinct(n, top):
    """Expected distinct values of n ids floor(top u^2): an id x is drawn with probability about 1 / (2 sqrt(x top))."""
    steps = 4096
    total = 0.0
    for i in range(steps):
        lo, hi = top * (i / steps) ** 2, top * ((i + 1) / steps) ** 2
        total += (hi - lo) * -math.expm1(-n / steps / (hi - lo))
    return min(total, n, top)


def work(case):
    op, b = case["op"], _BYTES[case["type"]]
    if op == "lookup":
        rows = case["table"] * -math.expm1(-case["ids"] / case["table"])      # distinct rows read
        return dict(bytes=int(4 * case["ids"] + rows * case["dim"] * b + case["ids"] * case["dim"] * _BYTES[case["out"]]), flops=case["ids"] * case["dim"])
    if op == "lookup_grad":
        rows = case["ids"] if case["sparse"] else case["table"]
        extra = 4 * case["ids"] if case["sparse"] else 0
        return dict(bytes=int(4 * case["ids"] + case["ids"] * case["dim"] * b + rows * case["dim"] * _BYTES[case["out"]] + extra),
                    flops=2 * case["ids"] * case["dim"])
    if op in ("attend", "attend_train"):
        e = _edges(case)
        qw, kw = case["heads"] * case["head_dim"], case["kv_heads"] * case["head_dim"]
        touched = _distinct(e * (1.0 - case["masked"]), case["src"])
        index = 4 * (case["dst"] + 1) + 4 * e
        forward = index + 2 * touched * kw * b + 2 * case["dst"] * qw * b + 4 * case["dst"] * case["heads"]
        if op == "attend":
            return dict(bytes=int(forward), flops=int(4 * e * qw))
        # the gradients need the inputs, the upstream gradient and the saved statistics once more only where they do not
        # stay on chip; counted once: q, k, v, dout in, out, lse, dq, dk, dv out
        backward = 2 * case["dst"] * qw * b + 2 * case["src"] * kw * b
        return dict(bytes=int(forward + backward), flops=int(14 * e * qw))
    n, v, d = case["rows"], case["vocab"], case["dim"]
    return dict(bytes=int(2 * (n * d + v * d) * b + 16 * n), flops=6 * n * v * d)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "lookup":
        return torch.index_select(s["table"], 0, s["ids"]).double() * float(case["scale"])
    if op == "lookup_grad":
        order = torch.argsort(s["ids"].long(), stable=True)
        ids, counts = torch.unique_consecutive(s["ids"][order], return_counts=True)
        total = torch.segment_reduce(s["dout"].double()[order], "sum", lengths=counts, axis=0) * float(case["scale"])
        if case["sparse"]:
            grad = torch.zeros(case["ids"], case["dim"], dtype=torch.float64, device="cuda")
            grad[:ids.numel()] = total
            return dict(ids=None, count=None, grad=grad)
        grad = torch.zeros(case["table"], case["dim"], dtype=torch.float64, device="cuda")
        grad[ids.long()] = total
        return grad
    if op in ("attend", "attend_train"):
        return _exact_attend(s, case, op == "attend_train")
    h, w = s["hidden"].double(), s["table"].double()
    valid = s["labels"] >= 0
    y = s["labels"].long().clamp(min=0)[:, None]
    z = torch.mm(h, w.t()) * float(case["scale"])
    lse = torch.logsumexp(z, 1)
    loss = (lse - z.gather(1, y)[:, 0]) * valid
    g = s["dloss"].double() * valid * float(case["scale"])
    z = torch.exp(z.sub_(lse[:, None]))
    z.scatter_add_(1, y, torch.full_like(lse, -1.0)[:, None])
    z.mul_(g[:, None])
    return dict(loss=loss, lse=lse, dhidden=torch.mm(z, w), dtable=torch.mm(z.t(), h))


def _exact_attend(s, case, train):
    """Head by head, so that 64-bit copies of the gathered rows stay small."""
    n, hq, hk, d = case["dst"], case["heads"], case["kv_heads"], case["head_dim"]
    length = (s["indptr"][1:] - s["indptr"][:-1]).long()
    row = torch.arange(n, device="cuda").repeat_interleave(length)
    row, col = row[s["indices"] >= 0], s["indices"][s["indices"] >= 0].long()
    new = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, lse, dq, dk, dv = new(n, hq, d), new(n, hq), new(n, hq, d), new(case["src"], hk, d), new(case["src"], hk, d)
    for h in range(hq):
        qh, kh, vh = s["q"][:, h].double(), s["k"][:, h * hk // hq].double()[col], s["v"][:, h * hk // hq].double()[col]
        z = torch.einsum("ed,ed->e", qh[row], kh) / math.sqrt(d)
        high = torch.full((n,), -math.inf, dtype=torch.float64, device="cuda").scatter_reduce_(0, row, z, "amax")
        e = torch.exp(z - high[row])
        den = new(n).index_add_(0, row, e)
        lse[:, h] = high + den.log()
        e /= den[row]
        o = new(n, d).index_add_(0, row, e[:, None] * vh)
        out[:, h] = o
        if train:
            go = s["dout"][:, h].double()
            gz = e * (torch.einsum("ed,ed->e", go[row], vh) - (go * o).sum(1)[row]) / math.sqrt(d)
            dq[:, h] = new(n, d).index_add_(0, row, gz[:, None] * kh)
            dk[:, h * hk // hq] += new(case["src"], d).index_add_(0, col, gz[:, None] * qh[row])
            dv[:, h * hk // hq] += new(case["src"], d).index_add_(0, col, e[:, None] * go[row])
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv) if train else dict(out=out, lse=lse)
