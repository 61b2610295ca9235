"""Workloads of the operators around an attention layer: its norm, its cache in 8 bits, the attention that reads the cache, gradient clipping.

Each case is one pass of one operator, in the sizes that training and serving on the graphs of ``workloads/`` meet:

* ``norm``        root-mean-square norm of a layer's rows with the residual's addition, forward and backward
* ``norm_coded``  the same norm, forward only, its result in 8 bits with a scale per group of columns, and read back
* ``cache``       key and value rows of some nodes quantised into a cache as they are written, rows of a next batch read back
* ``serve``       softmax attention of a block's destinations over key and value rows that a cache holds in 8 bits
* ``clip``        the norm over all gradients of a step, and the gradients scaled to a largest norm

What is held in 8 bits is e4m3 with a scale per block of rows and head, the smallest power of two 2^e (e >= -127) with
|x| <= 448 * 2^e for all x of the block; a scale is held as the byte e + 127.  ``run`` computes a pass in elementary tensor
operations (32 bits, rounded once), or, where ``own`` is true, by the package's kernels.  ``exact`` is the same from the
definition in 64 bits.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
_TYPES = {F32: torch.float32, BF16: torch.bfloat16}
_BYTES = {F32: 4, BF16: 2}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the seeds of one small batch behind a layer of 4 heads of 16: latency counts
        dict(name="norm_seeds", op="norm", rows=64, dim=64, residual=True, type=F32),
        # wide odd rows: normalised bag-of-words features, no residual
        dict(name="norm_wide_odd", op="norm", rows=4096, dim=1433, residual=False, type=F32),
        # all input nodes of a batch of 8,192 seeds
        dict(name="norm_batch_large", op="norm", rows=2031616, dim=128, residual=True, type=BF16),
        # the input-side destinations of such a batch while serving: one scale per row and 32 columns
        dict(name="norm_coded_batch", op="norm_coded", rows=262144, dim=128, groups=4, residual=True, type=BF16),
        # a few served nodes refresh their rows of a small cache, one scale per row and head
        dict(name="cache_few", op="cache", rows=2708, heads=8, head_dim=16, block=1, written=64, read=384, type=F32),
        # the destinations of a batch put their key and value rows into the cache, the next batch's input nodes are read
        dict(name="cache_batch", op="cache", rows=2449029, heads=8, head_dim=32, block=16, written=262144, read=2031616, type=BF16),
        # serving a handful of seeds: one hop of 5 neighbours
        dict(name="serve_few", op="serve", dst=64, rows=2708, longest=5, skew=0.2, empty=0.05, masked=0.0, heads=4, kv_heads=4, head_dim=16, block=1, type=F32),
        # one node against its whole neighbourhood, shared key/value heads
        dict(name="serve_one_hub", op="serve", dst=1, rows=736389, longest=200011, skew=0.0, empty=0.0, masked=0.05, heads=8, kv_heads=2, head_dim=64, block=64, type=BF16),
        # input-side block of a batch of 8,192 seeds (fan-out 20)
        dict(name="serve_batch_large", op="serve", dst=262144, rows=2449029, longest=20, skew=0.2, empty=0.02, masked=0.0, heads=4, kv_heads=4, head_dim=32, block=16, type=BF16),
        # all gradients of the small training example: two tables, two layers
        dict(name="clip_example", op="clip", table=2708, dim=64, layers=2, touched=0, spread=1.0, type=F32),
        # a table of input vectors and one of context vectors, dense f32 gradients
        dict(name="clip_dense", op="clip", table=169343, dim=128, layers=3, touched=0, spread=30.0, type=F32),
        # touched rows of a large input table (their number is known on the device alone) beside a dense context table, bf16
        dict(name="clip_touched", op="clip", table=736389, dim=128, layers=3, touched=2031616, spread=30.0, type=BF16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_coded", "cache", "cache", "serve", "serve", "clip", "clip"])
    kind = rng.choice([F32, BF16])
    if op == "norm":
        dim = rng.choice([_log_int(rng, 8, 4096), 8 * _log_int(rng, 1, 512), 64, 128])
        return dict(op=op, rows=min(_log_int(rng, 1, 2031616), 130000000 // dim), dim=dim, residual=rng.random() < 0.7, type=kind)
    if op == "norm_coded":
        groups, width = rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 33, 64, 100, 128])
        return dict(op=op, rows=min(_log_int(rng, 1, 1015808), 100000000 // (groups * width)), dim=groups * width, groups=groups,
                    residual=rng.random() < 0.7, type=kind)
    if op == "cache":
        heads, head_dim = rng.choice([1, 2, 4, 8]), rng.choice([8, 16, 24, 32, 33, 64, 100, 128])
        rows = min(_log_int(rng, 64, 2449029), 600000000 // (heads * head_dim))
        most = min(2031616, 260000000 // (heads * head_dim))
        return dict(op=op, rows=rows, heads=heads, head_dim=head_dim, block=rng.choice([1, 4, 16, 64]), written=min(_log_int(rng, 1, most), rows // 2),
                    read=_log_int(rng, 64, most), type=kind)
    if op == "serve":
        head_dim = rng.choice([8, 16, 24, 32, 33, 64, 100, 128])
        kv = rng.choice([h for h in (1, 2, 4, 8) if h * head_dim <= 256])
        heads = kv * rng.choice([1, 1, 2, 4])
        width = heads * head_dim
        if rng.random() < 0.35:             # whole neighbourhoods: few long rows among short ones, down to one row alone
            dst = rng.choice([1, _log_int(rng, 1, 4096)])
            longest = min(_log_int(rng, 64, 200011), 300000000 // width)
            skew = 0.0 if dst == 1 else 30.0
            dst = max(1, min(dst, 300000000 // (width * max(1, longest // 30))))
        else:
            dst, longest, skew = _log_int(rng, 1, 262144), rng.randint(1, 32), 0.2
            dst = max(1, min(dst, 500000000 // (width * longest)))
        return dict(op=op, dst=dst, rows=min(_log_int(rng, 64, 2449029), 300000000 // (kv * head_dim)), longest=longest, skew=skew,
                    empty=rng.choice([0.0, 0.05, 0.3]) if dst > 1 else 0.0, masked=rng.choice([0.0, 0.1]), heads=heads, kv_heads=kv, head_dim=head_dim,
                    block=rng.choice([1, 16, 64]), type=kind)
    dim = rng.choice([16, 33, 64, 100, 128, 256])
    touched = rng.choice([0, min(_log_int(rng, 64, 2031616), 260000000 // dim)])
    return dict(op="clip", table=min(_log_int(rng, 64, 736389), 94000000 // dim), dim=dim, layers=rng.choice([1, 2, 3, 6, 12]), touched=touched,
                spread=rng.choice([1.0, 30.0]), type=kind)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _rows_of_many_sizes(g, rows, heads, head_dim, dtype):
    """Key and value rows as a layer gives them: normal within a node, nodes of different sizes."""
    size = torch.exp2(torch.rand(rows, 1, 1, generator=g, device="cuda") * 4.0 - 2.0)
    return (torch.randn(rows, heads, head_dim, generator=g, device="cuda") * size).to(dtype)


def _skewed(g, n, top):
    """n ids below `top`, low ones far more often (the endpoint distribution of a power-law graph)."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (u * u * top).long().clamp_(max=top - 1).int()


def _pitch(head_dim):
    """Bytes a head's codes take in a row: whole pieces of 16, the rest zero."""
    return (head_dim + 15) // 16 * 16


def _exponent(top):
    """e of the smallest 2^e >= top / 448, -127 at least (and for top = 0)."""
    part, e = torch.frexp(top)                               # top = part 2^e, part in [1/2, 1);  448 = 7/8 2^9
    e = e - torch.where(part <= 0.875, 9, 8)
    return torch.where(top > 0, e, -127).clamp(min=-127)


def _power(e):
    """2^e, exactly: put together from its bits (in 64, where 2^-127 is an ordinary number)."""
    return ((e.long() + 1023) << 52).view(torch.float64).float()


def _cache_of(x, block):
    """A cache that holds the rows x: codes [rows, heads, pitch], scales [blocks, heads]."""
    rows, heads, dim = x.shape
    blocks = (rows + block - 1) // block
    top = torch.zeros(blocks * block, heads, device="cuda")
    top[:rows] = x.float().abs().amax(2)
    e = _exponent(top.view(blocks, block, heads).amax(1))
    codes = torch.zeros(rows, heads, _pitch(dim), dtype=torch.float8_e4m3fn, device="cuda")
    codes[:, :, :dim] = (x.float() * _power(-e).repeat_interleave(block, 0)[:rows, :, None]).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def prepare(case, seed):
    g, t = _generator(seed), _TYPES[case["type"]]
    op = case["op"]
    if op in ("norm", "norm_coded"):
        shape = (case["rows"], case["dim"])
        s = dict(case=case, x=_normal(g, shape, t), weight=1.0 + 0.2 * torch.randn(case["dim"], generator=g, device="cuda"))
        if case["residual"]:
            s["residual"] = _normal(g, shape, t, 2.0)
        if op == "norm":
            s["dout"] = _normal(g, shape, t)
            if case["residual"]:
                s["dhidden"] = _normal(g, shape, t)
        return s
    if op == "cache":
        codes, scales = _cache_of(_rows_of_many_sizes(g, case["rows"], case["heads"], case["head_dim"], torch.bfloat16), case["block"])
        ids = torch.randperm(case["rows"], generator=g, device="cuda")[:case["written"]].int()
        return dict(case=case, codes=codes, scales=scales, ids=ids, new=_rows_of_many_sizes(g, case["written"], case["heads"], case["head_dim"], t),
                    wanted=_skewed(g, case["read"], case["rows"]))
    if op == "serve":
        n = case["dst"]
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        length = ((case["longest"] + 1) * u ** case["skew"]).long().clamp_(max=case["longest"])
        length[torch.rand(n, generator=g, device="cuda") < case["empty"]] = 0
        indptr = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        indptr[1:] = torch.cumsum(length, 0).int()
        edges = int(indptr[-1])
        # the frequent nodes lie anywhere in the cache
        perm = torch.randperm(case["rows"], generator=g, device="cuda").int()
        indices = perm[_skewed(g, edges, case["rows"]).long()]
        if case["masked"]:
            indices[torch.rand(edges, generator=g, device="cuda") < case["masked"]] = -1
        # one cache row: the node's key heads, then its value heads
        codes, scales = _cache_of(_rows_of_many_sizes(g, case["rows"], 2 * case["kv_heads"], case["head_dim"], torch.bfloat16), case["block"])
        return dict(case=case, indptr=indptr, indices=indices, codes=codes, scales=scales, q=_normal(g, (n, case["heads"], case["head_dim"]), t))
    # the gradients of a step, parameter by parameter: tables, then the layers' projections and norms; of sizes that differ
    d, spread = case["dim"], case["spread"]
    shapes = [(case["table"], d)] + [x for _ in range(case["layers"]) for x in ((d, 3 * d), (d, d), (d,))]
    s = dict(case=case, grads=[_normal(g, shape, t if i == 0 else torch.float32, spread / math.sqrt(shape[0] * d) * (1 + i % 3)) for i, shape in enumerate(shapes)],
             max_norm=1.0, count=None)
    if case["touched"]:
        s["grads"].insert(0, _normal(g, (case["touched"], d), t, spread / math.sqrt(case["touched"] * d)))
        s["count"] = torch.tensor([max(1, case["touched"] * 7 // 8)], dtype=torch.int32, device="cuda")
        s["grads"][0][int(s["count"]):] = 0                  # what the touched rows' gradient has behind them
    else:
        s["grads"].insert(0, _normal(g, (case["table"], d), t, spread / math.sqrt(case["table"] * d)))
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_norm_forward(s):
    t = s["x"].dtype
    h = (s["x"].float() + s["residual"].float()).to(t) if "residual" in s else s["x"]
    x = h.float()
    inv = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    return h, x, inv, x * inv * s["weight"]


def _plain_norm(s):
    t = s["x"].dtype
    h, x, inv, y = _plain_norm_forward(s)
    dy = s["dout"].float()
    g = dy * s["weight"]
    dx = g * inv - x * (inv * inv * inv * (g * x).mean(1, keepdim=True))
    dweight = (dy * x * inv).sum(0, dtype=torch.float64).float()
    if "residual" not in s:
        return dict(out=y.to(t), dx=dx.to(t), dweight=dweight)
    return dict(hidden=h, out=y.to(t), dx=(dx + s["dhidden"].float()).to(t), dweight=dweight)


def _plain_norm_coded(s):
    c = s["case"]
    h, _, _, y = _plain_norm_forward(s)
    y = y.view(c["rows"], c["groups"], -1)
    e = _exponent(y.abs().amax(2))
    values = (y * _power(-e)[..., None]).to(torch.float8_e4m3fn).float() * _power(e)[..., None]
    values = values.bfloat16()                               # a code times a power of two is a bf16 number
    return dict(values=values, hidden=h) if "residual" in s else dict(values=values)


def _plain_cache(s):
    """The rows that `wanted` has after the write, and the scales; the state's cache is changed."""
    c, block, t = s["case"], s["case"]["block"], _TYPES[s["case"]["type"]]
    rows, d = c["rows"], c["head_dim"]
    ids = s["ids"].long()
    new = s["new"].float()
    blocks = s["scales"].shape[0]
    need = (_exponent(new.abs().amax(2)) + 127).to(torch.uint8)
    top = torch.zeros(blocks, c["heads"], dtype=torch.uint8, device="cuda")
    top = top.scatter_reduce(0, (ids // block)[:, None].expand_as(need), need, "amax")
    # a block keeps its scale for the rows that are not written, if there are any
    lengths = torch.full((blocks,), block, device="cuda")
    lengths[-1] = rows - (blocks - 1) * block
    fresh = torch.bincount(ids // block, minlength=blocks) == lengths
    after = torch.where(fresh[:, None], top, torch.maximum(top, s["scales"]))
    raised = ((after > s["scales"]) & ~fresh[:, None]).any(1).nonzero()[:, 0]
    at = (raised[:, None] * block + torch.arange(block, device="cuda")).flatten()
    at = at[at < rows]
    ratio = _power(s["scales"][at // block].int() - after[at // block].int())
    s["codes"][at] = (s["codes"][at].float() * ratio[..., None]).to(torch.float8_e4m3fn)
    e = after.int() - 127
    s["codes"][ids, :, :d] = (new * _power(-e[ids // block])[..., None]).to(torch.float8_e4m3fn)
    s["scales"].copy_(after)
    wanted = s["wanted"].long()
    values = s["codes"][wanted][:, :, :d].float() * _power(e[wanted // block])[..., None]
    return dict(values=values.to(t), scales=s["scales"])


def _plain_serve(s):
    c, t = s["case"], _TYPES[s["case"]["type"]]
    n, hk, d = c["dst"], c["kv_heads"], c["head_dim"]
    keep = s["indices"] >= 0
    dst = torch.repeat_interleave(torch.arange(n, device="cuda"), (s["indptr"][1:] - s["indptr"][:-1]).long())[keep]
    row = s["indices"][keep].long()
    kv = s["codes"][row][:, :, :d].float() * _power(s["scales"][row // c["block"]].int() - 127)[..., None]
    k, v = kv[:, :hk].repeat_interleave(c["heads"] // hk, 1), kv[:, hk:].repeat_interleave(c["heads"] // hk, 1)
    score = (s["q"].float()[dst] * k).sum(-1) * (1.0 / math.sqrt(d))
    top = torch.full((n, c["heads"]), -math.inf, device="cuda").scatter_reduce(0, dst[:, None].expand_as(score), score, "amax")
    weight = torch.exp(score - top[dst])
    # a row of a hundred thousand terms: sums in 64 bits
    total = torch.zeros(n, c["heads"], dtype=torch.float64, device="cuda").index_add_(0, dst, weight.double())
    p = weight / total.float()[dst]
    out = torch.zeros(n, c["heads"], d, device="cuda").index_add_(0, dst, p[..., None] * v)
    return dict(out=out.to(t), lse=top + torch.log(total).float())


def _plain_clip(s):
    grads = s["grads"]
    if s["count"] is not None:
        here = torch.arange(grads[0].shape[0], device="cuda") < s["count"]
        grads = [torch.where(here[:, None], grads[0], 0)] + grads[1:]
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads]).sum().sqrt().float()
    scale = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return dict(norm=norm.view(1), grads=[(g.float() * scale).to(g.dtype) for g in grads])


# ------------------------------------------------------------------------------------------------ the package's operators
def _workspace(s, size):
    """The state's workspace, made at the first pass as a program does before its loop."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(size(), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_run(s):
    import paper_2406_17918_b200 as gs

    c = s["case"]
    op = c["op"]
    if op == "norm":
        ws = _workspace(s, lambda: gs.gs_rms_norm_workspace_bytes(c["rows"], c["dim"]))
        out, hidden = gs.gs_rms_norm_forward(s["x"], s["weight"], residual=s.get("residual"), eps=EPS)
        dx, dweight = gs.gs_rms_norm_backward(hidden, s["dout"], ws, weight=s["weight"], dhidden=s.get("dhidden"), eps=EPS)
        return dict(hidden=hidden, out=out, dx=dx, dweight=dweight) if c["residual"] else dict(out=out, dx=dx, dweight=dweight)
    if op == "norm_coded":
        if "coded" not in s:
            s["coded"] = gs.gs_coded_rows(c["rows"], c["groups"], c["dim"] // c["groups"], block=1, device="cuda")
        coded, hidden = gs.gs_rms_norm_coded(s["x"], s["coded"], s["weight"], residual=s.get("residual"), eps=EPS)
        values = gs.gs_coded_read(coded, num_rows=c["rows"], out_dtype=torch.bfloat16)
        return dict(values=values, hidden=hidden) if c["residual"] else dict(values=values)
    if op == "cache":
        if "cache" not in s:
            s["cache"] = gs.CodedRows(s["codes"], s["scales"], c["head_dim"], c["block"])
        gs.gs_coded_write(s["cache"], s["new"], ids=s["ids"])
        return dict(values=gs.gs_coded_read(s["cache"], ids=s["wanted"], out_dtype=_TYPES[c["type"]]), scales=s["scales"])
    if op == "serve":
        ws = _workspace(s, lambda: gs.gs_coded_attention_workspace_bytes(c["dst"], s["indices"].numel(), c["heads"], c["head_dim"]))
        if "cache" not in s:
            s["cache"] = gs.CodedRows(s["codes"], s["scales"], c["head_dim"], c["block"])
            s["k"], s["v"] = s["cache"].heads(0, c["kv_heads"]), s["cache"].heads(c["kv_heads"], 2 * c["kv_heads"])
        out, lse = gs.gs_coded_attention_forward(s["indptr"], s["indices"], s["q"], s["k"], s["v"], ws, max_row=c["longest"])
        return dict(out=out, lse=lse)
    ws = _workspace(s, lambda: gs.gs_grad_workspace_bytes(len(s["grads"])))
    if "clipped" not in s:
        s["clipped"] = [torch.zeros_like(g) for g in s["grads"]]
    counts = None if s["count"] is None else [s["count"]] + [None] * (len(s["grads"]) - 1)
    norm = gs.gs_grad_clip(s["grads"], s["max_norm"], ws, out=s["clipped"], counts=counts)
    return dict(norm=norm, grads=s["clipped"])


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "norm":
        return _plain_norm(state)
    if op == "norm_coded":
        return _plain_norm_coded(state)
    if op == "cache":
        return _plain_cache(state)
    if op == "serve":
        return _plain_serve(state)
    return _plain_clip(state)


# ------------------------------------------------------------------------------------------------ work
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
    if op == "norm":
        n, d = case["rows"], case["dim"]
        # x, dout in, out, dx out; with a residual also the residual and its gradient in, the sum out
        return dict(bytes=(7 if case["residual"] else 4) * n * d * b + 8 * d, flops=16 * n * d)
    if op == "norm_coded":
        n, d = case["rows"], case["dim"]
        # the codes and scales are written and read once, the values they stand for written
        coded = d + case["groups"]
        return dict(bytes=n * ((3 if case["residual"] else 1) * d * b + 2 * coded + 2 * d) + 4 * d, flops=8 * n * d)
    if op == "cache":
        width = case["heads"] * case["head_dim"]
        return dict(bytes=int(case["written"] * (4 + width * (b + 1)) + _distinct(case["read"], case["rows"]) * width + case["read"] * (4 + width * b)),
                    flops=4 * case["written"] * width + case["read"] * width)
    if op == "serve":
        f, s = case["longest"], case["skew"]
        mean = f if s == 0.0 else sum(1.0 - (k / (f + 1.0)) ** (1.0 / s) for k in range(1, f + 1))
        e = case["dst"] * (1.0 - case["empty"]) * mean
        qw = case["heads"] * case["head_dim"]
        touched = _distinct(e * (1.0 - case["masked"]), case["rows"])
        return dict(bytes=int(4 * (case["dst"] + 1) + 4 * e + touched * 2 * case["kv_heads"] * case["head_dim"] + 2 * case["dst"] * qw * b + 4 * case["dst"] * case["heads"]),
                    flops=int(4 * e * qw))
    d = case["dim"]
    tables = (case["touched"] * 7 // 8 if case["touched"] else case["table"]) * d * b + case["table"] * d * b
    layers = case["layers"] * (4 * d * d + d)
    return dict(bytes=2 * (tables + 4 * layers), flops=3 * (tables // b + layers))


# ------------------------------------------------------------------------------------------------ 64 bits
def _powers():
    """2^k, k = -127 .. 127: entry k + 127."""
    return torch.tensor([2.0 ** k for k in range(-127, 128)], dtype=torch.float64, device="cuda")


def _nearest_code(x, unit):
    """The e4m3 value next to x / unit (ties to even), times unit; |x| <= 448 unit."""
    v, powers = x / unit, _powers()
    low = torch.bucketize(v.abs().clamp(min=2.0 ** -6), powers, right=True) - 1
    step = powers[low] / 8.0
    return torch.round(v / step) * step * unit


def _unit(top):
    """The power of two of a block whose largest magnitude is `top`: the first of which 448 times is no less."""
    powers = _powers()
    return powers[torch.bucketize(top, 448.0 * powers)]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "norm_coded"):
        total = s["x"].double() + s["residual"].double() if "residual" in s else s["x"].double()
        h = total.to(s["x"].dtype).double()                  # what is normalised is the sum as it is kept
        rms = torch.sqrt((h.square().sum(1) / case["dim"] + EPS))[:, None]
        unit, w = h / rms, s["weight"].double()
        del h
        if op == "norm_coded":
            y = (unit * w).view(case["rows"], case["groups"], -1)
            r = dict(values=_nearest_code(y, _unit(y.abs().amax(2, keepdim=True))))
            if "residual" in s:
                r["hidden"] = total
            return r
        r = dict(out=unit * w)
        if "residual" in s:
            r["hidden"] = total
        dy = s["dout"].double()
        r["dweight"] = torch.einsum("nd,nd->d", dy, unit)
        dy *= w
        dx = (dy - unit * (torch.einsum("nd,nd->n", dy, unit) / case["dim"])[:, None]) / rms
        r["dx"] = dx + s["dhidden"].double() if "residual" in s else dx
        return r
    if op == "cache":
        rows, block, d = case["rows"], case["block"], case["head_dim"]
        old = _powers()[s["scales"].long()]
        blocks = old.shape[0]
        place = torch.full((blocks * block,), -1, dtype=torch.int64, device="cuda")
        place[s["ids"].long()] = torch.arange(case["written"], device="cuda")
        place = place.view(blocks, block)
        kept = (place < 0) & (torch.arange(blocks * block, device="cuda").view(blocks, block) < rows)
        size = torch.cat([s["new"].double().abs().amax(2), torch.zeros(1, case["heads"], dtype=torch.float64, device="cuda")])
        unit = _unit(size[place].amax(1))
        unit = torch.where(kept.any(1)[:, None], torch.maximum(unit, old), unit)
        unit = torch.where((place >= 0).any(1)[:, None], unit, old)
        w = s["wanted"].long()
        values = torch.empty(case["read"], case["heads"], d, dtype=torch.float64, device="cuda")
        for part in torch.split(torch.arange(case["read"], device="cuda"), 1 << 18):
            at = w[part]
            was = s["codes"][at][:, :, :d].double() * old[at // block][..., None]
            fresh = s["new"][place.view(-1)[at].clamp(min=0)].double()
            values[part] = _nearest_code(torch.where((place.view(-1)[at] >= 0)[:, None, None], fresh, was), unit[at // block][..., None])
        return dict(values=values, scales=None)
    if op == "serve":
        n, hq, hk, d = case["dst"], case["heads"], case["kv_heads"], case["head_dim"]
        length = (s["indptr"][1:] - s["indptr"][:-1]).long()
        row = torch.arange(n, device="cuda").repeat_interleave(length)
        row, col = row[s["indices"] >= 0], s["indices"][s["indices"] >= 0].long()
        unit = _powers()[s["scales"].long()]
        out, lse = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda"), torch.zeros(n, hq, dtype=torch.float64, device="cuda")
        for h in range(hq):                                  # head by head, so that 64-bit copies of the gathered rows stay small
            kh, vh = h * hk // hq, hk + h * hk // hq
            z = torch.einsum("ed,ed->e", s["q"][:, h].double()[row], s["codes"][:, kh, :d][col].double()) * unit[col // case["block"], kh] / math.sqrt(d)
            high = torch.full((n,), -math.inf, dtype=torch.float64, device="cuda").scatter_reduce_(0, row, z, "amax")
            e = torch.exp(z - high[row])
            den = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, row, e)
            lse[:, h] = high + den.log()
            e = e / den[row] * unit[col // case["block"], vh]
            out[:, h] = torch.zeros(n, d, dtype=torch.float64, device="cuda").index_add_(0, row, e[:, None] * s["codes"][:, vh, :d][col].double())
        return dict(out=out, lse=lse)
    first = case["touched"] if s["count"] is None else int(s["count"])
    flat = [g.double() for g in s["grads"]]
    if case["touched"]:
        flat[0][first:] = 0.0
    norm = math.sqrt(sum(float(torch.dot(g.reshape(-1), g.reshape(-1))) for g in flat))
    return dict(norm=torch.tensor([norm], dtype=torch.float64, device="cuda"), grads=[g * min(1.0, s["max_norm"] / (norm + 1e-6)) for g in flat])
