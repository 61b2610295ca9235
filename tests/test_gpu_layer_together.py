"""The operators around an attention layer used together: a training step with clipped gradients against 64-bit autograd, a served
layer over a cache in 8 bits against the same layer on what the cache holds, both captured and replayed, calls on another stream."""
import math
import os
import sys

import pytest
import torch

import paper_2406_17918_b200 as gs
from paper_2406_17918_b200.autograd import block_attention, embedding, rms_norm, table_cross_entropy

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _block(n, src, longest, g):
    lengths = torch.randint(0, longest + 1, (n,), generator=g, device="cuda")
    indptr = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    indptr[1:] = lengths.cumsum(0).int()
    return indptr, torch.randint(0, src, (int(indptr[-1]),), generator=g, device="cuda", dtype=torch.int32)


def _plain_attention(q, k, v, indptr, indices):
    n, heads, dim = q.shape
    dst = torch.repeat_interleave(torch.arange(n, device=q.device), (indptr[1:] - indptr[:-1]).long())
    src = indices.long()
    s = (q[dst] * k[src]).sum(-1) / dim ** 0.5
    top = torch.full((n, heads), -float("inf"), dtype=q.dtype, device=q.device).scatter_reduce(0, dst[:, None].expand_as(s), s.detach(), "amax")
    w = torch.exp(s - top[dst])
    total = torch.zeros(n, heads, dtype=q.dtype, device=q.device).index_add(0, dst, w)
    return torch.zeros(n, heads, dim, dtype=q.dtype, device=q.device).index_add(0, dst, (w / total[dst])[..., None] * v[src])


def test_a_training_step():
    """f32; a gradient passes through five 32-bit operators of at most a few hundred terms: 1e-4 of its norm is a hundred times
    their rounding, and the clipped gradient's factor is off by that of the norm."""
    g = _gen(0)
    n, src, width, vocab = 30, 80, 32, 90
    indptr, indices = _block(n, src, 12, g)
    ids = torch.randint(0, vocab, (src,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(-1, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    leaves = [torch.randn(s, generator=g, device="cuda") * 0.3 for s in ((vocab, width), (width, 3 * width), (vocab, width))] + [torch.ones(width, device="cuda")]
    mine, ref = [x.clone().requires_grad_() for x in leaves], [x.double().requires_grad_() for x in leaves]

    x = embedding(mine[0], ids, scale=2.0)
    qkv = (x @ mine[1]).view(src, 3, 4, 8)
    h = block_attention(qkv[:n, 0], qkv[:, 1], qkv[:, 2], indptr, indices, max_row=12)
    y, hidden = rms_norm(h.reshape(n, width), mine[3], residual=x[:n])
    (table_cross_entropy(y, mine[2], labels).sum() + (hidden ** 2).sum() * 1e-3).backward()
    grads = [p.grad for p in mine]
    norm = gs.gs_grad_clip(grads, 0.7, torch.empty(gs.gs_grad_workspace_bytes(4), dtype=torch.uint8, device="cuda"))

    xr = ref[0][ids.long()] * 2.0
    qr = (xr @ ref[1]).view(src, 3, 4, 8)
    hr = xr[:n] + _plain_attention(qr[:n, 0], qr[:, 1], qr[:, 2], indptr, indices).reshape(n, width)
    yr = ref[3] * hr / torch.sqrt((hr * hr).mean(1, keepdim=True) + 1e-6)
    keep = labels >= 0
    (torch.nn.functional.cross_entropy((yr @ ref[2].t())[keep], labels[keep].long(), reduction="sum") + (hr ** 2).sum() * 1e-3).backward()
    want = math.sqrt(sum(float((p.grad ** 2).sum()) for p in ref))
    assert want > 0.7 and abs(float(norm) - want) <= 1e-4 * want
    for a, b in zip(grads, ref):
        b = b.grad * (0.7 / want)
        assert (a.double() - b).norm() <= 2e-4 * b.norm()


@pytest.mark.parametrize("norm,max_norm", [("rms", 0.0), ("layer", 0.5), ("rms", 0.5)])
def test_the_example_with_norm_and_clipping(norm, max_norm):
    """It runs; the parameters' gradients of its last step have the norm they are clipped to, or less."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_context_nodes as example

    made, model = [], example.Model
    try:
        example.Model = lambda *a, **k: made.append(model(*a, **k)) or made[0]
        history = example.train("tiny", 3, log=lambda *_: None, norm=norm, max_norm=max_norm)
    finally:
        example.Model = model
    assert len(history) == 3 and all(math.isfinite(x) for x in history)
    grads = [p.grad for p in made[0].parameters()]
    total = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    assert math.isfinite(total) and total > 0 and (not max_norm or total <= max_norm * (1 + 2.0 ** -19))
    if norm == "rms":
        assert all(float(p.grad.abs().sum()) > 0 for p in made[0].norm)


class Served:
    """One layer: rows normalised, keys and values into the cache, attention over the cache, the result normalised into 8 bits."""

    def __init__(self, seed, t, nodes=3000, n=400, heads=4, dim=32):
        g = _gen(seed)
        self.t, self.heads, self.dim, self.n = t, heads, dim, n
        w = heads * dim
        self.indptr, self.indices = _block(n, nodes, 20, g)
        self.ids = torch.randperm(nodes, generator=g, device="cuda")[:n].int()
        self.x = torch.randn(n, w, generator=g, device="cuda").to(t)
        self.weight = torch.randn(w, generator=g, device="cuda")
        self.project = (torch.randn(w, 3 * w, generator=g, device="cuda") * w ** -0.5).to(t)
        self.cache = gs.gs_coded_rows(nodes, 2 * heads, dim, 16)
        gs.gs_coded_write(self.cache, torch.randn(nodes, 2 * heads, dim, generator=g, device="cuda"))
        self.k, self.v = self.cache.heads(0, heads), self.cache.heads(heads, 2 * heads)
        self.ws = torch.empty(gs.gs_coded_attention_workspace_bytes(n, self.indices.numel(), heads, dim), dtype=torch.uint8, device="cuda")
        self.result = gs.gs_coded_rows(n, heads, dim, 1)

    def fill(self, other):
        for name in ("x", "ids"):
            getattr(self, name).copy_(getattr(other, name))
        self.cache.codes.view(torch.uint8).copy_(other.cache.codes.view(torch.uint8))
        self.cache.scales.copy_(other.cache.scales)

    def step(self, stream=None):
        y, _ = gs.gs_rms_norm_forward(self.x, self.weight, stream=stream)
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            qkv = (y @ self.project).view(self.n, 3, self.heads, self.dim)
        gs.gs_coded_write(self.cache, qkv[:, 1:].reshape(self.n, 2 * self.heads, self.dim) if stream is None else self._kv(qkv, stream), ids=self.ids, stream=stream)
        out, lse = gs.gs_coded_attention_forward(self.indptr, self.indices, qkv[:, 0], self.k, self.v, self.ws, max_row=20, stream=stream)
        _, hidden = gs.gs_rms_norm_coded(out.view(self.n, -1), self.result, self.weight, residual=self.x, stream=stream)
        return dict(q=qkv[:, 0], out=out, lse=lse, hidden=hidden, codes=self.result.codes.view(torch.uint8), scales=self.result.scales,
                    cache=self.cache.codes.view(torch.uint8), cache_scales=self.cache.scales)

    def _kv(self, qkv, stream):
        with torch.cuda.stream(stream):
            return qkv[:, 1:].reshape(self.n, 2 * self.heads, self.dim)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_a_served_layer(t):
    """The typed attention over what the cache holds: both kernels are within their bounds of the same value."""
    s = Served(1, t)
    got = s.step()
    kv = gs.gs_coded_read(s.cache, out_dtype=t)               # e4m3 times a power of two is exact in both types
    ws = torch.empty(gs.gs_block_attention_workspace_bytes(s.n, 3000, s.indices.numel(), s.heads, s.heads, s.dim), dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(s.indptr, s.indices, got["q"], kv[:, :s.heads], kv[:, s.heads:], ws, max_row=20)
    step = 2.0 ** -7 if t == torch.bfloat16 else 2.0 ** -23
    assert ((got["out"].double() - out.double()).abs() <= 2 * step * out.double().abs() + 1e-5).all()
    ok = torch.isfinite(lse)
    assert torch.equal(torch.isfinite(got["lse"]), ok) and ((got["lse"] - lse)[ok].abs() <= 1e-5 * (1 + lse[ok].abs())).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_captured_and_replayed(t):
    """Replays on new contents, eager calls between them, two graphs that share the workspace: what eager calls give."""
    s, other = Served(2, t), Served(2, t)
    contents = [Served(k, t) for k in (2, 3, 4)]
    want = []
    for c in contents:
        other.fill(c)
        want.append({k: v.clone() for k, v in other.step().items()})
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = s.step()
        graphs.append((graph, got))
    for k, c in enumerate(contents):
        for graph, got in graphs:
            s.fill(c)
            graph.replay()
            for name in got:
                assert torch.equal(got[name], want[k][name]), name
        s.fill(c)
        eager = s.step()
        for name in eager:
            assert torch.equal(eager[name], want[k][name]), name


def test_another_stream():
    a, b = Served(5, torch.float32), Served(5, torch.float32)
    want = a.step()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)                             # the current stream is busy with other things
    got = b.step(side)
    side.synchronize()
    torch.cuda.synchronize()
    for name in want:
        assert torch.equal(got[name], want[name]), name


def test_training_calls_captured():
    """Norm forward and backward and the clipping in one graph, replayed on other contents."""
    g = _gen(6)
    n, d = 700, 96
    new = lambda: [torch.randn(n, d, generator=g, device="cuda") for _ in range(4)]  # noqa: E731
    held, w = new(), torch.randn(d, generator=g, device="cuda")
    nws = torch.empty(gs.gs_rms_norm_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
    gws = torch.empty(gs.gs_grad_workspace_bytes(3), dtype=torch.uint8, device="cuda")
    count = torch.tensor([n], dtype=torch.int32, device="cuda")

    def step(x, res, dy, dh):
        out, hid = gs.gs_rms_norm_forward(x, w, residual=res, count=count)
        dx, dw = gs.gs_rms_norm_backward(hid, dy, nws, weight=w, dhidden=dh, count=count)
        norm = gs.gs_grad_clip([dx, dw], 3.0, gws, counts=[count, None])
        return out, hid, dx, dw, norm

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*held)
    for live in (n, 123, 0):
        other = new()
        count.fill_(live)
        want = [t.clone() for t in step(*other)]
        for a, b in zip(held, other):
            a.copy_(b)
        graph.replay()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_refusals():
    g = _gen(7)
    x, w = torch.randn(6, 32, generator=g, device="cuda"), torch.ones(32, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    store = gs.gs_coded_rows(20, 2, 16, 4)
    for call in (lambda: gs.gs_rms_norm_forward(x.t(), w), lambda: gs.gs_rms_norm_forward(x, w[:31]), lambda: gs.gs_rms_norm_forward(x, w.half()),
                 lambda: gs.gs_rms_norm_forward(x, w, residual=x.bfloat16()), lambda: gs.gs_rms_norm_forward(x, w, residual=x[:5]), lambda: gs.gs_rms_norm_forward(x.half(), w),
                 lambda: gs.gs_rms_norm_forward(x, w, out=x.bfloat16()), lambda: gs.gs_rms_norm_forward(x, w, residual=x.cpu()), lambda: gs.gs_rms_norm_forward(x, w.cpu()),
                 lambda: gs.gs_rms_norm_backward(x, x[:, :31], ws), lambda: gs.gs_rms_norm_backward(x, x, ws, weight=w, dweight=w.bfloat16()),
                 lambda: gs.gs_rms_norm_backward(x, x, ws, dweight=w), lambda: gs.gs_rms_norm_backward(x, x, ws.float()),
                 lambda: gs.gs_rms_norm_coded(x, store, w), lambda: gs.gs_rms_norm_coded(x, gs.gs_coded_rows(5, 2, 16, 1), w), lambda: gs.gs_rms_norm_coded(x, gs.gs_coded_rows(9, 3, 16, 1), w),
                 lambda: gs.gs_coded_rows(10, 2, 16, 3), lambda: gs.gs_coded_rows(10, 2, 0, 1), lambda: gs.CodedRows(store.codes, store.scales, 15, 1),
                 lambda: gs.CodedRows(store.codes[:, :, :8], store.scales, 8, 4), lambda: gs.CodedRows(store.codes, store.scales.cpu(), 16, 4),
                 lambda: store.heads(1, 3), lambda: store.heads(1, 1), lambda: gs.gs_coded_write(store, x.view(6, 2, 16), first=15), lambda: gs.gs_coded_write(store, x.view(6, 2, 16), first=-1),
                 lambda: gs.gs_coded_write(store, x.view(6, 1, 32)), lambda: gs.gs_coded_write(store, x.view(6, 2, 16), ids=torch.arange(7, device="cuda").int()),
                 lambda: gs.gs_coded_write(store, x.view(6, 2, 16), ids=torch.arange(6, device="cuda")), lambda: gs.gs_coded_write(store, x.view(6, 2, 16).half()),
                 lambda: gs.gs_coded_read(store, first=21), lambda: gs.gs_coded_read(store, first=10, num_rows=11), lambda: gs.gs_coded_read(store, out_dtype=torch.float16),
                 lambda: gs.gs_coded_read(store, num_rows=4, out=torch.empty(3, 2, 16, device="cuda"))):
        with pytest.raises((TypeError, ValueError, gs.GsError)):
            call()
    assert (store.codes.view(torch.uint8) == 0).all()
    indptr, idx = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v = torch.randn(1, 2, 16, device="cuda"), store.heads(0, 1), store.heads(1, 2)
    for call in (lambda: gs.gs_coded_attention_forward(indptr, idx, q.half(), k, v, ws), lambda: gs.gs_coded_attention_forward(indptr, idx, q[:, :, :8], k, v, ws),
                 lambda: gs.gs_coded_attention_forward(indptr, idx, q, k, gs.gs_coded_rows(20, 1, 16, 1), ws), lambda: gs.gs_coded_attention_forward(indptr, idx.long(), q, k, v, ws),
                 lambda: gs.gs_coded_attention_forward(indptr, idx, torch.randn(1, 3, 16, device="cuda"), store, store, ws),
                 lambda: gs.gs_coded_attention_forward(torch.zeros(9, dtype=torch.int32, device="cuda"), idx, q, k, v, ws),
                 lambda: gs.gs_coded_attention_forward(indptr, idx, q, k, v, ws[:128]), lambda: gs.gs_coded_attention_forward(indptr, idx, q, k, v, ws, lse=torch.empty(1, 1, device="cuda"))):
        with pytest.raises((TypeError, ValueError, gs.GsError)):
            call()
    graph = torch.cuda.CUDAGraph()
    held = torch.zeros(4, device="cuda")
    with torch.cuda.graph(graph):
        held.add_(1)
        with pytest.raises(RuntimeError, match="captured"):
            gs.CodedRows(store.codes, store.scales, 16, 4)
