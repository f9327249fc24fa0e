"""The microscaled operators as they are used: a training step whose dense layer keeps its input in 8 bits, micro-batches
that share one output, the trained model served in 4 bits, and the same calls replayed from a HIP graph."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from helpers import small_problem
from oracle import mx

pytestmark = pytest.mark.gpu

TABLES = [(500, 16, 0), (300, 32, 0), (800, 8, 1), (90, 24, 0)]
FIELDS = [(0, 0), (1, 1), (2, 0), (1, 0), (3, 1)]


def problem(seed, B):
    pr = small_problem(seed, B=B, tables=TABLES, fields=FIELDS, max_len=6)
    return pr, torch.from_numpy(pr["ids"]).cuda(), torch.from_numpy(pr["offsets"]).cuda()


def new_layer(pr):
    from paper_2204_04903_amd.layer import PackedEmbedding
    layer = PackedEmbedding(TABLES, FIELDS)
    for t in range(len(TABLES)):
        layer.load_table(t, pr["Wt"][t])
    return layer


def quantized(x, fmt):
    return mx.decode(mx.encode(x.float().cpu().numpy(), fmt), fmt, x.shape[1])


def test_train_then_serve():
    from paper_2204_04903_amd.layer import ActivationCheckpoint, QuantizedEmbedding, QuantizedLinear
    B, N = 60, 48
    pr, ids, offs = problem(1, B)
    layer = new_layer(pr)
    W = torch.randn((N, layer.out_dim), generator=torch.Generator().manual_seed(1)).cuda() * 0.1
    for step in range(3):
        out = layer.forward(ids, offs, B)
        kept = ActivationCheckpoint(B, layer.out_dim).quantize(out)
        y = out @ W.t()
        grad_y = y - 1.0                                     # of half the squared distance from one
        seen = quantized(out, 1)
        out.fill_(float("nan"))                              # its memory is used for something else
        dw = kept.weight_grad(grad_y)
        ref = grad_y.double().cpu().numpy().T @ seen
        mag = np.abs(grad_y.double().cpu().numpy()).T @ np.abs(seen)
        assert (np.abs(dw.double().cpu().numpy() - ref) <= 1.01 * (3 * B + 1) * 2.0 ** -23 * mag).all()
        layer.backward_update(grad_y @ W, 0.05, 1e-8)
        W = W - 0.05 * dw
    assert layer.error_word() == 0
    serve = QuantizedEmbedding.from_layer(layer)
    try:
        dense = QuantizedLinear(W)
        x = serve.forward(ids, offs, B)
        y = dense.forward(x).double().cpu().numpy()
        xq, wq = quantized(x, 0), quantized(W, 0)
        assert (np.abs(y - xq @ wq.T) <= 1.01 * (layer.out_dim + 1) * 2.0 ** -23 * (np.abs(xq) @ np.abs(wq).T)).all()
        # and near what the full layer gives: a table's element is off by at most a quarter of itself or a sixth of its
        # block's largest (test_oracle_mx), and a pooled sum by the sum of that
        full = layer.forward(ids, offs, B).double().cpu().numpy()
        mags = [np.abs(layer.table_view(t).float().cpu().numpy().astype(np.float64)) for t in range(len(TABLES))]
        col = 0
        for f, (t, pool) in enumerate(FIELDS):
            D = TABLES[t][1]
            for b in range(B):
                q0, q1 = pr["offsets"][f * B + b], pr["offsets"][f * B + b + 1]
                rows = mags[t][pr["ids"][q0:q1] % TABLES[t][0]]
                off = np.maximum(0.25 * rows, rows.max(1, keepdims=True, initial=0) / 6).sum(0) / (max(q1 - q0, 1) if pool else 1)
                assert (np.abs(x[b, col:col + D].double().cpu().numpy() - full[b, col:col + D]) <= off + 1e-5).all()
            col += D
    finally:
        serve.close()
        layer.close()


def test_micro_batches_share_one_output():
    from paper_2204_04903_amd.layer import MicroBatchPipeline
    prs = [problem(20 + m, B) for m, B in enumerate((32, 20, 32))]
    layer = new_layer(prs[0][0])
    try:
        pipe = MicroBatchPipeline(layer, 32, max(len(p[0]["ids"]) for p in prs))
        out = torch.empty((32, layer.out_dim), device="cuda")
        W = torch.randn((12, layer.out_dim), generator=torch.Generator().manual_seed(3)).cuda()
        dw, ref, mag = torch.empty((12, layer.out_dim), device="cuda"), 0.0, 0.0
        for m, (pr, ids, offs) in enumerate(prs):
            t = pipe.submit(ids, offs, pr["B"])
            pooled = pipe.pool(t, out, keep=True)[:pr["B"]]
            grad_y = pooled @ W.t()
            seen = quantized(pooled, 1)
            out.zero_()
            t["kept"].weight_grad(grad_y, out=dw, accumulate=m > 0)
            pipe.backward_update(t, grad_y @ W, 0.01, 1e-8)
            g = grad_y.double().cpu().numpy()
            ref, mag = ref + g.T @ seen, mag + np.abs(g).T @ np.abs(seen)
            assert pipe.ctx_error(t) == 0
        assert (np.abs(dw.double().cpu().numpy() - ref) <= 1.01 * (3 * 84 + 3) * 2.0 ** -23 * mag).all()
    finally:
        layer.close()


def test_replayed_from_a_graph():
    from paper_2204_04903_amd.layer import ActivationCheckpoint, QuantizedEmbedding, QuantizedLinear
    B, N = 130, 70
    pr, ids, offs = problem(7, B)
    layer = new_layer(pr)
    serve = QuantizedEmbedding.from_layer(layer)
    try:
        dense = QuantizedLinear(torch.randn((N, layer.out_dim), device="cuda"), torch.randn(N, device="cuda"))
        grad_y = torch.randn((B, N), device="cuda")

        def step():
            x = serve.forward(ids, offs, B)
            kept = ActivationCheckpoint(B, layer.out_dim).quantize(x)
            return x, dense.forward(x), kept.weight_grad(grad_y), kept.dequantize(dtype=torch.bfloat16), dense.forward(x[:3])

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):                                   # two graphs of the same objects
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                got = step()
            graphs.append((g, got))
        for i in range(3):
            ids.copy_(torch.randint(0, 10 ** 6, ids.shape, device="cuda"))
            grad_y.normal_()
            want = [v.clone() for v in step()]
            for g, got in graphs:
                for v in got:
                    v.zero_()
                g.replay()
                torch.cuda.synchronize()
                for a, b in zip(got, want):
                    assert torch.equal(a, b)
        streams = [torch.cuda.Stream() for _ in graphs]      # and both at once
        torch.cuda.synchronize()
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            for a, b in zip(got, want):
                assert torch.equal(a, b)
        assert serve.error_word() == 0
    finally:
        serve.close()
        layer.close()


def test_on_a_stream_of_its_own():
    from paper_2204_04903_amd.layer import ActivationCheckpoint, QuantizedLinear
    x, w, g = torch.randn((700, 300), device="cuda"), torch.randn((90, 300), device="cuda"), torch.randn((700, 90), device="cuda")
    dense = QuantizedLinear(w)
    want = dense.forward(x), ActivationCheckpoint(700, 300).quantize(x).weight_grad(g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = dense.forward(x), ActivationCheckpoint(700, 300).quantize(x).weight_grad(g)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
