"""Operators on microscaled numbers that stand beside the packed embedding layer, as cases that can be timed.

A microscaled row is cut into blocks of 32 columns; a block has one power of two as its scale, the smallest with which
the block's largest magnitude is no larger than the format's largest value, and its elements are held in 4 bits
(mxfp4: 0, .5, 1, 1.5, 2, 3, 4, 6 and the sign) or in 8 (mxfp8: one sign bit, four of exponent, three of mantissa,
up to 448), each rounded to the nearest, ties to the even code.

  op  codec        a matrix is rounded to microscaled rows and read back: writing and reading an activation
                   checkpoint in 8 bits, or tables in 4
      lookup       the layer's pooled lookup from tables held in 4 bits (serving)
      linear       the product of the pooled output, rounded to 4 bits, with a dense layer's weights held in 4 bits
      weight_grad  the gradient of that dense layer's weights from the pooled output's 8-bit checkpoint, in
                   `parts` micro-batches that add to one gradient
  rows, cols, n    rows (samples); columns of the input; outputs of the dense layer
  src, dst         types of what is read and written: f32 or bf16
  the others       as in perf/cases.py: batch, fields, tables, dims, rows_lo/hi, len_lo/hi, seq_fields, seq_lo/hi, pool, alpha, hashed
"""
import math
import random
import zlib

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
BLOCK = 32
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_LOOKUP = dict(op="lookup", batch=64, fields=26, tables=26, dims="32", rows_lo=100_000, rows_hi=100_000, len_lo=1, len_hi=1,
               seq_fields=0, seq_lo=1, seq_hi=1, pool="sum", alpha=1.05, hashed=False)


def _lookup(**kw):
    return dict(_LOOKUP, **kw)


def listed():
    return [
        # the checkpoint of a small model's pooled output, eight fields of 16 columns: latency counts
        dict(name="small_checkpoint", op="codec", rows=512, cols=128, format="mxfp8", src="f32", dst="f32"),
        # ... of the thousand-field layer, read back for a dense part that computes in bf16
        dict(name="many_fields_checkpoint", op="codec", rows=2048, cols=12000, format="mxfp8", src="f32", dst="bf16"),
        # a trained bf16 table of a million rows on its way to a service, and back
        dict(name="table_codec", op="codec", rows=1_000_000, cols=32, format="mxfp4", src="bf16", dst="f32"),
        # one request of a ranking service: 26 one-hot fields, 64 candidates
        _lookup(name="serve_lookup"),
        # the wide model with multi-hot features: 200 fields, bags of 1 to 50 IDs, mean pooling, four packs
        _lookup(name="multihot_lookup", batch=4096, fields=200, tables=200, dims="8,16,32,64", rows_lo=25_000,
                rows_hi=2_500_000, len_hi=50, pool="mean", alpha=1.2),
        # behaviour sequences: 50 one-hot fields and 10 of 100 to 1000 IDs
        _lookup(name="sequence_lookup", batch=1024, fields=60, tables=60, dims="64", rows_lo=500_000, rows_hi=500_000,
                seq_fields=10, seq_lo=100, seq_hi=1000, alpha=1.1),
        # sizes that fit nothing: odd batch and dimensions, shared tables, empty bags, both poolings, hashed IDs
        _lookup(name="ragged_lookup", batch=3001, fields=37, tables=29, dims="10,24,48,100", rows_lo=700, rows_hi=900_000,
                len_lo=0, len_hi=19, pool="mixed", alpha=1.1, hashed=True),
        # the first dense layer for one sample of a service
        dict(name="one_sample_linear", op="linear", rows=1, cols=832, n=1024, src="f32", dst="f32", bias=True),
        # ... for an evaluation batch of the 26-field model
        dict(name="onehot_linear", op="linear", rows=8192, cols=832, n=1024, src="f32", dst="bf16", bias=True),
        # ... of the thousand-field model
        dict(name="many_fields_linear", op="linear", rows=2048, cols=12000, n=1024, src="f32", dst="f32", bias=True),
        # its weights' gradient: the 26-field model trained in bf16
        dict(name="onehot_weight_grad", op="weight_grad", rows=8192, cols=832, n=1024, src="bf16", parts=1),
        # ... and the thousand-field model in fp32, as four micro-batches
        dict(name="many_fields_weight_grad", op="weight_grad", rows=2048, cols=12000, n=1024, src="f32", parts=4),
    ]


# ---- microscaled rows: 4-byte words of codes, then one scale byte a block, then up to a multiple of `align` bytes ----
def _code_bytes(format, cols):
    return (cols + 7) // 8 * 4 if format == "mxfp4" else (cols + 3) // 4 * 4


def _row_bytes(format, cols, align=4):
    need = _code_bytes(format, cols) + (cols + BLOCK - 1) // BLOCK
    return (need + align - 1) // align * align


def _blocks(x):
    """x [R, C] in 32 bits as [R, blocks, 32], zeros behind the last column."""
    R, C = x.shape
    pad = -C % BLOCK
    return torch.nn.functional.pad(x.float(), (0, pad)).reshape(R, (C + pad) // BLOCK, BLOCK)


def _round(x, format):
    """(elements, exponents of the scales) of x [R, C]: [R, blocks, 32] and [R, blocks, 1]."""
    v = _blocks(x)
    m, e = torch.frexp(v.abs().amax(2, keepdim=True))
    if format == "mxfp4":
        t = e - 3 + (m > 0.75)                  # 6 = .75 * 2^3
    else:
        t = e - 9 + (m > 0.875)                 # 448 = .875 * 2^9
    t = torch.where(m == 0, -126, t.clamp(-126, 127))
    a = torch.ldexp(v, -t)
    size = a.abs()
    if format == "mxfp4":
        step = 0.5 + 0.5 * (size >= 2) + (size >= 4)
    else:
        step = torch.ldexp(torch.ones_like(a), (torch.frexp(size)[1] - 1).clamp(min=-6) - 3)
    return torch.round(a / step) * step, t


def _values(q, t, C):
    return torch.ldexp(q, t).reshape(q.shape[0], -1)[:, :C]


def _pack(x, format, align=4):
    """The bytes of x's microscaled rows, [R, row bytes]."""
    R, C = x.shape
    q, t = _round(x, format)
    q = q.reshape(R, -1)
    if format == "mxfp4":
        code = torch.tensor([0, 1, 2, 3, 4, 0, 5, 0, 6, 0, 0, 0, 7], dtype=torch.uint8, device=x.device)[(2 * q.abs()).long()]
        code = code | (q < 0).to(torch.uint8) * 8
        code = code[:, 0::2] | code[:, 1::2] * 16
    else:
        code = q.to(torch.float8_e4m3fn).view(torch.uint8)
    out = torch.zeros((R, _row_bytes(format, C, align)), dtype=torch.uint8, device=x.device)
    n, blocks = _code_bytes(format, C), t.shape[1]
    out[:, :n] = code[:, :n]
    out[:, n:n + blocks] = (t[:, :, 0] + 127).to(torch.uint8)
    return out


def _unpack(rows, format, C):
    """The values of microscaled rows [R, row bytes], in 32 bits."""
    n, blocks = _code_bytes(format, C), (C + BLOCK - 1) // BLOCK
    code = rows[:, :n]
    if format == "mxfp4":
        of = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=rows.device)
        of = torch.cat([of, -of])
        q = torch.stack([of[(code & 15).long()], of[(code >> 4).long()]], 2).reshape(rows.shape[0], -1)
    else:
        q = code.contiguous().view(torch.float8_e4m3fn).float()
    t = (rows[:, n:n + blocks].int() - 127).repeat_interleave(BLOCK, 1)[:, :C]
    return torch.ldexp(q[:, :C], t)


# ---- inputs ------------------------------------------------------------------------------------------------------
def _gen(case, seed, what):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 1009 + zlib.crc32(what.encode()))
    return g


def _activations(R, C, g):
    """Pooled outputs: every 8 columns of a size of their own, and a bag in 32 that is empty."""
    x = torch.randn((R, C), device=DEVICE, generator=g)
    n = (C + 7) // 8
    x *= (torch.randn(n, device=DEVICE, generator=g) - 3.0).exp_().repeat_interleave(8)[:C]
    return x * (torch.rand((R, n), device=DEVICE, generator=g) >= 1.0 / 32).repeat_interleave(8, 1)[:, :C]


def _matrix(case, seed):
    """What a codec, a linear or a weight_grad case reads: its matrix (rows, cols)."""
    g = _gen(case, seed, "matrix")
    if case.get("format") == "mxfp4":             # a table: rows as training left them, frequent ones larger
        x = torch.randn((case["rows"], case["cols"]), device=DEVICE, generator=g)
        x *= (0.7 * torch.randn((case["rows"], 1), device=DEVICE, generator=g) - 4.0).exp_()
    else:
        x = _activations(case["rows"], case["cols"], g)
    return x if case["op"] == "weight_grad" else x.to(_TYPE[case["src"]])


def _dense(case, seed):
    """A dense layer's weights [n, cols] and bias, and for weight_grad the gradient [rows, n] of its output."""
    g = _gen(case, seed, "dense")
    if case["op"] == "weight_grad":
        # samples weigh differently, and a rectifier behind the layer stops half of the gradient
        d = torch.randn((case["rows"], case["n"]), device=DEVICE, generator=g)
        d *= (torch.randn((case["rows"], 1), device=DEVICE, generator=g) - 7.0).exp_()
        return (d * (torch.rand(d.shape, device=DEVICE, generator=g) < 0.5)).to(_TYPE[case["src"]]), None
    w = torch.randn((case["n"], case["cols"]), device=DEVICE, generator=g) / math.sqrt(case["cols"])
    return w, torch.randn(case["n"], device=DEVICE, generator=g) * 0.1 if case["bias"] else None


def _shape(c):
    """(tables, fields, bag length range per field) of a lookup, from the case alone."""
    text = ",".join("%s=%s" % (k, c[k]) for k in ("fields", "tables", "dims", "rows_lo", "rows_hi", "pool"))
    rng = random.Random(zlib.crc32(text.encode()))
    dims = [int(d) for d in c["dims"].split(",")]
    pool = {"sum": (0,), "mean": (1,), "mixed": (0, 1)}[c["pool"]]
    tables = [(max(2, int(math.exp(rng.uniform(math.log(c["rows_lo"]), math.log(c["rows_hi"]))) + 0.5)), dims[t % len(dims)], 0)
              for t in range(c["tables"])]
    fields = [(f % c["tables"], pool[f % len(pool)]) for f in range(c["fields"])]
    one = c["fields"] - c["seq_fields"]
    return tables, fields, [(c["len_lo"], c["len_hi"])] * one + [(c["seq_lo"], c["seq_hi"])] * c["seq_fields"]


def _pack_dims(tables):
    """Packs are the distinct dimensions, ascending; a pack's tables are stacked in their order."""
    return sorted({d for _, d, _ in tables})


def _pack_rows(tables, dim):
    return sum(r for r, d, _ in tables if d == dim)


def _pack_values(case, seed, dim):
    """Pack `dim`'s stacked tables as training left them."""
    R = _pack_rows(_shape(case)[0], dim)
    g = _gen(case, seed, "pack %d" % dim)
    x = torch.randn((R, dim), device=DEVICE, generator=g)
    return x.mul_((0.7 * torch.randn((R, 1), device=DEVICE, generator=g) - 4.0).exp_())


def _mix64(x):
    """A 64-bit finaliser, on int64 tensors (products wrap, shifts are made logical)."""
    for shift, mult in ((30, 0xBF58476D1CE4E5B9), (27, 0x94D049BB133111EB), (31, None)):
        x = x ^ ((x >> shift) & ((1 << (64 - shift)) - 1))
        if mult is not None:
            x = x * (mult - (1 << 64))
    return x


def _batch(c, seed):
    """IDs and offsets of one batch: field-major bags, IDs by the case's law, hot ranks scattered over the rows."""
    tables, fields, lens = _shape(c)
    g = _gen(c, seed, "batch")
    F, B = len(fields), c["batch"]
    lo = torch.tensor([a for a, _ in lens], device=DEVICE)
    span = torch.tensor([b - a + 1 for a, b in lens], device=DEVICE)
    u = torch.rand((F, B), device=DEVICE, generator=g, dtype=torch.float64)
    n = (lo[:, None] + (u * span[:, None]).long()).reshape(-1)
    offsets = torch.zeros(F * B + 1, dtype=torch.int64, device=DEVICE)
    torch.cumsum(n, 0, out=offsets[1:])
    field = torch.repeat_interleave(torch.arange(F, device=DEVICE), n.view(F, B).sum(1))
    rows = torch.tensor([tables[t][0] for t, _ in fields], dtype=torch.int64, device=DEVICE)[field]
    u = torch.rand(field.shape[0], device=DEVICE, generator=g, dtype=torch.float64)
    if c["alpha"] == 0.0:
        rank = (u * rows).long()
    else:                                     # inverse of the bounded power law on [1, rows + 1)
        e = 1.0 - c["alpha"]
        rank = ((u * ((rows + 1.0) ** e - 1.0) + 1.0) ** (1.0 / e)).long() - 1
    rank = torch.minimum(rank.clamp_(min=0), rows - 1)
    shift = torch.tensor([7919 * (t + 1) for t, _ in fields], dtype=torch.int64, device=DEVICE)[field]
    if c["hashed"]:
        return _mix64(rank * -7046029254386353131 + (shift << 32)), offsets.to(torch.int32)
    mult = torch.tensor([int(r * 0.6180339887498949) | 1 for r, _, _ in tables], dtype=torch.int64, device=DEVICE)
    return (rank * mult[torch.tensor([t for t, _ in fields], device=DEVICE)[field]] + shift) % rows, offsets.to(torch.int32)


# ---- a pass ------------------------------------------------------------------------------------------------------
class _State:
    def __del__(self):
        emb = getattr(self, "emb", None)
        if emb is not None:
            emb.close()


def prepare(case, seed):
    """Inputs, and the tables, weights and checkpoint as bytes of microscaled rows; the framework's objects hold those bytes."""
    s = _State()
    s.case = c = dict(case)
    s.op = c["op"]
    if s.op == "lookup":
        tables, fields, _ = _shape(c)
        s.tables, s.fields, s.dims = tables, fields, _pack_dims(tables)
        s.ids, s.offsets = _batch(c, seed)
        s.packs = [_pack(_pack_values(c, seed, d), "mxfp4") for d in s.dims]
        first, s.base = {d: 0 for d in s.dims}, []
        for r, d, _ in tables:
            s.base.append(first[d])
            first[d] += r
        s.cols = np.concatenate([[0], np.cumsum([tables[t][1] for t, _ in fields])])
        if own:
            from paper_2204_04903_amd.layer import QuantizedEmbedding
            s.emb = QuantizedEmbedding(tables, fields, rows=s.packs)
        return s
    s.x = _matrix(c, seed)
    if s.op == "codec":
        s.format = c["format"]
    elif s.op == "linear":
        w, s.bias = _dense(c, seed)
        s.w = _pack(w, "mxfp4", 16)
    else:
        s.kept = _pack(s.x, "mxfp8", 16)
        s.x = None
        s.dy, _ = _dense(c, seed)
        step = (c["rows"] + c["parts"] - 1) // c["parts"]
        s.cuts = [(a, min(a + step, c["rows"])) for a in range(0, c["rows"], step)]
    if own:
        from paper_2204_04903_amd import binding as pk
        from paper_2204_04903_amd.layer import ActivationCheckpoint, MxRows, QuantizedLinear
        if s.op == "codec":
            s.mx = MxRows(c["rows"], c["cols"], pk.PK_MXFP4 if s.format == "mxfp4" else pk.PK_MXFP8, device=DEVICE)
        elif s.op == "linear":
            s.layer = QuantizedLinear(MxRows(c["n"], c["cols"], pk.PK_MXFP4, device=DEVICE, data=s.w), s.bias)
        else:
            s.parts = [ActivationCheckpoint(b - a, c["cols"], device=DEVICE, data=s.kept[a:b]) for a, b in s.cuts]
    return s


def run(s):
    c = s.case
    if s.op == "codec":
        if own:
            return {"values": s.mx.quantize(s.x).dequantize(dtype=_TYPE[c["dst"]])}
        return {"values": _values(*_round(s.x, s.format), c["cols"]).to(_TYPE[c["dst"]])}
    if s.op == "lookup":
        return {"out": s.emb.forward(s.ids, s.offsets, c["batch"]) if own else _plain_lookup(s)}
    if s.op == "linear":
        if own:
            return {"y": s.layer.forward(s.x, dtype=_TYPE[c["dst"]])}
        y = _values(*_round(s.x, "mxfp4"), c["cols"]) @ _unpack(s.w, "mxfp4", c["cols"]).t()
        return {"y": (y if s.bias is None else y + s.bias).to(_TYPE[c["dst"]])}
    assert s.op == "weight_grad"
    dw = None
    for i, (a, b) in enumerate(s.cuts):
        if own:
            dw = s.parts[i].weight_grad(s.dy[a:b], out=dw, accumulate=i > 0)
        else:
            g = s.dy[a:b].float().t() @ _unpack(s.kept[a:b], "mxfp8", c["cols"])
            dw = g if dw is None else dw + g
    return {"dw": dw}


def _plain_lookup(s):
    """All packs' rows gathered, scaled, added up per bag in 64 bits (bags are long) and rounded once."""
    F, B = len(s.fields), s.case["batch"]
    dev = s.ids.device
    out = torch.empty((B, int(s.cols[-1])), device=dev)
    offsets = s.offsets.long()
    n = offsets[1:] - offsets[:-1]
    bag = torch.repeat_interleave(torch.arange(F * B, device=dev), n)
    of_field = lambda v: torch.tensor([v[t] for t, _ in s.fields], dtype=torch.int64, device=dev)
    f = bag // B
    rows = of_field([r for r, _, _ in s.tables])[f]
    high = (s.ids >> 1) & ((1 << 63) - 1)                       # IDs are unsigned: halves, so that the remainder is one of theirs
    key = (high % rows * 2 + (s.ids & 1)) % rows + of_field(s.base)[f]
    mean = torch.tensor([p == 1 for _, p in s.fields], device=dev)
    scale = torch.where(mean[:, None], 1.0 / n.view(F, B).clamp(min=1), torch.ones((), dtype=torch.float64, device=dev))
    dims = of_field([d for _, d, _ in s.tables])
    for p, d in enumerate(s.dims):
        mine = torch.nonzero(dims == d)[:, 0]
        pos = torch.nonzero(dims[f] == d)[:, 0]
        slot = torch.zeros(F, dtype=torch.int64, device=dev)
        slot[mine] = torch.arange(mine.shape[0], device=dev)
        acc = torch.zeros((mine.shape[0] * B, d), dtype=torch.float64, device=dev)
        acc.index_add_(0, slot[f[pos]] * B + bag[pos] % B, _unpack(s.packs[p][key[pos]], "mxfp4", d).double())
        acc = acc.view(-1, B, d) * scale[mine][:, :, None]
        col = torch.tensor(s.cols[:-1], device=dev)[mine]
        out[:, (col[:, None] + torch.arange(d, device=dev)).reshape(-1)] = acc.permute(1, 0, 2).reshape(B, -1).float()
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def _distinct(rows, n, alpha):
    """Expected number of distinct rows among n draws from the bounded power law over `rows` rows."""
    edge = np.unique(np.round(np.exp(np.linspace(0.0, math.log(rows + 1.0), 400)))).astype(np.float64)
    if alpha == 0.0:
        cum = (edge - 1.0) / rows
    else:
        e = 1.0 - alpha
        cum = (edge ** e - 1.0) / ((rows + 1.0) ** e - 1.0)
    width = np.diff(edge)
    return float(np.sum(width * -np.expm1(-n * np.diff(cum) / width)))


def _nnz(c):
    return c["batch"] * sum(lo + hi for lo, hi in _shape(c)[2]) / 2.0


def work(case):
    c = case
    size = {"f32": 4, "bf16": 2}
    if c["op"] == "lookup":
        tables, fields, lens = _shape(c)
        occ, nnz, out_dim, flops = [0.0] * len(tables), 0.0, 0, 0.0
        for (t, _), (lo, hi) in zip(fields, lens):
            m = c["batch"] * (lo + hi) / 2.0
            occ[t] += m
            nnz += m
            out_dim += tables[t][1]
            flops += m * tables[t][1]
        total = 8.0 * nnz + 4.0 * (len(fields) * c["batch"] + 1) + 4.0 * c["batch"] * out_dim
        total += sum(_distinct(r, m, c["alpha"]) * (_code_bytes("mxfp4", d) + (d + BLOCK - 1) // BLOCK)
                     for (r, d, _), m in zip(tables, occ) if m > 0)
        return {"bytes": total, "flops": flops}
    R, C = c["rows"], c["cols"]
    bytes4, bytes8 = (_code_bytes(f, C) + (C + BLOCK - 1) // BLOCK for f in ("mxfp4", "mxfp8"))
    if c["op"] == "codec":       # the rows are written and read
        return {"bytes": float(R) * (C * (size[c["src"]] + size[c["dst"]]) + 2 * (bytes4 if c["format"] == "mxfp4" else bytes8)),
                "flops": 4.0 * R * C}
    if c["op"] == "linear":
        return {"bytes": float(R) * C * size[c["src"]] + float(c["n"]) * (bytes4 + 4 * c["bias"]) + float(R) * c["n"] * size[c["dst"]],
                "flops": 2.0 * R * C * c["n"]}
    return {"bytes": float(R) * bytes8 + float(R) * c["n"] * size[c["src"]] + 4.0 * c["n"] * C,
            "flops": 2.0 * R * C * c["n"]}


# ---- from the definition, in 64 bits ---------------------------------------------------------------------------------
def _nearest(x, format):
    """Every element of x [R, C] as what its microscaled row holds for it: of all the format's values times the block's
    scale the nearest, of two as near the one with the even code."""
    if format == "mxfp4":
        grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        grid = [(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127]
    grid = torch.tensor(grid, dtype=torch.float64, device=x.device)
    y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    whole = x.shape[1] // BLOCK * BLOCK
    for a, b, k in ((0, whole, BLOCK), (whole, x.shape[1], x.shape[1] - whole)):
        if a == b:
            continue
        v = x[:, a:b].double().reshape(-1, k)
        top = v.abs().max(1, keepdim=True).values
        t = torch.ceil(torch.log2(top / grid[-1]))
        t = torch.where(torch.exp2(t - 1) * grid[-1] >= top, t - 1, t)           # (the logarithm is rounded: its neighbours are looked at)
        t = torch.where(torch.exp2(t) * grid[-1] < top, t + 1, t)
        s = torch.exp2(torch.where(top > 0, t, torch.zeros_like(t)).clamp(-126, 127))
        u = (v / s).abs()
        up = torch.searchsorted(grid, u).clamp(max=grid.shape[0] - 1)            # the first value that is not below it
        down = (up - 1).clamp(min=0)
        near, far = u - grid[down], grid[up] - u
        pick = torch.where((far < near) | ((far == near) & (up % 2 == 0)), up, down)
        y[:, a:b] = (grid[pick] * v.sign() * s).reshape(x.shape[0], b - a)
    return y


def exact(case, seed):
    c = case
    if c["op"] == "codec":
        return {"values": _nearest(_matrix(c, seed), c["format"])}
    if c["op"] == "linear":
        w, bias = _dense(c, seed)
        y = _nearest(_matrix(c, seed), "mxfp4").matmul(_nearest(w, "mxfp4").T.contiguous())
        return {"y": y if bias is None else y + bias.double()}
    if c["op"] == "weight_grad":
        return {"dw": _dense(c, seed)[0].double().T.contiguous().matmul(_nearest(_matrix(c, seed), "mxfp8"))}
    # a field's bags are differences of the running sum over its IDs' rows
    tables, fields, _ = _shape(c)
    B = c["batch"]
    ids, offsets = _batch(c, seed)
    offsets = offsets.long()
    first = offsets[::B].tolist()
    out, width = [None] * len(fields), []
    for d in _pack_dims(tables):
        stacked = _nearest(_pack_values(c, seed, d), "mxfp4").float()           # (held in 32 bits: the values have two digits)
        at = 0
        for t, (r, dim, _) in enumerate(tables):
            if dim != d:
                continue
            for f in range(t, len(fields), len(tables)):
                mine = ids[first[f]:first[f + 1]]
                row = torch.remainder(torch.remainder(mine, r) + (mine < 0) * ((1 << 64) % r), r)
                run_sum = torch.cat([torch.zeros((1, d), dtype=torch.float64, device=ids.device),
                                     stacked[at:at + r][row].double().cumsum(0)])
                edge = offsets[f * B:(f + 1) * B + 1] - first[f]
                bags = run_sum[edge[1:]] - run_sum[edge[:-1]]
                if fields[f][1] == 1:
                    bags = bags / (edge[1:] - edge[:-1]).clamp(min=1)[:, None]
                out[f] = bags
            at += r
    return {"out": torch.cat(out, 1)}


# ---- more cases of the same ranges -----------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return max(int(lo), min(int(hi), int(math.exp(rng.uniform(math.log(lo), math.log(hi))) + 0.5)))


def _one(rng):
    op = rng.choice(["codec", "lookup", "lookup", "linear", "weight_grad"])
    if op == "codec":
        return dict(op=op, rows=_log(rng, 1, 1_000_000), cols=_log(rng, 1, 12000), format=rng.choice(["mxfp4", "mxfp8"]),
                    src=rng.choice(["f32", "bf16"]), dst=rng.choice(["f32", "bf16"]))
    if op == "linear":
        return dict(op=op, rows=_log(rng, 1, 16384), cols=_log(rng, 8, 12000), n=_log(rng, 1, 2048),
                    src=rng.choice(["f32", "f32", "bf16"]), dst=rng.choice(["f32", "bf16"]), bias=rng.random() < 0.5)
    if op == "weight_grad":
        return dict(op=op, rows=_log(rng, 8, 16384), cols=_log(rng, 8, 12000), n=_log(rng, 1, 2048),
                    src=rng.choice(["f32", "bf16"]), parts=rng.choice([1, 1, 2, 4, 8]))
    alpha = rng.choice([0.0, round(rng.uniform(1.01, 1.3), 2), round(rng.uniform(1.01, 1.3), 2)])
    kind = rng.choice(["onehot", "multihot", "sequence", "ragged"])
    if kind == "onehot":
        F, rows = _log(rng, 4, 64), _log(rng, 1000, 1_000_000)
        return _lookup(batch=_log(rng, 1, 8192), fields=F, tables=F, dims=rng.choice(["4", "8", "16", "32", "64", "128"]),
                       rows_lo=rows, rows_hi=rows, alpha=alpha, hashed=rng.random() < 0.3)
    if kind == "multihot":
        F, lo = _log(rng, 20, 600), _log(rng, 1000, 25_000)
        return _lookup(batch=_log(rng, 64, 4096), fields=F, tables=F, dims=rng.choice(["8,16,32,64", "16,32", "8,16", "32", "4,16,128"]),
                       rows_lo=lo, rows_hi=100 * lo, len_hi=_log(rng, 2, 60), pool=rng.choice(["sum", "mean", "mixed"]), alpha=alpha,
                       hashed=rng.random() < 0.3)
    if kind == "sequence":
        F, hi, rows = _log(rng, 4, 80), _log(rng, 100, 1500), _log(rng, 20_000, 500_000)
        return _lookup(batch=_log(rng, 16, 1024), fields=F, tables=F, dims=rng.choice(["16", "32", "64", "128"]), rows_lo=rows, rows_hi=rows,
                       seq_fields=min(F, _log(rng, 1, 12)), seq_lo=max(1, hi // 10), seq_hi=hi, alpha=alpha, pool=rng.choice(["sum", "mean"]))
    F, lo = _log(rng, 5, 120), _log(rng, 50, 5000)
    return _lookup(batch=_log(rng, 1, 5000) | 1, fields=F, tables=max(1, F - rng.randrange(1 + F // 3)),
                   dims=rng.choice(["10,24,48,100", "3,20", "12,36,200", "5,16,48", "256,6", "1,33"]), rows_lo=lo, rows_hi=200 * lo,
                   len_lo=rng.choice([0, 0, 1]), len_hi=_log(rng, 1, 25), pool=rng.choice(["sum", "mean", "mixed"]), alpha=alpha,
                   hashed=rng.random() < 0.3)


def draw(rng):
    def room(c):
        return sum(r * d for r, d, _ in _shape(c)[0]) if c["op"] == "lookup" else 0
    top = [work(c) for c in listed()]
    most = {k: max(w[k] for w in top) for k in ("bytes", "flops")}
    lookups = [c for c in listed() if c["op"] == "lookup"]
    most_nnz, most_room = max(_nnz(c) for c in lookups), max(room(c) for c in lookups)
    while True:
        c = _one(rng)
        w = work(c)
        if w["bytes"] > most["bytes"] or w["flops"] > most["flops"]:
            continue
        if c["op"] == "codec" and c["rows"] * c["cols"] < 64:
            continue
        if c["op"] == "weight_grad" and c["parts"] > c["rows"]:
            continue
        if c["op"] != "lookup" or (_nnz(c) >= 16 and _nnz(c) <= most_nnz and room(c) <= most_room):
            return c
