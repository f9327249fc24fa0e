"""Buffer management around the C ABI: allocates the packed tables, the Adagrad
accumulators, the output and the workspace as torch device tensors and hands
their addresses to the library.  No arithmetic happens here."""
from __future__ import annotations

from typing import List, Sequence, Tuple

import numpy as np
import torch

from . import binding as pk


class PackedEmbedding:
    def __init__(self, tables: Sequence[Tuple[int, int, int]], fields: Sequence[Tuple[int, int]],
                 device: str = "cuda:0", **plan_opts):
        self.tables, self.fields = list(tables), list(fields)
        self.device = torch.device(device)
        self.plan = pk.pk_plan_create(self.tables, self.fields, **plan_opts)
        self.n_packs = pk.pk_plan_num_packs(self.plan)
        self.packs = [pk.pk_plan_pack_info(self.plan, p) for p in range(self.n_packs)]
        self.pack_fields = [pk.pk_plan_pack_fields(self.plan, p) for p in range(self.n_packs)]
        self.table_slot = [pk.pk_plan_table_slot(self.plan, t) for t in range(len(self.tables))]
        self.field_col = [pk.pk_plan_field_col(self.plan, f) for f in range(len(self.fields))]
        self.out_dim = pk.pk_plan_out_dim(self.plan)
        self.W: List[torch.Tensor] = []
        self.A: List[torch.Tensor] = []
        for info in self.packs:
            dt = torch.float32 if info["dtype"] == pk.PK_F32 else torch.bfloat16
            self.W.append(torch.empty((info["total_rows"], info["dim"]), dtype=dt, device=self.device))
            self.A.append(torch.zeros((info["total_rows"], info["dim"]), dtype=torch.float32, device=self.device))
        self.ws = None
        self.ws_bytes = 0
        self._shape = None

    def close(self):
        if self.plan:
            pk.pk_plan_destroy(self.plan)
            self.plan = None

    def table_view(self, t: int) -> torch.Tensor:
        p, base = self.table_slot[t]
        return self.W[p][base:base + self.tables[t][0]]

    def acc_view(self, t: int) -> torch.Tensor:
        p, base = self.table_slot[t]
        return self.A[p][base:base + self.tables[t][0]]

    def load_table(self, t: int, values: np.ndarray) -> None:
        """values: float32 [rows, dim], or uint16 bf16 bit patterns for a bf16 table."""
        values = np.ascontiguousarray(values)
        if self.tables[t][2] == pk.PK_BF16:
            v = torch.from_numpy(values.view(np.int16)).view(torch.bfloat16)
        else:
            v = torch.from_numpy(values)
        self.table_view(t).copy_(v.to(self.device))

    def _ensure_ws(self, B: int, nnz: int) -> None:
        need = pk.pk_workspace_bytes(self.plan, B, nnz)
        if self.ws is None or self.ws_bytes < need:
            self.ws = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
            self.ws_bytes = need
        self._shape = (B, nnz)

    def forward(self, ids: torch.Tensor, offsets: torch.Tensor, B: int, out: torch.Tensor = None) -> torch.Tensor:
        nnz = int(ids.shape[0])
        self._ensure_ws(B, nnz)
        if out is None:
            out = torch.empty((B, self.out_dim), dtype=torch.float32, device=self.device)
        stream = torch.cuda.current_stream(self.device).cuda_stream
        pk.pk_forward(self.plan, self.W, ids, offsets, B, nnz, out, out.stride(0), self.ws, self.ws_bytes, stream)
        return out

    def backward_update(self, grad_out: torch.Tensor, lr: float, eps: float) -> None:
        B, nnz = self._shape
        stream = torch.cuda.current_stream(self.device).cuda_stream
        pk.pk_backward_update(self.plan, self.W, self.A, grad_out, grad_out.stride(0), B, nnz, lr, eps, self.ws,
                              self.ws_bytes, stream)

    def ctx(self, p: int) -> dict:
        """Pack p's saved context copied to numpy (synchronises)."""
        B, nnz = self._shape
        d = pk.pk_ctx_pack(self.plan, self.ws, B, nnz, p)
        base = self.ws.data_ptr()

        def grab(addr, n, dtype):
            off = addr - base
            return self.ws[off:off + 4 * n].view(dtype).cpu().numpy().copy()

        k = len(self.pack_fields[p])
        return dict(
            nnz_p=d["nnz_p"], n_unique=d["n_unique"],
            keys=grab(d["keys"], d["nnz_p"], torch.int32).view(np.uint32),
            unique=grab(d["unique"], d["n_unique"], torch.int32).view(np.uint32),
            inverse=grab(d["inverse"], d["nnz_p"], torch.int32),
            packed_offsets=grab(d["packed_offsets"], k * B + 1, torch.int32),
            seg_offsets=grab(d["seg_offsets"], d["n_unique"] + 1, torch.int32),
        )

    def error_word(self) -> int:
        return pk.pk_ctx_error(self.plan, self.ws)

    def partition(self, p: int, n_owners: int):
        """Sec. II-D Partition of pack p's distinct keys by owner (row mod n_owners), after a forward pass.
        Returns device tensors (part_keys [nnz] int32 bits of uint32, part_index [nnz] int32, part_offsets
        [n_owners + 1] int32); only the first part_offsets[-1] entries of the first two are meaningful."""
        B, nnz = self._shape
        need = pk.pk_partition_scratch_bytes(self.plan, nnz, n_owners)
        scratch = torch.empty(need, dtype=torch.uint8, device=self.device)
        keys = torch.empty(max(nnz, 1), dtype=torch.int32, device=self.device)
        index = torch.empty(max(nnz, 1), dtype=torch.int32, device=self.device)
        offsets = torch.empty(n_owners + 1, dtype=torch.int32, device=self.device)
        stream = torch.cuda.current_stream(self.device).cuda_stream
        pk.pk_partition_unique(self.plan, self.ws, self.ws_bytes, B, nnz, p, n_owners, keys, index, offsets, scratch,
                               need, stream)
        return keys, index, offsets


class MicroBatchPipeline:
    """D-Interleaving of the layer (Sec. III-C): micro-batches pass through it one after the other, and the
    dedup of the next one (integer work that reads no table) is enqueued on a second stream while the current
    one is pooled and updated on the caller's stream.  Two workspaces, sized for a micro-batch, alternate.
    Scheduling only: every step runs in the library's kernels.

        t = pipe.submit(ids0, offsets0, B0)
        for m in range(M):
            nxt = pipe.submit(ids[m + 1], offsets[m + 1], B[m + 1]) if m + 1 < M else None
            pipe.pool(t, out[m]); ...; pipe.backward_update(t, grad[m], lr, eps)
            t = nxt

    The tensors handed to `submit` must stay alive until the micro-batch has been updated."""

    def __init__(self, layer: PackedEmbedding, max_B: int, max_nnz: int):
        self.layer = layer
        self.ws_bytes = pk.pk_workspace_bytes(layer.plan, max_B, max_nnz)
        self.ws = [torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=layer.device) for _ in range(2)]
        self.side = torch.cuda.Stream(device=layer.device)
        self.ev_inputs = [torch.cuda.Event() for _ in range(2)]
        self.ev_dedup = [torch.cuda.Event() for _ in range(2)]
        self.count = 0

    def submit(self, ids: torch.Tensor, offsets: torch.Tensor, B: int) -> dict:
        """Enqueue the dedup of a micro-batch.  It starts once everything enqueued so far on the caller's
        stream has run: the inputs are there, and the workspace's previous micro-batch has been updated."""
        layer, slot = self.layer, self.count % 2
        self.count += 1
        nnz = int(ids.shape[0])
        if pk.pk_workspace_bytes(layer.plan, B, nnz) > self.ws_bytes:
            raise ValueError("micro-batch larger than the pipeline was sized for")
        main = torch.cuda.current_stream(layer.device)
        self.ev_inputs[slot].record(main)
        self.side.wait_event(self.ev_inputs[slot])
        pk.pk_forward_dedup(layer.plan, ids, offsets, B, nnz, self.ws[slot], self.ws_bytes, self.side.cuda_stream)
        self.ev_dedup[slot].record(self.side)
        return dict(slot=slot, B=B, nnz=nnz)

    def pool(self, t: dict, out: torch.Tensor, keep: bool = False) -> torch.Tensor:
        """keep: the pooled output is also kept in 8 bits, as t["kept"] (an ActivationCheckpoint), for the gradient of the
        weights that multiply it; the micro-batches can then share one `out`."""
        layer = self.layer
        main = torch.cuda.current_stream(layer.device)
        main.wait_event(self.ev_dedup[t["slot"]])
        pk.pk_forward_pool(layer.plan, layer.W, t["B"], t["nnz"], out, out.stride(0), self.ws[t["slot"]],
                           self.ws_bytes, main.cuda_stream)
        if keep:
            t["kept"] = ActivationCheckpoint(t["B"], layer.out_dim, device=layer.device).quantize(out[:t["B"], :layer.out_dim])
        return out

    def backward_update(self, t: dict, grad_out: torch.Tensor, lr: float, eps: float) -> None:
        layer = self.layer
        main = torch.cuda.current_stream(layer.device)
        pk.pk_backward_update(layer.plan, layer.W, layer.A, grad_out, grad_out.stride(0), t["B"], t["nnz"], lr, eps,
                              self.ws[t["slot"]], self.ws_bytes, main.cuda_stream)

    def ctx_error(self, t: dict) -> int:
        return pk.pk_ctx_error(self.layer.plan, self.ws[t["slot"]])


_MX_DTYPE = {torch.float32: pk.PK_F32, torch.bfloat16: pk.PK_BF16}


def _device(device) -> torch.device:
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device


def _matrix(x: torch.Tensor, name: str, rows: int, cols: int, device, dtypes=_MX_DTYPE) -> int:
    """Checks a matrix argument; returns its row stride in elements."""
    if x.dim() != 2 or x.shape[0] != rows or x.shape[1] != cols:
        raise ValueError(f"{name} must be [{rows}, {cols}], got {list(x.shape)}")
    if x.dtype not in dtypes:
        raise ValueError(f"{name} must be one of {list(dtypes)}, got {x.dtype}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, expected {device}")
    s0, s1 = x.stride()
    if rows == 0 or cols == 0:
        return cols
    if cols > 1 and s1 != 1:
        raise ValueError(f"{name}: neighbouring columns must be neighbours in memory")
    if rows > 1 and s0 < cols:
        raise ValueError(f"{name}: rows overlap")
    return s0 if rows > 1 else cols


def _enqueue(device, call, *args) -> None:
    """The library's call on the device's current stream, with the device current."""
    if device.type != "cuda":
        raise ValueError(f"the library computes on a GPU, not on {device}")
    stream = torch.cuda.current_stream(device.index).cuda_stream
    if torch.cuda.current_device() == device.index:
        call(*args, stream)
    else:
        with torch.cuda.device(device):
            call(*args, stream)


class MxRows:
    """A matrix as microscaled rows (4- or 8-bit elements, one scale per 32 columns) in one device buffer.

        rows = MxRows(n_rows, cols, pk.PK_MXFP4).quantize(x)      # x: fp32 or bf16 [n_rows, cols]
        y = rows.dequantize()                                     # fp32, or dtype=torch.bfloat16

    `data`: a uint8 tensor [n_rows, stride] that holds (or will hold) the rows; else one is allocated whose rows are
    `align` bytes apart or a multiple of that.  Buffer management only."""

    def __init__(self, n_rows: int, cols: int, format: int, device: str = "cuda:0", data: torch.Tensor = None, align: int = 16):
        self.n_rows, self.cols, self.format = int(n_rows), int(cols), int(format)
        self.device = _device(device)
        need = pk.pk_mx_row_bytes(self.format, self.cols)
        if data is None:
            stride = (need + align - 1) // align * align
            data = torch.empty((self.n_rows, stride), dtype=torch.uint8, device=self.device)
        stride = data.stride(0) if data.dim() == 2 and data.shape[0] > 1 else data.shape[-1]
        if (data.dim() != 2 or data.dtype != torch.uint8 or data.shape[0] != self.n_rows or data.shape[1] < need or
                data.device != self.device or (data.shape[1] > 1 and data.stride(1) != 1) or stride < need or stride % 4 or
                data.data_ptr() % 4):
            raise ValueError(f"data must be uint8 [{self.n_rows}, >= {need}] on {self.device}, rows a multiple of 4 bytes apart")
        self.data, self.stride = data, stride

    def quantize(self, x: torch.Tensor) -> "MxRows":
        stride = _matrix(x, "x", self.n_rows, self.cols, self.device)
        _enqueue(self.device, pk.pk_mx_quantize, x, _MX_DTYPE[x.dtype], stride, self.n_rows, self.cols, self.format, self.data, self.stride)
        return self

    def dequantize(self, out: torch.Tensor = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        if out is None:
            out = torch.empty((self.n_rows, self.cols), dtype=dtype, device=self.device)
        stride = _matrix(out, "out", self.n_rows, self.cols, self.device)
        _enqueue(self.device, pk.pk_mx_dequantize, self.data, self.stride, self.n_rows, self.cols, self.format, out, _MX_DTYPE[out.dtype], stride)
        return out


class ActivationCheckpoint(MxRows):
    """The input of a dense layer (the pooled output, say) kept in 8 bits from the forward to the backward pass.

        kept = ActivationCheckpoint(B, layer.out_dim).quantize(out)      # out's memory can be used again
        ...
        dw = kept.weight_grad(grad_y)                                    # [N, cols] = grad_y^T times the kept input
        dw = kept.weight_grad(grad_y, out=dw, accumulate=True)           # a further micro-batch's share"""

    def __init__(self, n_rows: int, cols: int, device: str = "cuda:0", data: torch.Tensor = None):
        super().__init__(n_rows, cols, pk.PK_MXFP8, device=device, data=data)

    def weight_grad(self, grad_y: torch.Tensor, out: torch.Tensor = None, accumulate: bool = False) -> torch.Tensor:
        if grad_y.dim() != 2:
            raise ValueError("grad_y must have two dimensions")
        N = int(grad_y.shape[1])
        grad_stride = _matrix(grad_y, "grad_y", self.n_rows, N, self.device)
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs out")
            out = torch.empty((N, self.cols), dtype=torch.float32, device=self.device)
        out_stride = _matrix(out, "out", N, self.cols, self.device, (torch.float32,))
        ws_bytes = pk.pk_mx_weight_grad_workspace_bytes(self.n_rows, N, self.cols)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)       # (the allocator's: free again when the stream is past it)
        _enqueue(self.device, pk.pk_mx_weight_grad, grad_y, _MX_DTYPE[grad_y.dtype], grad_stride, self.data, self.stride, self.n_rows, N, self.cols,
                 out, out_stride, accumulate, ws, ws_bytes)
        return out


class QuantizedLinear:
    """A dense layer with its weights in 4 bits; its input is rounded to 4 bits on the way in.

        dense = QuantizedLinear(weight, bias)            # weight: fp32 or bf16 [N, K]; bias: fp32 [N] or None
        y = dense.forward(out)                           # out: fp32 or bf16 [M, K]; y: fp32, or dtype=torch.bfloat16

    `weight` may be an MxRows of PK_MXFP4 rows instead.  The layer keeps the weights in rows of its own, `dense.weight`, that begin on
    128-byte lines: what is written to `weight` later does not change it, `dense.weight.quantize(...)` does.  Buffer management only."""

    def __init__(self, weight, bias: torch.Tensor = None):
        if isinstance(weight, MxRows) and weight.format != pk.PK_MXFP4:
            raise ValueError("weight rows must be PK_MXFP4")
        self.N, self.K = (weight.n_rows, weight.cols) if isinstance(weight, MxRows) else (int(n) for n in weight.shape)
        # (whole lines a row: what the product reads of one is what it needs)
        self.weight = MxRows(self.N, self.K, pk.PK_MXFP4, device=weight.device, align=128)
        self.device = self.weight.device
        if isinstance(weight, MxRows):
            need = pk.pk_mx_row_bytes(pk.PK_MXFP4, self.K)
            self.weight.data[:, :need].copy_(weight.data[:, :need])
        else:
            self.weight.quantize(weight)
        if bias is not None and (bias.dtype != torch.float32 or bias.shape != (self.N,) or bias.device != self.device or
                                 (self.N > 1 and bias.stride(0) != 1)):
            raise ValueError(f"bias must be fp32 [{self.N}], contiguous, on {self.device}")
        self.bias = bias

    def forward(self, x: torch.Tensor, out: torch.Tensor = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        if x.dim() != 2:
            raise ValueError("x must have two dimensions")
        M = int(x.shape[0])
        x_stride = _matrix(x, "x", M, self.K, self.device)
        if out is None:
            out = torch.empty((M, self.N), dtype=dtype, device=self.device)
        out_stride = _matrix(out, "out", M, self.N, self.device)
        ws_bytes = pk.pk_mx_linear_workspace_bytes(M, self.N, self.K)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)
        _enqueue(self.device, pk.pk_mx_linear, x, _MX_DTYPE[x.dtype], x_stride, M, self.weight.data, self.weight.stride, self.N, self.K, self.bias, out,
                 _MX_DTYPE[out.dtype], out_stride, ws, ws_bytes)
        return out


class QuantizedEmbedding:
    """The layer for serving: its tables in 4 bits (0.53 bytes a column from 32 columns on), pooled lookups only.

        serve = QuantizedEmbedding.from_layer(layer)     # or QuantizedEmbedding(tables, fields) and load_table
        out = serve.forward(ids, offsets, B)             # as PackedEmbedding.forward

    `rows`: the packs' tables as microscaled rows where they are there already, uint8 [total_rows, pk_mx_row_bytes] each.
    Buffer management only."""

    def __init__(self, tables: Sequence[Tuple[int, int, int]], fields: Sequence[Tuple[int, int]], device: str = "cuda:0",
                 rows: Sequence[torch.Tensor] = None, **plan_opts):
        self.tables, self.fields = list(tables), list(fields)
        self.device = _device(device)
        self.plan = pk.pk_plan_create(self.tables, self.fields, **plan_opts)
        try:
            self._hold(rows)
        except BaseException:
            self.close()                                     # (nobody else can: the caller gets no object)
            raise

    def _hold(self, rows) -> None:
        self.n_packs = pk.pk_plan_num_packs(self.plan)
        self.packs = [pk.pk_plan_pack_info(self.plan, p) for p in range(self.n_packs)]
        self.table_slot = [pk.pk_plan_table_slot(self.plan, t) for t in range(len(self.tables))]
        self.field_col = [pk.pk_plan_field_col(self.plan, f) for f in range(len(self.fields))]
        self.out_dim = pk.pk_plan_out_dim(self.plan)
        if rows is not None and len(rows) != self.n_packs:
            raise ValueError(f"rows must be a list of {self.n_packs} packs")
        # (rows stand close together: a lookup reads single rows, and what it reads is what it costs)
        self.T = [MxRows(k["total_rows"], k["dim"], pk.PK_MXFP4, device=self.device, data=rows[p] if rows is not None else None, align=4)
                  for p, k in enumerate(self.packs)]
        for m in self.T:
            if m.stride != pk.pk_mx_row_bytes(m.format, m.cols):
                raise ValueError("a pack's rows must be pk_mx_row_bytes apart")
        self._T = [m.data for m in self.T]
        self.error = torch.zeros(1, dtype=torch.int32, device=self.device)

    @classmethod
    def from_layer(cls, layer: PackedEmbedding, **plan_opts) -> "QuantizedEmbedding":
        """The tables of a trained layer, rounded to 4 bits (plan_opts: as the layer's, where they change its packs)."""
        if isinstance(layer, HybridEmbedding):
            raise ValueError("rows in a Hot-storage are newer than the tables: quantize a PackedEmbedding")
        q = cls(layer.tables, layer.fields, device=layer.device, **plan_opts)
        try:
            if [(k["dim"], k["dtype"], k["total_rows"]) for k in q.packs] != [(k["dim"], k["dtype"], k["total_rows"]) for k in layer.packs]:
                raise ValueError("the layer was made with other plan options")
            for t in range(len(q.tables)):
                q.load_table(t, layer.table_view(t))
        except BaseException:
            q.close()
            raise
        return q

    def close(self):
        if self.plan:
            pk.pk_plan_destroy(self.plan)
            self.plan = None

    def load_table(self, t: int, values: torch.Tensor) -> None:
        """values: fp32 or bf16 [rows, dim]; rounded to 4 bits (a copy on the host is moved to the device first)."""
        p, base = self.table_slot[t]
        n, m = self.tables[t][0], self.T[p]
        MxRows(n, m.cols, m.format, device=self.device, data=m.data[base:base + n]).quantize(values.to(self.device))

    def forward(self, ids: torch.Tensor, offsets: torch.Tensor, B: int, out: torch.Tensor = None) -> torch.Tensor:
        for x, name, dt, n in ((ids, "ids", torch.int64, None), (offsets, "offsets", torch.int32, len(self.fields) * B + 1)):
            if x.dtype != dt or x.dim() != 1 or x.device != self.device or not x.is_contiguous() or (n is not None and x.shape[0] != n):
                raise ValueError(f"{name} must be contiguous {dt} on {self.device}" + (f", {n} of them" if n is not None else ""))
        if out is None:
            out = torch.empty((B, self.out_dim), dtype=torch.float32, device=self.device)
        stride = _matrix(out, "out", B, self.out_dim, self.device, (torch.float32,))
        _enqueue(self.device, pk.pk_mx_forward, self.plan, self._T, ids, offsets, B, ids.shape[0], out, stride, self.error)
        return out

    def error_word(self) -> int:
        """Bit 0: some call's offsets were rejected since the word was last read (reading clears it).  Synchronises the device, whatever
        streams the calls were on, and is not to be called while another thread makes some."""
        torch.cuda.synchronize(self.device)
        w = int(self.error.item())
        if w:
            self.error.zero_()
            torch.cuda.synchronize(self.device)              # (a call that follows on another stream may raise it again)
        return w


class HybridEmbedding(PackedEmbedding):
    """The layer with a Hot-storage in front of its tables (HybridHash): the tables and accumulators are the
    Cold-storage, in pinned host memory when `cold_on_host`, and the `hot_rows[p]` most queried rows of pack p
    live in device memory.  Buffer management only."""

    def __init__(self, tables, fields, hot_rows: Sequence[int], warmup_iters: int, flush_iters: int,
                 cold_on_host: bool = True, device: str = "cuda:0", **plan_opts):
        self.tables, self.fields = list(tables), list(fields)
        self.device = torch.device(device)
        self.plan = pk.pk_plan_create(self.tables, self.fields, **plan_opts)
        self.n_packs = pk.pk_plan_num_packs(self.plan)
        self.packs = [pk.pk_plan_pack_info(self.plan, p) for p in range(self.n_packs)]
        self.pack_fields = [pk.pk_plan_pack_fields(self.plan, p) for p in range(self.n_packs)]
        self.table_slot = [pk.pk_plan_table_slot(self.plan, t) for t in range(len(self.tables))]
        self.field_col = [pk.pk_plan_field_col(self.plan, f) for f in range(len(self.fields))]
        self.out_dim = pk.pk_plan_out_dim(self.plan)
        self.warmup_iters, self.flush_iters, self.itr = int(warmup_iters), int(flush_iters), 0
        self.W, self.A, self.hh = [], [], []
        for p, info in enumerate(self.packs):
            dt = torch.float32 if info["dtype"] == pk.PK_F32 else torch.bfloat16
            R, D, k = info["total_rows"], info["dim"], int(hot_rows[p])
            if cold_on_host:
                Wc = torch.empty((R, D), dtype=dt, pin_memory=True)
                Ac = torch.zeros((R, D), dtype=torch.float32, pin_memory=True)
            else:
                Wc = torch.empty((R, D), dtype=dt, device=self.device)
                Ac = torch.zeros((R, D), dtype=torch.float32, device=self.device)
            self.W.append(Wc)
            self.A.append(Ac)
            self.hh.append(dict(
                W_cold=Wc, A_cold=Ac, hot_rows=k,
                W_hot=torch.empty((max(k, 1), D), dtype=dt, device=self.device),
                A_hot=torch.empty((max(k, 1), D), dtype=torch.float32, device=self.device),
                slot_of=torch.empty(R, dtype=torch.int32, device=self.device),
                hot_row=torch.empty(max(k, 1), dtype=torch.int32, device=self.device),
                fcounter=torch.empty(R, dtype=torch.int32, device=self.device)))
        self.scratch_bytes = pk.pk_hh_scratch_bytes(self.plan, self.hh)
        self.scratch = torch.empty(self.scratch_bytes + 256, dtype=torch.uint8, device=self.device)
        self.ws, self.ws_bytes, self._shape = None, 0, None
        pk.pk_hh_init(self.plan, self.hh, torch.cuda.current_stream(self.device).cuda_stream)

    def load_table(self, t: int, values: np.ndarray) -> None:
        values = np.ascontiguousarray(values)
        if self.tables[t][2] == pk.PK_BF16:
            v = torch.from_numpy(values.view(np.int16)).view(torch.bfloat16)
        else:
            v = torch.from_numpy(values)
        self.table_view(t).copy_(v)

    def forward(self, ids, offsets, B: int, out=None):
        nnz = int(ids.shape[0])
        self._ensure_ws(B, nnz)
        if out is None:
            out = torch.empty((B, self.out_dim), dtype=torch.float32, device=self.device)
        stream = torch.cuda.current_stream(self.device).cuda_stream
        pk.pk_hh_forward(self.plan, self.hh, ids, offsets, B, nnz, out, out.stride(0), self.ws, self.ws_bytes, stream)
        return out

    def backward_update(self, grad_out, lr: float, eps: float) -> None:
        B, nnz = self._shape
        stream = torch.cuda.current_stream(self.device).cuda_stream
        pk.pk_hh_backward_update(self.plan, self.hh, grad_out, grad_out.stride(0), B, nnz, lr, eps, self.ws,
                                 self.ws_bytes, stream)

    def end_iteration(self, want_counts: bool = True):
        """Alg. 1's bookkeeping for the batch just processed; returns (queried, hits, flushed)."""
        B, nnz = self._shape
        stream = torch.cuda.current_stream(self.device).cuda_stream
        r = pk.pk_hh_end_iteration(self.plan, self.hh, self.itr, self.warmup_iters, self.flush_iters, B, nnz, self.ws,
                                   self.ws_bytes, self.scratch, self.scratch_bytes, stream, want_counts)
        self.itr += 1
        return r

    def hot_count(self, p: int) -> int:
        return pk.pk_hh_hot_count(self.plan, p)
