"""Device-side objects for running layers through the C ABI.

DeviceGraph uploads a sampled subgraph's CSR and runs the per-subgraph
preparation (transposed values, aggregation plan).  SageStack holds the
weights and activations of an L-layer GraphSAGE stack and chains the
layers (Algorithm 1's layer loop: forward l = 1..L, backward l = L..1 with
each layer's dX feeding the layer below).  Only buffer management and calls
into libgnnprop happen here.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np
import torch

from . import gnnprop as G


def _round_up(a: int, b: int) -> int:
    return (a + b - 1) // b * b


def padded(t: torch.Tensor, ld: int) -> torch.Tensor:
    """Copy a (rows, cols) tensor into a (rows, ld) buffer; returns the
    (rows, cols) view with row stride ld."""
    rows, cols = t.shape
    buf = torch.zeros((rows, ld), dtype=t.dtype, device=t.device)
    buf[:, :cols] = t
    return buf[:, :cols]


class _Rows:
    """A (rows, ld) float32 device buffer that grows on demand; view(n) is
    the first n rows, `cols` wide, at row stride ld."""

    def __init__(self, cols: int, ld: int, device):
        self.cols, self.ld, self.device = cols, ld, device
        self.buf = torch.empty((1, ld), device=device)

    def view(self, n: int) -> torch.Tensor:
        if n > self.buf.shape[0]:
            self.buf = torch.empty((n, self.ld), device=self.device)
        return self.buf[:n, : self.cols]


def _grown(buf: Optional[torch.Tensor], nbytes: int, device) -> torch.Tensor:
    """buf if it holds nbytes, else a new byte buffer of that size (>= 256)."""
    if buf is not None and buf.numel() >= nbytes:
        return buf
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


class DeviceGraph:
    def __init__(self, csr, device: str = "cuda"):
        self.n = int(csr.n)
        self.nnz = int(csr.nnz)
        self.device = device
        self.indptr = torch.from_numpy(np.ascontiguousarray(csr.indptr)).to(device)
        self.indices = torch.from_numpy(np.ascontiguousarray(csr.indices)).to(device)
        self.values = torch.from_numpy(np.ascontiguousarray(csr.values, np.float32)).to(device)
        # at least one element so that data pointers are never NULL
        self.values_t = torch.empty(max(self.nnz, 1), dtype=torch.float32, device=device)
        if self.nnz == 0:
            self.indices = torch.empty(1, dtype=torch.int32, device=device)
            self.values = torch.empty(1, dtype=torch.float32, device=device)
        self.plan = torch.empty(max(G.gnn_plan_bytes(self.n, self.nnz), 256),
                                dtype=torch.uint8, device=device)

    @classmethod
    def on_device(cls, n: int, indptr: torch.Tensor, indices: torch.Tensor,
                  values: torch.Tensor, nnz: Optional[int] = None,
                  values_t: Optional[torch.Tensor] = None,
                  plan: Optional[torch.Tensor] = None) -> "DeviceGraph":
        """Wraps a CSR already in device memory (int32 indptr of n + 1,
        int32 indices and float32 values holding at least nnz entries);
        values_t / plan buffers are allocated unless given (large enough)."""
        g = cls.__new__(cls)
        g.n = int(n)
        g.nnz = int(indices.numel()) if nnz is None else int(nnz)
        g.device = indptr.device
        g.indptr, g.indices, g.values = indptr, indices, values
        g.values_t = values_t if values_t is not None else \
            torch.empty(max(g.nnz, 1), dtype=torch.float32, device=g.device)
        need = G.gnn_plan_bytes(g.n, g.nnz)
        g.plan = plan if plan is not None and plan.numel() >= need else \
            torch.empty(max(need, 256), dtype=torch.uint8, device=g.device)
        return g

    def struct(self) -> G.gnn_csr:
        return G.make_csr(self.n, self.nnz, self.indptr, self.indices, self.values,
                          self.values_t, self.plan)

    def prepare(self, stream=None):
        """Per-subgraph preparation: the work plan and (A_s)^T values, one
        launch."""
        G.gnn_csr_prepare(self.struct(), self.plan, self.values_t, stream)

    def validate(self, symmetric: bool = True) -> int:
        return G.gnn_csr_validate(self.struct(), symmetric)


class FullGraphDevice:
    """A full training graph resident in device memory with its features
    and labels; builds minibatch subgraphs from host node lists (the
    induction of Algorithms 2 / 3 and Algorithm 1's feature and label
    lookup, all in libgnnprop)."""

    def __init__(self, full, X: Optional[np.ndarray] = None,
                 labels: Optional[np.ndarray] = None, norm: int = G.GNN_NORM_ROW,
                 device: str = "cuda"):
        self.n, self.nnz = int(full.n), int(full.nnz)
        self.deg = np.asarray(full.degrees(), np.int64)
        self.device, self.norm = device, norm
        self.indptr = torch.from_numpy(np.ascontiguousarray(full.indptr, np.int64)).to(device)
        self.indices = torch.from_numpy(np.ascontiguousarray(full.indices, np.int32)).to(device)
        if self.nnz == 0:
            self.indices = torch.empty(1, dtype=torch.int32, device=device)
        self.map = torch.full((max(self.n, 1),), -1, dtype=torch.int32, device=device)
        self.X = None if X is None else \
            torch.from_numpy(np.ascontiguousarray(X, np.float32)).to(device)
        self.labels = None if labels is None else \
            torch.from_numpy(np.ascontiguousarray(labels, np.float32)).to(device)
        # side by side, read back by one copy (the status word's upper half
        # stays 0)
        self.meta = torch.zeros(2, dtype=torch.int64, device=device)
        self.nnz_out = self.meta[:1]
        self.status = self.meta.view(torch.int32)[2:3]

    def capacity(self, nodes: np.ndarray) -> int:
        """Entries the induced subgraph of `nodes` can hold at most."""
        return int(self.deg[nodes].sum()) + len(nodes)

    def induce(self, nodes: np.ndarray, stream=None, pad: int = 16):
        """Subgraph on the sorted, distinct host node list `nodes`: returns
        (DeviceGraph prepared for propagation, X_s, labels_s).  Reads the
        entry count back (one synchronisation)."""
        nodes = np.ascontiguousarray(nodes, np.int32)
        n_s = len(nodes)
        cap = self.capacity(nodes) if n_s else 0
        nd = torch.from_numpy(nodes).to(self.device) if n_s else \
            torch.empty(1, dtype=torch.int32, device=self.device)
        ip = torch.empty(n_s + 1, dtype=torch.int32, device=self.device)
        ix = torch.empty(max(cap, 1), dtype=torch.int32, device=self.device)
        vals = torch.empty(max(cap, 1), dtype=torch.float32, device=self.device)
        ws = torch.empty(max(G.gnn_induce_workspace_bytes(n_s), 256), dtype=torch.uint8,
                         device=self.device)
        G.gnn_induce_subgraph(self.n, self.nnz, self.indptr, self.indices, n_s, nd,
                              self.norm, self.map, cap, ip, ix, vals, self.nnz_out,
                              self.status, ws, stream)
        Xs = Ts = None
        if self.X is not None:
            f = self.X.shape[1]
            Xs = torch.empty((max(n_s, 1), _round_up(f, pad)), device=self.device)[:n_s, :f]
            G.gnn_gather_rows(n_s, nd, f, self.X, self.X.stride(0), self.n, Xs,
                              Xs.stride(0), stream)
        if self.labels is not None:
            C = self.labels.shape[1]
            Ts = torch.empty((n_s, C), device=self.device)
            G.gnn_gather_rows(n_s, nd, C, self.labels, self.labels.stride(0), self.n, Ts,
                              C, stream)
        nnz, st = self.meta.tolist()
        if st:
            raise ValueError("gnn_induce_subgraph status %d (1: id out of range, 2: ids "
                             "not ascending, 4: over capacity)" % st)
        dg = DeviceGraph.on_device(n_s, ip, ix[: max(nnz, 1)], vals[: max(nnz, 1)])
        dg.nnz = nnz
        dg.nodes = nd
        dg.prepare(stream)
        return dg, Xs, Ts


class _Slot:
    """Buffers of one subgraph in flight through the pipeline."""

    def __init__(self, max_nodes: int, cap: int, f: int, C: int, pad: int, device):
        self.host_nodes = torch.empty(max_nodes, dtype=torch.int32).pin_memory()
        self.host_meta = torch.zeros(2, dtype=torch.int64).pin_memory()
        self.nodes = torch.empty(max(max_nodes, 1), dtype=torch.int32, device=device)
        self.indptr = torch.empty(max_nodes + 1, dtype=torch.int32, device=device)
        self.indices = torch.empty(max(cap, 1), dtype=torch.int32, device=device)
        self.values = torch.empty(max(cap, 1), dtype=torch.float32, device=device)
        self.values_t = torch.empty(max(cap, 1), dtype=torch.float32, device=device)
        self.plan = torch.empty(max(G.gnn_plan_bytes(max_nodes, cap), 256),
                                dtype=torch.uint8, device=device)
        self.meta = torch.zeros(2, dtype=torch.int64, device=device)  # nnz, status
        self.ws = torch.empty(max(G.gnn_induce_workspace_bytes(max_nodes), 256),
                              dtype=torch.uint8, device=device)
        self.X = torch.empty((max(max_nodes, 1), _round_up(f, pad)), device=device)
        self.T = torch.empty((max(max_nodes, 1), max(C, 1)), device=device)
        self.induced = torch.cuda.Event()
        self.consumed = torch.cuda.Event()
        self.n = 0
        self.sid = -1


class SubgraphPipeline:
    """Algorithm 8 on one GPU.  A pool of host sampler threads keeps node
    lists ready (gnn_sampler_pool); each subgraph is induced and its rows
    gathered on a preparation stream while the previous subgraph trains on
    the caller's stream, with `depth` sets of buffers in rotation.

        sub = pipe.next()       # (DeviceGraph prepared, X_s, T_s, id)
        ...launch the iteration on sub...
        pipe.release()          # after launching: frees the slot for reuse
                                # and starts preparing the following subgraph
    """

    def __init__(self, full_dev: FullGraphDevice, pool, max_nodes: int, depth: int = 2,
                 pad: int = 16):
        assert depth >= 2
        self.full, self.pool = full_dev, pool
        self.max_nodes = int(max_nodes)
        deg = np.sort(full_dev.deg)[::-1]
        cap = int(deg[: self.max_nodes].sum()) + self.max_nodes  # any max_nodes nodes fit
        f = full_dev.X.shape[1] if full_dev.X is not None else 1
        C = full_dev.labels.shape[1] if full_dev.labels is not None else 1
        dev = full_dev.device
        self.cap = cap
        self.slots = [_Slot(self.max_nodes, cap, f, C, pad, dev) for _ in range(depth)]
        self.prep = torch.cuda.Stream(device=dev)
        self.k = 0
        self._issue(self.slots[0])

    def _issue(self, s: _Slot):
        sid, nodes = self.pool.next()
        n = len(nodes)
        if n > self.max_nodes:
            raise ValueError("subgraph of %d nodes exceeds max_nodes %d" % (n, self.max_nodes))
        s.n, s.sid = n, sid
        s.host_nodes[:n].copy_(torch.from_numpy(nodes))
        full = self.full
        with torch.cuda.stream(self.prep):
            self.prep.wait_event(s.consumed)  # the iteration that last used s is done
            s.nodes[:n].copy_(s.host_nodes[:n], non_blocking=True)
            G.gnn_induce_subgraph(full.n, full.nnz, full.indptr, full.indices, n, s.nodes,
                                  full.norm, full.map, self.cap, s.indptr, s.indices,
                                  s.values, s.meta[0:1], s.meta[1:2].view(torch.int32), s.ws,
                                  self.prep.cuda_stream)
            if full.X is not None:
                G.gnn_gather_rows(n, s.nodes, full.X.shape[1], full.X, full.X.stride(0),
                                  full.n, s.X, s.X.stride(0), self.prep.cuda_stream)
            if full.labels is not None:
                G.gnn_gather_rows(n, s.nodes, full.labels.shape[1], full.labels,
                                  full.labels.stride(0), full.n, s.T, s.T.stride(0),
                                  self.prep.cuda_stream)
            s.host_meta.copy_(s.meta, non_blocking=True)
            s.induced.record(self.prep)

    def next(self):
        s = self.slots[self.k % len(self.slots)]
        s.induced.synchronize()
        nnz, status = int(s.host_meta[0]), int(s.host_meta[1])
        if status:
            raise ValueError("gnn_induce_subgraph status %d" % status)
        cur = torch.cuda.current_stream()
        cur.wait_event(s.induced)
        dg = DeviceGraph.on_device(s.n, s.indptr[: s.n + 1], s.indices, s.values, nnz=nnz,
                                   values_t=s.values_t, plan=s.plan)
        dg.prepare(cur.cuda_stream)
        f = self.full.X.shape[1] if self.full.X is not None else 0
        C = self.full.labels.shape[1] if self.full.labels is not None else 0
        return dg, s.X[: s.n, :f], s.T[: s.n, :C], s.sid

    def release(self):
        s = self.slots[self.k % len(self.slots)]
        s.consumed.record(torch.cuda.current_stream())
        self.k += 1
        self._issue(self.slots[self.k % len(self.slots)])


class SageStack:
    """Weights, activations and gradients of an L-layer stack on one graph."""

    def __init__(self, graph: DeviceGraph, params: Sequence, f_in: int,
                 order: int = 0, flags: int = 0, pad: int = 16,
                 fuse_masks: bool = False, device: str = "cuda"):
        """fuse_masks: in the backward pass layer l > 0 writes its dX already
        masked by its input's sign (the ReLU mask of layer l - 1), which layer
        l - 1 then takes as its masked dY, so no separate masking pass runs
        below the top layer.  The dX buffers of layers l > 0 then hold those
        masked gradients; the first layer's dX is always the plain one.  Off
        by default: the mask read lands in the tail of the dX product, where
        it costs about what the masking pass it replaces does."""
        self.order, self.flags, self.pad = order, flags, pad
        self.fuse_masks = fuse_masks
        self.device = device
        self.layers = []
        f = f_in
        for p in params:
            h = p.w_self.shape[1]
            assert p.w_self.shape == (f, h) == p.w_neigh.shape
            L = {"f_in": f, "h": h}
            L["W_self"] = torch.from_numpy(np.ascontiguousarray(p.w_self)).to(device)
            L["W_neigh"] = torch.from_numpy(np.ascontiguousarray(p.w_neigh)).to(device)
            L["b_self"] = None if p.b_self is None else \
                torch.from_numpy(np.ascontiguousarray(p.b_self)).to(device)
            L["b_neigh"] = None if p.b_neigh is None else \
                torch.from_numpy(np.ascontiguousarray(p.b_neigh)).to(device)
            L["dW_self"] = torch.empty((f, h), device=device)
            L["dW_neigh"] = torch.empty((f, h), device=device)
            L["db_self"] = torch.empty(h, device=device) if p.b_self is not None else None
            L["db_neigh"] = torch.empty(h, device=device) if p.b_neigh is not None else None
            L["_Y"] = _Rows(2 * h, _round_up(2 * h, pad), device)
            L["_dX"] = _Rows(f, _round_up(f, pad), device)
            L["saved"] = None
            self.layers.append(L)
            f = 2 * h
        self.f_in = f_in
        self.workspace = None
        self.inputs: List[Optional[torch.Tensor]] = [None] * len(self.layers)
        self.bind(graph)

    def bind(self, graph: DeviceGraph):
        """Moves the stack to another (prepared) subgraph: activation and
        gradient views of its size, saved state and workspace grown as
        needed.  Weights and their gradients are kept."""
        self.g = graph
        self.n = graph.n
        ws_bytes = 0
        for i, L in enumerate(self.layers):
            L["Y"] = L["_Y"].view(self.n)
            L["dX"] = L["_dX"].view(self.n)
            lay = self._layer(i, _round_up(L["f_in"], self.pad))
            L["saved"] = _grown(L["saved"], G.gnn_prop_saved_bytes(graph.struct(), lay),
                                self.device)
            ws_bytes = max(ws_bytes, G.gnn_prop_workspace_bytes(graph.struct(), lay))
        self.workspace = _grown(self.workspace, ws_bytes, self.device)
        self.inputs = [None] * len(self.layers)

    def _layer(self, i: int, ld_x: int, extra_flags: int = 0) -> G.gnn_layer:
        L = self.layers[i]
        return G.make_layer(L["f_in"], L["h"], ld_x, L["Y"].stride(0) if self.n else 2 * L["h"],
                            L["dX"].stride(0) if self.n else L["f_in"], self.order,
                            self.flags | extra_flags)

    def forward(self, X: torch.Tensor, stream=None) -> torch.Tensor:
        csr = self.g.struct()
        x = X
        for i, L in enumerate(self.layers):
            self.inputs[i] = x
            ld_x = x.stride(0) if self.n else L["f_in"]
            G.gnn_prop_fwd(csr, self._layer(i, ld_x), x, L["W_self"], L["W_neigh"],
                           L["b_self"], L["b_neigh"], L["Y"], L["saved"],
                           self.workspace, stream)
            x = L["Y"]
        return x

    def backward(self, dY: torch.Tensor, want_dx_first: bool = True, stream=None):
        csr = self.g.struct()
        d = dY
        for i in reversed(range(len(self.layers))):
            L = self.layers[i]
            x = self.inputs[i]
            ld_x = x.stride(0) if self.n else L["f_in"]
            extra = 0
            if self.fuse_masks:
                if i < len(self.layers) - 1:
                    extra |= G.GNN_FLAG_DY_MASKED
                if i > 0:
                    extra |= G.GNN_FLAG_DX_MASKED
            lay = self._layer(i, ld_x, extra)
            # the upstream gradient must share Y's row stride
            if self.n and d.stride(0) != L["Y"].stride(0):
                d = padded(d.contiguous(), L["Y"].stride(0))
            dx = L["dX"] if (i > 0 or want_dx_first) else None
            G.gnn_prop_bwd(csr, lay, x, L["W_self"], L["W_neigh"], L["Y"], d,
                           L["saved"], dx, L["dW_self"], L["dW_neigh"],
                           L["db_self"], L["db_neigh"], self.workspace, stream)
            d = dx
        return self.layers[0]["dX"] if want_dx_first else None


def _stream_object(stream):
    """torch's object of a stream argument (None: the current stream)."""
    if stream is None:
        return torch.cuda.current_stream()
    return torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream


def _on_current(t: torch.Tensor) -> bool:
    return t.is_cuda and t.get_device() == torch.cuda.current_device()


class ParamSet:
    """AdamW on a set of tensors, one launch a step: their moments (in 32
    bits, or in 8 with a scale for each 256 elements), the plan that lists
    them and the norm of their gradients.  Weights and gradients are
    contiguous float32 tensors that stay where they are.  The constructor
    returns when moments and plan are written, so that the first step may be on
    any stream; later steps on another stream than the last one's have to wait
    for it, as for whatever writes the gradients."""

    def __init__(self, weights: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                 weight_decay: Sequence[float], state_bits: int = 32):
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        if not len(weights) == len(grads) == len(weight_decay):
            raise ValueError("as many gradients and decays as weights")
        for t in list(weights) + list(grads):
            if t.dtype != torch.float32 or not t.is_contiguous() or not _on_current(t):
                raise ValueError("weights and gradients must be contiguous float32 tensors on "
                                 "the current device")
        for w, g in zip(weights, grads):
            if w.shape != g.shape or w.device != g.device:
                raise ValueError("a weight and its gradient differ in shape or device")
        self.weights, self.grads, self.state_bits = list(weights), list(grads), state_bits
        device = weights[0].device if weights else "cuda"
        kind = torch.float32 if state_bits == 32 else torch.uint8
        self.state = []  # (m, v), or with 8 bits (m, v, their scales)
        for w in self.weights:
            st = tuple(torch.zeros(w.numel(), dtype=kind, device=device) for _ in range(2))
            if state_bits == 8:
                blocks = (w.numel() + G.GNN_STATE_BLOCK - 1) // G.GNN_STATE_BLOCK
                st += tuple(torch.zeros(blocks, device=device) for _ in range(2))
            self.state.append(st)
        self.params = G.make_params(
            [(w, g) + st + (None,) * (4 - len(st)) + (float(d),)
             for w, g, st, d in zip(self.weights, self.grads, self.state, weight_decay)],
            state_bits)
        self.plan = torch.empty(G.gnn_params_plan_bytes(self.params), dtype=torch.uint8,
                                device=device)
        self.params.plan = self.plan.data_ptr()
        self.norm = torch.zeros(1, device=device)
        self.ws = torch.empty(max(G.gnn_grad_norm_workspace_bytes(self.params), 256),
                              dtype=torch.uint8, device=device)
        G.gnn_params_build_plan(self.params, self.plan)
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()

    def grad_norm(self, stream=None) -> torch.Tensor:
        """Norm of all gradients (one float, on the device)."""
        G.gnn_grad_norm(self.params, self.norm, self.ws, stream)
        return self.norm

    def step(self, t: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
             max_norm: Optional[float] = None, seed: int = 0, stream=None):
        """AdamW step t (from 1).  With max_norm the gradients are scaled down
        to that norm where theirs is larger, and a step whose norm is not
        finite changes nothing (the device decides that: to count only steps
        that were taken, read `norm`).  seed: of the 8-bit moments' rounding."""
        norm = self.grad_norm(stream) if max_norm is not None else None
        G.gnn_adamw_step(self.params, lr, betas[0], betas[1], eps, t, norm,
                         max_norm if max_norm is not None else 1.0, seed, stream)


class Trainer:
    """One training iteration of Algorithm 1 on a prepared subgraph: the
    stack's forward pass, the classifier and loss (Section 3.1), the backward
    pass from the classifier's input gradient down (Section 5.1), then SGD,
    Adam or AdamW on every weight.  policy_step is the same iteration with the
    clipped policy loss in the place of the classifier's.  All arithmetic runs
    in libgnnprop; the loss stays on the device (read it with `loss.item()`
    when needed)."""

    def __init__(self, graph: DeviceGraph, params: Sequence, f_in: int, w_mlp,
                 multilabel: bool, optimizer: str = "adam", lr: float = 0.01,
                 betas=(0.9, 0.999), eps: float = 1e-8, order: int = 0,
                 flags: int = 0, pad: int = 16, fuse_masks: bool = False,
                 want_probs: bool = False, keep_xm: bool = False,
                 device: str = "cuda", weight_decay: Optional[float] = None,
                 max_norm: Optional[float] = None, state_bits: int = 32, seed: int = 0):
        """want_probs / keep_xm: keep the class probabilities Y / the MLP
        output X_MLP = ReLU(X^(L) W_MLP) of the last iteration in `probs` /
        `xm` (n x C views).
        With optimizer "adamw": weight_decay (0.01 unless given) of the weight
        matrices (biases do not decay), max_norm to clip the norm of all
        gradients, state_bits 8 for moments of one byte and the seed of their
        rounding.  `t` counts the iterations, those too that change nothing
        because their gradients' norm is not finite."""
        if optimizer not in ("sgd", "adam", "adamw"):
            raise ValueError("optimizer must be 'sgd', 'adam' or 'adamw'")
        if optimizer != "adamw" and (weight_decay is not None or max_norm is not None or
                                     state_bits != 32):
            raise ValueError("weight_decay, max_norm and state_bits go with 'adamw'")
        if max_norm is not None and not max_norm > 0:
            raise ValueError("max_norm must be above 0")
        self.max_norm, self.seed = max_norm, seed
        self.stack = SageStack(graph, params, f_in, order, flags, pad, fuse_masks, device)
        self.kind = G.GNN_LOSS_SIGMOID if multilabel else G.GNN_LOSS_SOFTMAX
        self.flags = flags & (G.GNN_FLAG_BF16 | G.GNN_FLAG_F32_MFMA)
        self.optimizer, self.lr, self.betas, self.eps = optimizer, lr, betas, eps
        self.device = device
        top = self.stack.layers[-1]
        self.f_top = 2 * top["h"]
        self.C = int(w_mlp.shape[1])
        assert w_mlp.shape == (self.f_top, self.C)
        self.W_mlp = torch.from_numpy(np.ascontiguousarray(w_mlp, np.float32)).to(device)
        self.dW_mlp = torch.empty_like(self.W_mlp)
        # the classifier writes dX^(L) at the top layer's Y stride, which is
        # the stride the stack's backward pass expects
        self._dX_top = _Rows(self.f_top, top["_Y"].ld, device)
        ld_p = _round_up(self.C, 4)
        self._probs = _Rows(self.C, ld_p, device) if want_probs else None
        self._xm = _Rows(self.C, ld_p, device) if keep_xm else None
        self.loss = torch.zeros(1, device=device)
        self.cls_ws = None
        self.bind(graph, rebind_stack=False)
        # Every weight, gradient and optimizer moment lives in one flat
        # buffer (tensors at 256-byte offsets, zero padding between them), so
        # that one update launch covers the whole model.  (weight, gradient)
        # pairs in a fixed order: W_MLP, then per layer W_self, W_neigh
        # (, b_self, b_neigh).
        names = [(None, "W_mlp", "dW_mlp")]
        for L in self.stack.layers:
            names += [(L, "W_self", "dW_self"), (L, "W_neigh", "dW_neigh")]
            if L["b_self"] is not None:
                names += [(L, "b_self", "db_self"), (L, "b_neigh", "db_neigh")]
        get = lambda L, k: getattr(self, k) if L is None else L[k]
        offs, total = [], 0
        for L, wk, _ in names:
            offs.append(total)
            total += _round_up(get(L, wk).numel(), 64)
        self.flat_w = torch.zeros(max(total, 64), device=device)
        self.flat_g = torch.zeros(max(total, 64), device=device)
        self.pairs = []
        for (L, wk, gk), o in zip(names, offs):
            w = get(L, wk)
            wv = self.flat_w[o: o + w.numel()].view(w.shape)
            wv.copy_(w)
            gv = self.flat_g[o: o + w.numel()].view(w.shape)
            if L is None:
                setattr(self, wk, wv)
                setattr(self, gk, gv)
            else:
                L[wk], L[gk] = wv, gv
            self.pairs.append((wv, gv))
        self.state = None
        if optimizer == "adam":
            self.flat_m = torch.zeros_like(self.flat_w)
            self.flat_v = torch.zeros_like(self.flat_w)
            self.state = [(self.flat_m[o: o + w.numel()].view(w.shape),
                           self.flat_v[o: o + w.numel()].view(w.shape))
                          for (w, _), o in zip(self.pairs, offs)]
        if optimizer == "adamw":
            decay = 0.01 if weight_decay is None else float(weight_decay)
            self.params = ParamSet([w for w, _ in self.pairs], [g for _, g in self.pairs],
                                   [decay if w.dim() == 2 else 0.0 for w, _ in self.pairs],
                                   state_bits)
            self.state = self.params.state
        self.t = 0
        # the policy's logits, their gradient, log-probabilities and workspace,
        # made when first used
        self._Z, self._dZ = _Rows(self.C, ld_p, device), _Rows(self.C, ld_p, device)
        self.policy_out = torch.zeros(3, device=device)
        self.logp = self._logp = torch.empty(0, device=device)
        self.policy_ws = None
        self._policy_streams = set()  # handles of the streams they were used on

    def bind(self, graph: DeviceGraph, rebind_stack: bool = True):
        """Moves the iteration to another prepared subgraph (weights and
        optimizer state are kept)."""
        if rebind_stack:
            self.stack.bind(graph)
        self.n = graph.n
        self.dX_top = self._dX_top.view(self.n)
        self.probs = self._probs.view(self.n) if self._probs is not None else None
        self.xm = self._xm.view(self.n) if self._xm is not None else None
        self.cls_ws = _grown(self.cls_ws, G.gnn_classifier_workspace_bytes(
            self.n, self.f_top, self.C), self.device)

    def step(self, X: torch.Tensor, targets: torch.Tensor, stream=None) -> torch.Tensor:
        """X: n x f_in (any row stride); targets: n x C 0/1 floats."""
        top = self.stack.forward(X, stream)
        ld_top = top.stride(0) if self.n else self.f_top
        ld_t = targets.stride(0) if self.n else self.C
        G.gnn_classifier(self.n, self.f_top, self.C, self.kind, self.flags, top, ld_top,
                         self.W_mlp, targets, ld_t, self.xm,
                         self.xm.stride(0) if self.xm is not None else self.C, self.probs,
                         self.probs.stride(0) if self.probs is not None else self.C,
                         self.loss, self.dW_mlp, self.dX_top,
                         self.dX_top.stride(0) if self.n else self.f_top, self.cls_ws,
                         stream)
        self.stack.backward(self.dX_top, want_dx_first=False, stream=stream)
        self._update(stream)
        return self.loss

    def _update(self, stream):
        self.t += 1
        if self.optimizer == "sgd":
            G.gnn_sgd_step(self.flat_w.numel(), self.flat_w, self.flat_g, self.lr, stream)
        elif self.optimizer == "adam":
            G.gnn_adam_step(self.flat_w.numel(), self.flat_w, self.flat_g, self.flat_m,
                            self.flat_v, self.lr, self.betas[0], self.betas[1], self.eps,
                            self.t, stream)
        else:
            self.params.step(self.t, self.lr, self.betas, self.eps, self.max_norm, self.seed,
                             stream)

    def _per_row(self, name: str, t: Optional[torch.Tensor], dtype=torch.float32):
        if t is not None and (t.dtype != dtype or t.shape != (self.n,) or
                              not t.is_contiguous() or not _on_current(t)):
            raise ValueError("%s must be %d contiguous values of %s on the current device" %
                             (name, self.n, dtype))
        return t

    def _policy_buffers(self, stream):
        """Makes the policy's buffers, if the present ones are too small, in the
        memory of the stream that they are used on, and keeps their memory from
        other use, once they are replaced, until every stream that used them
        is done."""
        n, C, f = self.n, self.C, self.f_top
        need = max(G.gnn_policy_workspace_bytes(n, C), G.gnn_gemm_workspace_bytes(n, C, f),
                   G.gnn_gemm_workspace_bytes(f, C, n), G.gnn_gemm_workspace_bytes(n, f, C), 256)
        if self.policy_ws is None or self.policy_ws.numel() < need or self._Z.buf.shape[0] < n:
            with torch.cuda.stream(_stream_object(stream)):
                self._Z = _Rows(C, self._Z.ld, self.device)
                self._dZ = _Rows(C, self._dZ.ld, self.device)
                for rows in (self._Z, self._dZ):
                    rows.view(n)
                self._logp = torch.empty(n, device=self.device)
                self.policy_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            self._policy_streams.clear()
        handle = G._stream(stream)
        if handle not in self._policy_streams:
            for t in (self._Z.buf, self._dZ.buf, self._logp, self.policy_ws):
                t.record_stream(_stream_object(stream))
            self._policy_streams.add(handle)

    def _logits(self, X: torch.Tensor, stream):
        """(X^(L), its row stride, logits Z = X^(L) W_MLP, their row stride)."""
        n, C, f = self.n, self.C, self.f_top
        self._policy_buffers(stream)
        top, Z = self.stack.forward(X, stream), self._Z.view(n)
        ld_top = top.stride(0) if n else f
        G.gnn_gemm(False, False, n, C, f, top, ld_top, self.W_mlp, C, Z, self._Z.ld, self.flags,
                   self.policy_ws, stream)
        return top, ld_top, Z, self._Z.ld

    def action_logp(self, X: torch.Tensor, actions: torch.Tensor, stream=None) -> torch.Tensor:
        """Log-probability of each row's action (n int32; outside [0, C): 0)
        under the present weights: a new tensor, to be kept as old_logp or
        ref_logp.  stream: where all of it runs (the current one unless given);
        what the call reads has to be ready there, and what it gives is."""
        self._per_row("actions", actions, torch.int32)
        _, _, Z, ld = self._logits(X, stream)
        if stream is None:
            logp = torch.empty(self.n, device=self.device)
        else:
            with torch.cuda.stream(_stream_object(stream)):
                logp = torch.empty(self.n, device=self.device)
            logp.record_stream(torch.cuda.current_stream())
        G.gnn_action_logp(self.n, self.C, Z, ld, actions, logp, self.policy_ws, stream)
        return logp

    def policy_step(self, X: torch.Tensor, actions: torch.Tensor, advantage: torch.Tensor,
                    old_logp: Optional[torch.Tensor] = None,
                    ref_logp: Optional[torch.Tensor] = None,
                    weight: Optional[torch.Tensor] = None, clip=(0.2, 0.2), beta: float = 0.0,
                    stream=None) -> torch.Tensor:
        """One iteration with the clipped policy loss (gnn_policy_loss) on the
        logits X^(L) W_MLP: forward, loss, backward, update.  Each row's action
        (n int32; outside [0, C): the row is left out), advantage, old_logp
        (None: on-policy), ref_logp (with beta), weight (None: 1/n).  Returns
        three floats on the device: loss, KL and clipped share (weighted sums);
        the n rows' log-probabilities are in `logp`.  stream: as in
        action_logp."""
        for name, t in (("advantage", advantage), ("old_logp", old_logp),
                        ("ref_logp", ref_logp), ("weight", weight)):
            self._per_row(name, t)
        self._per_row("actions", actions, torch.int32)
        n, C, f = self.n, self.C, self.f_top
        top, ld_top, Z, ld = self._logits(X, stream)
        dZ, self.logp = self._dZ.view(n), self._logp[:n]
        G.gnn_policy_loss(n, C, Z, ld, actions, advantage, old_logp, ref_logp, weight, clip[0],
                          clip[1], beta, self.policy_out, self.logp, dZ, ld, self.policy_ws,
                          stream)
        G.gnn_gemm(True, False, f, C, n, top, ld_top, dZ, ld, self.dW_mlp, C, self.flags,
                   self.policy_ws, stream)
        G.gnn_gemm(False, True, n, f, C, dZ, ld, self.W_mlp, C, self.dX_top,
                   self.dX_top.stride(0) if n else f, self.flags, self.policy_ws, stream)
        self.stack.backward(self.dX_top, want_dx_first=False, stream=stream)
        self._update(stream)
        return self.policy_out
