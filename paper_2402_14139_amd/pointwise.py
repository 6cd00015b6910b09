"""A pointwise residual block over channels-last activations, trained from a quantised activation cache: group norm with its
activation (or layer norm over a pixel's channels), a widening linear layer (activation, dropout), a linear layer back with dropout and
the residual sum.  Host bookkeeping only: every arithmetic step but the example's squared-error loss is a call of include/nf.h.

    h = act(GN(x)) or LN(x);  a = D1(act(h W1^T + b1));  y = x + D2(a W2^T + b2)

The products run in the activations' type or on 4-bit operands (``mx``), forward and backward; weights are updated by SGD or, made orthogonal, by
``muon``; ``predict`` serves rows of any number from weights in 4 bits.

``python -m paper_2402_14139_amd.pointwise`` fits such blocks to a map that another one computes, from quantised caches.
"""
from __future__ import annotations

import math

import torch

from . import binding as nf

TYPES = {nf.NF_F32: torch.float32, nf.NF_BF16: torch.bfloat16, nf.NF_F16: torch.float16}


def _check(name: str, t, T, device, rows: int, row: int):
    """The kernels see addresses only: ``t`` has to hold ``rows`` dense rows of ``row`` elements of type ``T`` there."""
    if t.device != device or t.dtype != T or not t.is_contiguous() or t.shape[:1] != (rows,) or t.numel() != rows * row:
        raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}; want {rows} dense rows of {row} {T} on {device}")


class QuantisedCache:
    """``capacity`` rows of n elements in 8 or 4 bits, with their labels (nf_qcache_write / nf_qcache_read)."""

    def __init__(self, fmt, capacity: int, n: int, device="cuda"):
        code, scale = nf.nf_qcache_row_bytes(fmt, n)
        self.fmt, self.capacity, self.n = fmt, capacity, n
        self.codes = torch.empty((capacity, code), dtype=torch.uint8, device=device)
        self.scales = torch.empty((capacity, scale), dtype=torch.uint8, device=device)
        self.labels = torch.zeros(capacity, dtype=torch.int32, device=device)

    def write(self, dtype, first: int, x, labels):
        _check("x", x, TYPES[dtype], self.codes.device, x.shape[0], self.n)
        _check("labels", labels, torch.int32, self.codes.device, x.shape[0], 1)
        nf.nf_qcache_write(self.fmt, dtype, self.codes, self.scales, self.labels, self.capacity, self.n, first, x.shape[0], x,
                           labels)

    def read(self, dtype, idx, x_out, labels_out):
        B = idx.shape[0]
        _check("idx", idx, torch.int64, self.codes.device, B, 1)
        _check("x_out", x_out, TYPES[dtype], self.codes.device, B, self.n)
        _check("labels_out", labels_out, torch.int32, self.codes.device, B, 1)
        nf.nf_qcache_read(self.fmt, dtype, self.codes, self.scales, self.labels, self.capacity, self.n, 0, idx, B,
                          x_out, labels_out)


def workspace_bytes(norm, up, down, B: int, HW: int = 0) -> int:
    """Bytes for batches of 1 to ``B`` maps of ``HW`` pixels (a group norm's own): fewer rows are cut into other parts and may want more than many do."""
    group = isinstance(norm, nf.GroupNormDesc)
    HW = norm.HW if group else HW
    sums = lambda b: nf.nf_groupnorm_workspace_bytes(norm, b) if group else nf.nf_layernorm_workspace_bytes(norm, b * HW)  # noqa: E731
    return max(max(sums(b), *(nf.nf_linear_workspace_bytes(d, b * HW) for d in (up, down))) for b in range(1, B + 1))


class Rows4:
    """Room for matrices in 4 bits of up to ``rows`` x ``n`` elements: (codes, exponents) as the calls take them."""

    def __init__(self, rows: int, n: int, device="cuda"):
        code, scale = nf.nf_qcache_row_bytes(nf.NF_Q_E2M1, n)
        self.pair = tuple(torch.empty(rows * b, dtype=torch.uint8, device=device) for b in (code, scale))


def mx_workspace_bytes(up, down, B: int, HW: int) -> int:
    """Bytes for the 4-bit products of 1 to ``B`` * ``HW`` rows forward and of 1 to ``B`` maps backward.  How sums are cut into parts changes with the
    tiles of rows, 64 at least, and wants most at a tile's last row."""
    most = 0
    for_dx = [nf.LinearDesc(dtype=d.dtype, K=d.N, N=d.K, act=nf.NF_ACT_NONE) for d in (up, down)]
    for M in range(64, B * HW + 64, 64):
        most = max(most, *(nf.nf_mx_linear_workspace_bytes(d, M) for d in (up, down)), *(nf.nf_mx_product_workspace_bytes(d, M) for d in for_dx))
    for M in range(HW, B * HW + 1, HW):
        for d in (up, down):
            most = max(most, nf.nf_mx_product_workspace_bytes(nf.LinearDesc(dtype=nf.NF_F32, K=M, N=d.K, act=nf.NF_ACT_NONE), d.N))
    return most


MUON_STEPS = [(3.4445, -4.7750, 2.0315)] * 5   # drives singular values to between 0.7 and 1.2


class PointwiseBlock:
    """Parameters (fp32; the weights also in the activations' type), gradients and buffers of one block for batches of up to
    ``B`` maps of ``HW`` pixels and ``C`` channels, ``H`` hidden ones.  ``norm``: "group" (of ``groups`` groups, with the activation
    behind it) or "layer"; ``mx``: products on 4-bit operands."""

    kept = False   # the buffers hold what backward() reads: from forward() to the next predict() or backward()
    of = None   # its batch, and its step where that chooses masks
    v = muon_ws = None   # muon()'s momentum and workspace, from its first call on
    captured = False   # that call was recorded into a graph

    def __init__(self, dtype, B: int, HW: int, C: int, H: int, groups: int, act=nf.NF_ACT_GELU, p: float = 0.0, seed: int = 0,
                 device="cuda", norm: str = "group", mx: bool = False):
        if norm not in ("group", "layer"):
            raise ValueError(f"norm: {norm!r}; want 'group' or 'layer'")
        if not torch.cuda.is_available():
            raise RuntimeError("PointwiseBlock needs a GPU: the library has no CPU path")
        self.kind, self.mx = norm, mx
        self.dtype, self.B, self.HW, self.C, self.H, self.p, self.seed = dtype, B, HW, C, H, p, seed
        T = TYPES[dtype]
        if norm == "group":
            self.norm = nf.GroupNormDesc(dtype=dtype, C=C, G=groups, act=act, HW=HW, eps=1e-5)
        else:
            self.ln = nf.LayerNormDesc(dtype=dtype, C=C, eps=1e-5)
        self.up = nf.LinearDesc(dtype=dtype, K=C, N=H, act=act)
        self.down = nf.LinearDesc(dtype=dtype, K=H, N=C, act=nf.NF_ACT_NONE)
        g = torch.Generator().manual_seed(seed)
        self.p32 = {"gamma": torch.ones(C), "beta": torch.zeros(C), "W1": torch.randn(H, C, generator=g) / math.sqrt(C),
                    "b1": torch.zeros(H), "W2": torch.randn(C, H, generator=g) / math.sqrt(H), "b2": torch.zeros(C)}
        self.p32 = {k: v.to(device) for k, v in self.p32.items()}
        self.grad = {k: torch.zeros_like(v) for k, v in self.p32.items()}
        self.w = {k: self.p32[k].to(T) for k in ("W1", "W2")}
        M = B * HW
        new = lambda *s, d=T: torch.empty(s, dtype=d, device=device)  # noqa: E731
        self.h, self.z1, self.a, self.y = new(M, C), new(M, H), new(M, H), new(M, C)
        self.dz2, self.da, self.dh, self.dx = new(M, C), new(M, H), new(M, C), new(M, C)
        stats = (B, groups) if norm == "group" else (M,)
        self.mean, self.rstd = new(*stats, d=torch.float32), new(*stats, d=torch.float32)
        room = workspace_bytes(self.norm if norm == "group" else self.ln, self.up, self.down, B, HW)
        self.orth = nf.orth_desc(MUON_STEPS)
        self.unmoved = torch.ones((), dtype=torch.bool, device=device)   # no update has run on momentum that was made in a capture
        if mx:
            room = max(room, mx_workspace_bytes(self.up, self.down, B, HW))
            # gradients by rows and by columns, a layer's input by columns: the wider layer's size
            wide = max(C, H)
            self.dz_rows, self.dz_cols, self.in_cols = Rows4(M, wide, device), Rows4(wide, M, device), Rows4(wide, M, device)
            # the weights by rows (forward) and by columns (gradients)
            self.q = {k: (Rows4(*self.p32[k].shape, device), Rows4(*self.p32[k].t().shape, device)) for k in ("W1", "W2")}
        self.ws = torch.empty(max(room, 1), dtype=torch.uint8, device=device)
        if mx:
            self.pack()

    def _maps(self, name: str, t, B: int):
        if not 1 <= B <= self.B:
            raise ValueError(f"{name}: a batch of {B}; this block's buffers hold 1 to {self.B}")
        _check(name, t, TYPES[self.dtype], self.ws.device, B, self.HW * self.C)

    def _not_own(self, x):
        if x.untyped_storage().data_ptr() == self.y.untyped_storage().data_ptr():
            raise ValueError("x: this block's own results, whose place the new ones take; clone them")

    def _drop(self, which: int, step: int):
        return nf.DropoutDesc(p=self.p, seed=self.seed * 2 + which, step=step) if self.p else None

    def pack(self):
        """The weights in 4 bits, from their fp32 values; sgd() and muon() do it by themselves."""
        for k, (rows, cols) in self.q.items():
            nf.nf_mx_quantise(nf.NF_F32, *self.p32[k].shape, self.p32[k], *rows.pair, *cols.pair)

    def _normalise(self, x, M, h, keep: bool):
        P = self.p32
        if self.kind == "group":
            nf.nf_groupnorm_fwd(self.norm, M // self.HW, x, P["gamma"], P["beta"], h, self.mean, self.rstd, self.ws)
        else:
            nf.nf_layernorm_fwd(self.ln, M, x, P["gamma"], P["beta"], h, self.mean if keep else None, self.rstd if keep else None)

    def _linear(self, d, M, x, name, r, drop, y, z):
        b = self.p32["b" + name[1]]
        if self.mx:
            nf.nf_mx_linear_fwd(d, M, x, *self.q[name][0].pair, b, r, drop, y, z, self.ws)
        else:
            nf.nf_linear_fwd(d, M, x, self.w[name], b, r, drop, y, z, self.ws)

    def _linear_back(self, d, M, dz, x, name, dx):
        dW = self.grad[name]
        if not self.mx:
            nf.nf_linear_bwd(d, M, dz, x, self.w[name], dx, dW, self.ws)
            return
        nf.nf_mx_quantise(self.dtype, M, d.N, dz, *self.dz_rows.pair, *self.dz_cols.pair)
        nf.nf_mx_quantise(self.dtype, M, d.K, x, None, None, *self.in_cols.pair)
        for_dx = nf.LinearDesc(dtype=self.dtype, K=d.N, N=d.K, act=nf.NF_ACT_NONE)
        for_dW = nf.LinearDesc(dtype=nf.NF_F32, K=M, N=d.K, act=nf.NF_ACT_NONE)
        nf.nf_mx_product(for_dx, M, *self.dz_rows.pair, *self.q[name][1].pair, None, None, dx, self.ws)
        nf.nf_mx_product(for_dW, d.N, *self.dz_cols.pair, *self.in_cols.pair, None, None, dW, self.ws)

    def forward(self, x, step: int = 0, train: bool = True):
        """y [B, HW, C] of x [B, HW, C]; ``step`` chooses the dropout masks, which ``train=False`` leaves out."""
        B = x.shape[0]
        self._maps("x", x, B)
        self._not_own(x)
        M = B * self.HW
        d1, d2 = (self._drop(0, step), self._drop(1, step)) if train else (None, None)
        self._normalise(x, M, self.h, True)
        self._linear(self.up, M, self.h, "W1", None, d1, self.a, self.z1)
        self._linear(self.down, M, self.a, "W2", x, d2, self.y, None)
        self.kept = train or not self.p   # backward() applies the masks
        self.of = (B, step if self.p else None)
        return self.y[:M].view(B, self.HW, self.C)

    def backward(self, x, dy, step: int = 0):
        """Gradients of the parameters (``grad``) and of x but for the residual's part, which is dy itself; once for every forward()."""
        B = x.shape[0]
        self._maps("x", x, B)
        self._maps("dy", dy, B)
        if not self.kept:
            raise RuntimeError("backward: no forward() before it, one without its dropout, or its buffers taken since by predict() or another backward()")
        if self.of not in (None, (B, step if self.p else None)):
            raise RuntimeError(f"backward: a batch of {B} in step {step}; forward() before it had (batch, step) {self.of}")
        M, P, g = B * self.HW, self.p32, self.grad
        nf.nf_linear_bwd_epilogue(self.down, M, dy, None, self._drop(1, step), self.dz2, g["b2"], self.ws)
        self._linear_back(self.down, M, self.dz2, self.a, "W2", self.da)
        self.kept = False
        nf.nf_linear_bwd_epilogue(self.up, M, self.da, self.z1, self._drop(0, step), self.a, g["b1"], self.ws)  # a is not needed again
        self._linear_back(self.up, M, self.a, self.h, "W1", self.dh)
        if self.kind == "group":
            nf.nf_groupnorm_bwd(self.norm, B, self.dh, x, P["gamma"], P["beta"], self.mean, self.rstd, self.dx, g["gamma"], g["beta"],
                                self.ws)
        else:
            nf.nf_layernorm_bwd(self.ln, M, self.dh, x, P["gamma"], self.mean, self.rstd, None, self.dx, g["gamma"], g["beta"], self.ws)
        return self.dx[:M].view(B, self.HW, self.C)

    def predict(self, x):
        """y of rows x [rows, C], up to the block's pixels and down to a single one, from weights in 4 bits; nothing is kept for a backward pass,
        nor what a forward() before it kept."""
        if self.kind != "layer" or not self.mx:
            raise ValueError("predict: rows by themselves, from weights in 4 bits: the block wants norm='layer' and mx=True")
        rows = x.shape[0]
        if not 1 <= rows <= self.B * self.HW:
            raise ValueError(f"x: {rows} rows; this block's buffers hold 1 to {self.B * self.HW}")
        _check("x", x, TYPES[self.dtype], self.ws.device, rows, self.C)
        self._not_own(x)
        self.kept = False
        self._normalise(x, rows, self.h, False)
        self._linear(self.up, rows, self.h, "W1", None, None, self.a, None)
        self._linear(self.down, rows, self.a, "W2", x, None, self.y, None)
        return self.y[:rows]

    def _renew(self):
        for k, v in self.w.items():
            v.copy_(self.p32[k])
        if self.mx:
            self.pack()

    def sgd(self, lr: float):
        names = list(self.p32)
        nf.nf_sgd_update(lr, 0.0, [self.p32[k] for k in names], [self.grad[k] for k in names], None)
        self._renew()

    def prepare_muon(self):
        """Momentum and workspace for muon(), whose first call does it by itself; a block that is updated otherwise goes without."""
        if self.v is not None:
            return
        weights = [self.p32[k] for k in ("W1", "W2")]
        room = nf.nf_orthogonalise_workspace_bytes(self.orth, [w.shape for w in weights])
        self.captured = self.ws.is_cuda and torch.cuda.is_current_stream_capturing()
        self.muon_ws = torch.empty(room, dtype=torch.uint8, device=self.ws.device)
        # zeros written in a capture would be written by every replay
        self.v = [torch.empty_like(w) if self.captured else torch.zeros_like(w) for w in weights]

    def muon(self, lr: float, sgd_lr: float, momentum: float = 0.95, weight_decay: float = 0.0):
        """The weights' update made orthogonal, with its momentum; the other parameters' by SGD at ``sgd_lr``.  Where the first call is recorded into a
        graph, updates clear the momentum unless one has run, a pass over it more: prepare_muon() before the capture spares that."""
        self.prepare_muon()
        names, others = ("W1", "W2"), [k for k in self.p32 if k not in ("W1", "W2")]
        d = nf.MuonDesc(lr=lr, momentum=momentum, weight_decay=weight_decay, nesterov=1, orth=self.orth)
        if self.captured:
            for v in self.v:
                v.masked_fill_(self.unmoved, 0.0)
            self.unmoved.fill_(False)
        nf.nf_muon_update(d, [self.p32[k] for k in names], [self.grad[k] for k in names], self.v, self.muon_ws)
        nf.nf_sgd_update(sgd_lr, 0.0, [self.p32[k] for k in others], [self.grad[k] for k in others], None)
        self._renew()


def fit(dtype=nf.NF_BF16, fmt=nf.NF_Q_INT8, items=256, B=64, HW=64, C=64, H=128, groups=8, epochs=6, lr=0.5, p=0.0, seed=3,
        norm="group", mx=False, muon_lr=0.0):
    """Trains a block towards another one's outputs on rows of a quantised cache; the mean loss of every epoch.  ``muon_lr``: the weights' updates are
    made orthogonal, at this rate."""
    T = TYPES[dtype]
    teacher = PointwiseBlock(dtype, B, HW, C, H, groups, seed=seed, norm=norm)
    block = PointwiseBlock(dtype, B, HW, C, H, groups, p=p, seed=seed + 1, norm=norm, mx=mx)
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = QuantisedCache(fmt, items, HW * C)
    labels = torch.arange(items, dtype=torch.int32, device="cuda")
    for first in range(0, items, B):
        rows = min(B, items - first)
        x = torch.randn((rows, HW * C), generator=g, device="cuda").to(T)
        cache.write(dtype, first, x, labels[first:first + rows].clone())
    x, lab = torch.empty((B, HW, C), dtype=T, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    losses, step = [], 0
    for _ in range(epochs):
        order, total = torch.randperm(items, generator=g, device="cuda"), 0.0
        for first in range(0, items - B + 1, B):
            cache.read(dtype, order[first:first + B].clone(), x, lab)   # clone: 16-byte aligned
            want = teacher.forward(x, train=False)
            got = block.forward(x, step)
            off = got.float() - want.float()
            block.backward(x, (off * (2.0 / off.numel() * C)).to(T), step)
            block.muon(muon_lr, lr / C) if muon_lr else block.sgd(lr / C)
            total += off.square().mean().item()
            step += 1
        losses.append(total / (items // B))
    return losses


if __name__ == "__main__":
    for name, fmt in (("int8", nf.NF_Q_INT8), ("e4m3", nf.NF_Q_E4M3), ("e2m1", nf.NF_Q_E2M1)):
        print(name, " ".join(f"{v:.4f}" for v in fit(fmt=fmt)))
    for name, more in (("layer norm", dict()), ("orthogonal updates", dict(muon_lr=0.02)), ("and 4-bit products", dict(muon_lr=0.02, mx=True))):
        print(name, " ".join(f"{v:.4f}" for v in fit(norm="layer", **more)))
