"""A recurrent core for policies that have to remember, from the library's sequence-memory operators (no arithmetic of the core lives here).

The core turns features that a program has into features that remember (the library's own policies go from frames to logits in one call, without it):

    u  = x W_in^T + b_in                 [T,N,2I]: what is remembered, and a gate z
    c  = silu(short convolution of u's first half)
    p  = c W_proj^T                      [T,N,R+2S]: what the step sizes come from, B, C
    dt = p[.., :R] W_dt^T
    h  = selective scan of (c, dt, A, B, C), read out as v, gated by z
    y  = v W_out^T + b_out + x

A learner runs it over a whole storage (`forward`, `backward`), an actor a step at a time (`step`); both carry the same state (`State`).  `starts` marks the
steps that begin an episode; rows 1.. of a [T+1,N] array of starts are the `dones` of hts_returns_gae.  Parameters and gradients are flat binary32 vectors of
the same packing, for hts_adam_apply_static and the like; with bfloat16 operands `sync_params` refreshes the matrices' copies after an update.

`DeltaCore` is a block of the same interface around a memory that keys write and queries read, behind a layer norm, so that blocks can be stacked:

    n = layer norm of x                  [T,N,F]
    c = silu(short convolution of n W_in^T + b_in)     queries and keys [G,K] and values [H,V] of its heads
    g = n W_gate^T                       what the heads' decays and strengths come from, [2,H]
    h = gated delta rule of (q, k, v, g)
    y = h W_out^T + b_out + x

`optimizer` of a core is AdamW over its arrays (states in 32 or in 8 bits), which refreshes the matrices' copies as it updates them.

    python -m paper_2012_09849_amd.memory        # trains a small core of each kind to recall a cue, then acts with it step by step
"""
from __future__ import annotations

import torch

from . import binding as hts


def _meet(a, b):
    """Whether rows [M,F] of two tensors share memory."""
    (p, ld, m, size), (q, to, n, other) = ((t.data_ptr(), t.stride(0) * t.element_size(), t.shape[0], t.shape[1] * t.element_size()) for t in (a, b))
    if p + (m - 1) * ld + size <= q or q + (n - 1) * to + other <= p:
        return False
    # of the second one's rows the first that ends beyond a row's beginning begins before that row's end
    rows, theirs = p + torch.arange(m) * ld, q + torch.arange(n) * to
    first = torch.searchsorted(theirs + other, rows, right=True)
    there = first < n
    return bool((theirs[first[there]] < rows[there] + size).any())


class State:
    """What N sequences carry from call to call: the convolution's last inputs and the scan's states (zeros: nothing remembered)."""

    def __init__(self, core, N):
        with torch.cuda.stream(core.ctx.stream):               # where it is used
            self.conv = torch.zeros(N, core.width - 1, core.inner, device="cuda")
            self.h = torch.zeros(N, core.inner, core.states, device="cuda")

    def clone(self):
        other = object.__new__(State)
        other.conv, other.h = self.conv.clone(), self.h.clone()
        return other


class MemoryCore:
    """features F, inner I, states S of a channel, filter width W, rank R of the step sizes; up to max_steps x max_rows steps a call."""

    def __init__(self, features=512, inner=1024, states=16, width=4, rank=32, precision=hts.PRECISION_FP32, max_steps=1, max_rows=1, stream=None):
        self.features, self.inner, self.states, self.width, self.rank = features, inner, states, width, rank
        self.precision, self.dtype = precision, torch.bfloat16 if precision == hts.PRECISION_BF16 else torch.float32
        self.max_steps, self.max_rows = max_steps, max_rows
        F, I, S, R = features, inner, states, rank
        shapes = {"in.w": (2 * I, F), "in.b": (2 * I,), "conv.w": (I, width), "conv.b": (I,), "proj.w": (R + 2 * S, I), "dt.w": (I, R), "dt.b": (I,), "A": (I, S),
                       "skip": (I,), "out.w": (F, I), "out.b": (F,)}
        need = [hts.short_conv_workspace(max_steps, max_rows, I, width, precision=precision), hts.selective_scan_workspace(max_steps, max_rows, I, S, precision=precision)]
        self._make(shapes, ("in.w", "proj.w", "dt.w", "out.w"), need, stream)
        with torch.cuda.stream(self.ctx.stream):
            new = lambda k: torch.empty(max_steps * max_rows, k, dtype=self.dtype, device="cuda")  # noqa: E731
            self._u, self._c, self._p, self._dt, self._v = new(2 * I), new(I), new(R + 2 * S), new(I), new(I)

    def _make(self, shapes, matrices, need, stream):
        """The packing, the context and the parameters with their gradients.  matrices: what products read; need: bytes of workspace of the other calls."""
        self.shapes, self.matrices = shapes, matrices
        # every array of the packing begins at a multiple of 16 bytes
        self.offsets, self.P = {}, 0
        for name, shape in shapes.items():
            self.offsets[name] = self.P
            self.P += -(-torch.Size(shape).numel() // 4) * 4
        M = self.max_steps * self.max_rows
        self.ctx = hts.SeqContext(max(need + [hts.linear_workspace(M, *shapes[w], precision=self.precision) for w in matrices]), stream=stream)
        with torch.cuda.stream(self.ctx.stream):               # where they are used
            self.params = torch.zeros(self.P, device="cuda")
            self.grads = torch.zeros(self.P, device="cuda")
            self.p, self.g = self.views(self.params), self.views(self.grads)
            self.m = dict(self.p) if self.precision == hts.PRECISION_FP32 else {n: torch.zeros(shapes[n], dtype=self.dtype, device="cuda") for n in matrices}
        self._states, self._training = None, None

    def _states_needed(self, T, N):
        """Floats that a training forward call keeps of its states."""
        return hts.selective_scan_states(T, N, self.inner, self.states)

    def views(self, vector):
        """The packing's arrays, of a vector of P binary32 numbers."""
        return {n: vector[o:o + torch.Size(s).numel()].view(s) for (n, s), o in zip(self.shapes.items(), self.offsets.values())}

    def init_params(self, seed=0):
        """Small random projections; decays at -1 .. -S, step sizes between 1e-3 and 0.1."""
        g = torch.Generator().manual_seed(seed)
        p = self.views(torch.zeros(self.P))
        for name in ("in.w", "proj.w", "dt.w", "out.w", "conv.w"):
            p[name].copy_(torch.randn(p[name].shape, generator=g) / p[name].shape[1] ** 0.5)
        p["A"].copy_(-torch.arange(1, self.states + 1, dtype=torch.float32).expand(self.inner, -1))
        size = torch.exp(torch.rand(self.inner, generator=g) * 4.605 - 6.908)
        p["dt.b"].copy_(size + torch.log(-torch.expm1(-size)))
        p["skip"].fill_(1.0)
        self._put(p)

    def _put(self, p):
        with torch.cuda.stream(self.ctx.stream):
            for name, t in p.items():
                self.p[name].copy_(t)
        self.sync_params()

    def new_state(self, N):
        """What N sequences carry before their first step."""
        return State(self, N)

    def optimizer(self, bits=32, weight_decay=0.0):
        """hts.AdamW over the core's arrays and their gradients, on the core's stream: matrices decay, nothing else does; their copies are written with them.  bits: 32 or 8."""
        if bits not in (8, 32):
            raise hts.HtsError("optimizer: states have 32 or 8 bits")
        tensors = []
        with torch.cuda.stream(self.ctx.stream):
            for name, p in self.p.items():
                n, matrix = p.numel(), name in self.matrices
                if bits == 8:
                    state = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.zeros(hts.adamw_scales(n), device="cuda") for _ in range(2)]
                else:
                    state = [torch.zeros(n, device="cuda") for _ in range(2)]
                copy = self.m[name] if matrix and self.precision == hts.PRECISION_BF16 else None
                tensors.append(hts.AdamWTensor(p, self.g[name], *state, copy=copy, weight_decay=weight_decay if matrix else 0.0))
        return hts.AdamW(tensors, stream=self.ctx.stream)

    def sync_params(self):
        """After the parameters changed: the matrices in the operands' type, on the context's stream."""
        if self.precision == hts.PRECISION_BF16:
            with torch.cuda.stream(self.ctx.stream):
                for name, t in self.m.items():
                    t.copy_(self.p[name])

    def _rows(self, a, shape, name):
        """[T,N,F] as [T N, F], in its place."""
        T, N, _ = shape
        if not isinstance(a, torch.Tensor) or a.shape != shape or a.dtype is not self.dtype or (T > 1 and N > 1 and a.stride(0) != N * a.stride(1)):
            raise hts.HtsError(f"{name}: expected a {self.dtype} device tensor of shape {tuple(shape)} whose rows are one distance apart")
        return a.view(shape[0] * shape[1], shape[2])

    def _run(self, x, y, starts, lengths, state, states):
        self._training = None                                   # what a call before this one kept is overwritten
        T, N, F = x.shape
        I, S, R, M = self.inner, self.states, self.rank, x.shape[0] * x.shape[1]
        if T > self.max_steps or N > self.max_rows or F != self.features:
            raise hts.HtsError(f"x: at most [{self.max_steps},{self.max_rows},{self.features}]")
        c, xs, ys = self.ctx, self._rows(x, x.shape, "x"), self._rows(y, x.shape, "y")
        u, conv, p, dt, v = (a[:M] for a in (self._u, self._c, self._p, self._dt, self._v))
        steps = lambda a: a.view(T, N, a.shape[-1])  # noqa: E731
        c.hts_linear(xs, self.m["in.w"], u, bias=self.p["in.b"])
        c.hts_short_conv(steps(u)[:, :, :I], self.p["conv.w"], steps(conv), bias=self.p["conv.b"], act=hts.ACT_SILU, starts=starts, lengths=lengths, state_in=state.conv,
                         state_out=state.conv)
        c.hts_linear(conv, self.m["proj.w"], p)
        c.hts_linear(p[:, :R], self.m["dt.w"], dt)
        c.hts_selective_scan(steps(conv), steps(dt), self.p["A"], steps(p)[:, :, R:R + S], steps(p)[:, :, R + S:], steps(v), z=steps(u)[:, :, I:], skip=self.p["skip"],
                             dt_bias=self.p["dt.b"], starts=starts, lengths=lengths, h_in=state.h, h_out=state.h, states=states)
        c.hts_linear(v, self.m["out.w"], ys, bias=self.p["out.b"], residual=xs)

    def step(self, x, y, state, starts=None):
        """One step of N sequences: x, y [N,F], starts u8 [N]; the state moves on in its place.  (It takes the place of what a training call kept.)"""
        self._run(x[None], y[None], None if starts is None else starts[None], None, state, None)

    def forward(self, x, y, state, starts=None, lengths=None, train=False):
        """T steps of N sequences: x, y [T,N,F], all rows one distance apart, starts u8 [T,N], lengths i32 [N]; the state moves on in its place; y may take x's place.  train: what
        `backward` reads is kept until the next call, but for x, starts and lengths, which it reads where they are: they stay as they are until then, and y is not in x's place."""
        states = None
        if train:
            if _meet(self._rows(x, x.shape, "x"), self._rows(y, x.shape, "y")):
                raise hts.HtsError("forward: y shares memory with x, which backward reads")
            need = self._states_needed(x.shape[0], x.shape[1])
            with torch.cuda.stream(self.ctx.stream):          # where they are used
                if self._states is None or self._states.numel() < need:
                    self._states = torch.empty(need, device="cuda")
                begun = state.clone()
            states = self._states
        self._run(x, y, starts, lengths, state, states)
        if train:
            self._training = (x, starts, lengths, begun)

    def backward(self, dy, dx):
        """The gradients of dy [T,N,F] at the last forward(train=True): of the parameters into self.grads, of x into dx, which shares no memory with dy and x.  The state that
        the storage began with is a constant."""
        if self._training is None:
            raise hts.HtsError("backward: no forward(train=True) before it")
        x, starts, lengths, begun = self._training
        T, N, F = x.shape
        I, S, R, M, c, g = self.inner, self.states, self.rank, x.shape[0] * x.shape[1], self.ctx, self.g
        u, conv, p, dt, v = (a[:M] for a in (self._u, self._c, self._p, self._dt, self._v))
        new = lambda k: torch.empty(M, k, dtype=self.dtype, device="cuda")  # noqa: E731
        xs, dys, dxs = (self._rows(a, x.shape, name) for a, name in ((x, "x"), (dy, "dy"), (dx, "dx")))
        if _meet(dxs, dys) or _meet(dxs, xs):
            raise hts.HtsError("backward: dx shares memory with dy or x")
        steps = lambda a: a.view(T, N, a.shape[-1])  # noqa: E731
        with torch.cuda.stream(self.ctx.stream):
            du, dconv, dp, ddt, dv = new(2 * I), new(I), new(R + 2 * S), new(I), new(I)
        seq = dict(starts=starts, lengths=lengths)
        c.hts_linear_backward(v, self.m["out.w"], dys, dx=dv, dw=g["out.w"], db=g["out.b"])
        c.hts_selective_scan_backward(steps(conv), steps(dt), self.p["A"], steps(p)[:, :, R:R + S], steps(p)[:, :, R + S:], steps(dv), self._states, steps(dconv), steps(ddt),
                                      steps(dp)[:, :, R:R + S], steps(dp)[:, :, R + S:], g["A"], z=steps(u)[:, :, I:], dz=steps(du)[:, :, I:], skip=self.p["skip"],
                                      dskip=g["skip"], dt_bias=self.p["dt.b"], ddt_bias=g["dt.b"], h_in=begun.h, **seq)
        c.hts_linear_backward(p[:, :R], self.m["dt.w"], ddt, dx=dp[:, :R], dw=g["dt.w"])
        c.hts_linear_backward(conv, self.m["proj.w"], dp, add=dconv, dx=dconv, dw=g["proj.w"])
        c.hts_short_conv_backward(steps(u)[:, :, :I], self.p["conv.w"], steps(dconv), steps(du)[:, :, :I], g["conv.w"], db=g["conv.b"], bias=self.p["conv.b"],
                                  act=hts.ACT_SILU, state_in=begun.conv, **seq)
        c.hts_linear_backward(xs, self.m["in.w"], du, add=dys, dx=dxs, dw=g["in.w"], db=g["in.b"])

    def close(self):
        self.ctx.close()


class DeltaState:
    """What N sequences carry from call to call: the convolution's last inputs and the heads' states (zeros: nothing remembered)."""

    def __init__(self, core, N):
        with torch.cuda.stream(core.ctx.stream):               # where it is used
            self.conv = torch.zeros(N, core.width - 1, core.channels, device="cuda")
            self.h = torch.zeros(N, core.heads, core.keys, core.values, device="cuda")

    def clone(self):
        other = object.__new__(DeltaState)
        other.conv, other.h = self.conv.clone(), self.h.clone()
        return other


class DeltaCore(MemoryCore):
    """features F, H heads of K x V, G groups of queries and keys (default: one for each head), filter width W; up to max_steps x max_rows steps a call."""

    def __init__(self, features=512, heads=8, keys=128, values=128, groups=None, width=4, precision=hts.PRECISION_FP32, max_steps=1, max_rows=1, stream=None):
        self.features, self.heads, self.keys, self.values, self.groups, self.width = features, heads, keys, values, groups or heads, width
        self.precision, self.dtype = precision, torch.bfloat16 if precision == hts.PRECISION_BF16 else torch.float32
        self.max_steps, self.max_rows = max_steps, max_rows
        F, H, V, M = features, heads, values, max_steps * max_rows
        self.channels = C = 2 * self.groups * keys + H * V
        shapes = {"norm.w": (F,), "norm.b": (F,), "in.w": (C, F), "in.b": (C,), "conv.w": (C, width), "conv.b": (C,), "gate.w": (2 * H, F), "A": (H,), "a.b": (H,), "out.w": (F, H * V), "out.b": (F,)}
        need = [hts.layer_norm_workspace(M, F, precision=precision), hts.short_conv_workspace(max_steps, max_rows, C, width, precision=precision),
                hts.delta_rule_workspace(max_steps, max_rows, H, self.groups, keys, V, precision=precision)]
        self._make(shapes, ("in.w", "gate.w", "out.w"), need, stream)
        with torch.cuda.stream(self.ctx.stream):
            new = lambda k: torch.empty(M, k, dtype=self.dtype, device="cuda")  # noqa: E731
            self._n, self._u, self._c, self._g, self._v = new(F), new(C), new(C), new(2 * H), new(H * V)

    def new_state(self, N):
        return DeltaState(self, N)

    def _states_needed(self, T, N):
        return hts.delta_rule_states(T, N, self.heads, self.keys, self.values)

    def init_params(self, seed=0):
        """Small random projections; decays of a step between exp(-0.001) and exp(-1.6)."""
        g = torch.Generator().manual_seed(seed)
        p = self.views(torch.zeros(self.P))
        for name in ("in.w", "gate.w", "out.w", "conv.w"):
            p[name].copy_(torch.randn(p[name].shape, generator=g) / p[name].shape[1] ** 0.5)
        p["norm.w"].fill_(1.0)
        p["A"].copy_(-1 - 15 * torch.rand(self.heads, generator=g))
        size = torch.exp(torch.rand(self.heads, generator=g) * 4.605 - 6.908)
        p["a.b"].copy_(size + torch.log(-torch.expm1(-size)))
        self._put(p)

    def _parts(self, c, gates, T, N):
        """The convolution's channels and the gates as the rule reads them: q, k, v, a, b."""
        GK, H = self.groups * self.keys, self.heads
        c, gates = c.view(T, N, self.channels), gates.view(T, N, 2 * H)
        q, k = (c[:, :, i * GK:(i + 1) * GK].unflatten(2, (self.groups, self.keys)) for i in range(2))
        return q, k, c[:, :, 2 * GK:].unflatten(2, (H, self.values)), gates[:, :, :H], gates[:, :, H:]

    def _rule(self, starts, lengths, h):
        return dict(a_bias=self.p["a.b"], scale=self.keys ** -0.5, starts=starts, lengths=lengths, h_in=h)

    def _run(self, x, y, starts, lengths, state, states):
        self._training = None                                   # what a call before this one kept is overwritten
        T, N, F = x.shape
        M, c = T * N, self.ctx
        if T > self.max_steps or N > self.max_rows or F != self.features:
            raise hts.HtsError(f"x: at most [{self.max_steps},{self.max_rows},{self.features}]")
        xs, ys = self._rows(x, x.shape, "x"), self._rows(y, x.shape, "y")
        n, u, conv, gates, v = (a[:M] for a in (self._n, self._u, self._c, self._g, self._v))
        steps = lambda a: a.view(T, N, a.shape[-1])  # noqa: E731
        c.hts_layer_norm(xs, n, w=self.p["norm.w"], b=self.p["norm.b"])
        c.hts_linear(n, self.m["in.w"], u, bias=self.p["in.b"])
        c.hts_short_conv(steps(u), self.p["conv.w"], steps(conv), bias=self.p["conv.b"], act=hts.ACT_SILU, starts=starts, lengths=lengths, state_in=state.conv, state_out=state.conv)
        c.hts_linear(n, self.m["gate.w"], gates)
        c.hts_delta_rule(*self._parts(conv, gates, T, N), self.p["A"], steps(v).unflatten(2, (self.heads, self.values)), h_out=state.h, states=states,
                         **self._rule(starts, lengths, state.h))
        c.hts_linear(v, self.m["out.w"], ys, bias=self.p["out.b"], residual=xs)

    def backward(self, dy, dx):
        """As MemoryCore.backward."""
        if self._training is None:
            raise hts.HtsError("backward: no forward(train=True) before it")
        x, starts, lengths, begun = self._training
        T, N, F = x.shape
        M, c, g = T * N, self.ctx, self.g
        n, u, conv, gates, v = (a[:M] for a in (self._n, self._u, self._c, self._g, self._v))
        xs, dys, dxs = (self._rows(a, x.shape, name) for a, name in ((x, "x"), (dy, "dy"), (dx, "dx")))
        if _meet(dxs, dys) or _meet(dxs, xs):
            raise hts.HtsError("backward: dx shares memory with dy or x")
        steps = lambda a: a.view(T, N, a.shape[-1])  # noqa: E731
        heads = lambda a: steps(a).unflatten(2, (self.heads, self.values))  # noqa: E731
        with torch.cuda.stream(c.stream):
            dn, du, dconv, dgates, dv = (torch.empty_like(a) for a in (n, u, conv, gates, v))
        c.hts_linear_backward(v, self.m["out.w"], dys, dx=dv, dw=g["out.w"], db=g["out.b"])
        dq, dk, dvalues, da, db = self._parts(dconv, dgates, T, N)
        c.hts_delta_rule_backward(*self._parts(conv, gates, T, N), self.p["A"], heads(dv), self._states, dq, dk, dvalues, da, db, g["A"], da_bias=g["a.b"],
                                  **self._rule(starts, lengths, begun.h))
        c.hts_short_conv_backward(steps(u), self.p["conv.w"], steps(dconv), steps(du), g["conv.w"], db=g["conv.b"], bias=self.p["conv.b"], act=hts.ACT_SILU, state_in=begun.conv,
                                  starts=starts, lengths=lengths)
        c.hts_linear_backward(n, self.m["gate.w"], dgates, dx=dn, dw=g["gate.w"])
        c.hts_linear_backward(n, self.m["in.w"], du, add=dn, dx=dn, dw=g["in.w"], db=g["in.b"])
        c.hts_layer_norm_backward(xs, dn, w=self.p["norm.w"], add=dys, dx=dxs, dw=g["norm.w"], db=g["norm.b"])


def recall_storage(T, N, F, seed):
    """Episodes of about 12 steps whose first observation carries a cue of +1 or -1 in its first feature (every other feature is noise): observations
    [T,N,F], the cue of every step's episode [T,N], starts."""
    g = torch.Generator().manual_seed(seed)
    starts = (torch.rand(T, N, generator=g) < 1 / 12).to(torch.uint8)
    starts[0] = 1
    cue = torch.randint(0, 2, (T, N), generator=g).float() * 2 - 1
    for t in range(1, T):
        cue[t] = torch.where(starts[t] != 0, cue[t], cue[t - 1])
    x = torch.randn(T, N, F, generator=g) * 0.3
    x[:, :, 0] = torch.where(starts != 0, cue, torch.zeros(()))
    return x, cue, starts


def train_recall(core, updates, T=32, N=16, lr=3e-3, seed=1, optimizer=None):
    """The last feature of y learns to hold the episode's cue: mean squared errors of the updates.  optimizer: the core's AdamW, or Adam on the flat vectors."""
    F, losses, caller = core.features, [], torch.cuda.current_stream()
    core.ctx.stream.wait_stream(caller)
    with torch.cuda.stream(core.ctx.stream):                   # the storages and what is computed from them, where the core's calls read and write them
        if optimizer is None:
            opt, hp = hts.OptState(torch.zeros(core.P, device="cuda"), torch.zeros(core.P, device="cuda")), hts.HParams(lr=lr, max_grad_norm=1.0)
        else:
            hp = hts.AdamWHParams(lr=lr, max_grad_norm=1.0, seed=seed)
        for k in range(updates):
            x, cue, starts = (a.cuda() for a in recall_storage(T, N, F, seed + k))
            x = x.to(core.dtype)
            y, dy, dx = torch.empty_like(x), torch.zeros_like(x), torch.empty_like(x)
            core.forward(x, y, core.new_state(N), starts=starts, train=True)
            off = y[:, :, F - 1].float() - cue
            dy[:, :, F - 1] = (2 / off.numel()) * off
            losses.append((off * off).mean())
            core.backward(dy, dx)
            if optimizer is None:
                hts.hts_adam_apply_static(core.params, core.grads, opt, hp, core.ctx.stream)
                core.sync_params()
            else:
                optimizer.hts_adamw_step(hp)
        losses = [float(v) for v in losses]
    caller.wait_stream(core.ctx.stream)
    return losses


def _recall(core, optimizer=None):
    losses = train_recall(core, 200, optimizer=optimizer)
    print(f"recalling a cue: mean squared error {sum(losses[:5]) / 5:.3f} at first, {sum(losses[-5:]) / 5:.3f} after {len(losses)} updates")
    x, cue, starts = (a.cuda() for a in recall_storage(32, 16, 64, 12345))
    x, state = x.to(core.dtype), core.new_state(16)
    y = torch.empty(16, 64, dtype=core.dtype, device="cuda")
    right = 0
    for t in range(32):
        core.step(x[t], y, state, starts[t])
        right += int((y[:, 63].sign() == cue[t]).sum())
    print(f"acting step by step on episodes never seen: the cue's sign is right in {right} of {32 * 16} steps")


def main():
    core = MemoryCore(features=64, inner=128, precision=hts.PRECISION_BF16, max_steps=32, max_rows=16)         # on the current stream, as is all of the below
    core.init_params()
    _recall(core)
    core.close()
    core = DeltaCore(features=64, heads=4, keys=32, values=32, precision=hts.PRECISION_BF16, max_steps=32, max_rows=16)
    core.init_params()
    optimizer = core.optimizer(bits=8, weight_decay=0.01)
    _recall(core, optimizer)
    optimizer.close()
    core.close()


if __name__ == "__main__":
    main()
