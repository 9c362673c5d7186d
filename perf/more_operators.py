"""More operators of a policy's sequence memory and of its training, as cases that can be timed and compared: layer norm with its gradients, the
gated delta rule (long sequences, single steps, gradients), and AdamW over many tensors with states in 32 or in 8 bits, on the shapes of this
package's workloads (storages of 512 x 16 steps and environments, unrolls of 5, 512 features, 1024 inner channels) and on long prompts.

The plain forms compute in binary32 (binary64 for long sums) with elementary tensor operations and round once at the end; `exact` computes the
definitions step by step in binary64."""
import math

import torch

own = False


def listed():
    return [
        # one step of 16 environments: bound by latency
        {"name": "norm_16", "kind": "norm", "dtype": "bf16", "m": 16, "f": 512},
        # a storage of 512 x 16 before its projection
        {"name": "norm_8192", "kind": "norm", "dtype": "bf16", "m": 8192, "f": 512},
        # the gradients of a storage of wide rows, with what reaches the input past the block
        {"name": "norm_grad_8192", "kind": "norm_grad", "dtype": "bf16", "m": 8192, "f": 2048, "residual": True},
        # full precision at sizes that are no multiple of anything
        {"name": "norm_grad_odd_f32", "kind": "norm_grad", "dtype": "f32", "m": 1021, "f": 777, "residual": False},
        # one step of 32 environments: the memory is read, moved on and written
        {"name": "delta_step_32", "kind": "delta", "dtype": "bf16", "t": 1, "n": 32, "h": 8, "g": 8, "k": 128, "v": 128, "starts": True, "lengths": False},
        # an unroll of 5 steps of 16 environments in full precision
        {"name": "delta_unroll_5x16_f32", "kind": "delta", "dtype": "f32", "t": 5, "n": 16, "h": 4, "g": 4, "k": 64, "v": 64, "starts": True, "lengths": False},
        # one long prompt: little to work on at a time but time itself
        {"name": "delta_prompt_8192", "kind": "delta", "dtype": "bf16", "t": 8192, "n": 1, "h": 8, "g": 8, "k": 128, "v": 128, "starts": False, "lengths": False},
        # a storage of the learner, forward and backward
        {"name": "delta_train_512x16", "kind": "delta_train", "dtype": "bf16", "t": 512, "n": 16, "h": 8, "g": 8, "k": 128, "v": 128, "starts": True, "lengths": False},
        # ragged sequences in full precision, odd sizes, keys that two heads share
        {"name": "delta_train_129x5_f32", "kind": "delta_train", "dtype": "f32", "t": 129, "n": 5, "h": 6, "g": 3, "k": 37, "v": 53, "starts": True, "lengths": True},
        # the tensors of a small core: bound by latency
        {"name": "adamw_small", "kind": "adamw", "features": 64, "inner": 128, "layers": 1, "bits": 32, "grads": "f32", "clip": True},
        # those of one core of 512 features, with the bfloat16 copies of its matrices
        {"name": "adamw_core", "kind": "adamw", "features": 512, "inner": 1024, "layers": 1, "bits": 32, "grads": "f32", "clip": True},
        # a stack of cores, states in 8 bits, gradients in bfloat16
        {"name": "adamw_stack_8bit", "kind": "adamw", "features": 512, "inner": 1024, "layers": 24, "bits": 8, "grads": "bf16", "clip": True},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "norm_grad", "delta", "delta_train", "delta_train", "adamw"))
    if kind == "adamw":
        return {"kind": kind, "features": _log_uniform(rng, 24, 640), "inner": _log_uniform(rng, 48, 1280), "layers": _log_uniform(rng, 1, 8), "bits": rng.choice((8, 32)),
                "grads": rng.choice(("f32", "bf16")), "clip": rng.choice((True, False))}
    case = {"kind": kind, "dtype": rng.choice(("bf16", "bf16", "f32"))}
    if kind in ("norm", "norm_grad"):
        even = rng.choice((1, 8, 64))          # widths that are multiples of nothing, of a vector, of a wavefront
        f = max(even, _log_uniform(rng, 16, 8192) // even * even)
        case.update(m=_log_uniform(rng, 1, max(1, min(16384, 16777216 // f))), f=f)
        if kind == "norm_grad":
            case["residual"] = rng.choice((True, False))
        return case
    h = _log_uniform(rng, 1, 12)
    g = rng.choice([g for g in range(1, h + 1) if h % g == 0 and h // g <= 4])
    k, v = (rng.choice((128, 64, 32, _log_uniform(rng, 8, 128))) for _ in range(2))
    n = _log_uniform(rng, 1, 48)
    most = max(2, 512 * 16 * 8 * 128 * 128 // (n * h * max(k, 32) * max(v, 32)))
    t = 1 if kind == "delta" and rng.random() < 0.25 else _log_uniform(rng, 2, min(8192 if kind == "delta" else 1024, most))
    case.update(t=t, n=n, h=h, g=g, k=k, v=v, starts=rng.choice((True, False)), lengths=rng.choice((True, False)))
    return case


# ---- inputs -------------------------------------------------------------------------------------------------------
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
ADAMW = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "seed": 20202021}
BLOCK = 256          # entries that share a scale where states are held in 8 bits


def _sequence(case, g):
    """Which steps begin an episode (one in 100, as in the workloads' storages) and how many steps each sequence has (all, or a share of them; one has none)."""
    t, n = case["t"], case["n"]
    starts = (torch.rand(t, n, device="cuda", generator=g) < 0.01).to(torch.uint8) if case["starts"] else None
    lengths = None
    if case["lengths"]:
        lengths = (torch.rand(n, device="cuda", generator=g) * (t + 1)).floor().to(torch.int32).clamp_(max=t)
        lengths[0] = t
        if n > 2:
            lengths[n // 2] = 0
    return starts, lengths


def _shapes(case):
    """A core's tensors: matrices, whose bfloat16 copies are its operands, and the rest, which does not decay."""
    f, i = case["features"], case["inner"]
    return ((2 * i, f), (2 * i,), (i, 4), (i,), (64, i), (i, 32), (i,), (i, 16), (i,), (f, i), (f,))


def prepare(case, seed):
    kind = case["kind"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, device="cuda", generator=g)  # noqa: E731
    s = {"case": case}
    if kind in ("norm", "norm_grad"):
        dt, m, f = TYPES[case["dtype"]], case["m"], case["f"]
        s["x"] = (normal(m, f) * (0.5 + uniform(f)) + 0.3 * normal(m, 1)).to(dt)
        s["w"], s["b"] = 1 + 0.1 * normal(f), 0.1 * normal(f)
        if kind == "norm_grad":
            s["dy"] = normal(m, f).to(dt)
            s["add"] = normal(m, f).to(dt) if case["residual"] else None
    elif kind in ("delta", "delta_train"):
        dt = TYPES[case["dtype"]]
        t, n, h, gr, k, v = (case[c] for c in "tnhgkv")
        s["starts"], s["lengths"] = _sequence(case, g)
        mixed = torch.nn.functional.silu(normal(t, n, 2 * gr * k + h * v)).to(dt)        # what a convolution with an activation hands over holds all three
        s["q"], s["k"] = (mixed[:, :, i * gr * k:(i + 1) * gr * k].unflatten(2, (gr, k)) for i in range(2))
        s["v"] = mixed[:, :, 2 * gr * k:].unflatten(2, (h, v))
        gates = normal(t, n, 2 * h).to(dt)                                                 # one projection holds the decays' and the strengths' inputs
        s["a"], s["b"] = gates[:, :, :h], gates[:, :, h:]
        s["A"] = -1 - 15 * uniform(h)
        size = torch.exp(uniform(h) * math.log(100.0) + math.log(1e-3))                    # step sizes between 1e-3 and 0.1
        s["a_bias"] = size + torch.log(-torch.expm1(-size))                                # softplus of it gives them
        s["h"] = 0.3 * normal(n, h, k, v)
        s["scale"] = k ** -0.5
        if kind == "delta_train":
            s["dy"] = normal(t, n, h, v).to(dt)
            s["dh"] = 0.1 * normal(n, h, k, v)
    else:
        s["step"], s["tensors"] = 10, []
        for _ in range(case["layers"]):
            for shape in _shapes(case):
                matrix = len(shape) == 2 and shape[1] > 16
                e = torch.exp(1.5 * normal(*shape)) * 1e-3                                 # gradients of an entry have a size of their own
                t = {"p": normal(*shape) * 0.05, "g": (e * normal(*shape)).to(TYPES[case["grads"]]), "decay": 0.1 if matrix else 0.0,
                     "copy": torch.empty(shape, dtype=torch.bfloat16, device="cuda") if matrix else None}
                m, r = 0.3 * e * normal(*shape), e * (0.2 + uniform(*shape))
                if case["bits"] == 32:
                    t["m"], t["v"] = m, r * r
                else:
                    t["m"], t["m_scale"] = _held(m, 0.5)
                    t["v"], t["v_scale"] = _held(r, 0.5, positive=True)
                s["tensors"].append(t)
        s["grad_norm"] = torch.zeros(1, device="cuda")
        s["clip"] = 1.0 if case["clip"] else 0.0
    if own:
        _user(case, s)
    return s


def _user(case, s):
    """A program's context or optimiser, and the arrays that its calls write."""
    import paper_2012_09849_amd as hts
    kind = case["kind"]
    new32 = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
    if kind == "adamw":
        s["opt"] = hts.AdamW([hts.AdamWTensor(t["p"], t["g"], t["m"], t["v"], t.get("m_scale"), t.get("v_scale"), copy=t["copy"], weight_decay=t["decay"]) for t in s["tensors"]])
        s["opt"].step = s["step"]
        s["hp"] = hts.AdamWHParams(max_grad_norm=s["clip"], **ADAMW)
        return
    dt, precision = TYPES[case["dtype"]], hts.PRECISION_BF16 if case["dtype"] == "bf16" else hts.PRECISION_FP32
    new = lambda *shape: torch.empty(*shape, dtype=dt, device="cuda")  # noqa: E731
    if kind in ("norm", "norm_grad"):
        m, f = case["m"], case["f"]
        need = hts.layer_norm_workspace(m, f, precision=precision) if kind == "norm_grad" else 0        # (a forward call needs none)
        s["out"] = {"y": new(m, f)} if kind == "norm" else {"dx": new(m, f), "dw": new32(f), "db": new32(f)}
    else:
        t, n, h, gr, k, v = (case[c] for c in "tnhgkv")
        need = hts.delta_rule_workspace(t, n, h, gr, k, v, precision=precision)
        s["out"] = {"y": new(t, n, h, v), "h_out": new32(n, h, k, v)}
        if kind == "delta_train":
            s["states"] = new32(hts.delta_rule_states(t, n, h, k, v))
            s["grads"] = {"dq": new(t, n, gr, k), "dk": new(t, n, gr, k), "dv": new(t, n, h, v), "da": new(t, n, h), "db": new(t, n, h), "dA": new32(h), "da_bias": new32(h),
                          "dh_in": new32(n, h, k, v)}
    s["ctx"] = hts.SeqContext(need)


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    kind = s["case"]["kind"]
    if kind == "adamw":
        s["opt"].hts_adamw_step(s["hp"], grad_norm=s["grad_norm"])
        return _updated(s)
    ctx = s["ctx"]
    if kind == "norm":
        ctx.hts_layer_norm(s["x"], s["out"]["y"], w=s["w"], b=s["b"], eps=EPS)
        return s["out"]
    if kind == "norm_grad":
        ctx.hts_layer_norm_backward(s["x"], s["dy"], w=s["w"], add=s["add"], eps=EPS, **s["out"])
        return s["out"]
    ins = (s["q"], s["k"], s["v"], s["a"], s["b"], s["A"])
    more = {"a_bias": s["a_bias"], "scale": s["scale"], "starts": s["starts"], "lengths": s["lengths"], "h_in": s["h"]}
    if kind == "delta":
        ctx.hts_delta_rule(*ins, s["out"]["y"], h_out=s["out"]["h_out"], **more)
        return s["out"]
    ctx.hts_delta_rule(*ins, s["out"]["y"], h_out=s["out"]["h_out"], states=s["states"], **more)
    ctx.hts_delta_rule_backward(*ins, s["dy"], s["states"], dh_out=s["dh"], **more, **s["grads"])
    return {**s["out"], **s["grads"]}


def _updated(s):
    """What a step changed (of a stack the first core's and the last one's tensors); states in 8 bits as the numbers of that type, with their scales."""
    eight, held, of = s["case"]["bits"] == 8, s["tensors"], len(_shapes(s["case"]))
    shown = [0, 1, len(held) - 2, len(held) - 1]
    out = {"grad_norm": s["grad_norm"], "p": [t["p"] for t in (held if len(held) <= of else held[:of] + held[-of:])], "copy": [held[i]["copy"] for i in shown]}
    for name in ("m", "v"):
        out[name] = [held[i][name].view(torch.float8_e4m3fn) if eight else held[i][name] for i in shown]
        if eight:
            out[name + "_scale"] = [held[i][name + "_scale"] for i in shown]
    return out


# ---- the plain forms ----------------------------------------------------------------------------------------------
def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "adamw":
        return _plain_adamw(s)
    dt = TYPES[case["dtype"]]
    if kind in ("norm", "norm_grad"):
        x = s["x"].float()
        x = x - x.mean(1, keepdim=True)
        r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        x = x * r
        if kind == "norm":
            return {"y": (x * s["w"] + s["b"]).to(dt)}
        dy = s["dy"].float()
        g = dy * s["w"]
        dx = r * (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True))
        if s["add"] is not None:
            dx = dx + s["add"].float()
        return {"dx": dx.to(dt), "dw": (dy * x).double().sum(0).float(), "db": dy.double().sum(0).float()}
    if kind == "delta":
        y, h = _chunks(s, *(s[c].float() for c in ("q", "k", "v", "a", "b", "A", "a_bias", "h")))
        return {"y": y.to(dt), "h_out": h}
    with torch.enable_grad():
        leaves = [s[c].float().detach().clone().requires_grad_() for c in ("q", "k", "v", "a", "b", "A", "a_bias", "h")]
        y, h = _chunks(s, *leaves)
    dq, dk, dv, da, db, dA, dbias, dh = torch.autograd.grad((y, h), leaves, (s["dy"].float(), s["dh"]))
    return {"y": y.detach().to(dt), "h_out": h.detach(), "dq": dq.to(dt), "dk": dk.to(dt), "dv": dv.to(dt), "da": da.to(dt), "db": db.to(dt), "dA": dA, "da_bias": dbias, "dh_in": dh}


def _chunks(s, q, k, v, a, b, A, a_bias, state):
    """The rule over up to 64 steps at a time: within them what each step writes depends on the ones before it by a unit lower triangular matrix."""
    case = s["case"]
    t, n, h = (case[c] for c in "tnh")
    c = min(64, t)
    m = -(-t // c)
    at = torch.arange(t, device="cuda")[:, None]
    live = at < s["lengths"] if s["lengths"] is not None else torch.ones(t, n, dtype=torch.bool, device="cuda")
    fresh = (s["starts"] != 0) & live if s["starts"] is not None else torch.zeros_like(live)
    unit = lambda x: x * torch.rsqrt((x * x).sum(-1, keepdim=True) + 1e-6)  # noqa: E731
    heads = lambda x: x.repeat_interleave(h // case["g"], 2)  # noqa: E731
    x = a + a_bias
    decay = (x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))) * A * live[:, :, None]
    strength = torch.sigmoid(b) * live[:, :, None]

    def cut(x):          # [T,N,H,..] -> [chunks,N,H,c,..], zeros behind the end
        x = torch.cat([x, x.new_zeros((m * c - t, *x.shape[1:]))])
        return x.unflatten(0, (m, c)).movedim(1, 3)

    q, k, v, decay, strength = cut(heads(unit(q)) * s["scale"]), cut(heads(unit(k))), cut(v), cut(decay), cut(strength)[..., None]
    episode = cut(fresh.long()[:, :, None].expand(-1, -1, h)).cumsum(-1)
    far = decay.double().cumsum(-1)
    lower = torch.ones(c, c, dtype=torch.bool, device="cuda").tril()
    seen = (episode[..., :, None] == episode[..., None, :]) & lower
    ratio = torch.exp(torch.where(seen, far[..., :, None] - far[..., None, :], 0.0)).float() * seen
    kt = k.transpose(-1, -2).contiguous()
    before = strength * (k @ kt) * ratio * (~torch.eye(c, dtype=torch.bool, device="cuda"))
    # its inverse: that of blocks of 1, 2, 4 .. steps on the diagonal, from one size to the next
    row = torch.arange(c, device="cuda")
    inverse, size = torch.eye(c, device="cuda").expand_as(before), 1
    while size < c:
        of = row // size
        pair = (of[:, None] // 2 == of // 2) & (of[:, None] % 2 == 1) & (of % 2 == 0)
        inverse = inverse - inverse @ (before * pair) @ inverse
        size *= 2
    read = (q @ kt) * ratio
    kept = (torch.exp(far).float() * (episode == 0))[..., None]                        # of what was there before the chunk
    left = (torch.exp(far[..., -1:] - far).float() * (episode == episode[..., -1:]))[..., None]
    written = inverse @ (strength * v)
    undone = inverse @ (strength * kept * k)
    asked, late = kept * q, (left * k).transpose(-1, -2).contiguous()
    ys = []
    for i in range(m):
        u = written[i] - undone[i] @ state
        ys.append(asked[i] @ state + read[i] @ u)
        state = kept[i, :, :, -1:] * state + late[i] @ u
    y = torch.stack(ys).movedim(3, 1).flatten(0, 1)[:t]
    return y * live[:, :, None, None], state


def _random(seed, counter, tensor, step):
    """Philox4x32-10: four words of 32 bits for each counter."""
    low, k0, k1 = 0xFFFFFFFF, seed & 0xFFFFFFFF, seed >> 32
    c = [counter & low, torch.full_like(counter, tensor), torch.full_like(counter, step & low), torch.full_like(counter, step >> 32)]
    for _ in range(10):
        # 32 x 32 bits as two products of 16 x 32, which 64 bits with a sign hold
        both = []
        for word, by in ((c[0], 0xD2511F53), (c[2], 0xCD9E8D57)):
            mid = word * (by & 0xFFFF)
            top = word * (by >> 16) + (mid >> 16)
            both.append((top >> 16, ((top & 0xFFFF) << 16) | (mid & 0xFFFF)))
        c = [both[1][0] ^ c[1] ^ k0, both[1][1], both[0][0] ^ c[3] ^ k1, both[0][1]]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(c, -1)


def _held(x, part, positive=False):
    """x in 8 bits (e4m3, largest below 256 times a scale, a power of two for BLOCK entries): codes and scales.  part [0,1): how far up a value is moved before the bits
    below the last one are dropped.  positive: what is above zero stays so."""
    flat = x.flatten()
    n = flat.numel()
    rows = torch.cat([flat, flat.new_zeros(-n % BLOCK)]).view(-1, BLOCK)
    most = rows.abs().amax(1)
    power = torch.clamp(((most.view(torch.int32) >> 23) & 255) - 127 - 7, min=-126)
    scale = ((power + 127) << 23).view(torch.float32)
    by = ((127 - power) << 23).view(torch.float32)
    y = (rows * by[:, None]).flatten()[:n]
    e = torch.clamp(((y.view(torch.int32) >> 23) & 255) - 127, min=-6)
    digits = torch.floor(y.abs() * ((127 + 3 - e) << 23).view(torch.float32) + part).to(torch.int32)
    code = (e + 7) * 8 + digits - 8
    if positive:
        code = torch.where((y > 0) & (code == 0), torch.ones_like(code), code)
    code = code | torch.where(y < 0, 128, 0)
    return code.to(torch.uint8).view(x.shape), scale


def _given(code, scale):
    n = code.numel()
    return (code.view(torch.float8_e4m3fn).float().flatten() * scale.repeat_interleave(BLOCK)[:n]).view(code.shape)


def _plain_adamw(s):
    eight, hp = s["case"]["bits"] == 8, ADAMW
    s["step"] += 1
    single = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    b1, b2, lr = (single(hp[c]) for c in ("beta1", "beta2", "lr"))
    rest1, rest2 = single(1.0 - b1), single(1.0 - b2)
    size, root = single(lr / (1 - b1 ** s["step"])), single(1 / math.sqrt(1 - b2 ** s["step"]))
    norm = torch.stack([t["g"].double().square().sum() for t in s["tensors"]]).sum().sqrt().float()
    s["grad_norm"].copy_(norm.view(1))
    by = torch.clamp(s["clip"] / (norm + 1e-6), max=1.0) if s["clip"] > 0 else 1.0
    for i, t in enumerate(s["tensors"]):
        g = t["g"].float() * by
        m, r = (_given(t["m"], t["m_scale"]), _given(t["v"], t["v_scale"])) if eight else (t["m"], None)
        v = r * r if eight else t["v"]
        m = m * b1 + g * rest1
        v = v * b2 + g * rest2 * g
        r = torch.sqrt(v)
        p = t["p"] * single(1.0 - single(lr * single(t["decay"]))) - size * (m / (r * root + single(hp["eps"])))
        t["p"].copy_(p)
        if t["copy"] is not None:
            t["copy"].copy_(p)
        if eight:
            n = g.numel()
            word = _random(hp["seed"], torch.arange(-(-n // 4), device="cuda"), i, s["step"]).flatten()[:n]
            for name, x, part in (("m", m, word & 0xFFFF), ("v", r, word >> 16)):
                code, scale = _held(x, part.float() / 65536, positive=name == "v")
                t[name].copy_(code)
                t[name + "_scale"].copy_(scale)
        else:
            t["m"].copy_(m)
            t["v"].copy_(v)
    return _updated(s)


# ---- the definitions in binary64 ------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    wide = lambda x: None if x is None else x.double()  # noqa: E731
    if kind == "norm":
        return {"y": torch.nn.functional.layer_norm(wide(s["x"]), (case["f"],), wide(s["w"]), wide(s["b"]), EPS)}
    if kind == "norm_grad":
        with torch.enable_grad():
            x, w, b = (wide(s[c]).requires_grad_() for c in ("x", "w", "b"))
            dx, dw, db = torch.autograd.grad(torch.nn.functional.layer_norm(x, (case["f"],), w, b, EPS), (x, w, b), wide(s["dy"]))
        return {"dx": dx if s["add"] is None else dx + wide(s["add"]), "dw": dw, "db": db}
    if kind == "adamw":
        return _exact_adamw(case, s)
    t, n, h = (case[c] for c in "tnh")
    train = kind == "delta_train"
    if train and t * n * h * case["k"] * case["v"] > 1.5e9:
        return None
    length = s["lengths"] if s["lengths"] is not None else torch.full((n,), t, device="cuda")
    per = h // case["g"]
    names = ("q", "k", "v", "a", "b", "A", "a_bias", "h")
    with torch.set_grad_enabled(train):
        given = [wide(s[c]).clone().requires_grad_(train) for c in names]
        q, k, v, a, b, A, bias, state = given
        q, k = (x / torch.sqrt((x ** 2).sum(-1, keepdim=True) + 1e-6) for x in (q, k))
        q, k = (x[:, :, :, None].expand(-1, -1, -1, per, -1).flatten(2, 3) for x in (q, k))
        alpha, beta, ys = torch.exp(A * torch.nn.functional.softplus(a + bias, threshold=40)), torch.sigmoid(b), []
        for i, (qi, ki, vi, ai, bi) in enumerate(zip(*(x.unbind(0) for x in (q, k, v, alpha, beta)))):
            on = (i < length)[:, None, None]
            if s["starts"] is not None:
                ai = torch.where((s["starts"][i] != 0)[:, None], torch.zeros_like(ai), ai)
            moved = ai[..., None, None] * state
            wrong = vi - (ki[..., None] * moved).sum(-2)
            moved = moved + (bi[..., None] * ki)[..., None] * wrong[..., None, :]
            state = torch.where(on[..., None], moved, state)
            ys.append(torch.where(on, s["scale"] * (qi[..., None] * state).sum(-2), torch.zeros_like(vi)))
        y = torch.stack(ys)
    if not train:
        return {"y": y, "h_out": state}
    dq, dk, dv, da, db, dA, dbias, dh = torch.autograd.grad((y, state), given, (wide(s["dy"]), wide(s["dh"])))
    return {"y": y.detach(), "h_out": state.detach(), "dq": dq, "dk": dk, "dv": dv, "da": da, "db": db, "dA": dA, "da_bias": dbias, "dh_in": dh}


def _exact_adamw(case, s):
    """A step from the states as they are held.  What is rounded by random numbers has no value here."""
    eight, hp, step = case["bits"] == 8, ADAMW, s["step"] + 1
    norm = math.sqrt(sum(float((t["g"].double() ** 2).sum()) for t in s["tensors"]))
    by = min(1.0, s["clip"] / (norm + 1e-6)) if s["clip"] > 0 else 1.0
    for t in s["tensors"]:
        g = t["g"].double() * by
        if eight:
            m, r = (t[c].view(torch.float8_e4m3fn).double() for c in ("m", "v"))
            m, r = (x * t[c].double().repeat_interleave(BLOCK)[:x.numel()].view(x.shape) for x, c in ((m, "m_scale"), (r, "v_scale")))
            v = r ** 2
        else:
            m, v = t["m"].double(), t["v"].double()
        m, v = hp["beta1"] * m + (1 - hp["beta1"]) * g, hp["beta2"] * v + (1 - hp["beta2"]) * g ** 2
        update = (m / (1 - hp["beta1"] ** step)) / (torch.sqrt(v / (1 - hp["beta2"] ** step)) + hp["eps"])
        t["p"] = t["p"].double() - hp["lr"] * (update + t["decay"] * t["p"].double())
        t["copy"] = None if t["copy"] is None else t["p"]
        t["m"], t["v"] = m, v
    held, of = s["tensors"], len(_shapes(case))
    shown = [held[i] for i in (0, 1, len(held) - 2, len(held) - 1)]
    out = {"grad_norm": torch.tensor([norm], dtype=torch.float64), "p": [t["p"] for t in (held if len(held) <= of else held[:of] + held[-of:])], "copy": [t["copy"] for t in shown]}
    none = [None] * 4
    out.update({"m": none, "v": none, "m_scale": none, "v_scale": none} if eight else {"m": [t["m"] for t in shown], "v": [t["v"] for t in shown]})
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "adamw":
        sizes = [math.prod(shape) for shape in _shapes(case)]
        copied = sum(math.prod(shape) for shape in _shapes(case) if len(shape) == 2 and shape[1] > 16)
        n, g = sum(sizes), 2 if case["grads"] == "bf16" else 4
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": case["layers"] * (n * (8 + g + state) + 2 * copied), "flops": case["layers"] * n * 16}
    e = 2 if case["dtype"] == "bf16" else 4
    if kind in ("norm", "norm_grad"):
        m, f = case["m"], case["f"]
        if kind == "norm":
            return {"bytes": 2 * e * m * f + 8 * f, "flops": 8 * m * f}
        return {"bytes": e * m * f * (4 if case["residual"] else 3) + 12 * f, "flops": 18 * m * f}
    t, n, h, g, k, v = (case[c] for c in "tnhgkv")
    steps, masks = t * n, (t * n if case["starts"] else 0) + (4 * n if case["lengths"] else 0)
    inputs, state = e * steps * (2 * g * k + h * v + 2 * h) + masks, 4 * n * h * k * v
    # step by step: decay, what is there for the key, the write and the read, 7 operations an entry of the state
    forward = {"bytes": inputs + e * steps * h * v + 2 * state, "flops": 7 * steps * h * k * v}
    if kind == "delta":
        return forward
    # backward: the inputs and the output's gradient again, the gradients out
    return {"bytes": forward["bytes"] + 2 * inputs + e * steps * h * v + 3 * state, "flops": 3 * forward["flops"]}
