"""How many digits the gated delta rule's outputs and gradients have: each array's distance from binary64, as a whole, beside that of the same rule in binary32.

The rule is evaluated step by step on the same inputs by elementary operations, with gradients by torch's own differentiation, in binary64 and in binary32.  The kernels make the same
sums in chunks: for each of a value's K terms up to 64 more of the chunk's steps, twice (the substitution, the product with its result), in another order.  Roundings of either sign add
up by their root, so they are allowed sqrt((K + 128) / K) times binary32's own distance (2 u at least: an array of a few entries may be near by chance), four times (the sum's order is
chance, and one array is one draw), and 4 u for the roundings that the other one does not have (a factor's split, an exponential, the addition over heads).  An array of bfloat16 may be off
by its own rounding too, at most 2^-8 of each entry.  dA and da_bias are few numbers, sums over steps in which much may cancel: they may be off by what their terms may, added up by
its root, and by 16 u of the larger of the sum and the terms' root for the additions (six levels of a wavefront's, up to ten of the sequences' and chunks').
Nothing passes that is a part of 10^5 off: not zeros, another sign, a missing chunk, nor operands of fewer parts."""
import numpy as np
import pytest
import torch

from test_gpu_delta_rule import SHAPES, Case
from test_gpu_seq import hts  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NAMES = ("q", "k", "v", "a", "b", "A", "a_bias", "h_in")


def rule(c, kind, device="cpu"):
    """Outputs and gradients in that type."""
    T, N, G, H, K, V = c.shape
    here = lambda x: None if x is None else x.detach().to(device)  # noqa: E731
    p = {n: None if c.at[n] is None else here(c.at[n]).to(kind).requires_grad_() for n in NAMES}
    unit = (lambda x: x / torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6)) if c.more["normalize"] else (lambda x: x)
    q, k = (unit(p[n]).repeat_interleave(H // G, 2) for n in ("q", "k"))
    x = p["a"] + (0 if p["a_bias"] is None else p["a_bias"])
    step = x.clamp(min=0) + torch.log1p(torch.exp(-x.abs())) if c.more["softplus"] else x
    alpha, beta = torch.exp(step * p["A"]), torch.sigmoid(p["b"])
    S = p["h_in"] if p["h_in"] is not None else torch.zeros(N, H, K, V, dtype=kind, device=device)
    starts, lengths, ys, none = here(c.at["starts"]), here(c.at["lengths"]), [], torch.zeros((), dtype=kind, device=device)
    for t in range(T):
        al = alpha[t] if starts is None else torch.where((starts[t] != 0)[:, None], none, alpha[t])
        moved = al[:, :, None, None] * S
        z = p["v"][t] - (k[t][..., None] * moved).sum(2)
        new = moved + (beta[t][..., None] * k[t])[..., None] * z[:, :, None]
        y = c.more["scale"] * (q[t][..., None] * new).sum(2)
        if lengths is not None:
            on = (t < lengths)[:, None, None]
            new, y = torch.where(on[..., None], new, S), torch.where(on, y, none)
        S = new
        ys.append(y)
    y = torch.stack(ys)
    out = {"y": y, "h_out": S}
    leaves = {n: x for n, x in p.items() if x is not None}
    dh = c.at["dh_out"]
    total = (y * here(c.at["dy"]).to(kind)).sum() + (0 if dh is None else (S * here(dh).to(kind)).sum())
    for n, g in zip(leaves, torch.autograd.grad(total, list(leaves.values()))):      # (da before dA and da_bias)
        out["dh_in" if n == "h_in" else "d" + n] = g
    return {n: x.detach().double().cpu().numpy() for n, x in out.items()}


def check(c, device="cpu"):
    got, wide, single = c.run(), rule(c, torch.float64, device), rule(c, torch.float32, device)
    K, size = c.shape[4], np.linalg.norm
    a, A = c.at["a"].double().cpu().numpy(), c.at["A"].double().cpu().numpy()
    x = a + (0 if c.at["a_bias"] is None else c.at["a_bias"].double().cpu().numpy())
    step, rise = (np.logaddexp(0, x), 1 / (1 + np.exp(-x))) if c.more["softplus"] else (x, 1.0)
    terms = {"da_bias": wide["da"], "dA": wide["da"] / (A * rise) * step}
    share = {}
    for n in wide:
        off = got[n].double().cpu().numpy() - wide[n]
        if n in terms:
            root = np.sqrt((terms[n] ** 2).sum((0, 1)))
            room = share["da"] * root + 16 * U * np.maximum(root, np.abs(wide[n])) + U * np.abs(wide[n])
            assert (np.abs(off) <= room).all(), (n, off, room)
            continue
        most = size(wide[n])
        own = max(size(single[n] - wide[n]) / most, 2 * U) if most else 0.0
        share[n] = 4 * np.sqrt((K + 128) / K) * own + 4 * U
        room = share[n] + (2.0 ** -8 if got[n].dtype is torch.bfloat16 else U)
        assert size(off) <= room * most, (n, f"off by {size(off) / most:.2e}, binary32 by {own:.2e}, allowed {room:.2e}")
        # the test itself can tell (but a single number's length of one leaves 1e-6 of its gradient's terms, and none of their digits)
        assert (K == 1 or share[n] < 1e-3) and share[n] < 1e-5 * max(1.0, own / 2e-7), (n, share[n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,G,H,K,V", SHAPES)
@pytest.mark.parametrize("starts", [0.0, 0.1])
def test_digits(hts, dtype, T, N, G, H, K, V, starts):  # noqa: F811
    c = Case(hts, dtype, T, N, G, H, K, V, starts=starts)
    check(c)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,G,H,K,V,lengths", [(200, 4, 2, 4, 37, 53, [200, 0, 131, 64]), (400, 1, 1, 2, 128, 64, None), (900, 1, 1, 1, 32, 33, None), (330, 3, 2, 2, 64, 128, [330, 1, 257])])
@pytest.mark.parametrize("options", [{}, {"softplus": False, "normalize": False}])
def test_digits_of_many_chunks(hts, dtype, T, N, G, H, K, V, lengths, options):  # noqa: F811
    """Several chunks, in segments too; ragged; keys that heads share and that they do not; as they are and of length one."""
    c = Case(hts, dtype, T, N, G, H, K, V, lengths=lengths, starts=0.01, **options)
    check(c)
    c.ctx.close()


def test_digits_of_decays(hts):  # noqa: F811
    """Strong decays beside none: the last factor's gradients are sums of what passes a step, not differences of what does not."""
    for dtype in ("f32", "bf16"):
        c = Case(hts, dtype, 300, 2, 1, 2, 48, 40, softplus=False)
        a = np.abs(np.random.default_rng(3).normal(size=(300, 2, 2))) * 0.01
        a[::9] = 12.0
        a[2::7] = 0.0
        c.at["a"].copy_(torch.from_numpy(a))
        check(c)
        c.ctx.close()


def test_digits_of_a_storage(hts):  # noqa: F811
    """Sums over thousands of steps, in which whatever has one sign in every step would add up."""
    c = Case(hts, "bf16", 512, 16, 2, 2, 128, 128, starts=0.01)
    check(c, "cuda")
    c.ctx.close()
