"""The gated MLP in float64, with bounds on what the kernels' roundings can do to each output.

Bounds are propagated to first order through the formulas: `h` is half a step of the storage type (every value that is
stored or multiplied in it), `gamma(K)` the error of an fp32 sum of K products relative to the sum of their magnitudes
(K roundings of 2^-24), `act` the error of the activation's arithmetic.  |act'| <= 1.13 and |act''| <= 0.8 for SiLU and both GELUs.
A factor of 1.05 stands for the second-order terms (h is 2^-8 at most)."""

import math

import torch

U32 = 2.0 ** -24


def act_of(name, g):
    """act(g), act'(g)."""
    if name == "swiglu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if name == "geglu_erf":
        c = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def gamma(k):
    return (k + 2) * U32


def reference(name, w, x, dy=None):
    """{output: (value, bound)} in float64; gradients too where dy is given.  w, x, dy: tensors of the storage type."""
    dt = x.dtype
    h = torch.finfo(dt).eps / 2
    lost = 4e-6 if dt == torch.bfloat16 else 6e-7            # activation: exp2, rcp and the erf fit / fp32 library functions
    store = h if dt == torch.bfloat16 else 0.0               # intermediates kept in the storage type
    x, wgu, wd = x.double(), w["gate_up_w"].double(), w["down_w"].double()
    F, D, T = wd.shape[1], x.shape[1], x.shape[0]
    bgu = w["gate_up_b"].double() if "gate_up_b" in w else torch.zeros(2 * F, dtype=torch.float64, device=x.device)
    bd = w["down_b"].double() if "down_b" in w else torch.zeros(D, dtype=torch.float64, device=x.device)
    gu = x @ wgu.t() + bgu
    e = gamma(D) * (x.abs() @ wgu.abs().t() + bgu.abs())
    g, u, eg, eu = gu[:, :F], gu[:, F:], e[:, :F], e[:, F:]
    a, d = act_of(name, g)
    hid = a * u
    ea = 1.13 * eg + lost * (1 + g.abs())
    eh = ea * u.abs() + a.abs() * eu + store * hid.abs()
    y = hid @ wd.t() + bd
    out = {"y": (y, 1.05 * (eh @ wd.abs().t() + gamma(F) * (hid.abs() @ wd.abs().t() + bd.abs())) + h * y.abs())}
    if dy is None:
        return out
    dy = dy.double()
    ea, ed = 1.13 * eg + lost * (1 + g.abs()), 0.8 * eg + lost * (1 + g.abs())
    dh = dy @ wd
    edh = gamma(D) * (dy.abs() @ wd.abs())
    du, dg, hid = dh * a, dh * u * d, a * u
    kept = 2.0 ** -12 if dt == torch.bfloat16 else 0.0       # act(G) and U act'(G), saved with 12 bits of mantissa
    edu = edh * a.abs() + dh.abs() * (ea + kept * a.abs()) + store * du.abs()
    edg = edh * (u * d).abs() + dh.abs() * (eu * d.abs() + u.abs() * ed + kept * (u * d).abs()) + store * dg.abs()
    eh = ea * u.abs() + a.abs() * eu + store * hid.abs()
    dgu, edgu = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)

    def product(p, q, ep, k):
        v = p @ q
        return v, 1.05 * (ep @ q.abs() + gamma(k) * (p.abs() @ q.abs())) + h * v.abs()

    out["dx"] = product(dgu, wgu, edgu, 2 * F)
    out["gate_up_w"] = product(dgu.t(), x, edgu.t(), T)
    v = dy.t() @ hid
    out["down_w"] = (v, 1.05 * (dy.abs().t() @ eh + gamma(T) * (dy.abs().t() @ hid.abs())) + h * v.abs())
    if "gate_up_b" in w:
        v = dgu.sum(0)
        out["gate_up_b"] = (v, 1.05 * (edgu.sum(0) + gamma(T) * dgu.abs().sum(0)) + h * v.abs())
        v = dy.sum(0)
        out["down_b"] = (v, 1.05 * gamma(T) * dy.abs().sum(0) + h * v.abs())
    return out


# Roundings to bf16 on the way to each output, itself among them.  Each is off by h / sqrt(3) at most in the mean square
# (uniform within half a step of the smallest value of its binade), they are independent and products keep them relative, so
# the difference has 1.2 sqrt(n / 3) h of the output's norm: 1.2 for sums of unlike terms.
ROUNDINGS = {"y": 2, "dx": 2, "gate_up_w": 2, "down_w": 2, "gate_up_b": 2, "down_b": 1}


def check(got, want, norms=True):
    for n, (v, bound) in want.items():
        diff = (got[n].double() - v).abs()
        assert got[n].shape == v.shape, n
        assert bool((diff <= bound).all()), (n, float((diff - bound).max()), float(diff.max()))
        if norms and got[n].dtype == torch.bfloat16 and v.numel() >= 64:
            limit = 1.2 * math.sqrt(ROUNDINGS[n] / 3) * 2.0 ** -8
            rel = float(diff.norm() / v.norm())
            assert rel <= limit, (n, rel, limit)


def make(T, D, F, dtype, bias, seed, device="cuda:0", std=None):
    g = torch.Generator(device=device).manual_seed(seed)

    def randn(*s, std=1.0):
        return (torch.randn(s, generator=g, device=device, dtype=torch.float32) * std).to(dtype)

    std = D ** -0.5 if std is None else std
    w = {"gate_up_w": randn(2 * F, D, std=std), "down_w": randn(D, F, std=F ** -0.5)}
    if bias:
        w["gate_up_b"], w["down_b"] = randn(2 * F, std=0.5), randn(D, std=0.5)
    return w, randn(T, D), randn(T, D)
