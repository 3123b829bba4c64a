"""The recurrence in 64 bits, row by row, with bounds on what 32 bits may lose; packed sequences to try.

u = 2^-24 is half a step of float32.  A gate's a and 1 - a come from e = exp(-|gate|): v_exp_f32 2 u and its correction 1 u; 1 + e
1 u and e's share 1.5 u; v_rcp_f32 2 u: a within 4.5 u, e a within 8.5 u.  So a term a h + (1 - a) x is within 10 u of each part before
it is added, and 1 u after it; where rows are joined in pieces, a product of decays is rounded once a row as well, and once or
twice more for every 16.  The error of h_t is at most E_t = |a_t| E_(t-1) + 13 u M_t, with M_t = |a_t| M_(t-1) + |u_t|; the same for
l, from the end.  dgate is a product of five factors of which a and 1 - a have 8.5 u each and four roundings: 24 u."""
import numpy as np
import torch

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def terms(x, gate, mode):
    if mode == "given":
        return gate, x, np.ones_like(gate)
    with np.errstate(over="ignore"):
        e = np.exp(-np.abs(gate))
    big, small = 1 / (1 + e), e / (1 + e)
    a, rest = np.where(gate >= 0, big, small), np.where(gate >= 0, small, big)
    return a, rest * x, rest


def forward(x, gate, starts, initial, mode):
    """y, last, and for each row the state before it; then the same of the errors."""
    n, d = x.shape
    s = len(starts) - 1
    a, u, _ = terms(x, gate, mode)
    y, last, before = np.zeros((n, d)), np.zeros((s, d)), np.zeros((n, d))
    ey, elast, ebefore = np.zeros((n, d)), np.zeros((s, d)), np.zeros((n, d))
    for q in range(s):
        h = np.zeros(d) if initial is None else initial[q].copy()
        m, e = np.abs(h), np.zeros(d)
        for t in range(starts[q], starts[q + 1]):
            before[t], ebefore[t] = h, e
            h = a[t] * h + u[t]
            m = np.abs(a[t]) * m + np.abs(u[t])
            e = np.abs(a[t]) * e + 13 * U * m
            y[t], ey[t] = h, e
        last[q], elast[q] = h, e
    return y, last, before, ey, elast, ebefore


def backward(x, gate, dy, dlast, starts, before, ebefore, mode):
    n, d = x.shape
    s = len(starts) - 1
    a, _, rest = terms(x, gate, mode)
    dx, dg, di = np.zeros((n, d)), np.zeros((n, d)), np.zeros((s, d))
    ex, eg, ei = np.zeros((n, d)), np.zeros((n, d)), np.zeros((s, d))
    for q in range(s):
        c = np.zeros(d) if dlast is None else dlast[q].copy()
        mc, ec = np.abs(c), np.zeros(d)
        for t in range(starts[q + 1] - 1, starts[q] - 1, -1):
            l, ml = dy[t] + c, np.abs(dy[t]) + mc
            el = ec + 13 * U * ml
            dx[t], ex[t] = rest[t] * l, np.abs(rest[t]) * (el + 10 * U * ml)
            if mode == "given":
                dg[t] = l * before[t]
                eg[t] = el * np.abs(before[t]) + ml * (ebefore[t] + 2 * U * np.abs(before[t]))
            else:
                f, size = a[t] * rest[t], np.abs(before[t]) + np.abs(x[t])
                dg[t] = l * (before[t] - x[t]) * f
                eg[t] = f * (el * size + ml * ebefore[t] + 24 * U * ml * size)
            c, mc, ec = a[t] * l, np.abs(a[t]) * ml, np.abs(a[t]) * el
        di[q], ei[q] = c, ec
    return dx, dg, di, ex, eg, ei


def close(got, want, err, name):
    """`got` within the error `err` of `want`, and half a step of its type (the smallest steps of half precision are 2^-24)."""
    assert tuple(got.shape) == want.shape, name
    dt = got.dtype
    g = got.double().cpu().numpy()
    half = 0.0 if dt == torch.float32 else torch.finfo(dt).eps / 2
    floor = {torch.float32: 1e-36, torch.bfloat16: 1e-36, torch.float16: 2.0 ** -25}[dt]
    bound = err + half * (np.abs(want) + err) + floor
    bad = ~(np.abs(g - want) <= bound)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: {g[bad][0]} for {want[bad][0]} within {bound[bad][0]}"


def lengths(kind, seed=0):
    rng = np.random.default_rng(seed)
    return {
        "none": [], "empty": [0], "one": [1], "empties": [0, 0, 5, 0, 0, 0, 1, 0], "ones": [1] * 70, "sixteen": [16], "seventeen": [17],
        "around": [15, 1, 16, 48, 1, 31, 33, 2, 0, 63, 65], "long": [1500], "two": [700, 801],
        "many": rng.integers(0, 40, 60).tolist(), "mixed": [900, 0, 1, 300, 2, 0, 0, 77, 256, 255, 257],
        "emptyrun": [20] + [0] * 300 + [20],
    }[kind]


def problem(kind, d, dtype, seed, lead=0, behind=0, pad=0, big=1.5):
    """x, gate, dy (rows `pad` further apart than they are long), starts, and a generator."""
    L = lengths(kind, seed)
    starts = np.concatenate([[0], np.cumsum(L)]).astype(np.int64) + lead
    n = int(starts[-1]) + behind
    gen = torch.Generator().manual_seed(seed)

    def rows(f):
        a = f(torch.randn(n, d + pad, generator=gen)).to(DT[dtype]).cuda()
        return a[:, :d]

    return n, starts, gen, rows


def to64(a):
    return a.double().cpu().numpy()
