"""The losses over a vocabulary on sizes whose products run on the large tiles, compared with 64-bit products on the GPU: rings
that go round many times, K ranges with their join, dx and dw in one launch in either order, several passes over the rows.

Hidden states and head have a mean of their own, so that a part of a sum that is left out, or taken twice, shows: a token's
sum of p w, an id's sum of p x, are of the size of w and x, far above the bounds. The bounds are those of test_loss_gpu.py.
"""
import numpy as np
import pytest

from paper_2607_05895_amd import native

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _inputs(n, v, h, dtype, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(n, h, generator=g, device="cuda") + 0.7).to(dtype)
    w = ((torch.randn(v, h, generator=g, device="cuda") * 1.2 + 0.6) / h ** 0.5).to(dtype)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    t[torch.rand(n, generator=g, device="cuda") < 0.1] = -100
    return x, w, t


def _teacher(n, v, k, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    ids = torch.randint(0, v, (n, k), generator=g, device="cuda")
    ids[torch.rand(n, k, generator=g, device="cuda") < 0.1] = -1
    return ids, 5 - torch.cumsum(torch.rand(n, k, generator=g, device="cuda"), 1)


def _weights(kind, labels, n, v, temperature):
    """(q as n x v doubles, where targets are, sum of q log q, which tokens count) of the definition."""
    import torch
    q = torch.zeros(n, v, dtype=torch.float64, device="cuda")
    if kind == "xent":
        on = labels >= 0
        q[torch.nonzero(on)[:, 0], labels[on]] = 1.0
        return q, q > 0, torch.zeros(n, dtype=torch.float64, device="cuda"), on
    ids, lg = labels
    filled = ids >= 0
    on = filled.any(1)
    s = torch.where(filled, lg.double() / temperature, -torch.inf)
    s = torch.exp(s - torch.where(on, s.amax(1), 0.0)[:, None])
    s = s / torch.where(on, s.sum(1), 1.0)[:, None]
    ent = torch.where(s > 0, s * torch.log(torch.where(s > 0, s, 1.0)), 0.0).sum(1)
    at = torch.where(filled, ids, 0)
    q.scatter_add_(1, at, torch.where(filled, s, 0.0))
    hit = torch.zeros(n, v, dtype=torch.float64, device="cuda").scatter_add_(1, at, filled.double()) > 0
    return q, hit, ent, on


def _compare(kind, got, x, w, labels, temperature=1.0):
    import torch
    n, h = x.shape
    v = w.shape[0]
    bf16 = x.dtype == torch.bfloat16
    inv_t = 1.0 / temperature
    q, hit, ent, on = _weights(kind, labels, n, v, temperature)
    x64, w64 = x.double() * on[:, None], w.double()
    dr = (x64.abs() @ w64.abs().T).amax(1) * (2 * (h + 8) * U * inv_t)
    z = (x64 @ w64.T) * inv_t
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    token = torch.where(on, ent + (q * (lse[:, None] - z)).sum(1), 0.0)
    far = torch.where(hit, (top[:, None] - z).abs(), 0.0).amax(1)
    tol = 2 * dr + 2.0 ** -17 + 2.0 ** -18 * (token.abs() + far + lse - top)
    assert bool(((got["token_loss"].double() - token).abs() <= torch.where(on, tol, 0.0)).all())
    count = on.sum().double()
    assert abs(float(got["loss"]) - float(token.sum() / count)) <= 2.0 ** -15 * float(token.abs().sum() / count)
    p = torch.exp(z - lse[:, None])
    del z
    g = (on.double() * (inv_t / count))[:, None]
    dz = g * (p - q)
    del q
    eps = (2 * dr + 2.0 ** -16)[:, None] + torch.where(hit, 0.0, 2.0 ** -11 * float(np.log(2)) if bf16 else 0.0)
    half = 2.0 ** -8 if bf16 else U
    ddz = g * (p * eps + torch.where(hit, (p + 1.0) * 2.0 ** -18, 2.0 ** -60))
    del p, eps, hit
    ddz = ddz + half * (dz.abs() + ddz)
    worst = []
    for name, acc, a, b, e in (("dx", v, dz, w64, ddz), ("dw", n, dz.T.contiguous(), x64, ddz.T.contiguous())):
        if name not in got:
            continue
        want = a @ b
        tol = e @ b.abs() + 2 * (acc + 8) * U * (a.abs() @ b.abs())
        tol = tol + half * (want.abs() + tol)
        err = (got[name].double() - want).abs()
        worst.append(f"{name} {float((err / tol.clamp(min=1e-37)).max()):.2f}")
        assert bool((err <= tol.clamp(min=1e-37)).all()), (name, worst)
        # the bound tells a sum without a twentieth of its terms apart (except over 2^20 ids: an eighth by fp32 sums alone)
        assert acc > 1 << 16 or float(tol.mean()) < 0.05 * float((a.abs() @ b.abs()).mean())
        # fp32, as a whole: logits near 0.42 sqrt(h) < 20, summed in 3 h / 16 < 400 steps that round by 2^-23 with either sign:
        # off by sqrt(400) 20 2^-23 < 2^-14, and p, dx and dw by as much of themselves (a lost second part: 2^-11)
        assert bf16 or float((got[name].double() - want).norm() / want.norm()) < 2.0 ** -14
    print("  worst share of the bound:", ", ".join(worst), flush=True)


def _run(kind, x, w, labels, outs, temperature, chunk_rows):
    import torch
    nan = float("nan")
    got = dict(loss=torch.full((), nan, device="cuda"), token_loss=torch.full((x.shape[0],), nan, device="cuda"))
    for name, t in (("dx", x), ("dw", w)):
        if name in outs:
            got[name] = torch.full_like(t, nan)
    if kind == "xent":
        native.linear_xent_t(x, w, labels, **got, chunk_rows=chunk_rows)
    else:
        native.linear_distill_t(x, w, *labels, **got, temperature=temperature, chunk_rows=chunk_rows)
    torch.cuda.synchronize()
    return got


SIZES = [  # n, v, h, rows of a pass, dtype
    (2048, 20000, 1032, 0, "bfloat16"), (2500, 20000, 1032, 1024, "bfloat16"), (777, 32003, 1001, 0, "bfloat16"),
    (777, 32003, 1001, 512, "bfloat16"), (6000, 4000, 520, 0, "bfloat16"), (300, 20003, 2048, 0, "bfloat16"),
    (1024, 20000, 768, 0, "float32"), (1300, 20000, 768, 512, "float32"), (1500, 5003, 2047, 0, "float32"),
]


@pytest.mark.parametrize("kind", ["xent", "distill"])
@pytest.mark.parametrize("n,v,h,chunk,dtype", SIZES)
def test_large_tiles_match_64_bits(n, v, h, chunk, dtype, kind):
    import torch
    x, w, t = _inputs(n, v, h, getattr(torch, dtype), n + v)
    labels, temperature = (t, 1.0) if kind == "xent" else (_teacher(n, v, 20, n), 1.7)
    for outs in (("dx", "dw"), ("dx",), ("dw",)):  # (each has tiles and K ranges of its own)
        print(kind, n, v, h, chunk, dtype, outs, flush=True)
        _compare(kind, _run(kind, x, w, labels, outs, temperature, chunk), x, w, labels, temperature)


def test_one_pass_beyond_2_gib_of_logits():
    """1100 tokens on 2^20 ids: 16-bit logits of 2.7 GB in one pass, whose places pass 32 bits."""
    import torch
    n, v, h = 1100, 1 << 20, 256
    x, w, t = _inputs(n, v, h, torch.bfloat16, 7)
    print(n, v, h, flush=True)
    _compare("xent", _run("xent", x, w, t, ("dx", "dw"), 1.0, 0), x, w, t)


@pytest.mark.parametrize("n,v,h", [(18000, 1 << 20, 64), (9000, 128256, 1032)])
def test_a_loss_alone_over_many_rows(n, v, h):
    """More rows than one pass with gradients takes (the first: than one without, too): tokens of every pass, and of their ends,
    against 64 bits; the same tokens alone; the reduced loss against their sum."""
    import torch
    x, w, t = _inputs(n, v, h, torch.bfloat16, 9)
    print(n, v, h, flush=True)
    got = _run("xent", x, w, t, (), 1.0, 0)
    rows = torch.unique(torch.cat([torch.arange(0, n, n // 90, device="cuda"), torch.arange(n - 8, n, device="cuda")] +
                                  [torch.arange(c - 3, c + 3, device="cuda") for c in (1024, 8192, 16384, 17152) if c + 3 < n]))
    xr, tr = x[rows], t[rows]
    z = xr.double() @ w.double().T
    lse = torch.logsumexp(z, 1)
    on = tr >= 0
    want = torch.where(on, lse - z.gather(1, tr.clamp(min=0)[:, None])[:, 0], 0.0)
    dr = (xr.double().abs() @ w.double().abs().T).amax(1) * (2 * (h + 8) * U)
    tol = 2 * dr + 2.0 ** -17 + 2.0 ** -18 * (want.abs() + (z.amax(1) - z.amin(1)) + float(np.log(v)))
    assert bool(((got["token_loss"][rows].double() - want).abs() <= torch.where(on, tol, 0.0)).all())
    sums = got["token_loss"].double().sum() / (t >= 0).sum()
    assert bool(torch.isfinite(got["token_loss"]).all()) and abs(float(got["loss"]) - float(sums)) <= 2.0 ** -20 * float(sums)
