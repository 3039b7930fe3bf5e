"""GPU parity of the losses over a vocabulary (mfsdp_linear_xent, mfsdp_linear_distill) against the fp64 oracle.

Bounds, from the operator's arithmetic (u = 2^-24, half a step of fp32; 2u where a matrix instruction may truncate):
* a logit is a sum of h products: |dz| <= 2 (h + 8) u (|x| |w|^T) / T =: d; each value of an fp32 operand is
  off by at most u (two fp16 parts), their products by 3 u, which the 16 u cover;
* a probability is off by 2 max_v d of its row and by 2^-16 (up to 2^8 roundings of its row's sum, exp2, factors); with
  bf16 inputs, for ids that are no targets, by the 16-bit logit's 2^-11 ln 2 as well;
* dz is then rounded (bf16: 2^-8 of it; fp32: u), and dx, dw are sums of v, n products of it, rounded once more.
"""
import numpy as np
import pytest

import synth
from oracle import losses as OL
from paper_2607_05895_amd import native
from tests.helpers import from_dev, to_dev

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = synth.F32, synth.BF16


def _say(*a):
    print(*a, flush=True)


def _inputs(rng, n, v, h, dtype, x_scale=1.0, w_scale=None):
    """x, w as stored, and as float64."""
    x = (rng.standard_normal((n, h)) * x_scale).astype(np.float32)
    w = (rng.standard_normal((v, h)) * (w_scale or 1.2 / np.sqrt(h))).astype(np.float32)
    if dtype == BF16:
        x, w = synth.f32_to_bf16_bits(x), synth.f32_to_bf16_bits(w)
        return x, w, synth.bf16_bits_to_f32(x).astype(np.float64), synth.bf16_bits_to_f32(w).astype(np.float64)
    return x, w, x.astype(np.float64), w.astype(np.float64)


def _labels(rng, n, v, ignored=0.2):
    t = rng.integers(0, v, n)
    t[rng.random(n) < ignored] = -100
    return t


def _teacher(rng, n, v, k, empty=0.1):
    ids = rng.integers(0, v, (n, k))
    lg = -np.cumsum(rng.random((n, k)), 1) + 5
    ids[rng.random((n, k)) < empty] = -1
    if n > 3:
        ids[1] = -1
    if k > 2:
        ids[0, 1] = ids[0, 0]
    return ids, lg.astype(np.float32)


def _call(kind, x, w, dtype, labels, outs=("loss", "token_loss", "lse", "dx", "dw"), fill=float("nan"), **kw):
    """The outputs of one call, as float64; every buffer is filled with `fill` first."""
    import torch
    xd, wd = to_dev(x, dtype), to_dev(w, dtype)
    n, v = x.shape[0], w.shape[0]
    f = lambda *s: torch.full(s, fill, dtype=torch.float32, device="cuda")  # noqa: E731
    bufs = dict(loss=f(1), token_loss=f(n), lse=f(n), dx=torch.full_like(xd, fill), dw=torch.full_like(wd, fill))
    given = {o: bufs[o] for o in outs}
    if kw.get("token_weight") is not None:
        kw["token_weight"] = to_dev(np.asarray(kw["token_weight"], np.float32), F32)
    if kind == "xent":
        native.linear_xent_t(xd, wd, torch.from_numpy(labels).cuda(), **given, **kw)
    else:
        ids, lg, lgt = labels
        native.linear_distill_t(xd, wd, torch.from_numpy(ids).cuda(), to_dev(lg, lgt), **given, **kw)
    torch.cuda.synchronize()
    return {o: from_dev(given[o]) for o in outs}


def _check(got, ref, x64, w64, dtype, q_cols, inv_t=1.0, z_loss=0.0, what=""):
    """got against the oracle's ref within the module's bounds. q_cols: n x v, where the targets are."""
    n, h = x64.shape
    v = w64.shape[0]
    on = ref.token_loss != 0
    x64 = np.where(on[:, None], x64, 0.0)
    d = 2 * (h + 8) * U * (np.abs(x64) @ np.abs(w64).T) * inv_t
    dr = d.max(1) if n else np.zeros(0)
    top = ref.z.max(1)
    lse = top + np.log(np.exp(ref.z - top[:, None]).sum(1))
    size = np.abs(ref.token_loss) + np.where(q_cols, np.abs(top[:, None] - ref.z), 0.0).max(1) + (lse - top) + z_loss * lse ** 2
    tol_l = (1 + 2 * z_loss * np.abs(lse)) * (2 * dr + 2.0 ** -17) + 2.0 ** -18 * size
    worst = {}

    def within(name, err, tol):
        tol = np.maximum(tol, 1e-37)
        worst[name] = float((err / tol).max()) if err.size else 0.0
        assert np.isfinite(err).all() and (err <= tol).all(), (what, name, worst[name])

    if "token_loss" in got:
        within("token_loss", np.abs(got["token_loss"] - ref.token_loss), np.where(on, tol_l, 0.0))
    if "lse" in got:
        within("lse", np.abs(got["lse"] - ref.lse), np.where(on, dr + 2.0 ** -17 + 2.0 ** -22 * np.abs(lse), 0.0))
    if "dx" in got or "dw" in got:
        p = np.exp(ref.z - lse[:, None])
        g = np.abs(ref.g)[:, None] * inv_t
        eps = (2 * dr + 2.0 ** -16)[:, None] + (np.where(q_cols, 0.0, 2.0 ** -11 * np.log(2)) if dtype == BF16 else 0.0)
        half = 2.0 ** -8 if dtype == BF16 else U
        pz = p * (1 + 2 * z_loss * np.abs(lse))[:, None]
        # (2^-60: codes end 2^-64 below the largest logit of their 64 columns; p - q is formed from terms up to 1)
        ddz = g * (pz * eps + np.where(q_cols, (pz + 1.0) * 2.0 ** -18, 2.0 ** -60))
        ddz = ddz + half * (np.abs(ref.dz) + ddz)
        for name, acc, out, e in (("dx", v, ref.dx, (ddz @ np.abs(w64), np.abs(ref.dz) @ np.abs(w64))),
                                  ("dw", n, ref.dw, (ddz.T @ np.abs(x64), np.abs(ref.dz).T @ np.abs(x64)))):
            if name in got:
                tol = e[0] + 2 * (acc + 8) * U * e[1]
                within(name, np.abs(got[name] - out), tol + half * (np.abs(out) + tol))
    _say(f"  {what}: worst share of the bound: " + ", ".join(f"{a} {b:.2f}" for a, b in worst.items()))


class _Ref:
    """The oracle's result with the factor g of each token's gradient."""

    def __init__(self, r, on, weight, reduction, scale):
        self.__dict__.update(r._asdict())
        a = np.where(on, 1.0 if weight is None else weight, 0.0)
        den = a.sum() if reduction == "mean" else 1.0
        self.g = np.zeros(len(a)) if den == 0 else scale * a / den
        # (a token that counts with a loss of exactly 0 is told apart from one that does not count)
        self.token_loss = np.where(on & (self.token_loss == 0), 1e-300, self.token_loss)


def _check_loss(got, ref, tol_rel=2.0 ** -15):
    size = max(abs(ref.loss), float((np.abs(ref.g) * np.abs(ref.token_loss)).sum()))
    assert abs(float(got["loss"][0]) - ref.loss) <= tol_rel * size + 1e-30, (float(got["loss"][0]), ref.loss)


SHAPES = [(1, 1, 1), (1, 300, 64), (3, 64, 8), (7, 1003, 97), (64, 1000, 64), (255, 257, 33), (256, 256, 32),
          (257, 513, 257), (130, 4100, 200), (600, 2049, 520),
          # few tokens on many ids: w is read as it lies
          (1, 4096, 64), (31, 4100, 72), (32, 4111, 264), (33, 5003, 200), (64, 4097, 8), (100, 9001, 136), (128, 4351, 1000),
          (17, 4500, 129)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v,h", SHAPES)
def test_xent_matches_the_oracle(n, v, h, dtype):
    rng = np.random.default_rng(n * 7 + v * 3 + h)
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype)
    t = _labels(rng, n, v)
    weight = rng.uniform(0.1, 2.0, n).astype(np.float32) if n % 2 else None
    red, scale, zl = ("mean", 1.0, 0.0) if h % 2 else ("sum", 0.37, 1e-3)
    _say(f"xent {n} x {v} x {h} {dtype}")
    got = _call("xent", x, w, dtype, t.astype(np.int32 if n % 2 else np.int64), reduction=red, scale=scale, z_loss=zl,
                token_weight=weight)
    r = OL.linear_xent(x64, w64, t, reduction=red, scale=scale, weight=weight, z_loss=zl)
    ref = _Ref(r, t >= 0, weight, red, scale)
    q = np.zeros((n, v), bool)
    q[np.nonzero(t >= 0)[0], t[t >= 0]] = True
    _check(got, ref, x64, w64, dtype, q, z_loss=zl, what=f"xent {n}x{v}x{h} {dtype}")
    _check_loss(got, ref)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v,h,k", [(1, 40, 16, 1), (5, 70, 24, 3), (33, 1003, 96, 5), (130, 600, 64, 64),
                                     (257, 2100, 136, 65), (40, 300, 72, 256), (20, 4500, 80, 7),
                                     (1, 4500, 72, 3), (70, 4111, 104, 33), (128, 5000, 320, 4)])
def test_distill_matches_the_oracle(n, v, h, k, dtype):
    rng = np.random.default_rng(n + v + h + k)
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype)
    ids, lg = _teacher(rng, n, v, k, empty=0.0 if n == 1 else 0.1)
    lgt = BF16 if k % 2 else F32
    lgs = synth.f32_to_bf16_bits(lg) if lgt == BF16 else lg
    lg64 = synth.bf16_bits_to_f32(lgs).astype(np.float64) if lgt == BF16 else lg.astype(np.float64)
    temp, red, scale = (2.0, "mean", 4.0) if n % 2 else (0.7, "sum", 1.0)
    weight = rng.uniform(0.1, 2.0, n).astype(np.float32) if n == 33 else None
    _say(f"distill {n} x {v} x {h}, {k} {dtype}")
    got = _call("distill", x, w, dtype, (ids.astype(np.int32 if n % 2 else np.int64), lgs, lgt), temperature=temp,
                reduction=red, scale=scale, token_weight=weight)
    r = OL.linear_distill(x64, w64, ids, lg64, temperature=temp, reduction=red, scale=scale, weight=weight)
    on = (ids >= 0).any(1)
    ref = _Ref(r, on, weight, red, scale)
    q = np.zeros((n, v), bool)
    rows = np.repeat(np.arange(n), k).reshape(n, k)
    q[rows[ids >= 0], ids[ids >= 0]] = True
    _check(got, ref, x64, w64, dtype, q, inv_t=1 / temp, what=f"distill {n}x{v}x{h},{k} {dtype}")
    _check_loss(got, ref)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v,h,chunk", [(9, 500, 4000, 0), (200, 700, 2100, 0), (300, 130, 3001, 256), (1, 60, 4096, 0)])
def test_long_rows_of_few_tiles(n, v, h, chunk, dtype):
    """The logits' products are cut into K ranges."""
    rng = np.random.default_rng(29)
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype)
    t = _labels(rng, n, v, 0.2 if n > 1 else 0.0)
    _say(n, v, h, chunk, dtype)
    ref = _Ref(OL.linear_xent(x64, w64, t), t >= 0, None, "mean", 1.0)
    q = np.zeros((n, v), bool)
    q[np.nonzero(t >= 0)[0], t[t >= 0]] = True
    got = _call("xent", x, w, dtype, t, chunk_rows=chunk)
    _check(got, ref, x64, w64, dtype, q, what=f"long rows {n}x{v}x{h} {dtype}")
    _check_loss(got, ref)
    only = _call("xent", x, w, dtype, t, outs=("loss", "token_loss", "lse"), chunk_rows=chunk)
    for o in only:
        np.testing.assert_array_equal(only[o], got[o])
    ids, lg = _teacher(rng, n, v, 20, empty=0.1 if n > 1 else 0.0)
    got = _call("distill", x, w, dtype, (ids, lg, F32), temperature=2.0)
    ref = _Ref(OL.linear_distill(x64, w64, ids, lg, temperature=2.0), (ids >= 0).any(1), None, "mean", 1.0)
    q[:] = False
    q[np.repeat(np.arange(n), 20).reshape(n, 20)[ids >= 0], ids[ids >= 0]] = True
    _check(got, ref, x64, w64, dtype, q, inv_t=0.5, what=f"distill long rows {n}x{v}x{h} {dtype}")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_chunks_of_rows_add_up(dtype):
    """Three passes over the rows, the last one ragged: dw is summed in fp32 across them."""
    rng = np.random.default_rng(21)
    n, v, h = 600, 700, 72
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype)
    t = _labels(rng, n, v)
    _say(f"chunks {dtype}")
    got = _call("xent", x, w, dtype, t, chunk_rows=200)
    ref = _Ref(OL.linear_xent(x64, w64, t), t >= 0, None, "mean", 1.0)
    q = np.zeros((n, v), bool)
    q[np.nonzero(t >= 0)[0], t[t >= 0]] = True
    _check(got, ref, x64, w64, dtype, q, what=f"chunks {dtype}")
    _check_loss(got, ref)
    ids, lg = _teacher(rng, n, v, 6)
    got = _call("distill", x, w, dtype, (ids, lg, F32), chunk_rows=1, temperature=1.5)
    ref = _Ref(OL.linear_distill(x64, w64, ids, lg, temperature=1.5), (ids >= 0).any(1), None, "mean", 1.0)
    q[:] = False
    q[np.repeat(np.arange(n), 6).reshape(n, 6)[ids >= 0], ids[ids >= 0]] = True
    _check(got, ref, x64, w64, dtype, q, inv_t=1 / 1.5, what=f"distill chunks {dtype}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("outs", [("loss",), ("token_loss",), ("lse",), ("dx",), ("dw",), ("loss", "dx"), ("lse", "dw")])
def test_each_output_alone_is_the_same(outs, dtype):
    rng = np.random.default_rng(22)
    x, w, _, _ = _inputs(rng, 70, 333, 40, dtype)
    t = _labels(rng, 70, 333)
    _say(outs, dtype)
    every = _call("xent", x, w, dtype, t)
    some = _call("xent", x, w, dtype, t, outs=outs)
    for o in outs:
        np.testing.assert_array_equal(some[o], every[o])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["xent", "distill"])
def test_tokens_that_do_not_count_may_hold_anything(kind, dtype):
    rng = np.random.default_rng(23)
    n, v, h = 40, 300, 48
    x, w, _, _ = _inputs(rng, n, v, h, dtype)
    t = _labels(rng, n, v, 0.5)
    ids, lg = _teacher(rng, n, v, 4)
    ids[t < 0] = -1
    labels = t if kind == "xent" else (ids, lg, F32)
    off = t < 0 if kind == "xent" else (ids < 0).all(1)
    _say(kind, dtype)
    clean = _call(kind, x, w, dtype, labels)
    bad = x.copy()
    junk = np.array([np.nan, np.inf, -np.inf, 3e38], np.float32)
    bad[off] = np.resize(synth.f32_to_bf16_bits(junk) if dtype == BF16 else junk, bad[off].shape)
    if kind == "distill":
        lg = lg.copy()
        lg[ids < 0] = np.nan
        labels = (ids, lg, F32)
    got = _call(kind, bad, w, dtype, labels)
    for o in got:
        np.testing.assert_array_equal(got[o], clean[o])
    assert not got["dx"][off].any() and not got["token_loss"][off].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["xent", "distill"])
@pytest.mark.parametrize("reduction", ["mean", "sum"])
def test_no_token_counts(kind, reduction, dtype):
    rng = np.random.default_rng(24)
    x, w, _, _ = _inputs(rng, 5, 70, 24, dtype)
    _say(kind, reduction, dtype)
    labels = np.full(5, -100) if kind == "xent" else (np.full((5, 3), -1), np.zeros((5, 3), np.float32), F32)
    got = _call(kind, x, w, dtype, labels, reduction=reduction)
    for o in got:
        assert not got[o].any(), o
    labels = np.zeros(0, np.int64) if kind == "xent" else (np.zeros((0, 3), np.int64), np.zeros((0, 3), np.float32), F32)
    got = _call(kind, x[:0], w, dtype, labels, reduction=reduction)
    assert got["loss"][0] == 0 and not got["dw"].any()


def test_a_teacher_of_minus_infinity_teaches_nothing():
    rng = np.random.default_rng(25)
    x, w, x64, w64 = _inputs(rng, 3, 50, 16, F32)
    ids = rng.integers(0, 50, (3, 3))
    lg = rng.standard_normal((3, 3)).astype(np.float32)
    lg[1] = -np.inf
    lg[2, 0] = -np.inf
    got = _call("distill", x, w, F32, (ids, lg, F32))
    with np.errstate(invalid="ignore"):
        r = OL.linear_distill(x64, w64, ids, lg)
    np.testing.assert_allclose(got["token_loss"], r.token_loss, rtol=1e-5, atol=1e-6)
    assert not got["dx"][1].any()
    np.testing.assert_allclose(got["dw"], r.dw, rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("kind", ["xent", "distill"])
def test_an_id_outside_the_vocabulary_gives_nan(kind):
    rng = np.random.default_rng(26)
    x, w, _, _ = _inputs(rng, 4, 70, 24, BF16)
    for bad in (70, 1 << 40, -3 if kind == "xent" else 1 << 31):
        t = np.array([3, bad, 5, 6], np.int64)
        got = _call(kind, x, w, BF16, t if kind == "xent" else (t[:, None], np.zeros((4, 1), np.float32), F32))
        assert np.isnan(got["token_loss"][1]) and np.isfinite(got["token_loss"][[0, 2, 3]]).all()
        assert np.isnan(got["loss"][0]) and np.isnan(got["dw"]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["xent", "distill"])
@pytest.mark.parametrize("n,v,h", [(40, 300, 48), (300, 700, 72), (40, 4500, 72)])
def test_a_token_does_not_take_digits_from_another(n, v, h, kind, dtype):
    """Hidden states of 1e20 in a token of weight 0, weights from 1e-12 to 1e12: every other token, and dw, within the same bounds."""
    rng = np.random.default_rng(28)
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype)
    odd = 3
    far = np.full(h, 1e20, np.float32)
    x[odd] = synth.f32_to_bf16_bits(far) if dtype == BF16 else far
    x64[odd] = 0.0  # (as the oracle sees it: what follows leaves this token out)
    weight = (10.0 ** rng.uniform(-12, 12, n)).astype(np.float32)
    weight[odd] = 0.0
    t = _labels(rng, n, v)
    t[odd] = 5
    ids, lg = _teacher(rng, n, v, 4)
    labels = t if kind == "xent" else (ids, lg, F32)
    _say(kind, n, v, h, dtype)
    got = _call(kind, x, w, dtype, labels, reduction="sum", token_weight=weight)
    if kind == "xent":
        r, on = OL.linear_xent(x64, w64, t, reduction="sum", weight=weight), t >= 0
        cols = [(i, [t[i]]) for i in range(n) if on[i]]
    else:
        r, on = OL.linear_distill(x64, w64, ids, lg.astype(np.float64), reduction="sum", weight=weight), (ids >= 0).any(1)
        cols = [(i, ids[i][ids[i] >= 0]) for i in range(n)]
    ref = _Ref(r, on, weight, "sum", 1.0)
    q = np.zeros((n, v), bool)
    for i, c in cols:
        q[i, c] = True
    for o in ("token_loss", "lse"):
        got[o][odd] = getattr(ref, o)[odd]
    _check(got, ref, x64, w64, dtype, q, what=f"{kind} {n}x{v}x{h} {dtype}")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_sure_token_keeps_its_digits(dtype):
    """Logits that are exact small integers: what is left of the loss and of the gradient at p near 1 is the softmax's
    own error. 300 ids 12 to 40 below the label: a loss of 1e-5 and less."""
    n, v, h = 6, 301, 32
    rng = np.random.default_rng(27)
    w = rng.integers(-1, 2, (v, h)).astype(np.float64)
    w[:, 0] = -1
    w[7] = 0
    w[7, 0] = 1
    x = np.zeros((n, h))
    x[:, 0] = np.arange(12, 12 + 2 * n, 2)
    x[:, 1:4] = rng.integers(-1, 2, (n, 3))
    bits = (lambda a: synth.f32_to_bf16_bits(a.astype(np.float32))) if dtype == BF16 else (lambda a: a.astype(np.float32))
    t = np.full(n, 7)
    got = _call("xent", bits(x), bits(w), dtype, t, reduction="sum")
    r = OL.linear_xent(x, w, t, reduction="sum")
    assert r.token_loss.max() < 1e-7
    # exp2 of a rounded argument up to 60: 60 * 2 u; the sum and the rest below 2^-18
    np.testing.assert_allclose(got["token_loss"], r.token_loss, rtol=2.0 ** -16, atol=0)
    # the label's row of dw is sum_r (p - 1) x_r, the others' sum_r p x_r
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -20
    scale = np.abs(r.dz).T @ np.abs(x)
    assert (np.abs(got["dw"] - r.dw) <= (2 * half + 2.0 ** -11) * scale + 1e-37).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [3e3, 1e30])
def test_large_logits_do_not_overflow(size, dtype):
    rng = np.random.default_rng(28)
    x, w, x64, w64 = _inputs(rng, 20, 200, 16, dtype, x_scale=size, w_scale=1.0)
    t = rng.integers(0, 200, 20)
    t[:10] = (x64 @ w64.T).argmax(1)[:10]
    got = _call("xent", x, w, dtype, t, reduction="sum")
    r = OL.linear_xent(x64, w64, t, reduction="sum")
    tol = 64 * U * (np.abs(x64) @ np.abs(w64).T).max(1)
    assert (np.abs(got["token_loss"] - r.token_loss) <= 2 * tol + 1e-6 * np.abs(r.token_loss)).all()
    assert np.isfinite(got["dx"]).all() and np.isfinite(got["dw"]).all()


@pytest.mark.parametrize("n,v,h", [(5, 400, 32), (300, 400, 32), (5, 4400, 32), (100, 4400, 32)])
def test_ids_of_minus_infinity_have_no_share(n, v, h):
    """128 ids and more in a row, whole softmax partials among them, whose logit overflows to -inf for every token."""
    rng = np.random.default_rng(30)
    x, w, x64, w64 = _inputs(rng, n, v, h, BF16)
    x[:, 0], x64[:, 0] = 0x4000, 2.0
    off = np.zeros(v, bool)
    off[60:200] = off[v - 3:] = True
    w[off] = 0
    w[off, 0] = 0xFF7F  # -3.4e38
    t = rng.choice(np.nonzero(~off)[0], n)
    _say(n, v, h)
    got = _call("xent", x, w, BF16, t)
    ref = _Ref(OL.linear_xent(x64, w64[~off], np.cumsum(~off)[t] - 1), np.ones(n, bool), None, "mean", 1.0)
    assert not got["dw"][off].any()
    got["dw"] = got["dw"][~off]
    q = np.zeros((n, int((~off).sum())), bool)
    q[np.arange(n), np.cumsum(~off)[t] - 1] = True
    _check(got, ref, x64, w64[~off], BF16, q, what=f"-inf {n}x{v}x{h}")
    _check_loss(got, ref)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v,h", [(3, 1 << 20, 8), (2, 300, 1 << 16)])
def test_longest_sides(n, v, h, dtype):
    rng = np.random.default_rng(33)
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype)
    t = np.array([v - 1, 0, v // 2])[:n]
    _say(n, v, h, dtype)
    got = _call("xent", x, w, dtype, t)
    ref = _Ref(OL.linear_xent(x64, w64, t), t >= 0, None, "mean", 1.0)
    q = np.zeros((n, v), bool)
    q[np.arange(n), t] = True
    _check(got, ref, x64, w64, dtype, q, what=f"{n}x{v}x{h} {dtype}")
    _check_loss(got, ref)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_tokens_than_one_pass_takes(dtype):
    """65536 rows and a ragged second pass."""
    rng = np.random.default_rng(31)
    n, v, h = 66001, 90, 24
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype)
    t = _labels(rng, n, v)
    _say(n, v, h, dtype)
    got = _call("xent", x, w, dtype, t, reduction="sum")
    ref = _Ref(OL.linear_xent(x64, w64, t, reduction="sum"), t >= 0, None, "sum", 1.0)
    q = np.zeros((n, v), bool)
    q[np.nonzero(t >= 0)[0], t[t >= 0]] = True
    _check(got, ref, x64, w64, dtype, q, what=f"{n}x{v}x{h} {dtype}")
    _check_loss(got, ref)


def test_equal_logits():
    """Every logit equal (a head of equal rows): loss log v, whatever the size of the logits."""
    import torch
    w = torch.ones(777, 64, device="cuda")
    x = torch.tensor([0.0, 1.0, -50.0, 1e4], device="cuda")[:, None].expand(4, 64).contiguous()
    out = torch.empty(4, device="cuda")
    native.linear_xent_t(x, w, torch.tensor([0, 776, 64, 63], device="cuda"), token_loss=out)
    np.testing.assert_allclose(from_dev(out), np.full(4, np.log(777)), rtol=2.0 ** -20)


@pytest.mark.parametrize("kind", ["xent", "distill"])
def test_gradients_against_differences(kind):
    """fp32: (l(x + s d) - l(x - s d)) / 2 s along a direction against the gradient along it. The difference's own error
    (its s^2 term) is the oracle's; each loss is off by its bound."""
    rng = np.random.default_rng(29)
    n, v, h, s = 9, 130, 20, 2.0 ** -5
    x, w, x64, w64 = _inputs(rng, n, v, h, F32)
    t = _labels(rng, n, v)
    ids, lg = _teacher(rng, n, v, 4)
    labels = t if kind == "xent" else (ids, lg, F32)
    oracle = (lambda a, b: OL.linear_xent(a, b, t)) if kind == "xent" else (lambda a, b: OL.linear_distill(a, b, ids, lg))
    base = _call(kind, x, w, F32, labels)
    for which in ("dx", "dw"):
        d = rng.integers(-1, 2, x.shape if which == "dx" else w.shape).astype(np.float32)
        at = [(x + e * s * d, w) if which == "dx" else (x, w + e * s * d) for e in (1, -1)]
        up, dn = (float(_call(kind, a.astype(np.float32), b.astype(np.float32), F32, labels, outs=("loss",))["loss"][0])
                  for a, b in at)
        rup, rdn = (oracle(a.astype(np.float64), b.astype(np.float64)).loss for a, b in at)
        want = float((base[which] * d).sum())
        true = oracle(x64, w64)
        cut = abs((rup - rdn) / (2 * s) - float((getattr(true, which) * d).sum()))
        size = np.abs(true.token_loss).max()
        assert abs((up - dn) / (2 * s) - want) <= cut + 2.0 ** -15 * size / s + 2.0 ** -14 * np.abs(getattr(true, which) * d).sum()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nothing_is_written_past_the_outputs(dtype):
    """Outputs inside larger buffers: the elements around them stay as they were."""
    import torch
    rng = np.random.default_rng(30)
    n, v, h, pad = 37, 301, 45, 64
    x, w, _, _ = _inputs(rng, n, v, h, dtype)
    xd, wd = to_dev(x, dtype), to_dev(w, dtype)
    t = torch.from_numpy(_labels(rng, n, v)).cuda()
    big, outs = [], []
    for shape, dt in (((1,), torch.float32), ((n,), torch.float32), ((n,), torch.float32), ((n, h), xd.dtype),
                      ((v, h), xd.dtype)):
        num = int(np.prod(shape))
        b = torch.full((num + 2 * pad,), 7.0, dtype=dt, device="cuda")
        big.append((b, num))
        outs.append(b[pad:pad + num].view(shape))
    args = dict(zip(("loss", "token_loss", "lse", "dx", "dw"), outs))
    a = native.head_loss_args_t(xd, wd, **args)
    size = native.mfsdp_head_loss_workspace_size(a)
    ws = torch.full((size + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    native.linear_xent_t(xd, wd, t, **args, workspace=ws[256:256 + size])
    torch.cuda.synchronize()
    assert bool((ws[:256] == 0x5A).all()) and bool((ws[256 + size:] == 0x5A).all())
    for b, num in big:
        assert bool((b[:pad] == 7).all()) and bool((b[pad + num:] == 7).all())
        assert not bool((b[pad:pad + num] == 7).all())


def _bits(ts):
    import torch
    return [t.clone().view(torch.int16 if t.element_size() == 2 else torch.int32) for t in ts]


def test_repeated_calls_streams_and_replays_give_the_same_bits():
    """Eager twice, on another stream, and captured: three replays with eager work in between, on new inputs too."""
    import torch
    rng = np.random.default_rng(31)
    n, v, h = 300, 1500, 136
    x, w, _, _ = _inputs(rng, n, v, h, BF16)
    x2, _, _, _ = _inputs(rng, n, v, h, BF16)
    xd, wd, xd2 = to_dev(x, BF16), to_dev(w, BF16), to_dev(x2, BF16)
    ids, lg = _teacher(rng, n, v, 7)
    t = torch.from_numpy(_labels(rng, n, v)).cuda()
    ids, lg = torch.from_numpy(ids).cuda(), to_dev(lg, F32)

    def outs():
        return [torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros_like(xd), torch.zeros_like(wd)]

    def both(a, b, xx, ws):
        for kind, o in (("xent", a), ("distill", b)):
            kw = dict(loss=o[0], token_loss=o[1], dx=o[2], dw=o[3], workspace=ws)
            if kind == "xent":
                native.linear_xent_t(xx, wd, t, **kw)
            else:
                native.linear_distill_t(xx, wd, ids, lg, temperature=2.0, **kw)

    args = native.head_loss_args_t(xd, wd, dx=xd, dw=wd)
    new_ws = lambda: native.head_loss_workspace_t(args, 7)  # noqa: E731
    ws = new_ws()
    a, b = outs(), outs()
    both(a, b, xd, ws)
    first = _bits(a + b)
    both(a, b, xd2, ws)
    second = _bits(a + b)
    assert not torch.equal(first[2], second[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c, d, ws2 = outs(), outs(), new_ws()
        both(c, d, xd, ws2)
        on_side = _bits(c + d)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, on_side))
    xin, ws3 = xd.clone(), new_ws()
    e, f = outs(), outs()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        both(e, f, xin, ws3)
    for i, (src, want) in enumerate(((xd, first), (xd2, second), (xd, first))):
        xin.copy_(src)
        for o in e + f:
            o.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, _bits(e + f))), i
        both(a, b, xd2, ws)
        torch.cuda.synchronize()


@pytest.mark.parametrize("n,v,h,k,dtype", [(40, 5000, 136, 1, BF16), (128, 4200, 72, 6, BF16), (300, 1500, 136, 7, F32),
                                           (16, 700, 2112, 1, F32), (2048, 20000, 256, 1, BF16)])
def test_two_calls_at_once_and_replays(n, v, h, k, dtype):
    """Two streams with a workspace each, side by side; then two captured calls, replayed with eager work in between: the bits of
    a call alone."""
    import torch
    rng = np.random.default_rng(32)
    w = to_dev(_inputs(rng, 1, v, h, dtype)[1], dtype)
    xs = [to_dev(_inputs(rng, n, 1, h, dtype)[0], dtype) for _ in range(2)]
    t = torch.from_numpy(_labels(rng, n, v)).cuda()
    ids, lg = (torch.from_numpy(a).cuda() for a in _teacher(rng, n, v, k))
    _say(n, v, h, k, dtype)

    def outs():
        return [torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros_like(xs[0]), torch.zeros_like(w)]

    def call(x, o, ws):
        kw = dict(loss=o[0], token_loss=o[1], dx=o[2], dw=o[3], workspace=ws)
        if k == 1:
            native.linear_xent_t(x, w, t, **kw)
        else:
            native.linear_distill_t(x, w, ids, lg, **kw)

    args = native.head_loss_args_t(xs[0], w, dx=xs[0], dw=w)
    wss = [native.head_loss_workspace_t(args, k) for _ in range(2)]
    want = []
    for x in xs:
        o = outs()
        call(x, o, wss[0])
        want.append(_bits(o))

    def same(got):
        torch.cuda.synchronize()
        for o, bits in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(_bits(o), bits))
            for a in o:
                a.zero_()

    got, streams = [outs(), outs()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                call(xs[i], got[i], wss[i])
    same(got)
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(xs[i], got[i], wss[i])
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        same(got)
        call(xs[1], got[0], wss[0])


def test_helpers_refuse_what_does_not_fit():
    import torch
    x = torch.zeros(8, 32, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(70, 32, dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(8, dtype=torch.int64, device="cuda")
    loss = torch.zeros(1, device="cuda")
    native.linear_xent_t(x, w, t, loss=loss)
    with pytest.raises(ValueError, match="required"):
        native.linear_xent_t(x, w[:, :16].contiguous(), t, loss=loss)
    with pytest.raises(TypeError, match="dtype"):
        native.linear_xent_t(x, w.float(), t, loss=loss)
    with pytest.raises(TypeError, match="dtype"):
        native.linear_xent_t(x, w, t.float(), loss=loss)
    with pytest.raises(ValueError, match="shape"):
        native.linear_xent_t(x, w, t[:4], loss=loss)
    with pytest.raises(ValueError, match="contiguous"):
        native.linear_xent_t(w.t(), torch.zeros(9, 70, dtype=torch.bfloat16, device="cuda"), t, loss=loss)
    with pytest.raises(ValueError, match="shape"):
        native.linear_xent_t(x, w, t, dx=torch.zeros(8, 33, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError, match="dtype"):
        native.linear_xent_t(x, w, t, dw=torch.zeros(70, 32, device="cuda"))
    with pytest.raises(ValueError, match="one element"):
        native.linear_xent_t(x, w, t, loss=torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError, match="shape"):
        native.linear_distill_t(x, w, t[:, None], torch.zeros(8, 2, device="cuda"), loss=loss)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(native.MfsdpError, match="too small"):
        native.linear_xent_t(x, w, t, loss=loss, workspace=small)


@pytest.mark.parametrize("n,v,h", [(20, 40003, 1032), (50, 50257, 768), (128, 33001, 1544)])
def test_few_tokens_many_steps(n, v, h):
    """The products for a few tokens with more tiles than workgroups and rings that go round many times: the oracle's results, and
    the same bits from each of twenty calls, on a busy chip too."""
    import torch
    rng = np.random.default_rng(41)
    x, w, x64, w64 = _inputs(rng, n, v, h, BF16)
    t = _labels(rng, n, v)
    _say(n, v, h)
    got = _call("xent", x, w, BF16, t)
    ref = _Ref(OL.linear_xent(x64, w64, t), t >= 0, None, "mean", 1.0)
    q = np.zeros((n, v), bool)
    q[np.nonzero(t >= 0)[0], t[t >= 0]] = True
    _check(got, ref, x64, w64, BF16, q, what=f"few tokens {n}x{v}x{h}")
    _check_loss(got, ref)
    xd, wd, td = to_dev(x, BF16), to_dev(w, BF16), torch.from_numpy(t).cuda()
    args = native.head_loss_args_t(xd, wd, dx=xd, dw=wd)
    wss, streams = [native.head_loss_workspace_t(args) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty(n, device="cuda"), torch.empty_like(xd), torch.empty_like(wd)] for _ in range(2)]
    first = None
    torch.cuda.synchronize()
    for i in range(20):
        for s, ws, o in zip(streams, wss, outs):
            with torch.cuda.stream(s):
                native.linear_xent_t(xd, wd, td, token_loss=o[0], dx=o[1], dw=o[2], workspace=ws)
        torch.cuda.synchronize()
        bits = [_bits(o) for o in outs]
        first = first or bits[0]
        assert all(torch.equal(a, b) for o in bits for a, b in zip(o, first)), i


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("n,v", [(5, 70), (300, 400), (20, 4500)])
def test_a_teacher_logit_of_infinity_or_nan_gives_nan(n, v, value, dtype):
    """With gradients and without: its token's loss, dx and the reduced loss are NaN, the other tokens stay."""
    rng = np.random.default_rng(42)
    x, w, _, _ = _inputs(rng, n, v, 24, dtype)
    ids, lg = _teacher(rng, n, v, 5, empty=0.0)
    bad = lg.copy()
    bad[3, 2] = value
    _say(n, v, value, dtype)
    others = np.arange(n) != 3
    for lgt in (F32, BF16):
        store = (lambda a: synth.f32_to_bf16_bits(a)) if lgt == BF16 else (lambda a: a)
        clean = _call("distill", x, w, dtype, (ids, store(lg), lgt), reduction="sum")
        for outs in (("loss", "token_loss", "lse", "dx", "dw"), ("loss", "token_loss")):
            got = _call("distill", x, w, dtype, (ids, store(bad), lgt), outs=outs, reduction="sum")
            assert np.isnan(got["token_loss"][3]) and np.isnan(got["loss"][0]), outs
            np.testing.assert_array_equal(got["token_loss"][others], clean["token_loss"][others])
        got = _call("distill", x, w, dtype, (ids, store(bad), lgt), reduction="sum")
        assert np.isnan(got["dx"][3]).all() and np.isnan(got["dw"]).all()
        np.testing.assert_array_equal(got["dx"][others], clean["dx"][others])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_teacher_logits_over_a_small_temperature(dtype):
    """Finite teacher logits whose quotient by the temperature is beyond fp32: their softmax is still one."""
    rng = np.random.default_rng(43)
    n, v, h, temp = 9, 90, 24, 2.0 ** -10
    x, w, x64, w64 = _inputs(rng, n, v, h, dtype, x_scale=2.0 ** -10)
    ids = np.stack([rng.permutation(v)[:4] for _ in range(n)])
    lg = np.array([3e38, 2e38, -3e38, 3e38], np.float32) * np.ones((n, 1), np.float32)
    lg[1] = [1e37, 1e37, 1e37, -3e38]
    got = _call("distill", x, w, dtype, (ids, lg, F32), temperature=temp)
    ref = _Ref(OL.linear_distill(x64, w64, ids, lg.astype(np.float64), temperature=temp), np.ones(n, bool), None, "mean", 1.0)
    q = np.zeros((n, v), bool)
    q[np.arange(n)[:, None], ids] = True
    _check(got, ref, x64, w64, dtype, q, inv_t=1 / temp, what=f"small temperature {dtype}")
    _check_loss(got, ref)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_both_gradients_of_a_sure_token(dtype):
    """Small integers, exact in either type: the loss is near 0, and both gradients are sums of probabilities of e^-12 and
    less. A probability is off by 2^-16 (bf16, no target: its 16-bit code's 2^-11 ln 2 too); an element of dz by its parts, u of
    itself or 2^-40 of its row's largest (bf16: two parts, 2^-16, and p below 2^-64 of the label's is 0: the last token's logits
    are e^-44 = 2^-63.5 and less); then the sum and the result's rounding."""
    n, v, h = 6, 301, 32
    rng = np.random.default_rng(44)
    w = rng.integers(-1, 2, (v, h)).astype(np.float64)
    w[:, 0] = -1
    w[7] = 0
    w[7, 0] = 1
    x = np.zeros((n, h))
    x[:, 0] = np.arange(12, 12 + 2 * n, 2)
    x[:, 1:4] = rng.integers(-1, 2, (n, 3))
    store = (lambda a: synth.f32_to_bf16_bits(a.astype(np.float32))) if dtype == BF16 else (lambda a: a.astype(np.float32))
    t = np.full(n, 7)
    got = _call("xent", store(x), store(w), dtype, t, reduction="sum")
    r = OL.linear_xent(x, w, t, reduction="sum")
    np.testing.assert_allclose(got["token_loss"], r.token_loss, rtol=2.0 ** -16, atol=0)
    target = np.zeros((n, v), bool)
    target[:, 7] = True
    rel = 2.0 ** -16 + (2.0 ** -16 + np.where(target, 0.0, 2.0 ** -11 * np.log(2)) if dtype == BF16 else U)
    ddz = np.abs(r.dz) * rel + (np.where(target, 0.0, 2.0 ** -64) if dtype == BF16 else 2.0 ** -40 * np.abs(r.dz).max(1)[:, None])
    half = 2.0 ** -8 if dtype == BF16 else U
    for name, acc, want, e, size in (("dx", v, r.dx, ddz @ np.abs(w), np.abs(r.dz) @ np.abs(w)),
                                     ("dw", n, r.dw, ddz.T @ np.abs(x), np.abs(r.dz).T @ np.abs(x))):
        tol = e + 2 * (acc + 8) * U * size
        tol = tol + half * (np.abs(want) + tol) + 1e-37
        err = np.abs(got[name] - want)
        _say(dtype, name, "worst share of the bound:", float((err / tol).max()))
        assert (err <= tol).all(), name


@pytest.mark.parametrize("n,v,h", [(9, 300, 48), (300, 900, 136)])
def test_a_head_whose_rows_differ_widely(n, v, h):
    """fp32: rows of w from 1 down to 2^-30 of the largest, which no token holds likely, so that dx is made of the small ones. A
    value of w is held to u of itself or 2^-40 of the largest; x and dz each relative to their rows."""
    rng = np.random.default_rng(45)
    x, w, x64, w64 = _inputs(rng, n, v, h, F32)
    x64 = np.abs(x64) + 0.5
    x = x64.astype(np.float32)
    x64 = x.astype(np.float64)
    size = 2.0 ** -rng.integers(1, 31, v)
    w = (w64 * size[:, None]).astype(np.float32)
    w[:3] = -40.0 / h ** 0.5
    w64 = w.astype(np.float64)
    t = rng.integers(3, v, n)
    got = _call("xent", x, w, F32, t, reduction="sum")
    r = OL.linear_xent(x64, w64, t, reduction="sum")
    assert np.exp(r.z[:, :3] - r.lse[:, None]).max() < 2.0 ** -20
    lost = 2.0 ** -40 * np.abs(w64).max()
    dz_z = 2 * (h + 8) * U * (np.abs(x64) @ np.abs(w64).T) + lost * np.abs(x64).sum(1)[:, None]
    dr = dz_z.max(1)
    tol = 2 * dr + 2.0 ** -17 + 2.0 ** -18 * (np.abs(r.token_loss) + np.abs(r.z).max(1) + np.log(v))
    assert (np.abs(got["token_loss"] - r.token_loss) <= tol).all()
    p = np.exp(r.z - r.lse[:, None])
    q = np.zeros((n, v), bool)
    q[np.arange(n), t] = True
    ddz = p * (2 * dr + 2.0 ** -16)[:, None] + np.where(q, (p + 1) * 2.0 ** -18, 2.0 ** -60)
    ddz = ddz + U * (np.abs(r.dz) + ddz) + 2.0 ** -40 * np.abs(r.dz).max(1)[:, None]
    for name, acc, want, e, s in (("dx", v, r.dx, ddz @ np.abs(w64) + lost * np.abs(r.dz).sum(1)[:, None], np.abs(r.dz) @ np.abs(w64)),
                                  ("dw", n, r.dw, ddz.T @ np.abs(x64), np.abs(r.dz).T @ np.abs(x64))):
        tol = e + 2 * (acc + 8) * U * s
        tol = tol + U * (np.abs(want) + tol) + 1e-37
        err = np.abs(got[name] - want)
        _say(name, "worst share of the bound:", float((err / tol).max()))
        assert (err <= tol).all(), name


@pytest.mark.parametrize("n,v,h,k", [(64, 12289, 264, 1), (65, 12287, 264, 1), (65, 12288, 72, 1), (100, 13001, 136, 5), (128, 12300, 320, 33),
                                     (129, 12288, 72, 3), (128, 16384, 1000, 1)])
def test_around_the_limits_of_a_few_tokens(n, v, h, k):
    rng = np.random.default_rng(46)
    x, w, x64, w64 = _inputs(rng, n, v, h, BF16)
    _say(n, v, h, k)
    q = np.zeros((n, v), bool)
    if k == 1:
        t = _labels(rng, n, v)
        got = _call("xent", x, w, BF16, t, z_loss=1e-3)
        ref = _Ref(OL.linear_xent(x64, w64, t, z_loss=1e-3), t >= 0, None, "mean", 1.0)
        q[np.nonzero(t >= 0)[0], t[t >= 0]] = True
        _check(got, ref, x64, w64, BF16, q, z_loss=1e-3, what=f"limits {n}x{v}x{h}")
    else:
        ids, lg = _teacher(rng, n, v, k)
        got = _call("distill", x, w, BF16, (ids, lg, F32), temperature=1.5)
        ref = _Ref(OL.linear_distill(x64, w64, ids, lg, temperature=1.5), (ids >= 0).any(1), None, "mean", 1.0)
        q[np.repeat(np.arange(n), k).reshape(n, k)[ids >= 0], ids[ids >= 0]] = True
        _check(got, ref, x64, w64, BF16, q, inv_t=1 / 1.5, what=f"limits {n}x{v}x{h},{k}")
    _check_loss(got, ref)
