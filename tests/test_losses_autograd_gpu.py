"""The autograd front ends of the losses (paper_2607_05895_amd.losses) against the fp64 oracle: gradients of leaves through
them, and a training step that uses both losses and the owner's optimizer. Bounds: each product's rounding is that of
tests/test_loss_gpu.py; here relative Frobenius errors are compared, bf16 2^-8 per rounding (dz, the result, and one
more for a factor or a sum of two gradients), fp32 2^-17."""
import numpy as np
import pytest

import oracle
import synth
from oracle import losses as OL
from tests.helpers import from_dev, rel_fro, to_dev

pytestmark = pytest.mark.gpu
TOL = {synth.BF16: 4 * 2.0 ** -8, synth.F32: 2.0 ** -17}


def _leaf(arr, dtype):
    return to_dev(arr, dtype).clone().requires_grad_(True)


def _store(a, dtype):
    a = a.astype(np.float32)
    if dtype == synth.BF16:
        b = synth.f32_to_bf16_bits(a)
        return b, synth.bf16_bits_to_f32(b).astype(np.float64)
    return a, a.astype(np.float64)


@pytest.mark.parametrize("dtype", [synth.BF16, synth.F32])
def test_gradients_reach_the_leaves(dtype):
    import torch
    from paper_2607_05895_amd import losses
    rng = np.random.default_rng(1)
    B, T, v, h, k = 3, 50, 700, 72, 5
    xs, x = _store(rng.standard_normal((B, T, h)), dtype)
    ws, w = _store(rng.standard_normal((v, h)) / 8, dtype)
    t = rng.integers(0, v, (B, T))
    t[:, :7] = -100
    a = rng.uniform(0.2, 1.5, (B, T)).astype(np.float32)
    ids = rng.integers(0, v, (B, T, k))
    lg = rng.standard_normal((B, T, k)).astype(np.float32)
    dev = lambda z: torch.from_numpy(z).cuda()  # noqa: E731
    for name in ("xent", "distill"):
        X, W = _leaf(xs, dtype), _leaf(ws, dtype)
        if name == "xent":
            loss = losses.linear_cross_entropy(X, W, dev(t), token_weight=dev(a), z_loss=1e-3)
            r = OL.linear_xent(x.reshape(-1, h), w, t.reshape(-1), weight=a.reshape(-1), z_loss=1e-3)
        else:
            loss = losses.linear_distillation(X, W, dev(ids), dev(lg), temperature=2.0, scale=4.0, reduction="sum")
            r = OL.linear_distill(x.reshape(-1, h), w, ids.reshape(-1, k), lg.reshape(-1, k), temperature=2.0, scale=4.0,
                                  reduction="sum")
        (loss * 0.375).backward()
        assert abs(float(loss.detach()) - r.loss) <= 2.0 ** -14 * abs(r.loss)
        assert X.grad.shape == X.shape and X.grad.dtype == X.dtype
        assert rel_fro(from_dev(X.grad).reshape(-1, h), 0.375 * r.dx) <= TOL[dtype], name
        assert rel_fro(from_dev(W.grad), 0.375 * r.dw) <= TOL[dtype], name


def test_views_inner_results_and_what_needs_no_gradient():
    """A non-contiguous hidden view behind another operation; only one of the two leaves wants a gradient; no_grad."""
    import torch
    from paper_2607_05895_amd import losses
    rng = np.random.default_rng(2)
    v, h = 300, 48
    xs, x = _store(rng.standard_normal((2, 9, h)), synth.F32)
    ws, w = _store(rng.standard_normal((v, h)) / 7, synth.F32)
    t = torch.from_numpy(rng.integers(0, v, (2, 8))).cuda()
    X, W = _leaf(xs, synth.F32), to_dev(ws, synth.F32)
    loss = losses.linear_cross_entropy((2 * X)[:, :-1], W, t)
    loss.backward()
    r = OL.linear_xent(2 * x[:, :-1].reshape(-1, h), w, t.cpu().numpy().reshape(-1))
    want = np.zeros_like(x)
    want[:, :-1] = 2 * r.dx.reshape(2, 8, h)
    assert rel_fro(from_dev(X.grad), want) <= TOL[synth.F32]
    assert W.grad is None
    with torch.no_grad():
        again = losses.linear_cross_entropy((2 * X)[:, :-1], W, t)
    assert not again.requires_grad and float(again) == float(loss.detach())
    per = losses.token_losses((2 * X)[:, :-1], W, t)
    assert per.shape == t.shape and not per.requires_grad
    np.testing.assert_allclose(from_dev(per).reshape(-1), r.token_loss, rtol=1e-4, atol=1e-5)
    one = losses.token_losses((2 * X)[:1, :1], W, t[:1, :1])
    assert abs(float(one) - r.token_loss[0]) < 1e-4


def test_the_backward_pass_runs_once_and_shapes_are_checked():
    import torch
    from paper_2607_05895_amd import losses
    x = torch.randn(4, 16, device="cuda", requires_grad=True)
    w = torch.randn(40, 16, device="cuda", requires_grad=True)
    t = torch.arange(4, device="cuda")
    loss = losses.linear_cross_entropy(x, w, t)
    loss.backward(retain_graph=True)
    with pytest.raises(RuntimeError, match="once"):
        loss.backward()
    with pytest.raises(ValueError, match="shape"):
        losses.linear_cross_entropy(x, w, t[:3])
    with pytest.raises(ValueError, match="shape"):
        losses.linear_distillation(x, w, t[:, None], torch.zeros(4, 2, device="cuda"))
    with pytest.raises(ValueError, match="shape"):
        losses.token_losses(x, w, t[None])
    with pytest.raises(TypeError, match="dtype"):
        losses.linear_cross_entropy(x, w.bfloat16(), t)


@pytest.mark.parametrize("n", [1, 7, 8, 4097])
def test_scale_grad(n):
    import torch
    from paper_2607_05895_amd import native
    for dt in (torch.float32, torch.bfloat16):
        big = torch.randn(n + 16, device="cuda").to(dt)
        g = big[:n].clone()
        want = (g.float() * -0.3).to(dt)
        native.scale_grad_t(g, torch.tensor([-0.3], device="cuda"))
        assert torch.equal(g, want)
        native.scale_grad_t(g, torch.ones((), device="cuda"))
        assert torch.equal(g, want)


def test_a_training_step_with_both_losses_and_the_owner_optimizer():
    """hidden = body(x); loss = cross entropy + distillation; backward; OwnerMuon on body and head: their updated values
    against the oracle's gradients put through the oracle's optimizer."""
    import torch
    from paper_2607_05895_amd import losses
    from paper_2607_05895_amd.optim import OwnerMuon
    rng = np.random.default_rng(3)
    n, d, h, v, k = 96, 64, 80, 500, 4
    x0 = rng.standard_normal((n, d)).astype(np.float32)
    bs, body = _store(rng.standard_normal((h, d)) / 8, synth.F32)
    ws, head = _store(rng.standard_normal((v, h)) / 9, synth.F32)
    gs, bias = _store(rng.standard_normal(h) / 9, synth.F32)
    t = rng.integers(0, v, n)
    t[:9] = -100
    ids, lg = rng.integers(0, v, (n, k)), rng.standard_normal((n, k)).astype(np.float32)
    B, W, b = _leaf(bs, synth.F32), _leaf(ws, synth.F32), _leaf(gs, synth.F32)
    opt = OwnerMuon([B, W, b], lr=0.02, weight_decay=0.01, ns_dtype="f32", adamw_lr=1e-3, adamw_weight_decay=0.01)
    hidden = to_dev(x0, synth.F32) @ B.t() + b
    dev = lambda z: torch.from_numpy(z).cuda()  # noqa: E731
    loss = losses.linear_cross_entropy(hidden, W, dev(t)) + 0.5 * losses.linear_distillation(
        hidden, W, dev(ids), dev(lg), temperature=2.0, scale=4.0)
    loss.backward()
    opt.step()
    torch.cuda.synchronize()
    hid = x0.astype(np.float64) @ body.T + bias
    r1 = OL.linear_xent(hid, head, t)
    r2 = OL.linear_distill(hid, head, ids, lg, temperature=2.0, scale=4.0)
    assert abs(float(loss.detach()) - (r1.loss + 0.5 * r2.loss)) <= 1e-4
    dh = r1.dx + 0.5 * r2.dx
    grads = {"body": dh.T @ x0, "head": r1.dw + 0.5 * r2.dw}
    for p, p0, g in ((B, body, grads["body"]), (W, head, grads["head"])):
        assert rel_fro(from_dev(p.grad), g) <= 1e-4
        want, _, O = oracle.muon_step(p0, g, np.zeros_like(p0), lr=0.02, weight_decay=0.01, momentum=0.95, nesterov=True,
                                      a=synth.NS_COEFFS[0], b=synth.NS_COEFFS[1], c=synth.NS_COEFFS[2], ns_steps=5)
        # the orthogonalisation multiplies a relative error of small singular directions by up to 3.4445^5
        f = 0.02 * max(1.0, p0.shape[0] / p0.shape[1]) ** 0.5
        assert np.linalg.norm(from_dev(p.detach()) - want) <= 2e-2 * f * np.linalg.norm(O)
    g = dh.sum(0)
    want, _, _ = oracle.adamw_step(bias, g, np.zeros(h), np.zeros(h), lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                                   weight_decay=0.01, step=1)
    assert np.abs(from_dev(b.detach()) - want).max() <= 1e-5


@pytest.mark.parametrize("dtype", [synth.BF16, synth.F32])
def test_no_token_at_all(dtype):
    """An empty batch: loss 0, the head's gradient 0, the hidden states' gradient empty; on a stream of its own."""
    import torch
    from paper_2607_05895_amd import losses
    rng = np.random.default_rng(4)
    W = _leaf(_store(rng.standard_normal((300, 48)), dtype)[0], dtype)
    X = torch.empty((2, 0, 48), dtype=W.dtype, device="cuda", requires_grad=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        loss = losses.linear_cross_entropy(X, W, torch.empty((2, 0), dtype=torch.int64, device="cuda"))
        loss.backward()
        nll = losses.token_losses(X, W, torch.empty((2, 0), dtype=torch.int64, device="cuda"))
    torch.cuda.synchronize()
    assert float(loss.detach()) == 0.0 and nll.shape == (2, 0)
    assert X.grad.shape == X.shape and not W.grad.any()


@pytest.mark.parametrize("dtype", [synth.BF16, synth.F32])
def test_shifted_views(dtype):
    """Next-token labels: ids[1:] beside hidden[:-1], and views that begin in the middle of 16 bytes, give what copies give."""
    import torch
    from paper_2607_05895_amd import losses
    rng = np.random.default_rng(5)
    T, v, h = 38, 500, 18
    hid, w = (_leaf(_store(rng.standard_normal(s), dtype)[0], dtype) for s in ((T, h), (v + 1, h)))
    ids = torch.from_numpy(rng.integers(0, v, T)).cuda()
    a = torch.rand(T, device="cuda")
    top, lg = torch.randint(0, v, (T, 3), device="cuda"), torch.randn(T, 3, device="cuda")

    def grads(loss):
        return [loss.detach(), *torch.autograd.grad(loss, (hid, w))]

    got = grads(losses.linear_cross_entropy(hid[1:], w[1:], ids[1:], token_weight=a[1:]))
    want = grads(losses.linear_cross_entropy(hid[1:].clone(), w[1:].clone(), ids[1:].clone(), token_weight=a[1:].clone()))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    got = grads(losses.linear_distillation(hid[1:], w[1:], top[1:], lg[1:]))
    want = grads(losses.linear_distillation(hid[1:].clone(), w[1:].clone(), top[1:].clone(), lg[1:].clone()))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert torch.equal(losses.token_losses(hid[:-1], w, ids[1:]), losses.token_losses(hid[:-1].clone(), w, ids[1:].clone()))


def test_token_weights_of_another_shape_are_refused():
    """As many weights in another order of dimensions belong to other tokens; the tokens' shape and one dimension do not."""
    import torch
    from paper_2607_05895_amd import losses
    B, T, v, h = 2, 3, 40, 16
    x, w = torch.randn(B, T, h, device="cuda"), torch.randn(v, h, device="cuda")
    t, ids, lg = (torch.randint(0, v, s, device="cuda") for s in ((B, T), (B, T, 2), (B, T, 2)))
    a = torch.rand(B, T, device="cuda")
    calls = (lambda a: losses.linear_cross_entropy(x, w, t, token_weight=a, reduction="sum"),
             lambda a: losses.linear_distillation(x, w, ids, lg.float(), token_weight=a, reduction="sum"))
    for call in calls:
        assert float(call(a)) == float(call(a.reshape(-1)))
        for bad in (a.t(), a[:, :2], a[None], a[:1], a.reshape(1, -1), a[0, 0]):
            with pytest.raises(ValueError, match="token_weight"):
                call(bad)


@pytest.mark.parametrize("dtype", [synth.BF16, synth.F32])
def test_captured_forward_and_backward(dtype):
    """Both losses and their gradients in one graph, replayed on new inputs with eager work in between: the eager bits."""
    import torch
    from paper_2607_05895_amd import losses
    rng = np.random.default_rng(6)
    n, v, h = 70, 900, 72
    xs = [to_dev(_store(rng.standard_normal((n, h)), dtype)[0], dtype) for _ in range(2)]
    w = _leaf(_store(rng.standard_normal((v, h)) / 8, dtype)[0], dtype)
    t = torch.from_numpy(rng.integers(0, v, n)).cuda()
    ids, lg = torch.from_numpy(rng.integers(0, v, (n, 4))).cuda(), torch.randn(n, 4, device="cuda")
    x = xs[0].clone().requires_grad_(True)

    def step():
        loss = 0.75 * losses.linear_cross_entropy(x, w, t) + losses.linear_distillation(x, w, ids, lg, temperature=2.0)
        return [loss.detach().clone(), *torch.autograd.grad(loss, (x, w))]

    want = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in (0, 1):
            with torch.no_grad():
                x.copy_(xs[i])
            want.append([a.clone() for a in step()])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for i in (0, 1, 0):
        with torch.no_grad():
            x.copy_(xs[i])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])), i
        losses.token_losses(xs[1], w, t)
        torch.cuda.synchronize()
