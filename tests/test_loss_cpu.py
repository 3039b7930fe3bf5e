"""Host-side tests of the losses over a vocabulary that need no GPU: refusals before anything is enqueued, and the size
of the workspace."""
import ctypes

import pytest
import torch

from paper_2607_05895_amd import native

FAKE = 1 << 20  # a 16-byte aligned non-NULL address; never dereferenced (validation fails first)


def _args(**kw):
    d = dict(x=FAKE, w=FAKE * 2, n=64, v=1000, h=128, dtype=native.BF16, reduction=native.MEAN, scale=1.0,
             token_weight=None, loss=FAKE * 3, token_loss=None, lse=None, dx=FAKE * 4, dw=FAKE * 5, chunk_rows=0)
    d.update(kw)
    return native.HeadLoss(**d)


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(n=(1 << 28) + 1), dict(v=0), dict(v=(1 << 20) + 1), dict(h=0), dict(h=(1 << 20) + 1), dict(dtype=2),
    dict(dtype=-1), dict(reduction=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(chunk_rows=-1),
])
def test_bad_arguments_are_refused_by_every_entry(bad):
    a = _args(**bad)
    for call in (lambda: native.mfsdp_linear_xent(a, FAKE, 8, -100, 0.0, FAKE * 16, 1 << 50),
                 lambda: native.mfsdp_linear_distill(a, FAKE, 8, FAKE, native.F32, 4, 1.0, FAKE * 16, 1 << 50),
                 lambda: native.mfsdp_head_loss_workspace_size(a)):
        with pytest.raises(native.MfsdpError) as ei:
            call()
        assert ei.value.status == native.E_INVALID


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(w=None), dict(x=FAKE + 8), dict(w=FAKE + 2), dict(loss=FAKE + 4), dict(token_loss=FAKE + 4),
    dict(lse=FAKE + 4), dict(dx=FAKE + 2), dict(dw=FAKE + 2), dict(token_weight=FAKE + 4),
    dict(loss=None, dx=None, dw=None),
])
def test_bad_pointers_are_refused(bad):
    a = _args(**bad)
    for call in (lambda: native.mfsdp_linear_xent(a, FAKE, 8, -100, 0.0, FAKE * 16, 1 << 50),
                 lambda: native.mfsdp_linear_distill(a, FAKE, 8, FAKE, native.F32, 4, 1.0, FAKE * 16, 1 << 50)):
        with pytest.raises(native.MfsdpError) as ei:
            call()
        assert ei.value.status == native.E_INVALID


@pytest.mark.parametrize("targets,size,z_loss", [(None, 8, 0.0), (FAKE + 8, 8, 0.0), (FAKE, 2, 0.0), (FAKE, 8, -1.0),
                                                 (FAKE, 8, float("nan")), (FAKE, 8, float("inf"))])
def test_bad_labels_are_refused(targets, size, z_loss):
    with pytest.raises(native.MfsdpError) as ei:
        native.mfsdp_linear_xent(_args(), targets, size, -100, z_loss, FAKE * 16, 1 << 50)
    assert ei.value.status == native.E_INVALID


@pytest.mark.parametrize("ids,size,logits,dt,k,temp", [
    (None, 8, FAKE, 0, 4, 1.0), (FAKE, 8, None, 0, 4, 1.0), (FAKE, 1, FAKE, 0, 4, 1.0), (FAKE, 8, FAKE, 3, 4, 1.0),
    (FAKE, 8, FAKE, 0, 0, 1.0), (FAKE, 8, FAKE, 0, 257, 1.0), (FAKE, 8, FAKE, 0, 4, 0.0), (FAKE, 8, FAKE, 0, 4, -1.0),
    (FAKE, 8, FAKE, 0, 4, float("nan")), (FAKE, 8, FAKE, 0, 4, float("inf")), (FAKE + 4, 8, FAKE, 0, 4, 1.0),
    (FAKE, 8, FAKE + 4, 0, 4, 1.0),
])
def test_bad_teachers_are_refused(ids, size, logits, dt, k, temp):
    with pytest.raises(native.MfsdpError) as ei:
        native.mfsdp_linear_distill(_args(), ids, size, logits, dt, k, temp, FAKE * 16, 1 << 50)
    assert ei.value.status == native.E_INVALID


@pytest.mark.parametrize("ws,bytes_", [(None, 1 << 50), (FAKE * 16 + 16, 1 << 50), (FAKE * 16, 1 << 10)])
def test_bad_workspaces_are_refused(ws, bytes_):
    for call in (lambda: native.mfsdp_linear_xent(_args(), FAKE, 8, -100, 0.0, ws, bytes_),
                 lambda: native.mfsdp_linear_distill(_args(), FAKE, 8, FAKE, native.F32, 4, 1.0, ws, bytes_)):
        with pytest.raises(native.MfsdpError) as ei:
            call()
        assert ei.value.status == native.E_WORKSPACE


def test_null_arguments_are_refused():
    assert native.lib().mfsdp_linear_xent(None, FAKE, 8, -100, 0.0, FAKE, 1 << 40, None) == native.E_INVALID
    assert native.lib().mfsdp_head_loss_workspace_size(None, 1) == 0


def test_workspace_does_not_hold_the_logits():
    """128256 ids: beyond one chunk of rows the workspace grows by a few words per token, and without gradients it is
    that of the packed operands."""
    size = lambda **kw: native.mfsdp_head_loss_workspace_size(_args(v=128256, h=4096, **kw))  # noqa: E731
    a, b = size(n=1 << 16), size(n=1 << 18)
    assert (b - a) / ((1 << 18) - (1 << 16)) <= 32
    assert a - size(n=1 << 16, chunk_rows=512) > 1.8 * (1 << 30)   # the chunk's logits
    assert size(n=1 << 16, dx=None, dw=None) < 3 * (1 << 30)
    for n in (1, 255, 257):
        assert size(n=n) < 4 * (1 << 30)


@pytest.mark.parametrize("dtype", [native.BF16, native.F32])
@pytest.mark.parametrize("n,v,h", [(1, 1, 1), (48, 128256, 4096), (200, 5000, 130), (1024, 20000, 4096), (70000, 3000, 64)])
def test_fewer_outputs_never_need_more_workspace(n, v, h, dtype):
    size = lambda **kw: native.mfsdp_head_loss_workspace_size(_args(n=n, v=v, h=h, dtype=dtype, **kw))  # noqa: E731
    both = size()
    for fewer in (dict(dx=None), dict(dw=None), dict(dx=None, dw=None)):
        assert size(**fewer) <= both


def test_cpu_tensors_are_refused():
    x, w, t = torch.zeros(4, 8), torch.zeros(16, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        native.linear_xent_t(x, w, t, loss=torch.zeros(1))
    with pytest.raises(ValueError, match="CUDA"):
        native.linear_distill_t(x, w, t[:, None], torch.zeros(4, 1), loss=torch.zeros(1))


def test_front_ends_refuse_cpu_tensors():
    from paper_2607_05895_amd import losses
    x, w, t = torch.zeros(2, 4, 8), torch.zeros(16, 8), torch.zeros(2, 4, dtype=torch.int64)
    for call in (lambda: losses.linear_cross_entropy(x, w, t), lambda: losses.token_losses(x, w, t),
                 lambda: losses.linear_distillation(x, w, t[..., None], torch.zeros(2, 4, 1))):
        with pytest.raises(ValueError, match="GPU"):
            call()


@pytest.mark.parametrize("grad,numel,dt,factor", [(FAKE, -1, 0, FAKE), (FAKE, 4, 2, FAKE), (None, 4, 0, FAKE),
                                                  (FAKE, 4, 0, None), (FAKE + 4, 4, 0, FAKE)])
def test_bad_scale_arguments_are_refused(grad, numel, dt, factor):
    with pytest.raises(native.MfsdpError) as ei:
        native.mfsdp_scale_grad(grad, numel, dt, factor)
    assert ei.value.status == native.E_INVALID


def test_struct_matches_the_header():
    """8-byte fields and pairs of 4-byte ones: no padding anywhere."""
    assert ctypes.sizeof(native.HeadLoss) == 8 * 14


@pytest.mark.parametrize("scale", [1e39, -1e39, 1e300])
def test_a_scale_beyond_fp32_is_refused(scale):
    a = _args(scale=scale)
    for call in (lambda: native.mfsdp_linear_xent(a, FAKE, 8, -100, 0.0, FAKE * 16, 1 << 50),
                 lambda: native.mfsdp_linear_distill(a, FAKE, 8, FAKE, native.F32, 4, 1.0, FAKE * 16, 1 << 50),
                 lambda: native.mfsdp_head_loss_workspace_size(a)):
        with pytest.raises(native.MfsdpError, match="fp32") as ei:
            call()
        assert ei.value.status == native.E_INVALID


@pytest.mark.parametrize("scale,temperature", [(1.0, 1e-39), (1.0, 1e-300), (1.0, 1e39), (1.0, 1e300), (1e30, 1e-9), (-1e30, 1e-9)])
def test_a_temperature_beyond_fp32_is_refused(scale, temperature):
    """1 / temperature infinite or denormal, scale / temperature infinite: the results would be NaN or 0. (A workspace that
    is too small: a call that is not refused for its temperature is refused for that.)"""
    with pytest.raises(native.MfsdpError, match="temperature") as ei:
        native.mfsdp_linear_distill(_args(scale=scale), FAKE, 8, FAKE, native.F32, 4, temperature, FAKE * 16, 1 << 10)
    assert ei.value.status == native.E_INVALID


@pytest.mark.parametrize("temperature", [1e-37, 1e-3, 1e3, 1e37])
def test_far_temperatures_are_taken(temperature):
    with pytest.raises(native.MfsdpError, match="too small"):
        native.mfsdp_linear_distill(_args(), FAKE, 8, FAKE, native.F32, 4, temperature, FAKE * 16, 1 << 10)


def test_a_z_loss_beyond_fp32_is_refused():
    with pytest.raises(native.MfsdpError, match="z_loss") as ei:
        native.mfsdp_linear_xent(_args(), FAKE, 8, -100, 1e39, FAKE * 16, 1 << 10)
    assert ei.value.status == native.E_INVALID


def test_one_token_more_than_a_call_takes_is_refused():
    size = lambda n: native.mfsdp_head_loss_workspace_size(_args(n=n))  # noqa: E731
    assert size(1 << 25) > 0
    for n in ((1 << 25) + 1, 1 << 26):
        with pytest.raises(native.MfsdpError) as ei:
            size(n)
        assert ei.value.status == native.E_INVALID
        with pytest.raises(native.MfsdpError) as ei:
            native.mfsdp_linear_xent(_args(n=n), FAKE, 8, -100, 0.0, FAKE * 16, 1 << 50)
        assert ei.value.status == native.E_INVALID


def _size(k=1, **kw):
    return native.mfsdp_head_loss_workspace_size(_args(**kw), k)


OUTPUTS = [dict(), dict(dx=None), dict(dw=None), dict(dx=None, dw=None)]
SIDES = [(1, 1), (128, 64), (300, 64), (1000, 64), (4000, 128), (2000, 2048), (4096, 8), (4095, 264), (12287, 264), (12288, 264), (9001, 8192), (5000, 130), (400, 4000),
         (50257, 768), (128256, 4096), (128256, 4095), (128256, 32768), (1 << 20, 64), (90, 1 << 20)]


@pytest.mark.parametrize("dtype", [native.BF16, native.F32])
@pytest.mark.parametrize("v,h", SIDES)
def test_fewer_tokens_never_need_more_workspace(v, h, dtype):
    """A workspace sized for the largest batch serves every smaller one: few tokens, one pass, several passes."""
    counts = sorted({c + d for c in (1, 32, 64, 128, 256, 384, 512, 777, 1024, 2048, 4096, 6000, 8192, 8371, 8448, 10000, 16384,
                                     20000, 65536, 70000, 1 << 20, 1 << 25) for d in (-1, 0, 1) if 0 < c + d <= 1 << 25})
    for outs in OUTPUTS:
        for chunk in (0, 256, 5000):
            last = 0
            for n in counts:
                now = _size(n=n, v=v, h=h, dtype=dtype, chunk_rows=chunk, **outs)
                assert now >= last, (n, outs, chunk, last, now)
                last = now


@pytest.mark.parametrize("dtype", [native.BF16, native.F32])
def test_fewer_outputs_and_slots_never_need_more_workspace_at_any_size(dtype):
    import random
    rng = random.Random(5)
    log = lambda hi: int(2 ** rng.uniform(0, hi))  # noqa: E731
    sizes = [(log(18), log(20), log(15)) for _ in range(1500)] + [(65536, 1 << 20, 64), (65536, 128256, 32768)]
    for n, v, h in sizes:
        kw = dict(n=n, v=v, h=h, dtype=dtype, chunk_rows=rng.choice((0, 0, 256, 4096)))
        k = rng.randint(2, 256)
        both = _size(k, **kw)
        for outs in OUTPUTS[1:]:
            some = _size(k, **kw, **outs)
            assert some <= both, (kw, outs, some, both)
            assert _size(k, **kw, dx=None, dw=None) <= some, (kw, outs)
        assert _size(rng.randint(1, k), **kw) <= both
        fewer = dict(kw, n=rng.randint(1, n))
        assert _size(k, **fewer) <= both, (kw, fewer)


def test_one_pass_where_several_would_need_more_workspace():
    """A few rows beyond 2 GiB of logits: their logits take less than dw's sum over two passes, which is left out."""
    kw = dict(v=128256, h=4096)
    most = 8192
    total = 4 * 128256 * 4096
    assert _size(n=most + 1, **kw) - _size(n=most, **kw) < total // 10
    assert _size(n=65536, **kw) > _size(n=65536, dw=None, **kw) + total - 1
    # (asked for by the caller: 256 rows a pass and the sum)
    assert _size(n=1024, chunk_rows=256, **kw) > total
