"""The work that the loss operators' performance is measured on: the losses over a vocabulary that a training or scoring
program computes from hidden states ``x`` (n x h) and an output head ``w`` (v x h), with the gradients of both.

Kinds

* ``xent``     softmax cross entropy with the tokens' labels (some of them ignored), mean over the labelled tokens
* ``distill``  KL divergence from a teacher's ``k`` top logits a token (some slots empty) at a temperature

``grads`` says whether the gradients of x and w are computed as well; without them it is an evaluation or a scoring pass.
"""
from __future__ import annotations

import math

import torch

own = False

IGNORE = -100
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # scoring the next token of one sequence: the head is read once, and nothing else counts
        dict(name="xent_score_one_token", kind="xent", n=1, v=128256, h=4096, k=1, dtype="bf16", grads=False),
        # the smallest training call: a toy model in a test or a tutorial, where the launches count
        dict(name="xent_toy_f32", kind="xent", n=64, v=1000, h=64, k=1, dtype="f32", grads=True),
        # a GPT-2-small micro-batch of four sequences of 1024
        dict(name="xent_gpt2_4k", kind="xent", n=4096, v=50257, h=768, k=1, dtype="bf16", grads=True),
        # the same model trained in fp32, one sequence
        dict(name="xent_gpt2_1k_f32", kind="xent", n=1024, v=50257, h=768, k=1, dtype="f32", grads=True),
        # odd sizes everywhere: a ragged batch over a vocabulary and a width that divide by nothing
        dict(name="xent_odd", kind="xent", n=777, v=32003, h=1001, k=1, dtype="bf16", grads=True),
        # a Llama-3-8B head, one sequence of 8192 tokens: the main training case
        dict(name="xent_llama_8k", kind="xent", n=8192, v=128256, h=4096, k=1, dtype="bf16", grads=True),
        # evaluation (perplexity) on the same head
        dict(name="xent_llama_4k_eval", kind="xent", n=4096, v=128256, h=4096, k=1, dtype="bf16", grads=False),
        # a few tokens: the labelled end of one short instruction sample, fine-tuning step
        dict(name="xent_llama_48", kind="xent", n=48, v=128256, h=4096, k=1, dtype="bf16", grads=True),
        # a toy student
        dict(name="distill_toy", kind="distill", n=33, v=1003, h=96, k=5, dtype="bf16", grads=True),
        # a GPT-2-small student in fp32
        dict(name="distill_gpt2_f32", kind="distill", n=512, v=50257, h=768, k=16, dtype="f32", grads=True),
        # a Llama-3-8B student on a sequence of 2048 with 32 teacher logits a token
        dict(name="distill_llama_2k", kind="distill", n=2048, v=128256, h=4096, k=32, dtype="bf16", grads=True),
        # how far a student is from its teacher on held-out text
        dict(name="distill_eval", kind="distill", n=1500, v=50257, h=2048, k=20, dtype="bf16", grads=False),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the listed ones' ranges: any token count, vocabulary and width, odd ones among them."""
    most = 8192 * 128256 * 4096
    while True:
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        n, v, h = _log_uniform(rng, 1, 8192), _log_uniform(rng, 300, 128256), _log_uniform(rng, 64, 4096)
        if rng.random() < 0.6:
            h = (h + 63) // 64 * 64
        if rng.random() < 0.4:
            n = (n + 127) // 128 * 128
        if n * v * h <= (most if dtype == "bf16" else most // 32):
            break
    kind = rng.choice(("xent", "xent", "distill"))
    return dict(kind=kind, n=n, v=v, h=h, k=1 if kind == "xent" else rng.choice((1, 3, 8, 20, 50)), dtype=dtype,
                grads=rng.random() < 0.75)


def prepare(case, seed):
    """Hidden states of unit variance (a final norm's output) that lean towards the head's rows of their labels, by a
    strength of its own for each token: from one that the model has no idea of to one that it holds the likeliest by far."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, v, h, k = case["n"], case["v"], case["h"], case["k"]
    dt = DTYPES[case["dtype"]]
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    w = (randn(v, h) * (1.2 / math.sqrt(h))).to(dt)
    # token frequencies fall with the index, as in a vocabulary built by merges
    ids = (rand(n, k) ** 3 * v).long().clamp_(max=v - 1)
    logits = -torch.cumsum(rand(n, k) * 1.5, dim=1) + 12.0          # a teacher's sorted logits
    temperature = 1.0 if case["kind"] == "xent" else 2.0
    lean = torch.softmax(logits / temperature, dim=1)
    towards = (w[ids.reshape(-1)].float().reshape(n, k, h) * lean[:, :, None]).sum(1)
    x = (randn(n, h) + rand(n, 1) * 9.0 * towards).to(dt)
    state = dict(kind=case["kind"], grads=case["grads"], x=x, w=w, temperature=temperature)
    if case["kind"] == "xent":
        targets = ids[:, 0].clone()
        if n > 1:
            targets[rand(n) < 0.1] = IGNORE                         # prompt and padding tokens
        state.update(targets=targets)
    else:
        empty = rand(n, k) < 0.05
        if n > 1:
            empty |= rand(n, 1) < 0.05                              # tokens that the teacher says nothing about
        state.update(ids=torch.where(empty, -1, ids), logits=logits.to(dt))
    return state


def run(state):
    x, w = state["x"], state["w"]
    if own:
        from paper_2607_05895_amd import native
        n = x.shape[0]
        loss = torch.empty((), dtype=torch.float32, device=x.device)
        token_loss = torch.empty(n, dtype=torch.float32, device=x.device)
        dx = torch.empty_like(x) if state["grads"] else None
        dw = torch.empty_like(w) if state["grads"] else None
        if state["kind"] == "xent":
            native.linear_xent_t(x, w, state["targets"], loss=loss, token_loss=token_loss, dx=dx, dw=dw,
                                 ignore_index=IGNORE, reduction="mean")
        else:
            native.linear_distill_t(x, w, state["ids"], state["logits"], loss=loss, token_loss=token_loss, dx=dx, dw=dw,
                                    temperature=state["temperature"], reduction="mean")
        out = dict(loss=loss, token_loss=token_loss)
        if state["grads"]:
            out.update(dx=dx, dw=dw)
        return out
    x32, w32 = x.float(), w.float()
    z = x32 @ w32.t() / state["temperature"]
    # the softmax's sum without its largest term, which is 1: a token that the model is sure of has a loss, and a gradient,
    # far below the last bit of that 1
    top, at = z.max(1, keepdim=True)
    e = torch.exp(z - top)
    rest = e.scatter(1, at, 0.0).sum(1, keepdim=True)
    if state["kind"] == "xent":
        valid = state["targets"] != IGNORE
        ids = torch.where(valid, state["targets"], 0)[:, None]
        q = valid.float()[:, None]
        log_q = torch.zeros_like(q)
    else:
        filled = state["ids"] >= 0
        valid = filled.any(1)
        ids = torch.where(filled, state["ids"], 0)
        t = torch.where(filled, state["logits"].float() / state["temperature"], -torch.inf)
        t = t - torch.where(valid, t.amax(1), 0.0)[:, None]
        q = torch.exp(t) / torch.where(valid, torch.exp(t).sum(1), 1.0)[:, None]
        log_q = torch.where(q > 0, torch.log(torch.where(q > 0, q, 1.0)), 0.0)
    z_ids = z.gather(1, ids)
    token_loss = torch.where(valid, (q * (log_q + (top - z_ids))).sum(1) + torch.log1p(rest[:, 0]), 0.0)
    count = valid.sum().clamp(min=1).float()
    out = dict(loss=token_loss.sum() / count, token_loss=token_loss)
    if state["grads"]:
        q_ids = torch.zeros_like(z).scatter_add(1, ids, q).gather(1, ids)        # of an id that fills several slots
        dz_ids = torch.expm1(z_ids - top) + (1 - q_ids) - q_ids * rest
        dz = e.scatter(1, ids, dz_ids) / (1 + rest)
        dz = torch.where(valid[:, None], dz, 0.0) / (count * state["temperature"])
        out.update(dx=(dz @ w32).to(x.dtype), dw=(dz.t() @ x32).to(w.dtype))
    return out


def work(case):
    n, v, h, k, grads = case["n"], case["v"], case["h"], case["k"], case["grads"]
    size = 2 if case["dtype"] == "bf16" else 4
    per_slot = 8 if case["kind"] == "xent" else 8 + size
    return {"bytes": (1 + grads) * (n + v) * h * size + n * k * per_slot + 4 * n + 4, "flops": (6 if grads else 2) * n * v * h}


def exact(case, seed):
    """The definition in 64 bits: log-probabilities of blocks of tokens, the gradients by differentiating the loss."""
    state = prepare(case, seed)
    w = state["w"].double().requires_grad_(case["grads"])
    n, rows = case["n"], max(1, (1 << 27) // case["v"])
    if state["kind"] == "xent":
        labelled = state["targets"] != IGNORE
    else:
        labelled = (state["ids"] >= 0).sum(1) > 0
    count = max(1, int(labelled.sum()))
    token_loss, dx, dw = [], [], torch.zeros_like(w) if case["grads"] else None
    for at in range(0, n, rows):
        part = slice(at, min(n, at + rows))
        x = state["x"][part].double().requires_grad_(case["grads"])
        logp = torch.log_softmax(torch.matmul(x, w.T) / state["temperature"], dim=-1)
        if state["kind"] == "xent":
            loss = -logp[torch.arange(x.shape[0], device=x.device), state["targets"][part].clamp(min=0)]
        else:
            empty = state["ids"][part] < 0
            teacher = (state["logits"][part].double() / state["temperature"]).masked_fill(empty, -1e300)
            log_q = torch.log_softmax(teacher, dim=-1)
            terms = log_q.exp() * (log_q - torch.take_along_dim(logp, state["ids"][part].clamp(min=0), 1))
            loss = terms.masked_fill(empty, 0.0).sum(-1)
        loss = loss * labelled[part]
        token_loss.append(loss.detach())
        if case["grads"]:
            gx, gw = torch.autograd.grad(loss.sum() / count, (x, w))
            dx.append(gx)
            dw += gw
    token_loss = torch.cat(token_loss)
    out = dict(loss=token_loss.sum() / count, token_loss=token_loss)
    if case["grads"]:
        out.update(dx=torch.cat(dx), dw=dw)
    return out
