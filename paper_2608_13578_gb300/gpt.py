"""A GPT-style decoder whose token mixer is the BCMT layer (Sec. 3), for
whole-model training steps.

The model follows the setting the paper trains (Sec. 4.1): a decoder-only
language model with learned absolute position embeddings, pre-LayerNorm
residual blocks (mixer, then a GELU MLP), a final LayerNorm, an untied LM head
and next-token cross-entropy, trained with AdamW.  The paper does not print its
block wiring; these are the standard choices, named as readings in the design
notes.  Only the mixer is this library: ``BCMTMixer`` calls the C ABI's forward
and backward kernels.  Embeddings (but see ``embed_scale``), LayerNorm, MLP, LM head,
loss and optimizer are PyTorch's own CUDA kernels.

``mixer="dense"`` swaps in ordinary dense causal attention of the same shape
(x W_qkv -> PyTorch SDPA with a causal mask -> W_O), the baseline the paper
compares against; ``honly=True`` is the HOnly ablation of Sec. 4.5 (no block
summaries and no memory: Y = H).  ``mixer="linear"`` is linear attention with a
decay per head (BCMT's exponential memory taken per token), by the library's
operators; its state makes the model a recurrent one, so ``generate`` reads a
batch of prompts in one pass and then decodes token by token at a cost that does
not grow with the length.

``embed_scale`` and ``dropout`` put the library's scaled embedding (with its
gradient by sorted tokens) and its counter-based dropout in place of PyTorch's
embedding and of no dropout; both are off by default.  The masks come from a counter
that every call in training mode moves on, and that is saved with the model.

``block_norm="layer"`` or ``"rms"`` ends each branch in one call of the library: the
branch's norm (``post_norm``) and gate (``branch_gate``, learned per channel), the
addition to the scaled residual, and the norm that the next branch starts with; the
names of the weights are those of PyTorch's norms.  ``make_optimizer(bits=...)`` gives
the library's AdamW, and ``beam_search`` is generation by its beam search.
"""

from __future__ import annotations

import math
from dataclasses import dataclass

import torch
import torch.nn as nn
import torch.nn.functional as F

from . import beam, lm_ops, norms, optim
from .layer import BCMTMixer


@dataclass(frozen=True)
class GPTConfig:
    vocab: int = 32000
    D: int = 512
    H: int = 8
    layers: int = 6
    mlp: int = 2048
    L: int = 64
    T: int = 1024
    mixer: str = "bcmt"          # "bcmt", "dense" or "linear"
    honly: bool = False
    decay: float = 0.8           # broadcast per-channel decay (Sec. 3.5)
    learn_decay: bool = False    # learned per-channel decay (Sec. 5, future work)
    embed_scale: float = 0.0     # > 0: the library's embedding, rows times this
    dropout: float = 0.0         # > 0: after the embedding and on both branches of a block
    dropout_seed: int = 0
    block_norm: str = ""         # "layer" or "rms": the library's norms around a block
    post_norm: bool = False      # a norm at the end of each branch, of the same kind
    branch_gate: float = 0.0     # > 0: a learned gate per channel on each branch, from this value
    residual_scale: float = 1.0  # what the residual is multiplied by at each addition


class Mixer(nn.Module):
    """The token mixer of one block: BCMT (Sec. 3.3-3.8), dense causal attention
    or linear attention with a decay per head."""

    def __init__(self, c: GPTConfig):
        super().__init__()
        D = c.D
        self.c = c
        std = 1.0 / math.sqrt(D)   # weights ~ N(0, 1/D)
        self.w_qkv = nn.Parameter(torch.randn(D, 3 * D) * std)
        self.w_o = nn.Parameter(torch.randn(D, D) * std)
        if c.mixer == "bcmt":
            self.w_p = nn.Parameter(torch.randn(D) * std)
            self.w_m = nn.Parameter(torch.randn(D, D) * std)
            self.w_g = nn.Parameter(torch.randn(D, D) * std)
            decay = torch.full((D,), c.decay, dtype=torch.float32)
            if c.learn_decay:
                self.decay = nn.Parameter(decay)
            else:
                self.register_buffer("decay", decay)
        elif c.mixer == "linear":
            # memories of about 32 to 512 tokens, in powers of two over the heads
            e = torch.linspace(5.0, 9.0, c.H) if c.H > 1 else torch.tensor([6.0])
            self.register_buffer("decay", 1.0 - torch.exp2(-e))
        elif c.mixer != "dense":
            raise ValueError(f"unknown mixer {c.mixer!r}")

    def _apply(self, fn, *args, **kwargs):
        # the decay stays fp32 whatever dtype the rest of the model takes (near 1
        # it would not survive bf16 and back)
        kept = self.decay.detach() if self.c.mixer == "linear" else None
        out = super()._apply(fn, *args, **kwargs)
        if kept is not None and self.decay.dtype != torch.float32:
            self.decay = kept.to(self.decay.device)
        if self.c.mixer == "bcmt" and self.decay.dtype != torch.float32:
            self.decay.data = self.decay.data.float()
        return out

    def forward(self, x):
        c = self.c
        if c.mixer == "bcmt":
            return BCMTMixer.apply(x, self.w_qkv, self.w_o, self.w_p, self.w_m, self.w_g,
                                   self.decay, c.L, c.H, c.honly)
        if c.mixer == "linear":
            return self.recurrent(x)[0]
        B, T, D = x.shape
        q, k, v = (x @ self.w_qkv).view(B, T, 3, c.H, D // c.H).permute(2, 0, 3, 1, 4)
        o = F.scaled_dot_product_attention(q, k, v, is_causal=True)
        return o.transpose(1, 2).reshape(B, T, D) @ self.w_o


    def recurrent(self, x, state=None, lengths=None):
        """Linear attention from a state [B, H, dh, dh] (None: from nothing):
        (output rows, last state).  lengths [B] int32: tokens per sequence."""
        B, T, D = x.shape
        q, k, v = (x @ self.w_qkv).view(B, T, 3, self.c.H, D // self.c.H).unbind(2)
        o, state = lm_ops.linear_attention(q, k, v, self.decay, lengths=lengths, state=state)
        return o.reshape(B, T, D) @ self.w_o, state


def _norm(c: GPTConfig):
    return nn.RMSNorm(c.D, eps=1e-5) if c.block_norm == "rms" else nn.LayerNorm(c.D)


class Block(nn.Module):
    def __init__(self, c: GPTConfig):
        super().__init__()
        self.c = c
        self.ln1 = _norm(c)
        self.mix = Mixer(c)
        self.ln2 = _norm(c)
        self.fc1 = nn.Linear(c.D, c.mlp)
        self.fc2 = nn.Linear(c.mlp, c.D)
        if c.post_norm:
            self.post1, self.post2 = _norm(c), _norm(c)
        if c.branch_gate > 0:
            self.gate1, self.gate2 = (nn.Parameter(torch.full((c.D,), c.branch_gate))
                                      for _ in range(2))

    def forward(self, x, drop=None, n=None, following=None):
        """drop(branch, residual, site): the branch with dropout, plus the residual.
        With the library's norms: n is this block's first norm of x, and the result (x, the
        norm of x by the module ``following``)."""
        if following is not None:
            return self._fused(x, self.mix(n), following, drop)
        if drop is not None:
            x = drop(self.mix(self.ln1(x)), x, 0)
            return drop(self.mlp(x), x, 1)
        x = x + self.mix(self.ln1(x))
        return x + self.mlp(x)

    def mlp(self, x):
        return self._mlp(self.ln2(x))

    def _mlp(self, n):
        return self.fc2(F.gelu(self.fc1(n)))

    def _end(self, branch, x, following, site, drop):
        """(residual, its norm by the module ``following``) after a branch."""
        if drop is not None:
            branch = drop(branch, None, site)
        post = getattr(self, f"post{site + 1}", None)
        return norms.residual_norm(
            branch, x, following.weight, getattr(following, "bias", None),
            post_weight=None if post is None else post.weight,
            post_bias=getattr(post, "bias", None), gate=getattr(self, f"gate{site + 1}", None),
            residual_scale=self.c.residual_scale, kind=self.c.block_norm, eps=following.eps)

    def _fused(self, x, branch, following, drop):
        x, n = self._end(branch, x, self.ln2, 0, drop)
        return self._end(self._mlp(n), x, following, 1, drop)

    def recurrent(self, x, state, lengths=None, drop=None, n=None, following=None):
        if following is not None:
            m, state = self.mix.recurrent(n, state, lengths)
            return *self._fused(x, m, following, drop), state
        m, state = self.mix.recurrent(self.ln1(x), state, lengths)
        if drop is not None:
            x = drop(m, x, 0)
            return drop(self.mlp(x), x, 1), state
        x = x + m
        return x + self.mlp(x), state


class GPT(nn.Module):
    def __init__(self, c: GPTConfig):
        super().__init__()
        self.c = c
        if c.block_norm not in ("",) + norms.KINDS:
            raise ValueError(f"block_norm must be empty or one of {norms.KINDS}, not {c.block_norm!r}")
        if not c.block_norm and (c.post_norm or c.branch_gate > 0 or c.residual_scale != 1.0):
            raise ValueError("post_norm, branch_gate and residual_scale need a block_norm")
        self.tok = nn.Embedding(c.vocab, c.D)
        self.pos = nn.Parameter(torch.randn(c.T, c.D) * 0.02)
        self.blocks = nn.ModuleList(Block(c) for _ in range(c.layers))
        self.ln_f = _norm(c)
        self.head = nn.Linear(c.D, c.vocab, bias=False)
        # calls that drew masks so far: part of the dropout's counter, on the device so
        # that a captured call draws new masks at each replay.  Saved where it is used, so
        # that a resumed run goes on with new masks
        self.register_buffer("drop_step", torch.zeros(1, dtype=torch.int64),
                             persistent=c.dropout > 0)

    def _load_from_state_dict(self, state_dict, prefix, *args):
        # weights are shared between models with and without dropout, and with files
        # that hold no counter
        key, own = prefix + "drop_step", dict(state_dict)
        if self.c.dropout > 0:
            own.setdefault(key, self.drop_step)
        else:
            own.pop(key, None)
        super()._load_from_state_dict(own, prefix, *args)

    def embed(self, ids):
        if self.c.embed_scale > 0:
            return lm_ops.embedding(ids, self.tok.weight, self.c.embed_scale)
        return self.tok(ids)

    def _masks(self):
        """The dropout of one call of the model: drop(x, residual, site).  Every call has
        masks of its own; a site's mask can be drawn again (a block run anew for its
        backward), since the call keeps its own copy of the counter."""
        step = self.drop_step.clone()
        self.drop_step += 1
        # places are 2^40 steps apart in the counter's upper half
        return lambda x, residual, site: lm_ops.dropout(
            x, self.c.dropout, self.c.dropout_seed, site << 40, residual=residual, step=step)

    def _start(self, x):
        """In training with dropout: (x with it, each block's drop); else (x, Nones)."""
        if not (self.training and self.c.dropout > 0):
            return x, [None] * len(self.blocks)
        drop = self._masks()
        return drop(x, None, 0), [lambda y, res, s, i=i: drop(y, res, 1 + 2 * i + s)
                                  for i in range(len(self.blocks))]

    def forward(self, ids):
        x, drops = self._start(self.embed(ids) + self.pos[: ids.shape[1]])
        if self.c.block_norm:
            first, after = self._norms()
            n = first(x)
            for blk, drop, following in zip(self.blocks, drops, after):
                x, n = blk(x, drop, n, following)
            return self.head(n)
        for blk, drop in zip(self.blocks, drops):
            x = blk(x) if drop is None else blk(x, drop)
        return self.head(self.ln_f(x))

    def _norms(self):
        """The first norm of the model and those that follow each block."""
        every = [blk.ln1 for blk in self.blocks] + [self.ln_f]
        return every[0], every[1:]

    def recurrent(self, ids, pos, states=None, lengths=None):
        """The model as a recurrence (``mixer="linear"``): tokens ids [B, n] at
        positions pos[b] .. pos[b] + n - 1 on top of the states of an earlier call
        (None: from nothing); lengths [B] int32: valid tokens of each row of ids.
        Dropout as in ``forward``: in training mode, with masks of this call's own.
        Returns (logits [B, n, vocab], states)."""
        if self.c.mixer != "linear":
            raise ValueError(f"mixer {self.c.mixer!r} has no recurrent form")
        at = pos[:, None] + torch.arange(ids.shape[1], device=ids.device)
        x, drops = self._start(self.embed(ids) + self.pos[at.clamp(max=self.c.T - 1)])
        out = []
        if self.c.block_norm:
            first, after = self._norms()
            n = first(x)
            for i, (blk, drop, following) in enumerate(zip(self.blocks, drops, after)):
                x, n, s = blk.recurrent(x, None if states is None else states[i], lengths, drop,
                                        n, following)
                out.append(s)
            return self.head(n), out
        for i, (blk, drop) in enumerate(zip(self.blocks, drops)):
            x, s = blk.recurrent(x, None if states is None else states[i], lengths, drop)
            out.append(s)
        return self.head(self.ln_f(x)), out


def build(c: GPTConfig, device="cuda", dtype=torch.bfloat16, seed: int = 0) -> GPT:
    torch.manual_seed(seed)
    return GPT(c).to(device=device, dtype=dtype)


def make_optimizer(model: GPT, lr: float = 3e-4, bits: int = 0, masters: bool = False):
    """AdamW: PyTorch's, or (bits 32 or 8) the library's with states of so many bits and,
    with masters, float32 values of bf16 weights."""
    if bits:
        return optim.AdamW(model.parameters(), lr=lr, weight_decay=0.1, bits=bits, masters=masters)
    if masters:
        raise ValueError("masters are kept by the library's optimizer: bits must be 32 or 8")
    return torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.1,
                             fused=next(model.parameters()).is_cuda)


def _clip_scale(params, clip: float):
    """clip / the gradients' norm where that is below 1, else 1: one float32 on the device."""
    # (float32 norms: those of bf16 gradients would be rounded to bf16, 8 bits)
    each = torch._foreach_norm([p.grad for p in params if p.grad is not None], 2, torch.float32)
    norm = torch.linalg.vector_norm(torch.stack(each))
    return (clip / (norm + 1e-6)).clamp(max=1.0)


def train_step(model: GPT, opt, ids, targets, clip: float = 0.0):
    """One optimisation step on next-token cross-entropy; returns the loss tensor.  clip > 0:
    gradients are scaled down to this norm (within the step of the library's optimizer)."""
    logits = model(ids)
    loss = F.cross_entropy(logits.reshape(-1, logits.shape[-1]), targets.reshape(-1))
    loss.backward()
    if clip > 0 and isinstance(opt, optim.AdamW):
        opt.step(grad_scale=_clip_scale(model.parameters(), clip))
    else:
        if clip > 0:
            torch.nn.utils.clip_grad_norm_(model.parameters(), clip)
        opt.step()
    opt.zero_grad(set_to_none=True)
    if model.c.mixer == "bcmt" and model.c.learn_decay:
        with torch.no_grad():
            for blk in model.blocks:
                blk.mix.decay.clamp_(0.0, 0.999)
    return loss


def _prompts(model, ids, new_tokens, lengths):
    """(sequences, tokens) of the prompts, after the checks of a generation."""
    B, n = ids.shape
    if model.c.mixer != "linear":
        raise ValueError(f"mixer {model.c.mixer!r} has no recurrent form")
    if n < 1 or new_tokens < 0:
        raise ValueError(f"prompts must have a token and new_tokens be >= 0 (got {n}, {new_tokens})")
    if lengths is not None:
        # read back here: a length past the prompts would index past their logits
        if lengths.shape != (B,) or not all(1 <= x <= n for x in lengths.tolist()):
            raise ValueError(f"lengths must be [{B}], each in 1 .. {n}")
    return B, n


@torch.no_grad()
def generate(model: GPT, ids, new_tokens: int, lengths=None):
    """Greedy continuation of the prompts ids [B, n] (``mixer="linear"``): the
    prompts in one pass, then one token of every sequence per step.  lengths [B]
    int32: the prompts' own lengths (default n, each at least 1); positions past
    the model's T share its last position embedding.  Returns
    [B, new_tokens].  What has no meaning (a prompt of no token, a length that is
    not in 1 .. n) raises ValueError."""
    B, n = _prompts(model, ids, new_tokens, lengths)
    if new_tokens == 0:
        return ids.new_empty(B, 0)
    was_training = model.training
    model.eval()
    try:
        pos = torch.zeros(B, dtype=torch.int64, device=ids.device)
        logits, states = model.recurrent(ids, pos, None, lengths)
        last = torch.full_like(pos, n) if lengths is None else lengths.long()
        tok = logits[torch.arange(B, device=ids.device), last - 1].argmax(-1, keepdim=True)
        out = [tok]
        for i in range(new_tokens - 1):
            logits, states = model.recurrent(tok, last + i, states)
            tok = logits[:, 0].argmax(-1, keepdim=True)
            out.append(tok)
        return torch.cat(out, dim=1)
    finally:
        model.train(was_training)


@torch.no_grad()
def beam_search(model: GPT, ids, new_tokens: int, beams: int, lengths=None, eos=None):
    """The continuations of the prompts that beam search finds (``mixer="linear"``):
    (tokens [B, beams, new_tokens], scores [B, beams]), the best first; a score is the sum
    of its tokens' log probabilities.  A beam that takes the token ``eos`` ends: it keeps its
    score and goes on with eos.  Prompts, lengths and positions as in ``generate``; what has
    no meaning raises ValueError.  Fewer continuations than beams (beams > vocab at the
    first token): the rest have a score of -inf."""
    B, n = _prompts(model, ids, new_tokens, lengths)
    if not 1 <= beams <= 32:
        raise ValueError(f"beams = {beams} must be in 1 .. 32")
    V, dev = model.c.vocab, ids.device
    if eos is not None and not 0 <= eos < V:
        raise ValueError(f"eos = {eos} must be in 0 .. {V - 1}")
    scores = torch.full((B, beams), -math.inf, device=dev)
    scores[:, 0] = 0.0   # one beam to begin with
    if new_tokens == 0 or B == 0:
        return ids.new_empty(B, beams, new_tokens), scores
    was_training = model.training
    model.eval()
    try:
        pos = torch.zeros(B, dtype=torch.int64, device=dev)
        logits, states = model.recurrent(ids, pos, None, lengths)
        last = torch.full_like(pos, n) if lengths is None else lengths.long()
        logits = logits[torch.arange(B, device=dev), last - 1].unsqueeze(1).expand(B, beams, V)
        states = [s.repeat_interleave(beams, 0) for s in states]
        last = last.repeat_interleave(beams)
        ended, steps = None, []
        for i in range(new_tokens):
            if i > 0:
                logits, states = model.recurrent(tokens.view(B * beams, 1), last + (i - 1), states)
                logits = logits.view(B, beams, V)
            scores, parents, tokens, now = beam.beam_select(logits, scores, ended, eos)
            steps.append((parents, tokens))
            ended = None if eos is None else now
            if i + 1 < new_tokens and beams > 1:
                states = beam.beam_reorder(states, parents)
        # the tokens of each beam, from its last one back
        out, at = [], None
        for parents, tokens in reversed(steps):
            out.append(tokens if at is None else tokens.gather(1, at))
            at = parents if at is None else parents.gather(1, at)
        return torch.stack(out[::-1], dim=2), scores
    finally:
        model.train(was_training)


def flops_per_token(c: GPTConfig) -> float:
    """Algorithmic forward+backward flops per token (3x the forward): the
    mixer's 10 D^2 + 2 D (L+1) + 2 D^2 / L (dense: L -> T; HOnly: no W_m, W_g;
    linear: 8 D^2 + 4 D dh for the state's update and its use), the MLP's 4 D m
    and the LM head's 2 D V."""
    D, L = c.D, (c.T if c.mixer == "dense" else c.L)
    mix = 8 * D * D + (4 * D * (D // c.H) if c.mixer == "linear" else 2 * D * (L + 1))
    if c.mixer == "bcmt" and not c.honly:
        mix += 2 * D * D + 2 * D * D / c.L
    return 3.0 * (c.layers * (mix + 4 * D * c.mlp) + 2 * D * c.vocab)
