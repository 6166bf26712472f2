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
"""

from __future__ import annotations

import math
from dataclasses import dataclass

import torch
import torch.nn as nn
import torch.nn.functional as F

from . import lm_ops
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


class Block(nn.Module):
    def __init__(self, c: GPTConfig):
        super().__init__()
        self.c = c
        self.ln1 = nn.LayerNorm(c.D)
        self.mix = Mixer(c)
        self.ln2 = nn.LayerNorm(c.D)
        self.fc1 = nn.Linear(c.D, c.mlp)
        self.fc2 = nn.Linear(c.mlp, c.D)

    def forward(self, x, drop=None):
        """drop(branch, residual, site): the branch with dropout, plus the residual."""
        if drop is not None:
            x = drop(self.mix(self.ln1(x)), x, 0)
            return drop(self.mlp(x), x, 1)
        x = x + self.mix(self.ln1(x))
        return x + self.mlp(x)

    def mlp(self, x):
        return self.fc2(F.gelu(self.fc1(self.ln2(x))))

    def recurrent(self, x, state, lengths=None, drop=None):
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
        self.tok = nn.Embedding(c.vocab, c.D)
        self.pos = nn.Parameter(torch.randn(c.T, c.D) * 0.02)
        self.blocks = nn.ModuleList(Block(c) for _ in range(c.layers))
        self.ln_f = nn.LayerNorm(c.D)
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
        for blk, drop in zip(self.blocks, drops):
            x = blk(x) if drop is None else blk(x, drop)
        return self.head(self.ln_f(x))

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
        for i, (blk, drop) in enumerate(zip(self.blocks, drops)):
            x, s = blk.recurrent(x, None if states is None else states[i], lengths, drop)
            out.append(s)
        return self.head(self.ln_f(x)), out


def build(c: GPTConfig, device="cuda", dtype=torch.bfloat16, seed: int = 0) -> GPT:
    torch.manual_seed(seed)
    return GPT(c).to(device=device, dtype=dtype)


def make_optimizer(model: GPT, lr: float = 3e-4):
    return torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.1,
                             fused=next(model.parameters()).is_cuda)


def train_step(model: GPT, opt, ids, targets):
    """One optimisation step on next-token cross-entropy; returns the loss tensor."""
    logits = model(ids)
    loss = F.cross_entropy(logits.reshape(-1, logits.shape[-1]), targets.reshape(-1))
    loss.backward()
    opt.step()
    opt.zero_grad(set_to_none=True)
    if model.c.mixer == "bcmt" and model.c.learn_decay:
        with torch.no_grad():
            for blk in model.blocks:
                blk.mix.decay.clamp_(0.0, 0.999)
    return loss


@torch.no_grad()
def generate(model: GPT, ids, new_tokens: int, lengths=None):
    """Greedy continuation of the prompts ids [B, n] (``mixer="linear"``): the
    prompts in one pass, then one token of every sequence per step.  lengths [B]
    int32: the prompts' own lengths (default n, each at least 1); positions past
    the model's T share its last position embedding.  Returns
    [B, new_tokens].  What has no meaning (a prompt of no token, a length that is
    not in 1 .. n) raises ValueError."""
    B, n = ids.shape
    if model.c.mixer != "linear":
        raise ValueError(f"mixer {model.c.mixer!r} has no recurrent form")
    if n < 1 or new_tokens < 0:
        raise ValueError(f"prompts must have a token and new_tokens be >= 0 (got {n}, {new_tokens})")
    if lengths is not None:
        # read back here: a length past the prompts would index past their logits
        if lengths.shape != (B,) or not all(1 <= x <= n for x in lengths.tolist()):
            raise ValueError(f"lengths must be [{B}], each in 1 .. {n}")
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
