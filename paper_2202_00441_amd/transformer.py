"""A transformer block whose training keeps little: few-bit activations in the
feed-forward part, attention that recomputes its probabilities, norms and rotary
positions that are recomputed from their inputs, dropout without masks, and AdamW
moments in 8 bits; and the same block served with its products in 8-bit integers.

    python -m paper_2202_00441_amd.transformer --layers 4 --width 1024 --heads 8 --kv-heads 2 --steps 20

trains a small stack on a synthetic task (predicting the next of a sequence of
tokens, each a fixed function of the two before) and prints the loss, the time per
step, the bytes that autograd and the optimizer hold, and a few greedily generated
tokens.
"""
from __future__ import annotations

import argparse
import copy
import json
import time

import torch
import torch.nn.functional as F

from .autograd import FewBitAct
from .block import attention, attention_fwd, qk_norm_rope, qk_norm_rope_fwd, rope_tables
from .optim import AdamW
from .residual import (Int8Linear, _drops, draw_seed, residual_norm, residual_norm_fwd,
                       residual_norm_int8)


class Cache:
    """Keys and values of every layer for up to `most` tokens of each sequence.  `lengths` has how many
    there are of each, on the device; `used`, known on the host, is what none of them passes."""

    def __init__(self, layers: int, batch: int, most: int, kv_heads: int, head_dim: int, dtype, device):
        shape = layers, batch, most, kv_heads, head_dim
        self.k, self.v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=device)
        self.batch, self.most, self.used = batch, most, 0


def _eps(norm: torch.nn.RMSNorm) -> float:
    """What the norm adds to the mean square; without a number of its own torch's takes fp32's step for 16-bit types too."""
    return torch.finfo(torch.promote_types(norm.weight.dtype, torch.float32)).eps if norm.eps is None else norm.eps


class Block(torch.nn.Module):
    """x + attention(norm(x)), then x + feed-forward(norm(x))."""

    def __init__(self, width: int, heads: int, kv_heads: int, hidden: int, act: torch.nn.Module):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, width // heads
        self.norm1, self.norm2 = torch.nn.RMSNorm(width), torch.nn.RMSNorm(width)
        self.qkv = torch.nn.Linear(width, (heads + 2 * kv_heads) * self.head_dim, bias=False)
        self.q_norm, self.k_norm = (torch.nn.Parameter(torch.ones(self.head_dim)) for _ in range(2))
        self.out = torch.nn.Linear(width, width, bias=False)
        self.up, self.act, self.down = torch.nn.Linear(width, hidden), act, torch.nn.Linear(hidden, width)

    def _heads(self, x):
        """Queries, keys and values: views of one projection."""
        return self.qkv(self.norm1(x)).unflatten(-1, (-1, self.head_dim)).split((self.heads, self.kv_heads, self.kv_heads), -2)

    def _rest(self, x, attended):
        x = x + self.out(attended.flatten(-2))
        return x + self.down(self.act(self.up(self.norm2(x))))

    def forward(self, x, cos, sin):
        q, k, v = self._heads(x)
        q, k = qk_norm_rope(q, k, self.q_norm, self.k_norm, cos, sin)
        return self._rest(x, attention(q, k, v, causal=True))

    def step(self, h, branch, cos, sin, p: float, seed, site: int):
        """The block on a residual stream h (None before the first) that the last branch has yet to be added
        to: dropout, addition and norm in one pass.  The stream and its new last branch; takes sites `site`
        and `site` + 1 of the seed."""
        h, y = residual_norm(branch, h, self.norm1.weight, _eps(self.norm1), p, seed, site)
        q, k, v = self.qkv(y).unflatten(-1, (-1, self.head_dim)).split((self.heads, self.kv_heads, self.kv_heads), -2)
        q, k = qk_norm_rope(q, k, self.q_norm, self.k_norm, cos, sin)
        branch = self.out(attention(q, k, v, causal=True).flatten(-2))
        h, y = residual_norm(branch, h, self.norm2.weight, _eps(self.norm2), p, seed, site + 1)
        return h, self.down(self.act(self.up(y)))

    def extend(self, x, cos, sin, cache: Cache, layer: int, at):
        """New tokens x [batch, new, width], the first of sequence b at place at[b] of the cache."""
        return self._rest(x, self._attend(*self._heads(x), cos, sin, cache, layer, at))

    def _attend(self, q, k, v, cos, sin, cache: Cache, layer: int, at):
        """Attention of new tokens over the cache, which takes up their keys and values."""
        places = at[:, None].long() + torch.arange(q.shape[1], device=q.device)
        q, k = qk_norm_rope_fwd(q, k, self.q_norm, self.k_norm, cos, sin, places)
        rows = torch.arange(q.shape[0], device=q.device)[:, None]
        cache.k[layer][rows, places] = k
        cache.v[layer][rows, places] = v
        attended, _ = attention_fwd(q, cache.k[layer], cache.v[layer], causal=True, k_len=at + q.shape[1])
        return attended


def _alias(module: torch.nn.Module) -> torch.nn.Module:
    """A module without children on the same memory, with parameters of its own: converting or moving one of the two
    leaves the other as it is."""
    other = copy.copy(module)
    other._parameters = {name: None if p is None else _alias_parameter(p) for name, p in module._parameters.items()}
    return other


def _alias_parameter(p: torch.nn.Parameter) -> torch.nn.Parameter:
    return torch.nn.Parameter(p.detach(), p.requires_grad)


class Int8Block(Block):
    """A block for serving: its four products in 8-bit integers, each from tokens that are laid out in 8 bits
    where they arise (by the norm, or by quantize_rows after attention and activation)."""

    def __init__(self, block: Block):
        torch.nn.Module.__init__(self)
        self.heads, self.kv_heads, self.head_dim = block.heads, block.kv_heads, block.head_dim
        self.norm1, self.norm2 = _alias(block.norm1), _alias(block.norm2)
        self.q_norm, self.k_norm = _alias_parameter(block.q_norm), _alias_parameter(block.k_norm)
        name = _act_name(block.act)
        self.qkv, self.out = Int8Linear(block.qkv), Int8Linear(block.out)
        self.up, self.down = Int8Linear(block.up, name), Int8Linear(block.down)
        self.act = torch.nn.Identity() if name else block.act       # else it is in the product's epilogue

    def forward(self, *args):
        raise RuntimeError("a block in 8-bit integers is for serving: extend")

    step = forward

    def extend(self, h, branch, cos, sin, cache: Cache, layer: int, at):
        """New tokens, as in Block.step; the stream and its last branch."""
        h, codes, scale = residual_norm_int8(branch, h, self.norm1.weight, _eps(self.norm1))
        heads = self.qkv(codes, scale).unflatten(-1, (-1, self.head_dim)).split((self.heads, self.kv_heads, self.kv_heads), -2)
        branch = self.out(self._attend(*heads, cos, sin, cache, layer, at).flatten(-2))
        h, codes, scale = residual_norm_int8(branch, h, self.norm2.weight, _eps(self.norm2))
        return h, self.down(self.act(self.up(codes, scale)))


def _act_name(act):
    """The activation's name where int8_linear forms it."""
    if isinstance(act, FewBitAct):
        return act.act if act.act in ("gelu", "silu") else None
    if isinstance(act, torch.nn.GELU) and act.approximate == "none":
        return "gelu"
    return "silu" if isinstance(act, torch.nn.SiLU) else None


class Transformer(torch.nn.Module):
    def __init__(self, tokens: int, width: int, layers: int, heads: int, kv_heads: int, hidden: int | None = None,
                 act: str = "gelu", bits: int | None = 3, most: int = 4096, dropout: float | None = None):
        """bits: of the few-bit activation; None: torch's own, which keeps its input.  dropout: of the
        embeddings and of every branch before it is added; a number, 0 too, takes dropout, addition and norm
        in one pass, None has torch's norms and no dropout."""
        super().__init__()
        few = FewBitAct(act, bits) if bits is not None else {"gelu": torch.nn.GELU, "silu": torch.nn.SiLU}[act]()
        self.embed = torch.nn.Embedding(tokens, width)
        self.blocks = torch.nn.ModuleList(Block(width, heads, kv_heads, hidden or 4 * width, few) for _ in range(layers))
        self.norm, self.head = torch.nn.RMSNorm(width), torch.nn.Linear(width, tokens, bias=False)
        self.most, self.dropout = most, dropout
        if dropout is not None and not 0.0 <= dropout <= 1.0:
            raise ValueError("dropout must be between 0 and 1")
        self._tables = None

    def _check_positions(self, n: int):
        if n > self.most:
            raise ValueError(f"the model has {self.most} positions, {n} are needed")

    def tables(self, device):
        if self._tables is None or self._tables[0].device != device:
            with torch.inference_mode(False):       # a later backward reads them too
                self._tables = rope_tables(self.most, self.blocks[0].head_dim, device=device)
        return self._tables

    def forward(self, tokens, seed=None):
        """Logits.  seed: of the dropout in training, a whole number or an int64 tensor of one element on
        the device (for captured graphs); without, one is drawn from torch's generator of the host."""
        self._check_positions(tokens.shape[1])
        x = self.embed(tokens)
        cos, sin = self.tables(x.device)
        if self.dropout is not None:
            p = self.dropout if self.training else 0.0
            seed = 0 if not _drops(p) else draw_seed() if seed is None else seed
            h = None
            for i, b in enumerate(self.blocks):
                h, x = b.step(h, x, cos, sin, p, seed, 2 * i)
            return self.head(residual_norm(x, h, self.norm.weight, _eps(self.norm), p, seed, 2 * len(self.blocks))[1])
        for b in self.blocks:
            x = b(x, cos, sin)
        return self.head(self.norm(x))

    def cache(self, batch: int, most: int) -> Cache:
        b, w = self.blocks[0], self.embed.weight
        return Cache(len(self.blocks), batch, most, b.kv_heads, b.head_dim, w.dtype, w.device)

    @torch.no_grad()
    def extend(self, tokens, cache: Cache):
        """Logits of new tokens [batch, new] after those in the cache, which takes them up."""
        if tokens.shape[1] == 0:
            raise ValueError("no tokens to extend with")
        if tokens.shape[0] != cache.batch:
            raise ValueError(f"the cache is of {cache.batch} sequences, not {tokens.shape[0]}")
        used = cache.used + tokens.shape[1]
        if used > cache.most:
            raise ValueError(f"the cache holds {cache.most} tokens of a sequence, {used} are needed")
        self._check_positions(used)
        x = self._extend(self.embed(tokens), cache)
        cache.lengths += tokens.shape[1]
        cache.used = used
        return self.head(x)

    def _extend(self, x, cache: Cache):
        """What the head takes, of new tokens' embeddings."""
        cos, sin = self.tables(x.device)
        for i, b in enumerate(self.blocks):
            x = b.extend(x, cos, sin, cache, i, cache.lengths)
        return self.norm(x)

    @torch.no_grad()
    def generate(self, tokens, new: int):
        """`new` tokens after each sequence of tokens [batch, prompt], greedily."""
        self._check_positions(tokens.shape[1] + new - 1)
        cache = self.cache(tokens.shape[0], tokens.shape[1] + new)
        out = [tokens[:, :0]]
        for _ in range(new):
            tokens = self.extend(tokens, cache)[:, -1:].float().argmax(-1)
            out.append(tokens)
        return torch.cat(out, 1)


class Int8Transformer(Transformer):
    """A transformer for serving, the blocks' products in 8-bit integers; embeddings, norms and head are on the
    model's own memory until one of the two is converted or moved.  cache, extend and generate are as there."""

    def __init__(self, model: Transformer):
        torch.nn.Module.__init__(self)
        self.embed, self.norm, self.head, self.most = _alias(model.embed), _alias(model.norm), _alias(model.head), model.most
        self.blocks = torch.nn.ModuleList(Int8Block(b) for b in model.blocks)
        self._tables = None

    def forward(self, *args):
        raise RuntimeError("a transformer in 8-bit integers is for serving: extend or generate")

    def _extend(self, x, cache: Cache):
        cos, sin = self.tables(x.device)
        h = None
        for i, b in enumerate(self.blocks):
            h, x = b.extend(h, x, cos, sin, cache, i, cache.lengths)
        return residual_norm_fwd(x, h, self.norm.weight, _eps(self.norm))[1]


def synthetic(batch: int, length: int, tokens: int, generator, device):
    """Sequences in which each token is a fixed function of the two before it."""
    x = torch.randint(0, tokens, (batch, length + 1), generator=generator, device=device)
    for i in range(2, length + 1):
        x[:, i] = (3 * x[:, i - 1] + 5 * x[:, i - 2] + 7) % tokens
    return x


def train(steps: int = 20, layers: int = 4, width: int = 1024, heads: int = 8, kv_heads: int = 2, batch: int = 8,
          length: int = 512, tokens: int = 64, bits: int | None = 3, state_bits: int = 8, lr: float = 3e-4,
          dtype=torch.bfloat16, device: str = "cuda", seed: int = 0, dropout: float | None = None) -> dict:
    """Trains the stack; losses, milliseconds per step, bytes held, and the model."""
    torch.manual_seed(seed)
    generator = torch.Generator(device=device).manual_seed(seed)
    model = Transformer(tokens, width, layers, heads, kv_heads, bits=bits, most=length + 64, dropout=dropout).to(device=device, dtype=dtype)
    opt = AdamW(model.parameters(), lr=lr, betas=(0.9, 0.95), weight_decay=0.1, state_bits=state_bits, master=dtype != torch.float32)
    losses, held, began = [], 0, time.perf_counter()
    for i in range(steps):
        x = synthetic(batch, length, tokens, generator, device)
        if i < 2:                   # from the second step on, where there is one
            torch.cuda.synchronize()
            began = time.perf_counter()
        before = torch.cuda.memory_allocated()
        loss = F.cross_entropy(model(x[:, :-1]).flatten(0, 1).float(), x[:, 1:].flatten())
        held = torch.cuda.memory_allocated() - before
        loss.backward()
        opt.step()
        opt.zero_grad(set_to_none=True)
        losses.append(loss.detach())
    torch.cuda.synchronize()
    ms = (time.perf_counter() - began) / max(1, steps - 1) * 1e3
    return {"losses": [float(v) for v in losses], "ms_per_step": ms, "held_for_backward": held, "optimizer_state": opt.state_bytes(),
            "parameters": sum(p.numel() for p in model.parameters()), "model": model}


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("steps", 20), ("layers", 4), ("width", 1024), ("heads", 8), ("kv-heads", 2), ("batch", 8), ("length", 512),
                        ("tokens", 64), ("state-bits", 8)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--bits", type=int, default=3, help="of the activation's codes; 0: torch's own activation")
    p.add_argument("--dropout", type=float, default=None, help="of embeddings and branches; takes addition and norm in one pass with it")
    p.add_argument("--int8", action="store_true", help="generate with the blocks' products in 8-bit integers")
    a = p.parse_args()
    r = train(a.steps, a.layers, a.width, a.heads, a.kv_heads, a.batch, a.length, a.tokens, a.bits or None, a.state_bits, dropout=a.dropout)
    model = r.pop("model")
    if a.int8:
        model = Int8Transformer(model)
    prompt = synthetic(2, 16, a.tokens, torch.Generator(device="cuda").manual_seed(1), "cuda")[:, :16]
    r["generated"] = model.generate(prompt, 8).tolist()
    print(json.dumps(r))


if __name__ == "__main__":
    main()
