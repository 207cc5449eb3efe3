"""AdamW whose moments take 8 bits per element (or 32), stepped by one kernel for
all tensors of a type (block.adamw_step)."""
from __future__ import annotations

import torch

from .block import ADAMW_BLOCK, adamw_blocks, adamw_step

_MOMENTS = {8: torch.float8_e4m3fn, 32: torch.float32}


class AdamW(torch.optim.Optimizer):
    """Adam with decoupled weight decay.

    state_bits: 8 (a byte per moment and element, a power of two per 256, rounded
    with dither) or 32.  master: keep fp32 weights of 16-bit parameters, whose
    rounded copies the parameters then are.  Gradients have the parameters' type or
    fp32; a parameter without one is left as it is, and its steps, by whose number the
    moments are corrected, are those in which it had one.  Steps are counted on the
    host: a step that is captured into a graph repeats its own corrections.

    The moments of a group's parameters of one type and device lie in flat buffers,
    made at the first step; adding a parameter group afterwards gives it buffers of
    its own.
    """

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 state_bits: int = 8, master: bool = False):
        if state_bits not in _MOMENTS:
            raise ValueError("state_bits must be 8 or 32")
        super().__init__(params, {"lr": lr, "betas": betas, "eps": eps, "weight_decay": weight_decay})
        self.state_bits, self.master = state_bits, master
        self._buckets = {}          # (group, dtype, device) -> buffers
        self._steps = 0

    # Copies and pickles have the buffers and counts too; codes go as bytes, since a pickle of torch's
    # does not hold tensors of an 8-bit floating-point type.
    def __getstate__(self) -> dict:
        own = {k: self.__dict__[k] for k in ("state_bits", "master", "_steps")}
        return {**super().__getstate__(), **own, "_buckets": self._viewed(torch.uint8)}

    def __setstate__(self, state: dict) -> None:
        super().__setstate__(state)
        self._buckets = self._viewed(_MOMENTS[8])

    def _viewed(self, dtype) -> dict:
        if self.state_bits != 8:
            return self._buckets
        return {key: {**b, "m": b["m"].view(dtype), "v": b["v"].view(dtype)} for key, b in self._buckets.items()}

    def _bucket(self, key) -> dict:
        """The buffers of a key: those there are, or new ones, which the caller keeps."""
        g, dtype, device = key
        params = [p for p in self.param_groups[g]["params"] if p.dtype == dtype and p.device == device]
        b = self._buckets.get(key)
        if b is not None and len(b["params"]) == len(params) and all(x is y for x, y in zip(b["params"], params)):
            return b
        if b is not None:
            raise RuntimeError("the parameters of a group must stay as they were at its first step")
        blocks = [adamw_blocks(p.numel()) for p in params]
        n, moments = sum(blocks), _MOMENTS[self.state_bits]
        b = {"params": params, "counts": [0] * len(params), "m": torch.zeros(n * ADAMW_BLOCK, device=device).to(moments)}
        b["v"] = torch.zeros_like(b["m"])
        b["ms"] = b["vs"] = b["master"] = None
        if self.state_bits == 8:
            b["ms"], b["vs"] = (torch.full((n,), 2.0 ** -125, device=device) for _ in range(2))
        if self.master and dtype != torch.float32:
            b["master"] = torch.zeros(n * ADAMW_BLOCK, device=device)
            at = 0
            for p, k in zip(params, blocks):
                b["master"][at:at + p.numel()] = _in_memory(p.detach())
                at += k * ADAMW_BLOCK
        return b

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        step = self._steps + 1
        for g, group in enumerate(self.param_groups):
            kinds = dict.fromkeys((p.dtype, p.device) for p in group["params"] if p.grad is not None)
            for n, (dtype, device) in enumerate(kinds):
                b = self._buckets[g, dtype, device] = self._bucket((g, dtype, device))
                grads, counts = [_like(p.grad, p) for p in b["params"]], tuple(b["counts"])
                # one call for each number of steps that parameters have had: as a rule they all have as many
                for count in dict.fromkeys(c for c, x in zip(counts, grads) if x is not None):
                    these = [x if c == count else None for c, x in zip(counts, grads)]
                    adamw_step(b["params"], these, b["m"], b["v"], b["ms"], b["vs"], b["master"],
                               lr=group["lr"], beta1=group["betas"][0], beta2=group["betas"][1], eps=group["eps"],
                               weight_decay=group["weight_decay"], step=count + 1, seed=(step << 8) + 16 * g + n)
                    b["counts"] = [c + (x is not None) for c, x in zip(b["counts"], these)]
        self._steps = step
        return loss

    def state_bytes(self) -> int:
        """Device memory of the moments, their scales and the master copies."""
        return sum(t.numel() * t.element_size() for b in self._buckets.values()
                   for t in (b["m"], b["v"], b["ms"], b["vs"], b["master"]) if t is not None)

    def state_dict(self) -> dict:
        """Hyperparameters, the step counts and the buffers as they are (8-bit moments in 8 bits)."""
        buffers = []
        for (g, dtype, _), b in self._buckets.items():
            buffers.append({"group": g, "dtype": str(dtype), "counts": list(b["counts"]), **{k: b[k] for k in ("m", "v", "ms", "vs", "master")}})
        groups = [{k: v for k, v in group.items() if k != "params"} | {"params": [tuple(p.shape) for p in group["params"]]}
                  for group in self.param_groups]
        return {"steps": self._steps, "state_bits": self.state_bits, "master": self.master, "groups": groups, "buffers": buffers}

    @torch.no_grad()
    def load_state_dict(self, state: dict) -> None:
        """The state of an optimizer over parameters of the same shapes and types in the same groups.  Parameters of
        a type that had not been stepped there begin anew here."""
        if state["state_bits"] != self.state_bits or state["master"] != self.master:
            raise ValueError("the state is of moments in another form")
        if [g["params"] for g in state["groups"]] != [[tuple(p.shape) for p in g["params"]] for g in self.param_groups]:
            raise ValueError("the state is of other parameters")
        wanted = {}
        for saved in state["buffers"]:
            kinds = {(p.dtype, p.device) for p in self.param_groups[saved["group"]]["params"] if str(p.dtype) == saved["dtype"]}
            if len(kinds) != 1:
                raise ValueError("the state is of parameters of other types")
            key = saved["group"], *kinds.pop()
            b = self._bucket(key)
            if any((b[k] is None) != (saved[k] is None) or (b[k] is not None and b[k].shape != saved[k].shape)
                   for k in ("m", "v", "ms", "vs", "master")):
                raise ValueError("the state is of other parameters")
            wanted[key] = b, saved
        self._buckets = {key: b for key, (b, _) in wanted.items()}
        for b, saved in wanted.values():
            # states without counts are of parameters that had a gradient in every step
            b["counts"] = list(saved.get("counts", [state["steps"]] * len(b["params"])))
            for k in ("m", "v", "ms", "vs", "master"):
                if b[k] is not None:
                    # codes go as bytes: a copy between 8-bit types would round
                    as_bytes = (b[k].view(torch.uint8), saved[k].view(torch.uint8)) if b[k].dtype == torch.float8_e4m3fn else (b[k], saved[k])
                    as_bytes[0].copy_(as_bytes[1])
        for group, saved in zip(self.param_groups, state["groups"]):
            group.update({k: v for k, v in saved.items() if k != "params"})
        self._steps = state["steps"]


def _in_memory(t):
    """The elements of a dense tensor in the order they have in memory."""
    order = sorted(range(t.dim()), key=lambda i: (-t.stride(i), -t.size(i)))
    return t.permute(order).reshape(-1)


def _like(grad, p):
    """The gradient in its parameter's layout (a copy where it has another)."""
    if grad is None or grad.stride() == p.stride() or (grad.is_contiguous() and p.is_contiguous()):
        return grad
    return torch.empty_strided(p.size(), p.stride(), dtype=grad.dtype, device=grad.device).copy_(grad)
