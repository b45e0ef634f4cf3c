"""The weight update of a training step: gradient norm, clipping and AdamW on all tensors of a model, three launches a step.

The paper trains its models without naming the optimiser (section 8.1); AdamW is what a training program of this kind uses.
"""
from __future__ import annotations

import torch

from . import binding as B


class AdamW:
    """AdamW over many tensors.

    entries       one dict a tensor as for binding.ParamTable.  States that are not given are made: zeros, of `bits` bits
    lr            learning rate: a number, or a float32 device tensor of one element, read when a step runs (a captured step
                  then follows a schedule)
    max_norm      the gradients of a step are scaled down to this norm; 0: no clipping
    bits          32 or 8: bits of the states that are made here.  Tensors of fewer than 4096 elements get 32 in any case: they
                  are the biases and scales of a model, whose states cost nothing and whose blocks would mix few values
    step          steps taken so far (a run that goes on)
    rounding_seed   how 8-bit states are rounded.  Not 0: without bias, by draws that depend on this seed, the step, the tensor and the
                  element alone.  0: to the nearest code, with which second moments freeze after a few hundred steps (a gradient
                  that changes its size later leads to steps several times too small or too large).  None: 1 where 8-bit states
                  are made here, 0 where any are given - a run that goes on is told the seed that it began with

    A step whose gradients hold an infinity or NaN changes nothing (state.skipped counts them).
    """

    SMALL = 4096

    def __init__(self, entries: list, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, max_norm: float = 0.0, bits: int = 32, step: int = 0,
                 rounding_seed: int | None = None):
        if bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        full, made, given = [], False, False
        for e in entries:
            e = dict(e)
            if e.get("param") is not None and e.get("m") is None:
                n, dev = e["grad"].numel(), e["grad"].device
                if bits == 8 and n >= self.SMALL:
                    made = True
                    blocks = (n + B.STATE_BLOCK - 1) // B.STATE_BLOCK
                    e["m"], e["v"] = torch.zeros(n, dtype=torch.int8, device=dev), torch.zeros(n, dtype=torch.uint8, device=dev)
                    e["m_scale"], e["v_scale"] = (torch.zeros(blocks, dtype=torch.float32, device=dev) for _ in range(2))
                else:
                    e["m"], e["v"] = (torch.zeros(n, dtype=torch.float32, device=dev) for _ in range(2))
            elif e.get("param") is not None and e["m"].dtype == torch.int8:
                given = True
            full.append(e)
        self.table = B.ParamTable(full)
        self.state = B.StepState(step)
        self.lr, self.betas, self.eps, self.max_norm = lr, betas, eps, max_norm
        self.rounding_seed = int(made and not given) if rounding_seed is None else rounding_seed
        self.ws = B.Workspace()

    @classmethod
    def of(cls, model, weight_decay: float = 0.0, **kw) -> "AdamW":
        """For a MaskedGNN or ResSAGEPlus: its parameters and the gradients that its backward pass writes.  Weight matrices decay, biases
        and the scale and shift of a normalisation do not.  bfloat16 weights get a float32 copy that is updated in their place."""
        entries = []
        for p, g in zip(model.params, model.grads):
            for name, t in p.items():
                e = {"param": t, "grad": g["d" + name], "weight_decay": weight_decay if t.dim() == 2 else 0.0}
                if t.dtype == torch.bfloat16:
                    e["master"] = t.float()
                entries.append(e)
        return cls(entries, **kw)

    def step(self, grad_scale: float = 1.0) -> B.StepState:
        """One step on the current stream.  grad_scale: factor of all gradients (1 / number of batches they were added up over)."""
        on_device = isinstance(self.lr, torch.Tensor)
        B.gnn_grad_norm(self.table, self.state, grad_scale, self.max_norm, ws=self.ws)
        B.gnn_adamw_step(self.table, 0.0 if on_device else self.lr, self.betas, self.eps, state=self.state,
                         lr_device=self.lr if on_device else None, rounding_seed=self.rounding_seed)
        return self.state
