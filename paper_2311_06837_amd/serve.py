"""A trained MaskedGNN answers with its weights and activations in 8-bit integers.

The order of calls is the forward pass of the model (paper section 2.1's layer equation under section 6's masks), with
gnn_linear_i8_fwd in the place of gnn_linear_fwd: aggregation in the model's type, the feature transform in integers.
Every layer aggregates first.  A model that transforms its narrowing layers first gathers narrower rows, which is worth more than the
integers: ms of model.forward / Int8Answers.forward 13.8 / 20.4 (GraphSAGE 602-256-256-41, float32, 114M edges),
31.2 / 30.5 (GCN 100-256-256-47, float32, 125M), 5.7 / 6.7 (GraphSAGE of eight layers of 128, bfloat16, 20M).
"""
from __future__ import annotations

import torch

from . import binding as B
from .model import MaskedGNN


class Int8Answers:
    """Logits of a MaskedGNN's targets from 8-bit weights.

    model   its graph, active sets (build_active_sets or step has run), input and parameters are used; its activations are not
            touched.  Layers run in the paper's order (aggregate, then transform), whatever the model's.
    refresh puts the model's present weights on the grid; call it again after an update of the weights.
    """

    def __init__(self, model):
        if not isinstance(model, MaskedGNN):
            raise TypeError("a MaskedGNN is needed")
        self.model = model
        n, dev = model.n, model.targets.device
        self.A = torch.zeros(n, max(model.ld[:-1]), dtype=model.dtype, device=dev)
        self.H = [torch.zeros(n, max(model.ld[1:]), dtype=model.dtype, device=dev) for _ in range(min(2, model.L))]
        self.weights = [{} for _ in model.params]
        self.ws = B.Workspace()
        self.refresh()

    def refresh(self):
        for w, p in zip(self.weights, self.model.params):
            for name in ("W_neigh", "W_self"):
                if name in p:
                    w[name] = B.gnn_quantize_weight(p[name], out=w.get(name), ws=self.ws)

    def forward(self) -> torch.Tensor:
        """Logits: a matrix whose rows of the targets hold them, in the first dims[-1] columns (valid until the next call)."""
        m = self.model
        if m.hop is None or not m.H or m.H[0] is None:
            raise RuntimeError("the model has no input or no active sets yet: set_input and step (or build_active_sets) come first")
        x = m.H[0]
        for l in range(1, m.L + 1):
            K, N, nl = m.dims[l - 1], m.dims[l], m.n_rows_of_layer(l)
            sage, w = m.kind == "sage", self.weights[l - 1]
            a = self.A.view(-1)[: m.n * m.ld[l - 1]].view(m.n, m.ld[l - 1])     # the stride of x: both are read with one
            h = self.H[l % len(self.H)].view(-1)[: m.n * m.ld[l]].view(m.n, m.ld[l])
            g_l, rs_l = (m.g, m.rs) if m.layer_sampling is None else (m.g_l[l], m.rs_l[l])
            B.gnn_masked_spmm_fwd(g_l, m.rows, nl, x, a, K, rs_l, m.cs, ws=self.ws)
            B.gnn_linear_i8_fwd(m.rows, nl, a, None, x if sage else None, None, K, w["W_neigh"], w.get("W_self"), m.params[l - 1]["bias"], h,
                                relu=l < m.L, ws=self.ws)
            x = h
        return x
