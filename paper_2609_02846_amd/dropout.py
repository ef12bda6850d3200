"""Dropout from a counter-based generator, as an autograd function and a
module.  The mask is a function of (seed, tensor_id, element index): the
backward pass computes it again, so nothing but the key is kept."""

import torch
from torch.autograd.function import once_differentiable

from .operators import dropout_forward, recorded


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, tensor_id):
        ctx.key = p, seed, tensor_id
        return dropout_forward(x, p, seed, tensor_id, residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        dy = dy.contiguous()
        dx = dropout_forward(dy, *ctx.key) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


def dropout(x, p, seed, tensor_id=0, residual=None):
    """[``residual`` +] dropout of ``x`` (bf16, fp16 or fp32), with gradients.
    ``p`` is taken to the nearest 2^-16; survivors are scaled by the
    reciprocal of what is kept."""
    x = x.contiguous()
    residual = None if residual is None else residual.contiguous()
    if recorded(x, residual):
        return _DropoutFn.apply(x, residual, float(p), int(seed), int(tensor_id))
    return dropout_forward(x, p, seed, tensor_id, residual)


class Dropout(torch.nn.Module):
    """Dropout with a key of its own for each call in training and tensor id
    ``layer_id``; in evaluation x (plus the residual) passes.

    Without ``seed`` a call's key comes from torch's CPU generator, so that
    ``torch.manual_seed`` and the generator's state bring a run's masks back,
    and a call that activation checkpointing repeats, with that state
    restored, draws the mask of the first.  With ``seed`` call c draws with key
    ``seed`` + c: modules of one seed need different ``layer_id``s, or all of
    them drop the same elements, and the seeds of ranks have to be further
    apart than a run has calls.  A call inside a backward pass, where
    checkpointing repeats one, is refused then: which call it repeats the
    count does not tell.  (A call captured in a graph holds its key: every replay
    drops the same elements.)"""

    def __init__(self, p=0.1, seed=None, layer_id=0):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must be in [0, 1]")
        self.p, self.seed, self.layer_id, self.calls = float(p), None if seed is None else int(seed), int(layer_id), 0

    def next_key(self):
        """The key of one call."""
        if self.seed is None:
            return torch.randint(-2 ** 63, 2 ** 63 - 1, (), device="cpu").item() & (2 ** 64 - 1)
        if torch._C._current_graph_task_id() != -1:
            raise RuntimeError("a module with a seed of its own counts its calls, and a call repeated in the backward "
                               "pass would draw another mask: leave seed out to checkpoint it")
        key = (self.seed + self.calls) & (2 ** 64 - 1)
        self.calls += 1
        return key

    def forward(self, x, residual=None):
        if not self.training:
            return x if residual is None else residual + x
        return dropout(x, self.p, self.next_key(), self.layer_id, residual)

    # The count goes with the parameters, so that a resumed run does not draw its
    # first masks again.
    def _save_to_state_dict(self, destination, prefix, keep_vars):
        super()._save_to_state_dict(destination, prefix, keep_vars)
        if self.seed is not None:
            destination[prefix + "calls"] = torch.tensor(self.calls, device="cpu")

    def _load_from_state_dict(self, state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, errors):
        super()._load_from_state_dict(state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, errors)
        key = prefix + "calls"
        if key in state_dict:
            self.calls = int(state_dict[key])
            if key in unexpected_keys:
                unexpected_keys.remove(key)

    def extra_repr(self):
        return f"p={self.p}"
