"""A worker's embedding block, from token IDs to activations and from their
gradients to the contribution it pushes, through the C ABI.

Alg. 1 (worker) of the paper: the worker pulls the rows of its batch, computes
a gradient and pushes it.  The block at the bottom of the worker's model is
the embedding: the rows are pulled once per distinct ID, expanded to the
batch's tokens and scaled, and layer-normalised.  On the way back the layer
norm's gradient gives the gradient of the expanded rows, which is added up by
ID; then every gradient of the model is scaled by the global norm over all of
them, the rows included, into what a push takes: one flat float32 vector of
dense gradients, the distinct IDs and one float32 row each.

The class owns the block's outputs and scratch (allocated once, reused every
step); the rows, the parameters and the model's other gradients are the
caller's tensors.  All calls of a step are enqueued on one stream, the current one
or ``stream`` (which the caller orders behind what makes the tensors on another);
the number of distinct IDs stays on the GPU until ``contribution`` reads it for the message's length,
and with it the error word: a step that went wrong has nothing to push.
"""
from __future__ import annotations

import torch

from . import (DERR_NONFINITE, MAX_D, GBAError, gba_clip_grads, gba_embedding_grad_rows, gba_embedding_grad_workspace_size, gba_embedding_lookup,
               gba_grad_norm_workspace_size, gba_layer_norm, gba_layer_norm_grad, gba_layer_norm_grad_workspace_size,
               gba_pull_rows, gba_pull_workspace_size, gba_tensor_list, _stream)


class StepError(GBAError):
    """A step without a contribution.  ``bits``: the error word, DERR_ID_RANGE (an
    ID outside the table) or DERR_NONFINITE (a norm that is infinite or not a
    number, with which no gradient was written)."""

    def __init__(self, bits: int):
        super().__init__(f"the step has no contribution to push: error word {bits}")
        self.bits = bits


class EmbeddingBlock:
    """``n`` tokens a batch, rows of width ``D`` of a table of ``R`` rows;
    activations of ``dtype``.  ``dense_grads``: the gradient tensors of the rest of
    the model (float32, bfloat16 or float16, kept where they are), which are
    clipped with the block's own and follow them in the contribution:
    [dweight, dbias, *dense_grads].  ``weight``, ``bias``: whether the layer norm has
    them; one that it lacks has no gradient, no part in the norm and no place in
    the contribution.  ``D`` is a width that can be pulled and pushed: a multiple of 4
    up to MAX_D."""

    def __init__(self, n: int, D: int, R: int, dense_grads=(), dtype=torch.bfloat16, scale: float = 1.0,
                 padding_id: int = -1, eps: float = 1e-5, max_norm: float = 1.0, device="cuda", weight: bool = True,
                 bias: bool = True):
        if D % 4 or not 4 <= D <= MAX_D:
            raise GBAError(f"D: rows that are pulled and pushed have a multiple of 4 up to {MAX_D} elements, not {D}")
        self.n, self.D, self.R = n, D, R
        self.weight, self.bias = bool(weight), bool(bias)
        self.scale, self.padding_id, self.eps, self.max_norm = scale, padding_id, eps, max_norm
        dev = torch.device(device)

        def new(*shape, kind=torch.float32):
            return torch.empty(shape, dtype=kind, device=dev)

        # the number of distinct rows and the error word, read together
        self._words = torch.zeros(2, dtype=torch.int64, device=dev)
        self.num_unique, self.err = self._words[:1], self._words[1:].view(torch.int32)[:1]
        # forward
        self.pulled_ids, self.inverse = new(n, kind=torch.int64), new(n, kind=torch.int32)
        self.pulled, self.num_pulled = new(n, D), new(1, kind=torch.int64)
        self.x, self.y = new(n, D, kind=dtype), new(n, D, kind=dtype)
        self.mean, self.rstd = new(n), new(n)
        # backward
        self.dx = new(n, D, kind=dtype)
        self.dweight, self.dbias = new(D) if weight else None, new(D) if bias else None
        self.unique_ids, self.row_grads = new(n, kind=torch.int64), new(n, D)
        # the contribution
        self.grads = [*[g for g in (self.dweight, self.dbias) if g is not None], *dense_grads]
        self.P = sum(g.numel() for g in self.grads)
        self.flat, self.rows, self.norm, self.coef = new(self.P), new(n, D), new(1), new(1)
        places = list(self.flat.split([g.numel() for g in self.grads]))
        # (the rows not in place: clipped twice, a step would be scaled twice)
        self.list = gba_tensor_list([*self.grads, self.row_grads], [*places, self.rows],
                                    [*[None] * len(self.grads), self.num_unique])
        # one scratch for all calls: they follow each other on the stream
        size = max(gba_pull_workspace_size(n, R), gba_layer_norm_grad_workspace_size(n, D),
                   gba_embedding_grad_workspace_size(n, D, R), gba_grad_norm_workspace_size(self.list))
        self.workspace = new(size, kind=torch.uint8)
        self._stream = None   # of the last step

    def _parameter(self, name, given, has):
        # else its gradient would be missing from the norm, or be that of a parameter which is not there
        if (given is not None) != has:
            raise GBAError(f"{name}: the block was made {'with' if has else 'without'} one ({name}={has})")

    def _batch(self, ids):
        # fewer would leave tokens of an earlier batch behind them
        if ids.numel() != self.n:
            raise GBAError(f"ids: expected {self.n}, got {ids.numel()}")

    def forward(self, ids, table, weight=None, bias=None, stream=None):
        """The batch's activations, [n, D]: layer_norm(scale * table[ids])."""
        self._batch(ids)
        if table.dim() != 2 or table.shape[1] != self.D:   # (the pulled rows lie one after the other)
            raise GBAError(f"table: expected rows of {self.D}, got {list(table.shape)}")
        self._parameter("weight", weight, self.weight)
        self._parameter("bias", bias, self.bias)
        gba_pull_rows(ids, table, self.pulled_ids, self.inverse, self.pulled, self.num_pulled, self.workspace, self.err,
                      stream=stream)
        gba_embedding_lookup(self.inverse, self.pulled, self.x, self.scale, self.err, stream=stream)
        gba_layer_norm(self.x, weight, bias, self.y, self.eps, self.mean, self.rstd, stream=stream)
        return self.y

    def backward(self, ids, dy, weight=None, stream=None):
        """From the activations' gradient: dweight, dbias, and the rows' gradient by ID."""
        self._batch(ids)
        self._parameter("weight", weight, self.weight)
        gba_layer_norm_grad(dy, self.x, self.mean, self.rstd, weight, self.dx, self.dweight, self.dbias, self.workspace,
                            stream=stream)
        gba_embedding_grad_rows(ids, self.dx, self.R, self.unique_ids, self.row_grads, self.num_unique, self.workspace,
                                self.scale, self.padding_id, self.err, stream=stream)

    def clip(self, stream=None):
        """Every gradient scaled by min(1, max_norm / norm): the dense ones into
        ``flat``, the rows (``row_grads``) into ``rows``."""
        self._stream = _stream(None) if stream is None else stream   # (the current one's handle)
        gba_clip_grads(self.list, self.max_norm, self.norm, self.workspace, self.coef, self.err, stream=stream)

    def contribution(self, stream=None):
        """(flat [P], IDs [U], rows [U, D]) to push; reads U, and so waits for the stream
        of the last ``clip``, or for ``stream`` (a graph replayed on another than it was
        recorded on).  Raises StepError where the step's IDs or norm were bad, and clears ``err``
        then: what the buffers hold is not this step's, and the next step begins
        without it.  (An ID outside the table in an earlier step, whose
        contribution was not asked for, is reported here too.)"""
        self._wait(self._stream if stream is None else stream)
        U, bits = self._words.tolist()
        if bits:
            self.err.zero_()
            torch.cuda.current_stream(self.err.device).synchronize()   # before a step on any stream
            # (left by an earlier step whose contribution was not asked for: this one's norm is finite)
            if float(self.coef.item()) != 0.0:
                bits &= ~DERR_NONFINITE
        if bits:
            raise StepError(bits)
        return self.flat, self.unique_ids[:U], self.rows[:U]

    def _wait(self, stream):
        if stream is None:
            raise GBAError("contribution: no step has been clipped")
        if not hasattr(stream, "synchronize"):
            if int(stream) == _stream(None):
                return   # what is read next waits for the current stream
            stream = torch.cuda.ExternalStream(int(stream), device=self.err.device)
        stream.synchronize()
