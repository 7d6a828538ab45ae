"""The tied table of an arena's replicas, at both ends of their models.

``TiedTable`` binds one tensor of a StackedArena (a decoder's ``wte``, [vocab, width]) to the calls that use it: rows of the
replicas' parameters go in (hdet_embed), the loss is taken against their bf16 copy (hdet_token_loss, or a loss of one's own from
hdet_token_scores), and the gradients are written where the update reads them.  It owns the workspaces and the copy, nothing else; all arithmetic but the
rounding of that copy is in the CUDA library.
"""
from __future__ import annotations

import torch

from . import binding as B
from .arena import StackedArena


class TiedTable:
    def __init__(self, arena: StackedArena, k: int, vocab: int, width: int, n_tokens: int, scale: float = 1.0,
                 use_mean: bool = False, piece_bytes: int = 0, scores: bool = False, n_top: int = 0):
        """Tensor ``k`` of ``arena`` as a [vocab, width] table for batches of up to ``n_tokens`` tokens per replica.

        ``use_mean``: the loss reads the one averaged bf16 copy that every converge writes (bf16_copy=True).  It is the average of the
        last converge, whatever has happened to the replicas since, so this is for a converge every step; and before the first loss the copy has
        to be there: one hdet_converge writes it.  Otherwise ``refresh`` rounds every replica's own parameters after each update.
        ``scores``: the workspace is enough for ``scores`` and ``scores_grad`` too, with up to ``n_top`` alternatives a token.
        """
        if arena.numels[k] != vocab * width:
            raise ValueError(f"tensor {k} has {arena.numels[k]} elements, not {vocab} x {width}")
        if arena.shared_grad:
            raise ValueError("the replicas' batches differ, so the arena needs one gradient per replica")
        self.arena, self.scale, self.piece_bytes = arena, float(scale), int(piece_bytes)
        self.table = arena.param_view(k, (vocab, width))
        self.grad = arena.grad_view(k, (vocab, width))
        self.use_mean = bool(use_mean)
        self.weight = arena.mean_view(k, (vocab, width)) if use_mean else torch.empty(
            (arena.n, vocab, width), dtype=torch.bfloat16, device=arena.device)
        n, dev = arena.n, arena.device
        tokens = torch.empty((n, n_tokens), dtype=torch.int32, device=dev)
        rows = torch.empty((n, n_tokens, width), dtype=torch.bfloat16, device=dev)
        need = [B.hdet_embed_grad_workspace(tokens, rows, self.grad)]
        # the loss alone, and with gradients of the hidden states in either type
        for d_hidden in (None, rows, torch.empty((n, n_tokens, width), dtype=torch.float32, device=dev)):
            need.append(B.hdet_token_loss_workspace(rows, self.weight, tokens, d_hidden=d_hidden, d_weight=None if d_hidden is None else self.grad,
                                                    piece_bytes=piece_bytes))
            if scores and d_hidden is not None:
                need.append(B.hdet_token_scores_grad_workspace(rows, self.weight, tokens, d_hidden=d_hidden, d_weight=self.grad, piece_bytes=piece_bytes))
        self.n_top = min(n_top, vocab) if scores else -1
        if scores:                       # fewer alternatives need no more
            need.append(B.hdet_token_scores_workspace(rows, self.weight, tokens, n_top=self.n_top))
        # the calls follow one another on one stream, so they share one workspace
        self.workspace = torch.empty((max(need),), dtype=torch.uint8, device=dev)
        self.refresh()

    def refresh(self) -> None:
        """Rounds the replicas' parameters to the bf16 copy that the loss reads; call it after every update."""
        if not self.use_mean:
            self.weight.copy_(self.table)

    def embed(self, tokens, out) -> None:
        """out [N, T, width] = scale * the replicas' rows of tokens [N, T]."""
        B.hdet_embed(tokens, self.table, out, scale=self.scale, stream=self._stream())

    def loss(self, hidden, targets, losses, d_hidden=None, token_loss=None, grad_scale: float = 1.0) -> None:
        """losses [N] = every replica's mean cross entropy of hidden [N, T, width] (bf16) against its table.  With ``d_hidden``
        (bfloat16 or float32) the gradients are taken too: the table's is written to the arena, over what was there."""
        B.hdet_token_loss(hidden, self.weight, targets, losses, self.workspace, token_loss=token_loss, d_hidden=d_hidden,
                          d_weight=None if d_hidden is None else self.grad, grad_scale=grad_scale, piece_bytes=self.piece_bytes,
                          stream=self._stream())

    def scores(self, hidden, targets, logprob=None, entropy=None, lse=None, top_ids=None, top_logprob=None) -> None:
        """Of hidden [N, T, width] (bf16) against the replicas' tables, whichever is given: log probabilities of targets [N, T] (None:
        none are given), entropies and normalisers [N, T], and the best alternatives [N, T, n_top] with their log probabilities."""
        if self.n_top < (0 if top_ids is None else top_ids.shape[-1]):
            raise ValueError("build the table with scores=True and n_top alternatives")
        B.hdet_token_scores(hidden, self.weight, targets, self.workspace, logprob=logprob, entropy=entropy, lse=lse, top_ids=top_ids,
                            top_logprob=top_logprob, stream=self._stream())

    def scores_grad(self, hidden, targets, lse, d_hidden, logprob=None, entropy=None, d_logprob=None, d_entropy=None,
                    accumulate: bool = False) -> None:
        """The gradients of a loss of log probabilities and entropies, given its own with respect to those and what ``scores`` left:
        ``d_hidden`` (bfloat16 or float32), and the table's to the arena, over what was there or, with ``accumulate``, added to it."""
        if self.n_top < 0:
            raise ValueError("build the table with scores=True")
        B.hdet_token_scores_grad(hidden, self.weight, targets, self.workspace, lse, logprob=logprob, entropy=entropy, d_logprob=d_logprob,
                                 d_entropy=d_entropy, d_hidden=d_hidden, d_weight=self.grad, accumulate=accumulate, piece_bytes=self.piece_bytes,
                                 stream=self._stream())

    def embed_grad(self, tokens, d_out) -> None:
        """Adds the lookup's gradient to the table's in the arena; call it after ``loss`` or ``scores_grad``.  (A bf16 gradient is rounded by each.)"""
        B.hdet_embed_grad(tokens, d_out, self.grad, self.workspace, scale=self.scale, accumulate=True, stream=self._stream())

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.arena.device).cuda_stream
