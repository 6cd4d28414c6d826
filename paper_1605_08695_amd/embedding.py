"""Embedding table of a language model (the embedding layer of Section 4.2): lookup of the batch's
tokens and the sparse SGD update by their gradients, beside the large-vocabulary heads in
``sampled``."""
from __future__ import annotations

import numpy as np
import torch

from . import ops


class EmbeddingTable:
    """Variable W (vocab x d, fp32 master + bf16 shadow), read by scaled lookups and trained with SGD
    on the rows that a batch names.  Token ids are int32; an id outside the vocabulary is padding: it
    looks up zeros and its gradient is left out."""

    def __init__(self, W: np.ndarray, lr: float, scale: float = 1.0, device="cuda"):
        dev = torch.device(device)
        self.vocab, self.d = W.shape
        self.lr = float(np.float32(lr))
        self.scale = float(np.float32(scale))
        # master weights start at their bf16 values (the values that lookups read)
        self.W = torch.from_numpy(np.asarray(W, np.float32)).to(torch.bfloat16).to(torch.float32).to(dev)
        self.W_lp = self.W.to(torch.bfloat16)

    def lookup(self, ids: torch.Tensor, out=None, stream=None) -> torch.Tensor:
        """scale * W[ids], bf16, ids' shape with d columns."""
        return ops.embedding_fwd(self.W_lp, ids, self.scale, out=out, stream=stream)

    def gradient(self, ids: torch.Tensor, dy: torch.Tensor, dW=None, beta: float = 0.0, stream=None) -> torch.Tensor:
        """The dense fp32 gradient of W for the gradient dy of a lookup of ids (for dense optimizers, and
        beta = 1 for a head that shares W and left its own gradient in dW)."""
        return ops.embedding_bwd(dy, ids, self.vocab, self.scale, dtable=dW, beta=beta, stream=stream)

    def update(self, ids: torch.Tensor, dy: torch.Tensor, stream=None) -> None:
        """SGD on the rows of ids for the gradient dy of their lookup, in place."""
        ops.embedding_apply_sgd(self.W, ids, dy, self.lr, self.scale, shadow=self.W_lp, stream=stream)
