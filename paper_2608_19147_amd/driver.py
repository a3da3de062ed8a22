"""Host-side bookkeeping of a speculative-decoding verify loop over one KV state.

The paper's stage never trims its cache when drafts are rejected: rejected rows
stay in place and later forwards ignore them through the attention mask
(Speculative Decoding via Mask-Based KV Rewind, "Mask-Based Rewind"), and beam
reordering gathers through beam_idx (Reaching Monolithic Parity: the beam_idx
Gather Injection).  This driver keeps, per cache slot, which physical rows are
valid, and builds each step's mask, positions and beam_idx:

* the mask covers the P physical rows plus the n new ones; new rows are
  visible (causality among them is applied by the kernels);
* a new token's position is the number of valid past rows plus its index,
  i.e. its index in the equivalent trimmed cache;
* after a step, slot b keeps its first (1 + a_b) new rows, where a_b is the
  number of leading accepted drafts; the rest become holes;
* when beam_idx reorders the slots, the per-slot valid masks are reordered the
  same way before the mask is built.

Only host metadata lives here; every step of the forward runs in the library.
"""
from __future__ import annotations

from typing import Optional

import numpy as np


class VerifyDriver:
    """Valid-row masks of ``n_slots`` cache slots that start with ``past`` valid rows."""

    def __init__(self, n_slots: int, past: int):
        self.n_slots = n_slots
        self.valid = np.ones((n_slots, past), np.uint8)
        self._nodes: Optional[int] = None                     # of the last tree_inputs, until its nodes are recorded

    @property
    def physical_len(self) -> int:
        return self.valid.shape[1]

    def step_inputs(self, n_new: int, beam_idx: Optional[np.ndarray] = None):
        """(positions [S, n], mask [S, P + n], beam_idx) of the next forward.
        Applies the reorder to the valid masks first (the reorder persists)."""
        if beam_idx is not None:
            beam_idx = np.asarray(beam_idx, np.int32)
            self.valid = self.valid[beam_idx]
        base = self.valid.sum(axis=1).astype(np.int32)
        positions = base[:, None] + np.arange(n_new, dtype=np.int32)[None, :]
        mask = np.concatenate([self.valid, np.ones((self.n_slots, n_new), np.uint8)], axis=1)
        return positions, mask, beam_idx

    def accept(self, drafts_ok: np.ndarray) -> np.ndarray:
        """Record the outcome of the last step: ``drafts_ok`` [S, n - 1] are the
        draft verdicts; slot b keeps the verified token plus the leading run of
        accepted drafts.  Returns the tokens kept per slot (1 + accepted)."""
        drafts_ok = np.asarray(drafts_ok, bool)
        s, k = drafts_ok.shape
        lead = np.argmin(np.concatenate([drafts_ok, np.zeros((s, 1), bool)], axis=1), axis=1)
        keep = (np.arange(k + 1)[None, :] <= lead[:, None]).astype(np.uint8)
        self.valid = np.concatenate([self.valid, keep], axis=1)
        return 1 + lead

    def tree_inputs(self, parents: np.ndarray, beam_idx: Optional[np.ndarray] = None):
        """(positions [S, n], mask_rows [S, n, P + n], beam_idx) of the forward that
        verifies a drafted tree per slot: parents [S, n], every node's parent before
        it, node 0 (the last accepted token) the root.  A node sees the slot's valid
        rows, its ancestors and itself; its position is the number of valid rows plus
        its depth.  Applies the reorder to the valid masks first (it persists, unless the
        call is refused)."""
        valid = self.valid
        if beam_idx is not None:
            beam_idx = np.asarray(beam_idx, np.int32)
            if beam_idx.shape != (self.n_slots,) or not ((beam_idx >= 0) & (beam_idx < self.n_slots)).all():
                raise ValueError("beam_idx must name a slot for each slot")
            valid = valid[beam_idx]
        parents = np.asarray(parents)
        s, n = parents.shape
        if s != self.n_slots or n < 1 or (n > 1 and not ((parents[:, 1:] >= 0) & (parents[:, 1:] < np.arange(1, n))).all()):
            raise ValueError("parents must be [slots, nodes], each node's parent before it")
        see = np.zeros((s, n, n), np.uint8)
        depth = np.zeros((s, n), np.int32)
        slot = np.arange(s)
        see[:, 0, 0] = 1
        for i in range(1, n):
            see[:, i] = see[slot, parents[:, i]]
            see[:, i, i] = 1
            depth[:, i] = depth[slot, parents[:, i]] + 1
        self.valid, self._nodes = valid, n
        past = np.broadcast_to(valid[:, None, :], (s, n, self.physical_len))
        positions = valid.sum(axis=1).astype(np.int32)[:, None] + depth
        return positions, np.concatenate([past, see], axis=2), beam_idx

    def accept_tree(self, keep: np.ndarray) -> np.ndarray:
        """Record which nodes of the last ``tree_inputs`` forward were accepted: keep
        [S, n] of ``Stage.tree_accept``.  Returns the nodes kept per slot."""
        keep = (np.asarray(keep) != 0).astype(np.uint8)
        if keep.ndim != 2 or keep.shape[0] != self.n_slots:
            raise ValueError("keep must be [slots, nodes]")
        if self._nodes not in (None, keep.shape[1]):
            raise ValueError(f"keep has {keep.shape[1]} nodes, the tree {self._nodes}")
        self.valid, self._nodes = np.concatenate([self.valid, keep], axis=1), None
        return keep.sum(axis=1).astype(np.int32)
