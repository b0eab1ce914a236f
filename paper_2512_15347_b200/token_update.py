"""Driver of the policy update on token trajectories: scores rows of logits, forms the clipped objective over ragged rows of
tokens and takes its gradient back to the logits.  Allocation and streams are torch's; every number is computed by the library's
kernels.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as B


def _empty(dev, *shape) -> torch.Tensor:
    return torch.empty(shape, device=dev, dtype=torch.float32)


class Scores(NamedTuple):
    """Of rows of logits: logp [rows, given tokens] or None, entropy [rows], top_ids / top_logp [rows, n_top] or None."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    top_ids: Optional[torch.Tensor]
    top_logp: Optional[torch.Tensor]


class Update(NamedTuple):
    """Of one update step: objective [1] (to be raised), its gradient dlogits, and what it was made of: logp, entropy, distill (None without a
    teacher), weight [tokens], stats [TOKEN_STATS]."""
    objective: torch.Tensor
    dlogits: torch.Tensor
    logp: torch.Tensor
    entropy: torch.Tensor
    distill: Optional[torch.Tensor]
    weight: torch.Tensor
    stats: torch.Tensor


def score(logits, ids=None, *, n_top: int = 0, temperature=None) -> Scores:
    """Log-probs of the given tokens, entropy and the n_top likeliest tokens of rows of logits: a rollout's own log-probs, or the lists
    that a teacher or a reference policy leaves for ``TokenUpdate.step``."""
    rows, dev = logits.shape[0], logits.device
    terms = B.make_token_terms(temperature=temperature, ids=ids, n_top=n_top)
    n_ids = terms._plain[2]
    logp = _empty(dev, rows, n_ids) if n_ids else None
    entropy = _empty(dev, rows)
    top = (torch.empty((rows, n_top), device=dev, dtype=torch.int32), _empty(dev, rows, n_top)) if n_top else (None, None)
    B.token_forward(logits, terms, logp=logp, entropy=entropy, top_ids=top[0], top_logp=top[1])
    return Scores(logp, entropy, *top)


def _gradient_room(logits) -> torch.Tensor:
    """Room for the gradient of logits [rows, vocab], contiguous where the logits' rows allow it.  Rows lie on the 16-byte offsets of the logits' rows, so
    that the kernels write whole units: of a padded vocabulary's slice each row is up to 15 bytes longer, not as long as the padded one."""
    rows, vocab = logits.shape
    size = logits.element_size()
    first = logits.data_ptr() % 16 // size
    pitch = vocab + ((logits.stride(0) - vocab) % (16 // size) if rows > 1 else 0)
    if first == 0 and pitch == vocab:
        return torch.empty((rows, vocab), device=logits.device, dtype=logits.dtype)
    return torch.empty(first + rows * pitch, device=logits.device, dtype=logits.dtype).as_strided((rows, vocab), (pitch, 1), first)


class TokenUpdate:
    """The settings of an objective (see pg_token_objective) and what its calls need besides: workspaces, a status word.

    ``step`` may be captured in a CUDA graph.  Calls run on the current stream; workspaces are a stream's or a graph's own, so calls on
    several streams and replays of several graphs may overlap."""

    def __init__(self, *, clip_low: float = 0.2, clip_high: float = 0.2, beta: float = 0.0, entropy_coef: float = 0.0, distill_coef: float = 0.0,
                 kind: str = "forward", norm: str = "rows"):
        if not torch.cuda.is_available():
            raise RuntimeError("the rollout library needs a CUDA device; there is no CPU path")
        self.dev = torch.device("cuda", torch.cuda.current_device())
        if kind not in B.DISTILL_KINDS or norm not in B.TOKEN_NORMS:
            raise ValueError(f"kind: one of {B.DISTILL_KINDS}, norm: one of {B.TOKEN_NORMS}")
        self.kind, self.entropy_coef, self.distill_coef = kind, entropy_coef, distill_coef
        self._rule = dict(clip_low=clip_low, clip_high=clip_high, beta=beta, norm=norm)
        self.status = torch.zeros(1, device=self.dev, dtype=torch.int32)
        self._spaces = {}

    def _space(self, nbytes: int) -> torch.Tensor:
        """The current stream's workspace.  A capture takes one of the graph's own memory, zeroed at each replay: graphs recorded on one
        stream may be replayed on several at once."""
        if torch.cuda.is_current_stream_capturing():
            return torch.zeros(nbytes, device=self.dev, dtype=torch.uint8)
        stream = B._stream(None)
        space = self._spaces.get(stream)
        if space is None or space.nbytes < nbytes:
            space = self._spaces[stream] = torch.zeros(nbytes, device=self.dev, dtype=torch.uint8)
        return space

    def step(self, logits, ids, start, adv, logp_old=None, *, logp_ref=None, teacher: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
             temperature=None, scale: float = 1.0, dlogits=None) -> Update:
        """One step on packed tokens: logits [tokens, vocab] of the positions that made ids [tokens], rows of tokens by start [rows + 1], their
        advantages adv [rows]; logp_old, logp_ref [tokens] log-probs of the rollout (None: this policy's own) and of a reference; teacher
        (ids, log-probs) [tokens, n] as ``score`` gives them, for distill_coef; dlogits (may be logits) receives the gradient, soonest where its
        rows lie on the 16-byte offsets of the logits' rows.  Without it the gradient lies so, contiguous where contiguous rows do."""
        n, dev = logits.shape[0], logits.device
        if self.distill_coef and teacher is None:
            raise ValueError("distill_coef without a teacher's lists")
        if self._rule["beta"] and logp_ref is None:
            raise ValueError("beta without logp_ref")
        if ids.numel() != n:
            raise ValueError("ids: one token for each row of logits")
        listed = dict(teacher_ids=teacher[0], teacher_logp=teacher[1], kind=self.kind) if teacher is not None else {}
        terms = B.make_token_terms(temperature=temperature, ids=ids, **listed)
        logp, entropy, dlogp, weight = (_empty(dev, n) for _ in range(4))
        distill = _empty(dev, n) if teacher is not None else None
        saved, objective, stats = _empty(dev, n, B.TOKEN_SAVED), _empty(dev, 1), _empty(dev, B.TOKEN_STATS)
        B.token_forward(logits, terms, logp=logp, entropy=entropy, distill=distill, saved=saved)
        dlogits = _gradient_room(logits) if dlogits is None else dlogits
        B.token_objective(start, logp, adv, objective, dlogp, self._space(B.token_objective_workspace_bytes(n)), logp_old=logp_old,
                          logp_ref=logp_ref, entropy=entropy, distill=distill, entropy_coef=self.entropy_coef, distill_coef=self.distill_coef,
                          scale=scale, weight=weight, stats=stats, status=self.status, **self._rule)
        B.token_backward(logits, terms, saved, dlogits, dlogp=dlogp, dentropy=weight if self.entropy_coef else None,
                         entropy_scale=self.entropy_coef, ddistill=weight if self.distill_coef else None, distill_scale=-self.distill_coef)
        return Update(objective, dlogits, logp, entropy, distill, weight, stats)

    def check(self) -> None:
        """Raises PgError if a step was given starts that do not ascend; synchronises."""
        B.kv_status(self.status)
