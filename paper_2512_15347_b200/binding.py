"""ctypes binding of libprogrpo.so: same names as the C ABI (minus the ``pg_`` prefix),
argument marshalling only.  Tensors are torch CUDA tensors (or raw integer addresses); every
computation happens inside the library's kernels.  There is no fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libprogrpo.so")

OK, EINVAL, ESTATE, ECUDA, ENONFINITE, ETIMEOUT, ENOMEM, ECAPACITY, EINDEX, EDEVICE = 0, -1, -2, -3, -4, -5, -6, -7, -8, -9
STATIC_MAX_ROWS, STATIC_MAX_PARTIALS = 8192, 65536
ENOPAGES = -10
VEL_F32, VEL_BF16 = 0, 1
F32, BF16, F16 = 0, 1, 2              # element types of the token calls
LOGITS_MAX_TOKENS, LOGITS_MAX_BIAS = 1048575, 2046
MAX_GROUP = 1024
TOKEN_MAX_VOCAB, TOKEN_MAX_TOP, TOKEN_MAX_LIST, TOKEN_SAVED, TOKEN_STATS = 1 << 20, 128, 256, 12, 5
DISTILL_KINDS = ("forward", "forward_rest", "reverse_rest")
TOKEN_NORMS = ("rows", "tokens", "sum")


class PgError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        msg = lib().pg_strerror(code).decode()
        extra = f" (cudaError {lib().pg_last_cuda_error()})" if code == ECUDA else ""
        super().__init__(f"{what}: {msg}{extra}")


class Config(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("n_expand", ctypes.c_int32),
                ("elems", ctypes.c_int32), ("n_steps", ctypes.c_int32),
                ("n_stages", ctypes.c_int32),
                ("stage_step", ctypes.POINTER(ctypes.c_int32)),
                ("stage_keep", ctypes.POINTER(ctypes.c_int32)),
                ("seed", ctypes.c_uint64), ("group_offset", ctypes.c_int32),
                ("vel_dtype", ctypes.c_int32), ("logp_mean", ctypes.c_int32),
                ("adv_eps", ctypes.c_float)]


class StepCoef(ctypes.Structure):
    _fields_ = [("c_x", ctypes.c_double), ("c_v", ctypes.c_double), ("noise_std", ctypes.c_double)]


class RolloutOutputs(ctypes.Structure):
    _fields_ = [("x_final", ctypes.c_void_p), ("logp", ctypes.c_void_p), ("keep_idx", ctypes.c_void_p),
                ("adv", ctypes.c_void_p), ("rewards", ctypes.c_void_p), ("traj_id", ctypes.c_void_p),
                ("n_final", ctypes.c_int32), ("n_logp", ctypes.c_int64), ("n_keep", ctypes.c_int64)]


class PreviewCoef(ctypes.Structure):
    _fields_ = [("p_x", ctypes.c_double), ("p_v", ctypes.c_double)]


class Described(ctypes.Structure):
    """A descriptor that holds the tensors it points to.  Its reference is made anew each time: kept in the descriptor it would be a cycle,
    and the tensors would stay until the garbage collector runs."""

    @property
    def _ref(self):
        return ctypes.byref(self)


class Kv(Described):
    """Descriptor of a paged key-value cache (``make_kv``)."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("n_layers", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_stride", ctypes.c_int64),
                ("layer_stride", ctypes.c_int64), ("table", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("n_rows", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("grown", ctypes.c_void_p)]


class LogitsRules(Described):
    """Sampling rules (``make_logits_rules``)."""
    _fields_ = [("tokens", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("max_tokens", ctypes.c_int32),
                ("n_tokens", ctypes.c_void_p), ("n_prompt", ctypes.c_void_p), ("repetition", ctypes.c_void_p),
                ("presence", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("temperature", ctypes.c_void_p),
                ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p), ("n_bias", ctypes.c_int32),
                ("mask", ctypes.c_void_p), ("mask_stride", ctypes.c_int64)]


class TokenTerms(Described):
    """What rows of logits are asked about (``make_token_terms``)."""
    _fields_ = [("temperature", ctypes.c_void_p), ("ids", ctypes.c_void_p), ("n_ids", ctypes.c_int32), ("n_top", ctypes.c_int32),
                ("teacher_ids", ctypes.c_void_p), ("teacher_logp", ctypes.c_void_p), ("n_teacher", ctypes.c_int32),
                ("kind", ctypes.c_int32)]


class TokenOut(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("logp", "lse", "entropy", "top_ids", "top_logp", "distill", "saved")]


class TokenGrads(ctypes.Structure):
    _fields_ = [("dlogp", ctypes.c_void_p), ("dentropy", ctypes.c_void_p), ("ddistill", ctypes.c_void_p),
                ("entropy_scale", ctypes.c_float), ("distill_scale", ctypes.c_float)]


class TokenBatch(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("start", "logp_new", "logp_old", "logp_ref", "adv", "entropy", "distill")] + \
               [(name, ctypes.c_float) for name in ("clip_low", "clip_high", "beta", "entropy_coef", "distill_coef", "scale")] + \
               [("norm", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2512_15347_b200.build` "
                          "(there is no CPU or PyTorch fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u64, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64,
                             ctypes.c_size_t)
    L.pg_rollout_init.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(vp)]
    L.pg_rollout_destroy.argtypes = [vp]
    L.pg_rollout_reset.argtypes = [vp, vp]
    L.pg_rollout_restore.argtypes = [vp, i32, i32, vp, vp]
    L.pg_rollout_status.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.pg_step.argtypes = [vp, i32, ctypes.POINTER(StepCoef), vp, vp, vp, vp, vp, vp]
    L.pg_step_reward.argtypes = [vp, i32, ctypes.POINTER(StepCoef), vp, vp, vp, vp, vp, vp, vp]
    L.pg_score.argtypes = [vp, ctypes.POINTER(PreviewCoef), vp, vp, vp, vp, vp]
    L.pg_preview.argtypes = [vp, ctypes.POINTER(PreviewCoef), vp, vp, vp, i32, vp]
    L.pg_score_preview.argtypes = [vp, ctypes.POINTER(PreviewCoef), vp, vp, vp, vp, i32, vp]
    L.pg_prune_ovf.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    L.pg_prune_uniform.argtypes = [vp, i32, vp, vp, vp]
    L.pg_group_stats.argtypes = [i32, i32, vp, ctypes.c_float, vp, vp, vp, vp]
    L.pg_compact.argtypes = [vp, vp, vp, vp, sz, vp]
    L.pg_advantages.argtypes = [vp, vp, vp, vp, vp, vp]
    L.pg_policy_logprob.argtypes = [vp, ctypes.POINTER(StepCoef), vp, vp, vp, vp, vp, vp, vp]
    L.pg_policy_objective.argtypes = [vp, i32, vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp, vp, vp, vp]
    L.pg_policy_backward.argtypes = [vp, ctypes.POINTER(StepCoef), vp, vp, vp, vp, vp, ctypes.c_double, vp, vp]
    L.pg_ovf_select_batched.argtypes = [i32, i32, i32, vp, vp, vp, vp, ctypes.c_float, vp, vp]
    L.pg_rollout_host_workspace_bytes.argtypes = [ctypes.POINTER(Config)]
    L.pg_rollout_host_workspace_bytes.restype = sz
    L.pg_rollout_host.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(StepCoef),
                                  ctypes.POINTER(PreviewCoef), vp, ctypes.POINTER(vp),
                                  ctypes.POINTER(vp), vp, vp, vp, vp, vp, vp, vp, sz]
    L.pg_rollout_host_on.argtypes = [vp, ctypes.POINTER(StepCoef), ctypes.POINTER(PreviewCoef), vp,
                                     ctypes.POINTER(vp), ctypes.POINTER(vp), vp, vp, vp, vp, vp, vp, vp, sz]
    L.pg_score_static.argtypes = [i32, i32, i32, ctypes.POINTER(PreviewCoef), vp, vp, vp, vp]
    L.pg_rollout_run_workspace_bytes.argtypes = [ctypes.POINTER(Config)]
    L.pg_rollout_run_workspace_bytes.restype = sz
    L.pg_rollout_run.argtypes = [vp, ctypes.POINTER(StepCoef), ctypes.POINTER(PreviewCoef), vp,
                                 ctypes.POINTER(vp), ctypes.POINTER(vp), vp, vp, sz,
                                 ctypes.POINTER(RolloutOutputs), vp]
    L.pg_rollout_traj_ids.argtypes = [vp, vp, vp]
    L.pg_selftest_bounded_wait.argtypes = [vp, vp]
    L.pg_survivor_rows.argtypes = [vp, vp, vp, vp]
    L.pg_survivor_logp.argtypes = [vp, vp, vp, vp, vp]
    L.pg_gather_rows.argtypes = [vp, vp, i32, i32, vp, vp, sz, vp]
    L.pg_philox_raw.argtypes = [i64, vp, vp, vp, vp]
    L.pg_normal_rows.argtypes = [u64, i32, i32, i32, i32, vp, vp, vp]
    pkv = ctypes.POINTER(Kv)
    L.pg_kv_attend_workspace_bytes.argtypes = [pkv, i32, i32]
    L.pg_kv_attend_workspace_bytes.restype = sz
    L.pg_kv_attend.argtypes = [pkv, i32, i32, vp, i64, vp, vp, i64, ctypes.c_float, i32, vp, vp, i64, vp, vp, sz,
                               vp, vp]
    L.pg_kv_extend.argtypes = [pkv, vp, i32, vp, vp, vp, vp, vp]
    L.pg_kv_append.argtypes = [pkv, i32, i32, vp, vp, i64, vp, vp, vp]
    L.pg_kv_fork_workspace_bytes.argtypes = [pkv, i32]
    L.pg_kv_fork_workspace_bytes.restype = sz
    L.pg_kv_fork.argtypes = [pkv, i32, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.pg_kv_pack_workspace_bytes.argtypes = [pkv]
    L.pg_kv_pack_workspace_bytes.restype = sz
    L.pg_kv_pack.argtypes = [pkv, vp, vp, vp, vp, vp, sz, vp, vp]
    L.pg_kv_status.argtypes = [vp, vp]
    L.pg_logits_process.argtypes = [i32, i32, i32, vp, i64, i32, vp, i64, ctypes.POINTER(LogitsRules), vp]
    L.pg_token_forward.argtypes = [i32, i32, i32, vp, i64, ctypes.POINTER(TokenTerms), ctypes.POINTER(TokenOut), vp]
    L.pg_token_backward.argtypes = [i32, i32, i32, vp, i64, ctypes.POINTER(TokenTerms), vp, ctypes.POINTER(TokenGrads), vp, i64, vp]
    L.pg_token_forward_backward.argtypes = [i32, i32, i32, vp, i64, ctypes.POINTER(TokenTerms), ctypes.POINTER(TokenOut),
                                            ctypes.POINTER(TokenGrads), vp, i64, vp]
    L.pg_token_objective_workspace_bytes.argtypes = [i32]
    L.pg_token_objective_workspace_bytes.restype = sz
    L.pg_token_objective.argtypes = [i32, i32, ctypes.POINTER(TokenBatch), vp, vp, vp, vp, vp, vp, sz, vp, vp]
    L.pg_selftest_token_waits.argtypes = [ctypes.c_uint32]
    for name in ("pg_token_forward", "pg_token_backward", "pg_token_forward_backward", "pg_token_objective",
                 "pg_kv_attend", "pg_kv_extend", "pg_kv_append", "pg_kv_fork", "pg_kv_pack", "pg_kv_status",
                 "pg_logits_process", "pg_selftest_token_waits"):
        getattr(L, name).restype = ctypes.c_int
    L.pg_strerror.argtypes = [ctypes.c_int]
    L.pg_strerror.restype = ctypes.c_char_p
    L.pg_last_cuda_error.restype = ctypes.c_int
    L.pg_launch_count.restype = ctypes.c_uint64
    for name in ("pg_rollout_init", "pg_rollout_destroy", "pg_rollout_reset", "pg_rollout_status",
                 "pg_step", "pg_score", "pg_prune_ovf", "pg_compact", "pg_advantages",
                 "pg_ovf_select_batched", "pg_rollout_host", "pg_rollout_traj_ids",
                 "pg_philox_raw", "pg_normal_rows", "pg_score_static", "pg_policy_logprob",
                 "pg_policy_objective", "pg_policy_backward", "pg_prune_uniform", "pg_group_stats", "pg_preview", "pg_rollout_run", "pg_rollout_restore", "pg_score_preview", "pg_rollout_host_on", "pg_step_reward"):
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def _p(t) -> Optional[int]:
    """Device (or host) address of a tensor; None -> NULL; ints pass through."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return t.data_ptr()


# The current stream's handle without building a Stream object (1.5 us a call), where torch offers it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and _device is not None:
            return _raw_stream(_device()) or None
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _check(rc: int, what: str):
    if rc != OK:
        raise PgError(rc, what)


def make_config(n_groups: int, n_expand: int, elems: int, n_steps: int,
                stages: Sequence[Sequence[int]], seed: int, vel_dtype: int, *, group_offset: int = 0,
                logp_mean: bool = False, adv_eps: float = 1e-6) -> Config:
    n = len(stages)
    steps = (ctypes.c_int32 * max(n, 1))(*[int(s) for s, _ in stages])
    keeps = (ctypes.c_int32 * max(n, 1))(*[int(k) for _, k in stages])
    cfg = Config(n_groups, n_expand, elems, n_steps, n,
                 ctypes.cast(steps, ctypes.POINTER(ctypes.c_int32)),
                 ctypes.cast(keeps, ctypes.POINTER(ctypes.c_int32)),
                 seed & 0xFFFFFFFFFFFFFFFF, group_offset, vel_dtype, 1 if logp_mean else 0, adv_eps)
    cfg._keepalive = (steps, keeps)
    return cfg


def rollout_init(cfg: Config) -> int:
    h = ctypes.c_void_p()
    _check(lib().pg_rollout_init(ctypes.byref(cfg), ctypes.byref(h)), "pg_rollout_init")
    return h.value


def rollout_destroy(h: int) -> None:
    _check(lib().pg_rollout_destroy(h), "pg_rollout_destroy")


def rollout_reset(h: int, stream=None) -> None:
    _check(lib().pg_rollout_reset(h, _stream(stream)), "pg_rollout_reset")


def rollout_restore(h: int, next_step: int, stages_done: int, traj_ids, stream=None) -> None:
    _check(lib().pg_rollout_restore(h, next_step, stages_done, _p(traj_ids), _stream(stream)),
           "pg_rollout_restore")


def rollout_status(h: int, raise_on_flags: bool = True):
    """(n_active, next_step, device_status); synchronises the device."""
    a, b, c = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    rc = lib().pg_rollout_status(h, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    if rc != OK and (raise_on_flags or rc not in (ENONFINITE, ETIMEOUT, EINDEX)):
        raise PgError(rc, "pg_rollout_status")
    return a.value, b.value, c.value


def step(h: int, step_index: int, coef, x_in, vel, src_rows, x_out, logp_out, stream=None) -> None:
    c = StepCoef(*coef)
    _check(lib().pg_step(h, step_index, ctypes.byref(c), _p(x_in), _p(vel), _p(src_rows), _p(x_out),
                         _p(logp_out), _stream(stream)), "pg_step")


def step_reward(h: int, step_index: int, coef, x_in, vel, src_rows, x_out, logp_out, reward_out,
                stream=None) -> None:
    """pg_step that also writes the mean of every updated latent (the final-reward stand-in)."""
    c = StepCoef(*coef)
    _check(lib().pg_step_reward(h, step_index, ctypes.byref(c), _p(x_in), _p(vel), _p(src_rows), _p(x_out),
                                _p(logp_out), _p(reward_out), _stream(stream)), "pg_step_reward")


def score(h: int, coef, x, vel, scores_out, preview_out=None, stream=None) -> None:
    c = PreviewCoef(*coef)
    _check(lib().pg_score(h, ctypes.byref(c), _p(x), _p(vel), _p(scores_out), _p(preview_out),
                          _stream(stream)), "pg_score")


def score_preview(h: int, coef, x, vel, scores_out, preview_out, stream=None) -> None:
    """Scores and the preview x_hat (fp32 or bf16 tensor, by its dtype) in one pass."""
    c = PreviewCoef(*coef)
    dt = VEL_BF16 if preview_out is not None and preview_out.dtype == torch.bfloat16 else VEL_F32
    _check(lib().pg_score_preview(h, ctypes.byref(c), _p(x), _p(vel), _p(scores_out), _p(preview_out), dt,
                                  _stream(stream)), "pg_score_preview")


def preview(h: int, coef, x, vel, out, stream=None) -> None:
    """x_hat = p_x x + p_v vel into `out` (fp32 or bf16 tensor)."""
    c = PreviewCoef(*coef)
    dt = VEL_BF16 if out.dtype == torch.bfloat16 else VEL_F32
    _check(lib().pg_preview(h, ctypes.byref(c), _p(x), _p(vel), _p(out), dt, _stream(stream)), "pg_preview")


def prune_ovf(h: int, stage: int, scores, keep_idx, src_rows=None, sel_var=None, stream=None) -> None:
    _check(lib().pg_prune_ovf(h, stage, _p(scores), _p(keep_idx), _p(src_rows), _p(sel_var),
                              _stream(stream)), "pg_prune_ovf")


def prune_uniform(h: int, stage: int, keep_idx, src_rows=None, stream=None) -> None:
    _check(lib().pg_prune_uniform(h, stage, _p(keep_idx), _p(src_rows), _stream(stream)), "pg_prune_uniform")


def group_stats(n_groups: int, n: int, scores, delta: float, mean=None, std=None, clustered_frac=None,
                stream=None) -> None:
    _check(lib().pg_group_stats(n_groups, n, _p(scores), delta, _p(mean), _p(std), _p(clustered_frac),
                                _stream(stream)), "pg_group_stats")


def compact(h: int, keep_idx, src, dst, row_bytes: int, stream=None) -> None:
    _check(lib().pg_compact(h, _p(keep_idx), _p(src), _p(dst), row_bytes, _stream(stream)),
           "pg_compact")


def advantages(h: int, rewards, adv, mean=None, std=None, stream=None) -> None:
    _check(lib().pg_advantages(h, _p(rewards), _p(adv), _p(mean), _p(std), _stream(stream)),
           "pg_advantages")


def policy_logprob(h: int, coef, x, x_next, vel, vel_ref, logp_out, kl_out=None, stream=None) -> None:
    c = StepCoef(*coef)
    _check(lib().pg_policy_logprob(h, ctypes.byref(c), _p(x), _p(x_next), _p(vel), _p(vel_ref),
                                   _p(logp_out), _p(kl_out), _stream(stream)), "pg_policy_logprob")


def policy_objective(h: int, n_steps: int, logp_new, logp_old, kl, adv, clip_eps: float, beta: float,
                     ratio, dlogp, objective, stream=None) -> None:
    _check(lib().pg_policy_objective(h, n_steps, _p(logp_new), _p(logp_old), _p(kl), _p(adv), clip_eps,
                                     beta, _p(ratio), _p(dlogp), _p(objective), _stream(stream)),
           "pg_policy_objective")


def policy_backward(h: int, coef, x, x_next, vel, vel_ref, dlogp, dkl: float, grad_vel, stream=None) -> None:
    c = StepCoef(*coef)
    _check(lib().pg_policy_backward(h, ctypes.byref(c), _p(x), _p(x_next), _p(vel), _p(vel_ref),
                                    _p(dlogp), dkl, _p(grad_vel), _stream(stream)), "pg_policy_backward")


def ovf_select_batched(n_groups: int, n: int, k: int, scores, keep_idx, kept_scores=None, adv=None,
                       adv_eps: float = 1e-6, status=None, stream=None) -> None:
    _check(lib().pg_ovf_select_batched(n_groups, n, k, _p(scores), _p(keep_idx), _p(kept_scores),
                                       _p(adv), adv_eps, _p(status), _stream(stream)),
           "pg_ovf_select_batched")


def score_static(n_rows: int, elems: int, vel_dtype: int, coef, x, vel, scores_out, stream=None) -> None:
    """pg_score without a handle and without any allocation: the reduction scratch is a fixed
    array inside the library (see pg_score_static for its limits and sharing rules)."""
    c = PreviewCoef(*coef)
    _check(lib().pg_score_static(n_rows, elems, vel_dtype, ctypes.byref(c), _p(x), _p(vel),
                                 _p(scores_out), _stream(stream)), "pg_score_static")


def survivor_rows(h: int, keep_idx_packed, rows_out, stream=None) -> None:
    """rows_out [T, G*K] int32: row of every final survivor at every step."""
    _check(lib().pg_survivor_rows(h, _p(keep_idx_packed), _p(rows_out), _stream(stream)), "pg_survivor_rows")


def survivor_logp(h: int, rows, logp_packed, logp_out, stream=None) -> None:
    """logp_out [T, G*K]: the survivors' entries of the packed per-step log-probs."""
    _check(lib().pg_survivor_logp(h, _p(rows), _p(logp_packed), _p(logp_out), _stream(stream)),
           "pg_survivor_logp")


def gather_rows(h: int, rows, n_out: int, n_in: int, src, dst, row_bytes: int, stream=None) -> None:
    _check(lib().pg_gather_rows(h, _p(rows), n_out, n_in, _p(src), _p(dst), row_bytes, _stream(stream)),
           "pg_gather_rows")


def selftest_bounded_wait(h: int, stream=None) -> None:
    """Makes the library's bounded device-side wait run out once (sets status bit 1)."""
    _check(lib().pg_selftest_bounded_wait(h, _stream(stream)), "pg_selftest_bounded_wait")


def rollout_traj_ids(h: int, dst, stream=None) -> None:
    _check(lib().pg_rollout_traj_ids(h, _p(dst), _stream(stream)), "pg_rollout_traj_ids")


def philox_raw(n: int, ctr, key, out, stream=None) -> None:
    _check(lib().pg_philox_raw(n, _p(ctr), _p(key), _p(out), _stream(stream)), "pg_philox_raw")


def normal_rows(seed: int, step_index: int, stream_id: int, n_rows: int, d: int, traj_id, out,
                stream=None) -> None:
    _check(lib().pg_normal_rows(seed & 0xFFFFFFFFFFFFFFFF, step_index, stream_id, n_rows, d,
                                _p(traj_id), _p(out), _stream(stream)), "pg_normal_rows")


def rollout_host_workspace_bytes(cfg: Config) -> int:
    return int(lib().pg_rollout_host_workspace_bytes(ctypes.byref(cfg)))


def rollout_host(cfg: Config, step_coefs, preview_coefs, x0, vel_steps, stage_scores, final_rewards,
                 x_final, logp, keep_idx, adv, traj_id, workspace) -> int:
    """Whole rollout from host tensors (see pg_rollout_host).  Returns the status code, raising
    for anything but OK / ENONFINITE."""
    sc = (StepCoef * len(step_coefs))(*[StepCoef(*c) for c in step_coefs])
    npc = max(len(preview_coefs), 1)
    pc = (PreviewCoef * npc)(*[PreviewCoef(*c) for c in preview_coefs])
    vs = (ctypes.c_void_p * len(vel_steps))(*[_p(v) for v in vel_steps])
    ss = None
    if stage_scores is not None:
        ss = (ctypes.c_void_p * max(len(stage_scores), 1))(*[_p(s) for s in stage_scores])
    rc = lib().pg_rollout_host(ctypes.byref(cfg), sc, pc, _p(x0), vs, ss, _p(final_rewards),
                               _p(x_final), _p(logp), _p(keep_idx), _p(adv), _p(traj_id),
                               _p(workspace), workspace.numel() * workspace.element_size())
    if rc not in (OK, ENONFINITE):
        raise PgError(rc, "pg_rollout_host")
    return rc


class HostArgs:
    """Marshalled arguments of pg_rollout_host_on, built once and reused call after call."""

    def __init__(self, step_coefs, preview_coefs, vel_steps, stage_scores=None):
        self.sc = (StepCoef * len(step_coefs))(*[StepCoef(*c) for c in step_coefs])
        self.pc = (PreviewCoef * max(len(preview_coefs), 1))(*[PreviewCoef(*c) for c in preview_coefs])
        self.vs = (ctypes.c_void_p * len(vel_steps))(*[_p(v) for v in vel_steps])
        self.ss = None
        if stage_scores is not None:
            self.ss = (ctypes.c_void_p * max(len(stage_scores), 1))(*[_p(s) for s in stage_scores])
        self.keep = (vel_steps, stage_scores)      # the host tensors must outlive the calls


def rollout_host_on(h: int, args: "HostArgs", x0, final_rewards, x_final, logp, keep_idx, adv, traj_id,
                    workspace) -> int:
    """Whole rollout from host tensors on an existing handle (see pg_rollout_host_on): no
    allocation per call.  Returns the status code, raising for anything but OK / ENONFINITE."""
    rc = lib().pg_rollout_host_on(h, args.sc, args.pc, _p(x0), args.vs, args.ss, _p(final_rewards),
                                  _p(x_final), _p(logp), _p(keep_idx), _p(adv), _p(traj_id),
                                  _p(workspace), workspace.numel() * workspace.element_size())
    if rc not in (OK, ENONFINITE):
        raise PgError(rc, "pg_rollout_host_on")
    return rc


def rollout_run_workspace_bytes(cfg: Config) -> int:
    return int(lib().pg_rollout_run_workspace_bytes(ctypes.byref(cfg)))


class RunArgs:
    """Marshalled arguments of pg_rollout_run, built once and reusable (e.g. under graph capture)."""

    def __init__(self, step_coefs, preview_coefs, vel_steps, stage_scores=None):
        self.sc = (StepCoef * len(step_coefs))(*[StepCoef(*c) for c in step_coefs])
        self.pc = (PreviewCoef * max(len(preview_coefs), 1))(*[PreviewCoef(*c) for c in preview_coefs])
        self.vs = (ctypes.c_void_p * len(vel_steps))(*[_p(v) for v in vel_steps])
        self.ss = None
        if stage_scores is not None:
            self.ss = (ctypes.c_void_p * max(len(stage_scores), 1))(*[_p(t) for t in stage_scores])
        self.keep = (vel_steps, stage_scores)
        self.out = RolloutOutputs()


def rollout_run(h: int, args: "RunArgs", x0, final_rewards, workspace, stream=None) -> RolloutOutputs:
    """pg_rollout_run: the whole schedule from device tensors, enqueued on one stream."""
    _check(lib().pg_rollout_run(h, args.sc, args.pc, _p(x0), args.vs, args.ss, _p(final_rewards),
                                _p(workspace), workspace.numel() * workspace.element_size(),
                                ctypes.byref(args.out), _stream(stream)), "pg_rollout_run")
    return args.out


# ---------------------------------------------------------------- token rollouts

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _want(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


# Every tensor of a call lies on one CUDA device, the current one (a cache's calls: the cache's).  What the kernels are given are bare
# addresses: one of host memory, or of another GPU's, would fault there.
_INT32 = torch.int32


def _current(dev: int) -> None:
    """Refuses a call for tensors of `dev` while another device is current."""
    now = _device() if _device is not None else torch.cuda.current_device()
    if now != dev:
        raise ValueError(f"tensors of cuda:{dev}, while cuda:{now} is the current device")


def _elsewhere(what: str, dev: int) -> ValueError:
    return ValueError(f"{what}: a tensor on cuda:{dev}")


def _i32(t, what: str, n: Optional[int] = None, dev: Optional[int] = None) -> Optional[int]:
    """Address of a contiguous int32 tensor (of n elements) on device dev (None: on any CUDA device)."""
    if t is None:
        return None
    if t.dtype is not _INT32 or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous int32 tensor")
    on = t.get_device()
    if on != dev and (dev is not None or on < 0):
        raise _elsewhere(what, max(dev or 0, 0))
    if n is not None and t.numel() != n:
        raise ValueError(f"{what}: {n} elements")
    return t.data_ptr()


def _space(t, dev: int) -> int:
    """Address of a workspace."""
    if not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"workspace: a contiguous tensor on cuda:{dev}")
    return t.data_ptr()


def make_kv(k, v, table, length, grown=None) -> Kv:
    """Descriptor of a paged cache over caller-owned tensors: k, v [layers, pages, kv heads, page size,
    head dim] (or without the layers), each page contiguous, the page and layer strides free; table
    [rows, max pages] and length [rows] int32; grown [rows] int32 (nullable) keeps which rows ``kv_extend`` found
    room in, so that new tokens of the others are left out.  Keeps references to all of them."""
    if k.dim() == 4:
        k, v = k[None], v[None]
    _want(k.dim() == 5 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and
          k.dtype in _DTYPES, "k and v: alike, [layers, pages, kv heads, page size, head dim], fp32, bf16 or fp16")
    dev = k.get_device()
    _want(dev >= 0 and v.get_device() == dev, "k and v: on one CUDA device")
    n_layers, n_pages, heads, page, dim = k.shape
    _want(k.stride()[2:] == (page * dim, dim, 1) or k[0, 0].is_contiguous(), "the elements of a page must be contiguous")
    _want(table.dim() == 2 and length.numel() == table.shape[0], "table [rows, max pages], length [rows]")
    c = Kv(k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], n_layers, n_pages, heads, page, dim,
           k.stride(1) if n_pages > 1 else heads * page * dim, k.stride(0) if n_layers > 1 else 0,
           _i32(table, "table", dev=dev), _i32(length, "length", dev=dev), table.shape[0], table.shape[1],
           _i32(grown, "grown", table.shape[0], dev))
    c._keepalive = (k, v, table, length, grown)
    c._plain = (k.dtype, table.shape[0], heads, dim, n_pages, table.shape[1], dev)   # plain values, cheaper to read than the fields
    return c


def _rows_of(t, dtype, heads: int, dim: int, what: str, rows: int, dev: int) -> int:
    """Row stride of [rows, heads, head dim] whose rows are contiguous inside."""
    if t.dtype is not dtype or t.shape != (rows, heads, dim):
        raise ValueError(f"{what}: [rows, heads, head dim] of the cache's type")
    if t.get_device() != dev:
        raise _elsewhere(what, dev)
    a, b, c = t.stride()
    if c != 1 or (b != dim and heads != 1) or (a < heads * dim and rows > 1):
        raise ValueError(f"{what}: contiguous inside a row, rows apart")
    return a if rows > 1 else 0


def kv_attend_workspace_bytes(kv: Kv, n_q_heads: int, group: int = 1) -> int:
    return int(lib().pg_kv_attend_workspace_bytes(kv._ref, n_q_heads, group))


def kv_attend(kv: Kv, layer: int, q, out, workspace, *, k_new=None, v_new=None, lse=None,
              scale: Optional[float] = None, group: int = 1, shared=None, status=None, stream=None) -> None:
    """Attention of one new token per row over the cache (see pg_kv_attend).  q, out [rows, query heads,
    head dim]; with k_new / v_new the rows' last token is stored on the way (not in a row that ``kv.grown`` says has no room for
    it); scale defaults to head_dim ** -0.5."""
    dtype, rows, kv_heads, dim, _, _, dev = kv._plain
    _current(dev)
    heads, k_at, v_at, new_stride = q.shape[1], None, None, 0
    q_stride = _rows_of(q, dtype, heads, dim, "q", rows, dev)
    out_stride = _rows_of(out, dtype, heads, dim, "out", rows, dev)
    if k_new is not None:
        new_stride = _rows_of(k_new, dtype, kv_heads, dim, "k_new", rows, dev)
        if v_new is None or new_stride != _rows_of(v_new, dtype, kv_heads, dim, "v_new", rows, dev):
            raise ValueError("k_new and v_new alike")
        k_at, v_at = k_new.data_ptr(), v_new.data_ptr()
    elif v_new is not None:
        raise ValueError("v_new without k_new")
    if lse is not None:
        if lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.numel() != rows * heads:
            raise ValueError("lse: [rows, query heads] fp32")
        if lse.get_device() != dev:
            raise _elsewhere("lse", dev)
        lse = lse.data_ptr()
    _check(lib().pg_kv_attend(kv._ref, layer, heads, q.data_ptr(), q_stride, k_at, v_at, new_stride,
                              dim ** -0.5 if scale is None else scale, group,
                              None if shared is None else _i32(shared, "shared", rows // max(group, 1), dev), out.data_ptr(), out_stride,
                              lse, _space(workspace, dev), workspace.nbytes, None if status is None else _i32(status, "status", None, dev),
                              _stream(stream)), "pg_kv_attend")


def kv_extend(kv: Kv, n_new, len_out, refs, refs_out, status=None, stream=None) -> None:
    """Room for n_new more tokens (an int for all rows, or int32 [rows]): lengths, pages, counts."""
    _, rows, _, _, pages, _, dev = kv._plain
    _current(dev)
    one = isinstance(n_new, int)
    _check(lib().pg_kv_extend(kv._ref, None if one else _i32(n_new, "n_new", rows, dev), n_new if one else 0,
                              _i32(len_out, "len_out", rows, dev), _i32(refs, "refs", pages, dev), _i32(refs_out, "refs_out", pages, dev),
                              _i32(status, "status", None, dev), _stream(stream)), "pg_kv_extend")


def kv_append(kv: Kv, layer: int, k_new, v_new, start=None, status=None, stream=None) -> None:
    """Keys and values [tokens, kv heads, head dim] of the rows' last tokens into one layer's pages;
    start [rows + 1] int32 says whose they are (None: one token per row)."""
    dtype, rows, kv_heads, dim, _, _, dev = kv._plain
    _current(dev)
    n = k_new.shape[0]
    stride = _rows_of(k_new, dtype, kv_heads, dim, "k_new", n, dev)
    if stride != _rows_of(v_new, dtype, kv_heads, dim, "v_new", n, dev):
        raise ValueError("k_new and v_new alike")
    _check(lib().pg_kv_append(kv._ref, layer, n, k_new.data_ptr(), v_new.data_ptr(), stride,
                              _i32(start, "start", rows + 1, dev), _i32(status, "status", None, dev), _stream(stream)), "pg_kv_append")


def kv_fork_workspace_bytes(kv: Kv, n_out: int) -> int:
    return int(lib().pg_kv_fork_workspace_bytes(kv._ref, n_out))


def kv_fork(kv: Kv, src_rows, table_out, len_out, refs, refs_out, workspace, status=None, stream=None) -> None:
    """New row i becomes a fork of old row src_rows[i]; rows without a fork give up their pages."""
    pages, width, dev = kv._plain[4:]
    _current(dev)
    n = 0 if src_rows is None else src_rows.numel()
    _check(lib().pg_kv_fork(kv._ref, n, _i32(src_rows, "src_rows", None, dev), _i32(table_out, "table_out", n * width, dev),
                            _i32(len_out, "len_out", n, dev), _i32(refs, "refs", pages, dev), _i32(refs_out, "refs_out", pages, dev),
                            _space(workspace, dev), workspace.nbytes, _i32(status, "status", None, dev), _stream(stream)), "pg_kv_fork")


def kv_pack_workspace_bytes(kv: Kv) -> int:
    return int(lib().pg_kv_pack_workspace_bytes(kv._ref))


def kv_pack(kv: Kv, refs, refs_out, table_out, workspace, page_map=None, status=None, stream=None) -> None:
    """Moves the pages in use to the front of the pool; the table and the counts follow."""
    _, rows, _, _, pages, width, dev = kv._plain
    _current(dev)
    _check(lib().pg_kv_pack(kv._ref, _i32(refs, "refs", pages, dev), _i32(refs_out, "refs_out", pages, dev),
                            _i32(table_out, "table_out", rows * width, dev), _i32(page_map, "page_map", pages, dev),
                            _space(workspace, dev), workspace.nbytes, _i32(status, "status", None, dev), _stream(stream)), "pg_kv_pack")


def kv_status(status, stream=None) -> None:
    """Raises PgError (EINDEX, ENOPAGES) if a call has flagged the status word; synchronises the stream."""
    _check(lib().pg_kv_status(_i32(status, "status"), _stream(stream)), "pg_kv_status")


TOKEN_WAITS = ("tiles", "stages", "queries", "scores", "weights", "products", "chunks")


def selftest_token_waits(*kinds: str) -> None:
    """Makes the named waits of the attention (``TOKEN_WAITS``) run out at once in the calls that follow; none: all wait again."""
    _check(lib().pg_selftest_token_waits(sum(1 << TOKEN_WAITS.index(k) for k in set(kinds))), "pg_selftest_token_waits")


def make_logits_rules(*, tokens=None, n_tokens=None, n_prompt=None, repetition=None, presence=None, frequency=None,
                      temperature=None, bias_ids=None, bias_values=None, mask=None) -> LogitsRules:
    """Rules for ``logits_process`` over caller-owned tensors (see pg_logits_rules): tokens [rows, most
    tokens] int32 (the rows may be strided), n_tokens / n_prompt [rows] int32, the penalties and the
    temperature [rows] fp32, bias_ids / bias_values [rows, n], mask [rows or 1, >= vocab / 32] int32."""
    r = LogitsRules()
    rows = dev = None

    def on(t, what):
        nonlocal dev
        dev = t.get_device() if dev is None else dev
        _want(dev >= 0 and t.get_device() == dev, f"{what}: all tensors of the rules on one CUDA device")

    def see(t, what):
        nonlocal rows
        on(t, what)
        _want(rows is None or rows == t.shape[0], f"{what}: one entry per row")
        rows = t.shape[0]

    if tokens is not None:
        _want(tokens.dim() == 2 and tokens.dtype == torch.int32 and (tokens.stride(1) == 1 or tokens.shape[1] <= 1),
              "tokens: [rows, most tokens] int32")
        see(tokens, "tokens")
        r.tokens, r.token_stride, r.max_tokens = tokens.data_ptr(), tokens.stride(0), tokens.shape[1]
    for name, t in (("n_tokens", n_tokens), ("n_prompt", n_prompt)):
        if t is not None:
            _want(t.dim() >= 1 and t.numel() == t.shape[0], f"{name}: [rows] int32")
            see(t, name)
            setattr(r, name, _i32(t, name))
    for name, t in (("repetition", repetition), ("presence", presence), ("frequency", frequency), ("temperature", temperature)):
        if t is not None:
            _want(t.dtype == torch.float32 and t.dim() == 1 and t.is_contiguous(), f"{name}: [rows] fp32")
            see(t, name)
            setattr(r, name, t.data_ptr())
    _want(bias_ids is None or bias_ids.dim() == 2, "bias_ids: [rows, n] int32")
    if bias_ids is not None and bias_ids.shape[1] > 0:
        _want(bias_values is not None and bias_values.shape == bias_ids.shape and bias_values.dtype == torch.float32 and
              bias_values.is_contiguous(), "bias_values: fp32, shaped like bias_ids")
        see(bias_ids, "bias_ids")
        on(bias_values, "bias_values")
        r.bias_ids, r.bias_values, r.n_bias = _i32(bias_ids, "bias_ids"), bias_values.data_ptr(), bias_ids.shape[1]
    if mask is not None:
        _want(mask.dim() == 2 and mask.dtype == torch.int32 and (mask.stride(1) == 1 or mask.shape[1] == 1), "mask: [rows or 1, words] int32")
        on(mask, "mask")
        if mask.shape[0] > 1:
            see(mask, "mask")
        r.mask, r.mask_stride = mask.data_ptr(), mask.stride(0) if mask.shape[0] > 1 else 0
    r._rows, r._mask_words, r._dev = rows, None if mask is None else mask.shape[1], dev
    r._keepalive = (tokens, n_tokens, n_prompt, repetition, presence, frequency, temperature, bias_ids, bias_values, mask)
    return r


def logits_process(logits, out, rules: LogitsRules, stream=None) -> None:
    """Applies the rules to logits [rows, vocab] (rows may be strided) into out (may be logits)."""
    rows, vocab = logits.shape
    from_type, to_type = _DTYPES.get(logits.dtype), _DTYPES.get(out.dtype)
    if from_type is None or to_type is None or out.shape != logits.shape:
        raise ValueError("logits and out: [rows, vocab], fp32, bf16 or fp16")
    (a, one), (b, one_out) = logits.stride(), out.stride()
    if (one != 1 or one_out != 1) and vocab > 1:
        raise ValueError("logits and out: contiguous rows")
    if rows <= 1:
        a = b = 0
    elif a < vocab or b < vocab:
        raise ValueError("logits and out: rows apart")
    dev = logits.get_device()
    if dev < 0 or out.get_device() != dev or (rules._dev is not None and rules._dev != dev):
        raise ValueError("logits, out and the rules: on one CUDA device")
    _current(dev)
    if rules._rows is not None and rules._rows != rows:
        raise ValueError("the rules are for another number of rows")
    if rules._mask_words is not None and rules._mask_words * 32 < vocab:
        raise ValueError("mask: too few words for the vocabulary")
    _check(lib().pg_logits_process(rows, vocab, from_type, logits.data_ptr(), a, to_type, out.data_ptr(), b, rules._ref,
                                   _stream(stream)), "pg_logits_process")


# ---------------------------------------------------------------- policy update on token trajectories

_FLOAT32 = torch.float32
_MOST = 2 ** 31 - 1                   # ctypes cuts what passes 32 bits without a word


def _f32(t, what: str, n: int, dev: int) -> int:
    """Address of a contiguous fp32 tensor of n elements on device dev."""
    if t.dtype is _FLOAT32 and t.numel() == n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    if t.get_device() != dev:
        raise _elsewhere(what, dev)
    raise ValueError(f"{what}: {n} contiguous fp32 elements")


def make_token_terms(*, temperature=None, ids=None, n_top: int = 0, teacher_ids=None, teacher_logp=None, kind: str = "forward") -> TokenTerms:
    """What ``token_forward`` and the others are asked about, over caller-owned tensors (see pg_token_terms): temperature [rows] fp32,
    ids [rows] or [rows, n] int32 given tokens, n_top alternatives, a teacher's list teacher_ids [rows, n] int32 with its
    log-probs teacher_logp [rows, n] fp32 and the kind of divergence (``DISTILL_KINDS``).  Keeps references to all of them."""
    r = TokenTerms()
    rows = dev = None

    def see(t, what):
        nonlocal rows, dev
        dev = t.get_device() if dev is None else dev
        _want(dev >= 0 and t.get_device() == dev, f"{what}: all tensors of the terms on one CUDA device")
        _want(rows is None or rows == t.shape[0], f"{what}: one entry per row")
        rows = t.shape[0]

    if temperature is not None:
        _want(temperature.dtype == torch.float32 and temperature.dim() == 1 and temperature.is_contiguous(), "temperature: [rows] fp32")
        see(temperature, "temperature")
        r.temperature = temperature.data_ptr()
    n_ids = 0
    if ids is not None:
        _want(ids.dim() in (1, 2), "ids: [rows] or [rows, n] int32")
        see(ids, "ids")
        n_ids = 1 if ids.dim() == 1 else ids.shape[1]
        _want(n_ids <= TOKEN_MAX_LIST, f"ids: at most {TOKEN_MAX_LIST} a row")
        r.ids, r.n_ids = _i32(ids, "ids") if n_ids else None, n_ids
    n_teacher = 0
    _want((teacher_ids is None) == (teacher_logp is None), "teacher_ids and teacher_logp: both or neither")
    if teacher_ids is not None:
        _want(teacher_ids.dim() == 2 and teacher_logp.shape == teacher_ids.shape and teacher_logp.dtype == torch.float32 and
              teacher_logp.is_contiguous(), "teacher_ids [rows, n] int32, teacher_logp fp32 of its shape")
        see(teacher_ids, "teacher_ids")
        see(teacher_logp, "teacher_logp")
        n_teacher = teacher_ids.shape[1]
        _want(n_teacher <= TOKEN_MAX_LIST, f"teacher_ids: at most {TOKEN_MAX_LIST} a row")
        if n_teacher:
            r.teacher_ids, r.teacher_logp, r.n_teacher = _i32(teacher_ids, "teacher_ids"), teacher_logp.data_ptr(), n_teacher
    _want(0 <= n_top <= TOKEN_MAX_TOP, f"n_top: 0..{TOKEN_MAX_TOP}")
    _want(kind in DISTILL_KINDS, f"kind: one of {DISTILL_KINDS}")
    r.n_top, r.kind = n_top, DISTILL_KINDS.index(kind)
    r._plain = (rows, dev, n_ids, n_top, n_teacher)
    r._keepalive = (temperature, ids, teacher_ids, teacher_logp)
    return r


def _token_rows(t, terms: TokenTerms, what: str):
    """(rows, vocab, type, row stride, device) of logits."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or t.dim() != 2:
        raise ValueError(f"{what}: [rows, vocab], fp32, bf16 or fp16")
    rows, vocab = t.shape
    dev = t.get_device()
    if rows > _MOST or vocab > _MOST:
        raise ValueError(f"{what}: rows and vocabulary in 32 bits")
    at, on = terms._plain[:2]
    if dev < 0 or (on is not None and on != dev):
        raise ValueError(f"{what} and the terms: on one CUDA device")
    if at is not None and at != rows:
        raise ValueError("the terms are for another number of rows")
    return rows, vocab, dtype, _row_stride(t, rows, vocab, what), dev


def _row_stride(t, rows: int, vocab: int, what: str) -> int:
    if t.is_contiguous():
        return 0
    a, one = t.stride()
    if (one != 1 and vocab > 1) or (rows > 1 and a < vocab):
        raise ValueError(f"{what}: contiguous rows, apart")
    return a if rows > 1 else 0


def _token_out(terms, rows, dev, logp, lse, entropy, top_ids, top_logp, distill, saved) -> TokenOut:
    _, _, n_ids, n_top, n_teacher = terms._plain
    o = TokenOut()
    if logp is not None:
        _want(n_ids > 0, "logp: the terms have no ids")
        o.logp = _f32(logp, "logp", rows * n_ids, dev)
    if lse is not None:
        o.lse = _f32(lse, "lse", rows, dev)
    if entropy is not None:
        o.entropy = _f32(entropy, "entropy", rows, dev)
    if top_ids is not None:
        _want(n_top > 0, "top_ids: the terms have no n_top")
        o.top_ids = _i32(top_ids, "top_ids", rows * n_top, dev)
    if top_logp is not None:
        _want(top_ids is not None, "top_logp without top_ids")
        o.top_logp = _f32(top_logp, "top_logp", rows * n_top, dev)
    if distill is not None:
        _want(n_teacher > 0, "distill: the terms have no teacher")
        o.distill = _f32(distill, "distill", rows, dev)
    if saved is not None:
        o.saved = _f32(saved, "saved", rows * TOKEN_SAVED, dev)
    return o


def _token_grads(terms, rows, dev, dlogp, dentropy, ddistill, entropy_scale, distill_scale) -> TokenGrads:
    _, _, n_ids, _, n_teacher = terms._plain
    g = TokenGrads()
    if dlogp is not None:
        _want(n_ids > 0, "dlogp: the terms have no ids")
        g.dlogp = _f32(dlogp, "dlogp", rows * n_ids, dev)
    if dentropy is not None:
        g.dentropy, g.entropy_scale = _f32(dentropy, "dentropy", rows, dev), entropy_scale
    if ddistill is not None:
        _want(n_teacher > 0, "ddistill: the terms have no teacher")
        g.ddistill, g.distill_scale = _f32(ddistill, "ddistill", rows, dev), distill_scale
    return g


def _token_dlogits(logits, dlogits, rows: int, vocab: int, dev: int) -> int:
    """Row stride of the gradient."""
    if dlogits.dtype is not logits.dtype or dlogits.shape != logits.shape or dlogits.get_device() != dev:
        raise ValueError("dlogits: like the logits")
    return _row_stride(dlogits, rows, vocab, "dlogits")


def token_forward(logits, terms: TokenTerms, *, logp=None, lse=None, entropy=None, top_ids=None, top_logp=None, distill=None, saved=None,
                  stream=None) -> None:
    """One pass over logits [rows, vocab] (rows may be strided) for whatever outputs are given (see pg_token_forward): logp [rows, given
    tokens], lse, entropy, distill [rows], top_ids (int32) / top_logp [rows, n_top], saved [rows, TOKEN_SAVED] for ``token_backward``."""
    rows, vocab, dtype, stride, dev = _token_rows(logits, terms, "logits")
    _current(dev)
    out = _token_out(terms, rows, dev, logp, lse, entropy, top_ids, top_logp, distill, saved)
    _check(lib().pg_token_forward(rows, vocab, dtype, logits.data_ptr(), stride, terms._ref, out, _stream(stream)), "pg_token_forward")


def token_backward(logits, terms: TokenTerms, saved, dlogits, *, dlogp=None, dentropy=None, ddistill=None, entropy_scale: float = 1.0,
                   distill_scale: float = 1.0, stream=None) -> None:
    """Gradient to the logits of what ``token_forward`` computed with the same terms (see pg_token_backward); dlogits may be logits."""
    rows, vocab, dtype, stride, dev = _token_rows(logits, terms, "logits")
    _current(dev)
    grads = _token_grads(terms, rows, dev, dlogp, dentropy, ddistill, entropy_scale, distill_scale)
    _check(lib().pg_token_backward(rows, vocab, dtype, logits.data_ptr(), stride, terms._ref, _f32(saved, "saved", rows * TOKEN_SAVED, dev),
                                   grads, dlogits.data_ptr(), _token_dlogits(logits, dlogits, rows, vocab, dev), _stream(stream)),
           "pg_token_backward")


def token_forward_backward(logits, terms: TokenTerms, dlogits, *, logp=None, lse=None, entropy=None, top_ids=None, top_logp=None,
                           distill=None, saved=None, dlogp=None, dentropy=None, ddistill=None, entropy_scale: float = 1.0,
                           distill_scale: float = 1.0, stream=None) -> None:
    """``token_forward`` and ``token_backward`` in one pass, for derivatives that are known before (see pg_token_forward_backward)."""
    rows, vocab, dtype, stride, dev = _token_rows(logits, terms, "logits")
    _current(dev)
    out = _token_out(terms, rows, dev, logp, lse, entropy, top_ids, top_logp, distill, saved)
    grads = _token_grads(terms, rows, dev, dlogp, dentropy, ddistill, entropy_scale, distill_scale)
    _check(lib().pg_token_forward_backward(rows, vocab, dtype, logits.data_ptr(), stride, terms._ref, out, grads, dlogits.data_ptr(),
                                           _token_dlogits(logits, dlogits, rows, vocab, dev), _stream(stream)), "pg_token_forward_backward")


def token_objective_workspace_bytes(n_tokens: int) -> int:
    if n_tokens > _MOST:
        raise ValueError("n_tokens: in 32 bits")
    return int(lib().pg_token_objective_workspace_bytes(n_tokens))


def token_objective(start, logp_new, adv, objective, dlogp, workspace, *, logp_old=None, logp_ref=None, entropy=None, distill=None,
                    clip_low: float = 0.2, clip_high: float = 0.2, beta: float = 0.0, entropy_coef: float = 0.0, distill_coef: float = 0.0,
                    scale: float = 1.0, norm: str = "rows", weight=None, ratio=None, stats=None, status=None, stream=None) -> None:
    """Clipped objective over ragged rows of tokens and its derivative (see pg_token_objective): start [rows + 1] int32, adv [rows], the
    other arrays [tokens], objective [1], stats [TOKEN_STATS], norm one of ``TOKEN_NORMS``."""
    dev = logp_new.get_device()
    if dev < 0:
        raise ValueError("logp_new: a CUDA tensor")
    _current(dev)
    rows, n = start.numel() - 1, logp_new.numel()
    if rows < 0:
        raise ValueError("start: [rows + 1] int32")
    if rows > _MOST or n > _MOST:
        raise ValueError("rows and tokens: in 32 bits")
    if norm not in TOKEN_NORMS:
        raise ValueError(f"norm: one of {TOKEN_NORMS}")
    b = TokenBatch()
    b.start, b.logp_new, b.adv = _i32(start, "start", rows + 1, dev), _f32(logp_new, "logp_new", n, dev), _f32(adv, "adv", rows, dev)
    if logp_old is not None:
        b.logp_old = _f32(logp_old, "logp_old", n, dev)
    if logp_ref is not None:
        b.logp_ref, b.beta = _f32(logp_ref, "logp_ref", n, dev), beta
    if entropy is not None:
        b.entropy, b.entropy_coef = _f32(entropy, "entropy", n, dev), entropy_coef
    if distill is not None:
        b.distill, b.distill_coef = _f32(distill, "distill", n, dev), distill_coef
    b.clip_low, b.clip_high, b.scale, b.norm = clip_low, clip_high, scale, TOKEN_NORMS.index(norm)
    _check(lib().pg_token_objective(rows, n, b, _f32(objective, "objective", 1, dev), _f32(dlogp, "dlogp", n, dev),
                                    None if weight is None else _f32(weight, "weight", n, dev), None if ratio is None else _f32(ratio, "ratio", n, dev),
                                    None if stats is None else _f32(stats, "stats", TOKEN_STATS, dev), _space(workspace, dev), workspace.nbytes,
                                    None if status is None else _i32(status, "status", None, dev), _stream(stream)), "pg_token_objective")


def strerror(code: int) -> str:
    return lib().pg_strerror(code).decode()


def launch_count() -> int:
    return int(lib().pg_launch_count())
