"""Thin ctypes binding of libmoshpit.so (see include/moshpit.h).

Argument marshalling only: every step of a round runs in the library's HIP
kernels.  PyTorch supplies device memory (the state tensor) and the stream.
There is no fallback: if the library is missing or a call fails, an exception
is raised.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoshpit.so")

F32, BF16 = 0, 1
SCHED_NONE, SCHED_IID, SCHED_REJOIN, SCHED_EXPLICIT = 0, 1, 2, 3
RUN_DEFAULT, RUN_FUSED = 0, 1

EXPORTS = [
    "moshpit_create", "moshpit_destroy", "moshpit_bind_state", "moshpit_round", "moshpit_round_dev",
    "moshpit_run", "moshpit_dist_to_mean", "moshpit_dist_to_mean_static", "moshpit_dist_to_mean_subset", "moshpit_group_keys", "moshpit_schedule_mask",
    "moshpit_dynamic_reset", "moshpit_dynamic_round", "moshpit_dynamic_keys", "moshpit_local_step", "moshpit_sgd_round", "moshpit_sgd_run", "moshpit_random_groups_round", "moshpit_random_permutation", "moshpit_refresh", "moshpit_refresh_donors", "moshpit_grouped_round", "moshpit_set_tuning", "moshpit_copy_probe", "moshpit_check_bf16_rounding", "moshpit_sync", "moshpit_last_error",
    "moshpit_embed", "moshpit_embed_grad", "moshpit_checkpoint", "moshpit_checkpoint_restore", "moshpit_weight_grad", "moshpit_token_logp",
    "moshpit_policy_loss", "moshpit_norm", "moshpit_norm_grad", "moshpit_dropout",
    "moshpit_attention", "moshpit_attention_grad", "moshpit_attention_cached",
]


class MoshpitError(RuntimeError):
    pass


class _CSchedule(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("down_rounds", ctypes.c_int32), ("p", ctypes.c_double),
                ("seed", ctypes.c_uint64), ("explicit_masks", ctypes.c_void_p), ("group_skip", ctypes.c_int32),
                ("refresh", ctypes.c_int32)]


@dataclass
class Schedule:
    kind: int = SCHED_NONE
    p: float = 0.0
    seed: int = 0
    down_rounds: int = 0
    explicit_masks: np.ndarray | None = None      # uint8 [rounds, N] for SCHED_EXPLICIT
    group_skip: bool = False                      # a group with an absent member skips the round
    refresh: bool = False                         # a returning peer first copies an up-to-date peer


_lib = None
_torch_module = None
_raw_stream = None


def _torch():
    """torch, imported at the first call that needs it (an import statement per call costs as much as a kernel's launch)."""
    global _torch_module, _raw_stream
    if _torch_module is None:
        import torch
        _torch_module, _raw_stream = torch, getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return _torch_module


def _current_stream(index: int) -> int:
    """Handle of device `index`'s current stream (torch's Stream object for it takes 2 us to make, as long as a launch)."""
    return _raw_stream(index) if _raw_stream else _torch().cuda.current_stream(index).cuda_stream


def load_library() -> ctypes.CDLL:
    """Load libmoshpit.so (built in-tree by __graft_entry__.build())."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise MoshpitError(f"{LIB_PATH} is missing: run `python __graft_entry__.py` to build it")
    lib = ctypes.CDLL(LIB_PATH)
    i64, i32, vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
    lib.moshpit_create.argtypes = [i64, i64, i32, i32, i32, ctypes.POINTER(vp)]
    lib.moshpit_destroy.argtypes = [vp]
    lib.moshpit_bind_state.argtypes = [vp, vp, i64, vp]
    lib.moshpit_round.argtypes = [vp, i64, vp]
    lib.moshpit_round_dev.argtypes = [vp, i64, vp]
    lib.moshpit_run.argtypes = [vp, i64, i32, ctypes.POINTER(_CSchedule), i32, vp, vp]
    lib.moshpit_dist_to_mean.argtypes = [vp, ctypes.POINTER(ctypes.c_double)]
    lib.moshpit_dist_to_mean_static.argtypes = [vp, i64, i64, i64, i32, vp, vp]
    lib.moshpit_dist_to_mean_subset.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_double)]
    lib.moshpit_group_keys.argtypes = [vp, i64, vp]
    lib.moshpit_schedule_mask.argtypes = [vp, ctypes.POINTER(_CSchedule), i64, i32, vp]
    lib.moshpit_dynamic_reset.argtypes = [vp]
    lib.moshpit_dynamic_round.argtypes = [vp, i64, ctypes.c_uint64, vp]
    lib.moshpit_dynamic_keys.argtypes = [vp, vp]
    lib.moshpit_local_step.argtypes = [vp, vp, vp, i64, ctypes.c_float]
    lib.moshpit_sgd_round.argtypes = [vp, i64, vp, vp, i64, ctypes.c_float]
    lib.moshpit_sgd_run.argtypes = [vp, i64, i32, ctypes.POINTER(_CSchedule), i32, vp, i64, ctypes.c_float, vp, vp]
    lib.moshpit_random_groups_round.argtypes = [vp, i64, ctypes.c_uint64, i32, vp]
    lib.moshpit_random_permutation.argtypes = [vp, i64, ctypes.c_uint64, vp]
    lib.moshpit_refresh.argtypes = [vp, i64, ctypes.c_uint64, vp, vp]
    lib.moshpit_refresh_donors.argtypes = [vp, i64, ctypes.c_uint64, vp, vp, vp]
    lib.moshpit_grouped_round.argtypes = [vp, vp, i64, i32, vp]
    lib.moshpit_set_tuning.argtypes = [vp, i32, i32, i32, i32, i32, i32]
    lib.moshpit_copy_probe.argtypes = [vp, vp, i64, vp]
    lib.moshpit_check_bf16_rounding.argtypes = [vp, vp]
    f32 = ctypes.c_float
    lib.moshpit_embed.argtypes = [vp, i64, i64, i64, vp, i64, f32, vp, i32, i64]
    lib.moshpit_embed_grad.argtypes = [vp, vp, i32, i64, vp, i64, f32, i32, vp, i64, i64, i64, i64]
    lib.moshpit_checkpoint.argtypes = [vp, vp, i32, i64, i64, i64, vp, vp]
    lib.moshpit_checkpoint_restore.argtypes = [vp, vp, vp, i64, i64, vp, i32, i64]
    lib.moshpit_weight_grad.argtypes = [vp, vp, i32, i64, vp, vp, i64, i64, i64, i32, vp, i64, i64]
    lib.moshpit_token_logp.argtypes = [vp, vp, i32, i64, vp, i64, i64, vp]
    lib.moshpit_policy_loss.argtypes = [vp, vp, i32, i64, vp, i64, i64, vp, vp, vp, vp, f32, f32, f32, vp, i64, vp, vp]
    lib.moshpit_norm.argtypes = [vp, vp, i32, i64, vp, i64, i64, i64, i64, f32, vp, i64, vp, i64, vp, vp]
    lib.moshpit_norm_grad.argtypes = [vp, vp, i32, i64, vp, i64, vp, i64, i64, i64, i64, f32, vp, i64, i32, vp, i64]
    lib.moshpit_dropout.argtypes = [vp, vp, i32, i64, vp, i64, i64, i64, ctypes.c_double, ctypes.c_uint64, vp, vp, i64]
    lib.moshpit_attention.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, vp, i64, i32, i32, i32, f32, vp, i64, vp]
    lib.moshpit_attention_grad.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, vp, i64, i32, i32, i32, f32, vp, i64, vp, i64, vp, i64]
    lib.moshpit_attention_cached.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, vp, i64, i64, i64, i32, i32, i32, f32, vp, i64]
    lib.moshpit_sync.argtypes = [vp]
    lib.moshpit_last_error.argtypes = [vp]
    lib.moshpit_last_error.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name != "moshpit_last_error":
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _c_schedule(s: Schedule | None, rounds: int, N: int):
    if s is None:
        return None, None
    keep = None
    ptr = None
    if s.kind == SCHED_EXPLICIT:
        keep = np.ascontiguousarray(s.explicit_masks, dtype=np.uint8)
        if keep.shape != (rounds, N):
            raise ValueError("explicit masks must have shape (rounds, N)")
        ptr = keep.ctypes.data
    return _CSchedule(s.kind, s.down_rounds, float(s.p), s.seed, ptr, 1 if s.group_skip else 0, 1 if s.refresh else 0), keep


class Moshpit:
    """One handle = one peer-state matrix of N = M^d rows with P parameters."""

    _bound = None                              # device index (None: the tensors') and handle of the bound stream

    def __init__(self, N: int, P: int, M: int, d: int, dtype: int):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        rc = self._lib.moshpit_create(N, P, M, d, dtype, ctypes.byref(self._h))
        if rc != 0:
            msg = self._lib.moshpit_last_error(None).decode()
            self._h = ctypes.c_void_p()
            raise MoshpitError(f"moshpit_create failed ({rc}): {msg}")
        self.N, self.P, self.M, self.d, self.dtype = N, P, M, d, dtype
        self._state = None

    # -- plumbing ---------------------------------------------------------
    def _check(self, rc: int, what: str) -> None:
        if rc != 0:
            raise MoshpitError(f"{what} failed ({rc}): {self._lib.moshpit_last_error(self._h).decode()}")

    def close(self) -> None:
        if self._h:
            self._lib.moshpit_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._state = self._bound = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C ABI, one method per entry point ------------------------------
    def bind_state(self, X, stream=None) -> None:
        """X: torch tensor [N, P] on the GPU (float32 or bfloat16), unit column stride."""
        torch = _torch()
        want = torch.float32 if self.dtype == F32 else torch.bfloat16
        if X.dtype != want or X.dim() != 2 or tuple(X.shape) != (self.N, self.P) or not X.is_cuda:
            raise ValueError("state tensor has the wrong dtype, shape or device")
        if X.stride(1) != 1:
            raise ValueError("state tensor must have unit column stride")
        if stream is None:
            stream = torch.cuda.current_stream(X.device)
        self._check(self._lib.moshpit_bind_state(self._h, X.data_ptr(), X.stride(0), stream.cuda_stream), "bind_state")
        self._state = (X, stream)              # keep both alive
        self._bound = (X.device.index, stream.cuda_stream)

    def bind_raw(self, ptr: int, row_stride: int, stream_handle: int = 0) -> None:
        self._check(self._lib.moshpit_bind_state(self._h, ptr, row_stride, stream_handle), "bind_state")
        self._state = (None, None)             # (the caller keeps the state alive; _stream() makes the stream's object)
        self._bound = (None, stream_handle)

    def _stream(self):
        """The bound stream as an object of torch's."""
        X, stream = self._state
        if stream is None:
            cuda, handle = _torch().cuda, self._bound[1]
            stream = cuda.ExternalStream(handle) if handle else cuda.default_stream()
            self._state = (X, stream)
        return stream

    def round(self, t: int, alive=None) -> None:
        if alive is None:
            self._check(self._lib.moshpit_round(self._h, t, None), "round")
            return
        a = np.ascontiguousarray(alive, dtype=np.uint8)
        if a.shape != (self.N,):
            raise ValueError("alive mask must have shape (N,)")
        self._check(self._lib.moshpit_round(self._h, t, a.ctypes.data), "round")

    def round_dev(self, t: int, alive_dev) -> None:
        """alive_dev: torch uint8 tensor [N] on the GPU, or None."""
        ptr = None
        if alive_dev is not None:
            if alive_dev.numel() != self.N or alive_dev.element_size() != 1 or not alive_dev.is_contiguous():
                raise ValueError("device mask must be N contiguous bytes")
            ptr = alive_dev.data_ptr()
        self._check(self._lib.moshpit_round_dev(self._h, t, ptr), "round_dev")

    def run(self, t0: int, rounds: int, schedule: Schedule | None = None, want_dist: bool = False,
            want_times: bool = False, flags: int = 0):
        cs, keep = _c_schedule(schedule, rounds, self.N)
        dist = np.zeros(rounds + 1, dtype=np.float64) if want_dist else None
        ms = np.zeros(rounds, dtype=np.float32) if want_times else None
        rc = self._lib.moshpit_run(self._h, t0, rounds, ctypes.byref(cs) if cs is not None else None, flags,
                                   dist.ctypes.data if want_dist else None, ms.ctypes.data if want_times else None)
        self._check(rc, "run")
        del keep
        return dist, ms

    def dist_to_mean(self) -> float:
        out = ctypes.c_double()
        self._check(self._lib.moshpit_dist_to_mean(self._h, ctypes.byref(out)), "dist_to_mean")
        return out.value

    def dist_to_mean_subset(self, present) -> float:
        """present: uint8 [N], non-zero = the row holds a peer (None = all rows)."""
        out = ctypes.c_double()
        ptr = None
        if present is not None:
            keep = np.ascontiguousarray(present, dtype=np.uint8)
            if keep.shape != (self.N,):
                raise ValueError("present mask must have shape (N,)")
            ptr = keep.ctypes.data
        self._check(self._lib.moshpit_dist_to_mean_subset(self._h, ptr, ctypes.byref(out)), "dist_to_mean_subset")
        return out.value

    def group_keys(self, t: int) -> np.ndarray:
        keys = np.empty(self.N, dtype=np.int32)
        self._check(self._lib.moshpit_group_keys(self._h, t, keys.ctypes.data), "group_keys")
        return keys

    def schedule_mask(self, schedule: Schedule | None, t0: int, rounds: int) -> np.ndarray:
        cs, keep = _c_schedule(schedule, rounds, self.N)
        masks = np.empty((rounds, self.N), dtype=np.uint8)
        rc = self._lib.moshpit_schedule_mask(self._h, ctypes.byref(cs) if cs is not None else None, t0, rounds,
                                             masks.ctypes.data)
        self._check(rc, "schedule_mask")
        del keep
        return masks

    def _alive_ptr(self, alive):
        if alive is None:
            return None, None
        a = np.ascontiguousarray(alive, dtype=np.uint8)
        if a.shape != (self.N,):
            raise ValueError("alive mask must have shape (N,)")
        return a, a.ctypes.data

    def dynamic_reset(self) -> None:
        self._check(self._lib.moshpit_dynamic_reset(self._h), "dynamic_reset")

    def dynamic_round(self, t: int, seed: int, alive=None) -> None:
        keep, ptr = self._alive_ptr(alive)
        self._check(self._lib.moshpit_dynamic_round(self._h, t, seed, ptr), "dynamic_round")

    def dynamic_keys(self) -> np.ndarray:
        keys = np.zeros((self.N, max(self.d - 1, 0)), dtype=np.int32)
        self._check(self._lib.moshpit_dynamic_keys(self._h, keys.ctypes.data if keys.size else None), "dynamic_keys")
        return keys

    def _grad(self, G):
        torch = _torch()
        want = torch.float32 if self.dtype == F32 else torch.bfloat16
        if G.dtype != want or tuple(G.shape) != (self.N, self.P) or G.stride(1) != 1 or not G.is_cuda:
            raise ValueError("gradient tensor must match the state's dtype, shape and device")
        return G.data_ptr(), G.stride(0)

    def local_step(self, G, gamma: float, alive=None) -> None:
        keep, ptr = self._alive_ptr(alive)
        gp, gs = self._grad(G)
        self._lend(G)
        self._check(self._lib.moshpit_local_step(self._h, ptr, gp, gs, gamma), "local_step")

    def sgd_round(self, t: int, G, gamma: float, alive=None) -> None:
        keep, ptr = self._alive_ptr(alive)
        gp, gs = self._grad(G)
        self._lend(G)
        self._check(self._lib.moshpit_sgd_round(self._h, t, ptr, gp, gs, gamma), "sgd_round")

    def sgd_run(self, t0: int, rounds: int, G, gamma: float, schedule: Schedule | None = None, want_dist: bool = False,
                want_times: bool = False, flags: int = 0):
        cs, keep = _c_schedule(schedule, rounds, self.N)
        gp, gs = self._grad(G)
        self._lend(G)
        dist = np.zeros(rounds + 1, dtype=np.float64) if want_dist else None
        ms = np.zeros(rounds, dtype=np.float32) if want_times else None
        rc = self._lib.moshpit_sgd_run(self._h, t0, rounds, ctypes.byref(cs) if cs is not None else None, flags, gp, gs,
                                       gamma, dist.ctypes.data if want_dist else None,
                                       ms.ctypes.data if want_times else None)
        self._check(rc, "sgd_run")
        del keep
        return dist, ms

    def random_groups_round(self, t: int, seed: int, group_size: int, alive=None) -> None:
        keep, ptr = self._alive_ptr(alive)
        self._check(self._lib.moshpit_random_groups_round(self._h, t, seed, group_size, ptr), "random_groups_round")

    def random_permutation(self, t: int, seed: int) -> np.ndarray:
        perm = np.empty(self.N, dtype=np.int32)
        self._check(self._lib.moshpit_random_permutation(self._h, t, seed, perm.ctypes.data), "random_permutation")
        return perm

    def _two_masks(self, prev, cur):
        a = np.ascontiguousarray(prev, dtype=np.uint8)
        b = np.ascontiguousarray(cur, dtype=np.uint8)
        if a.shape != (self.N,) or b.shape != (self.N,):
            raise ValueError("masks must have shape (N,)")
        return a, b

    def refresh(self, t: int, seed: int, alive_prev, alive_cur) -> None:
        a, b = self._two_masks(alive_prev, alive_cur)
        self._check(self._lib.moshpit_refresh(self._h, t, seed, a.ctypes.data, b.ctypes.data), "refresh")

    def refresh_donors(self, t: int, seed: int, alive_prev, alive_cur) -> np.ndarray:
        a, b = self._two_masks(alive_prev, alive_cur)
        donors = np.empty(self.N, dtype=np.int32)
        self._check(self._lib.moshpit_refresh_donors(self._h, t, seed, a.ctypes.data, b.ctypes.data,
                                                     donors.ctypes.data), "refresh_donors")
        return donors

    def grouped_round(self, index, group_size: int, alive=None) -> None:
        idx = np.ascontiguousarray(index, dtype=np.int32)
        keep, ptr = self._alive_ptr(alive)
        self._check(self._lib.moshpit_grouped_round(self._h, idx.ctypes.data, len(idx), group_size, ptr),
                    "grouped_round")

    def set_tuning(self, cols: int = 0, unroll: int = 0, nontemporal: int = -1, block: int = 0,
                   waves_per_cu: int = 0, order: int = -1) -> None:
        self._check(self._lib.moshpit_set_tuning(self._h, cols, unroll, nontemporal, block, waves_per_cu, order),
                    "set_tuning")

    # -- the local step of language-model peers --------------------------------
    # Calls are queued on the bound stream.  Where another one is current, the caller orders the two (what a call reads has to be written
    # by then, what it writes is there after a wait); memory is looked after here, so temporaries may be given and results dropped.
    @staticmethod
    def _type_code(dtype) -> int:
        torch = _torch()
        if dtype is torch.float32:
            return F32
        if dtype is torch.bfloat16:
            return BF16
        raise ValueError("activations must be float32 or bfloat16")

    def _lend(self, *tensors) -> None:
        """Tensors that the bound stream is to use (None among them is passed over).  Where another stream is current, the allocator
        is told so: their memory, once given back, is not given out again before the bound stream is through with it."""
        bound = self._bound
        if bound is not None and _current_stream(bound[0] if bound[0] is not None else tensors[0].device.index) != bound[1]:
            stream = self._stream()
            for x in tensors:
                if x is not None:
                    x.record_stream(stream)

    def _new(self, device, *wanted):
        """New tensors, one per (shape, dtype), out of the bound stream's memory: a block that another stream has just given back may
        still be in use there.  Where another stream is current it will use them, too, which the allocator is told."""
        torch, bound = _torch(), self._bound
        if bound is None or _current_stream(bound[0] if bound[0] is not None else device.index) == bound[1]:
            return [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in wanted]
        with torch.cuda.stream(self._stream()):
            new = [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in wanted]
        for x in new:
            x.record_stream(torch.cuda.current_stream(device))
        return new

    def _rows(self, x, name: str, T: int | None = None):
        """x: [N, T, width] on the GPU, unit column stride, row i * T + t at a constant stride.
        Returns (pointer, type code, T, width, row stride)."""
        if x.dim() != 3 or x.shape[0] != self.N or not x.is_cuda or (T is not None and x.shape[1] != T):
            raise ValueError(f"{name} must be a GPU tensor [N, {'T' if T is None else T}, width]")
        _, n, width = x.shape
        peer, row, col = x.stride()
        if width > 1 and col != 1:
            raise ValueError(f"{name} must have unit column stride")
        stride = row if n > 1 else peer if n == 1 else max(peer, width)      # (of no rows any stride will do)
        if n > 1 and peer != n * row or stride < width:
            raise ValueError(f"rows of {name} must lie at one constant distance over all peers and tokens")
        return x.data_ptr(), self._type_code(x.dtype), n, width, stride

    def _tokens(self, tokens):
        """tokens: int32 [N, T] on the GPU, contiguous."""
        torch = _torch()
        if tokens.dtype != torch.int32 or tokens.dim() != 2 or tokens.shape[0] != self.N or not tokens.is_cuda or not tokens.is_contiguous():
            raise ValueError("tokens must be a contiguous int32 GPU tensor [N, T]")
        return tokens.data_ptr(), tokens.shape[1]

    def _per_token(self, shape, *named):
        """Pointers of float32 GPU tensors [N, T]; named: (tensor, name) pairs."""
        f32 = _torch().float32
        for x, name in named:
            if x.dtype is not f32 or x.shape != shape or not x.is_cuda or not x.is_contiguous():
                raise ValueError(f"{name} must be a contiguous float32 GPU tensor {list(shape)}")
        return [x.data_ptr() for x, _ in named]

    def embed(self, tokens, column: int, vocab: int, width: int, scale: float = 1.0, out=None, dtype=None):
        """Token embeddings [N, T, width] from the tables [vocab, width] that start at parameter `column` of
        every peer.  out: tensor to write; without it a new one of `dtype` (the state's if not given)."""
        torch = _torch()
        tp, T = self._tokens(tokens)
        if out is None:
            dtype = dtype or (torch.float32 if self.dtype == F32 else torch.bfloat16)
            out, = self._new(tokens.device, ((self.N, T, width), dtype))
        op, code, _, w, stride = self._rows(out, "out", T)
        if w != width:
            raise ValueError("out must be [N, T, width]")
        self._lend(tokens, out)
        self._check(self._lib.moshpit_embed(self._h, column, vocab, width, tp, T, scale, op, code, stride), "embed")
        return out

    def embed_grad(self, dY, tokens, G, column: int, vocab: int, scale: float = 1.0, accumulate: bool = False) -> None:
        """Gradient of the tables for dY [N, T, width], into columns column.. of the gradient matrix G."""
        tp, T = self._tokens(tokens)
        yp, code, _, width, stride = self._rows(dY, "dY", T)
        gp, gs = self._grad(G)
        self._lend(dY, tokens, G)
        self._check(self._lib.moshpit_embed_grad(self._h, yp, code, stride, tp, T, scale, int(accumulate), gp, gs, column, vocab, width),
                    "embed_grad")

    def checkpoint(self, x):
        """x [N, T, width] in 8 bits: (codes int8 [N, T, width], scales uint8 [N, T, ceil(width / 32)])."""
        torch = _torch()
        xp, code, T, width, stride = self._rows(x, "x")
        self._lend(x)
        codes, scales = self._new(x.device, ((self.N, T, width), torch.int8), ((self.N, T, -(-width // 32)), torch.uint8))
        self._check(self._lib.moshpit_checkpoint(self._h, xp, code, self.N * T, width, stride, codes.data_ptr(), scales.data_ptr()),
                    "checkpoint")
        return codes, scales

    def _saved(self, codes, scales):
        torch = _torch()
        if codes.dtype != torch.int8 or scales.dtype != torch.uint8 or codes.dim() != 3 or codes.shape[0] != self.N or \
                tuple(scales.shape) != (*codes.shape[:2], -(-codes.shape[2] // 32)) or not codes.is_cuda or not scales.is_cuda or \
                not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be what checkpoint() returned")
        return codes.data_ptr(), scales.data_ptr()

    def checkpoint_restore(self, codes, scales, dtype=None, out=None):
        """The activations that codes and scales stand for, in `dtype` (float32 if not given) or into `out`."""
        torch = _torch()
        cp, sp = self._saved(codes, scales)
        if out is None:
            out, = self._new(codes.device, (codes.shape, dtype or torch.float32))
        op, code, T, width, stride = self._rows(out, "out", codes.shape[1])
        if width != codes.shape[2]:
            raise ValueError("out must have the shape of codes")
        self._lend(codes, scales, out)
        self._check(self._lib.moshpit_checkpoint_restore(self._h, cp, sp, self.N * T, width, op, code, stride), "checkpoint_restore")
        return out

    def weight_grad(self, dY, codes, scales, G, column: int, accumulate: bool = False) -> None:
        """Gradient [outs, ins] of a linear layer's weights for dY [N, T, outs] and the saved input [N, T, ins], into
        columns column.. of the gradient matrix G."""
        cp, sp = self._saved(codes, scales)
        yp, code, T, outs, stride = self._rows(dY, "dY", codes.shape[1])
        gp, gs = self._grad(G)
        self._lend(dY, codes, scales, G)
        self._check(self._lib.moshpit_weight_grad(self._h, yp, code, stride, cp, sp, T, outs, codes.shape[2], int(accumulate), gp, gs, column),
                    "weight_grad")

    def token_logp(self, logits, tokens):
        """Log-probabilities [N, T] (float32) of `tokens` under logits [N, T, vocab]."""
        torch = _torch()
        tp, T = self._tokens(tokens)
        zp, code, _, vocab, stride = self._rows(logits, "logits", T)
        self._lend(logits, tokens)
        logp, = self._new(logits.device, ((self.N, T), torch.float32))
        self._check(self._lib.moshpit_token_logp(self._h, zp, code, stride, tp, T, vocab, logp.data_ptr()), "token_logp")
        return logp

    def policy_loss(self, logits, tokens, old_logp, advantage, weight, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2,
                    kl_coef: float = 0.0, grad=None):
        """Clipped policy loss with a KL term: (stats [N, 3] = loss, KL, clipped weight of every peer; logp [N, T]).  The
        logits' gradient goes into `grad` (like logits; None: into the logits themselves)."""
        torch = _torch()
        tp, T = self._tokens(tokens)
        zp, code, _, vocab, stride = self._rows(logits, "logits", T)
        dp, dcode, _, dvocab, dstride = (zp, code, T, vocab, stride) if grad is None else self._rows(grad, "grad", T)
        if dcode != code or dvocab != vocab:
            raise ValueError("grad must have the type and shape of logits")
        shape = tokens.shape
        old, adv, w = self._per_token(shape, (old_logp, "old_logp"), (advantage, "advantage"), (weight, "weight"))
        ref = None if ref_logp is None else self._per_token(shape, (ref_logp, "ref_logp"))[0]
        self._lend(logits, tokens, old_logp, advantage, weight, ref_logp, grad)
        logp, stats = self._new(logits.device, ((self.N, T), torch.float32), ((self.N, 3), torch.float32))
        self._check(self._lib.moshpit_policy_loss(self._h, zp, code, stride, tp, T, vocab, old, ref, adv, w, clip_low, clip_high, kl_coef, dp,
                                                  dstride, logp.data_ptr(), stats.data_ptr()), "policy_loss")
        return stats, logp

    def _like(self, x, code: int, T: int, width: int, name: str):
        """Pointer and row stride of a further matrix of a call, of the type and shape of the first; None: (None, 0)."""
        if x is None:
            return None, 0
        p, c, _, w, stride = self._rows(x, name, T)
        if c != code or w != width:
            raise ValueError(f"{name} must have the type and shape of the input")
        return p, stride

    def norm(self, x, column: int, residual=None, eps: float = 1e-6, saved: bool = False, out=None, total=None):
        """Root-mean-square norm of h = x + residual [N, T, width] with the gain that starts at parameter `column` of every peer.
        Returns (y, h, saved): h is x where there is no residual, saved is what checkpoint(y) gives where that is wanted, else None."""
        torch = _torch()
        xp, code, T, width, stride = self._rows(x, "x")
        if residual is None:
            if total is not None:
                raise ValueError("without a residual x is the total itself")
        wanted = [((self.N, T, width), x.dtype)] * ((out is None) + (total is None and residual is not None))
        if saved:
            wanted += [((self.N, T, width), torch.int8), ((self.N, T, -(-width // 32)), torch.uint8)]
        rp, rs = self._like(residual, code, T, width, "residual")
        new = self._new(x.device, *wanted) if wanted else []
        out = new.pop(0) if out is None else out
        if residual is not None and total is None:
            total = new.pop(0)
        op, os_ = self._like(out, code, T, width, "out")
        hp, hs = self._like(total, code, T, width, "total")
        self._lend(x, residual, out, total)
        self._check(self._lib.moshpit_norm(self._h, xp, code, stride, rp, rs, T, column, width, eps, hp, hs, op, os_,
                                           *([t.data_ptr() for t in new] if saved else (None, None))), "norm")
        return out, x if residual is None else total, tuple(new) if saved else None

    def norm_grad(self, dY, x, G, column: int, eps: float = 1e-6, dtotal=None, accumulate: bool = False, out=None):
        """Backward pass of norm for dY [N, T, width]; x: the h that norm returned, dtotal: the gradient that reaches h elsewhere.  Returns
        h's gradient (in `out` if given); the gain's goes into columns column.. of the gradient matrix G."""
        yp, code, T, width, stride = self._rows(dY, "dY")
        xp, xs = self._like(x, code, T, width, "x")
        tp, ts = self._like(dtotal, code, T, width, "dtotal")
        gp, gs = self._grad(G)
        if out is None:
            out, = self._new(dY.device, ((self.N, T, width), dY.dtype))
        op, os_ = self._like(out, code, T, width, "out")
        self._lend(dY, x, dtotal, G, out)
        self._check(self._lib.moshpit_norm_grad(self._h, yp, code, stride, xp, xs, tp, ts, T, column, width, eps, op, os_, int(accumulate), gp, gs),
                    "norm_grad")
        return out

    def dropout(self, x, p: float, seed: int, step=None, residual=None, out=None):
        """residual + dropout(x) for x [N, T, width]; the mask follows from seed (0 .. 2^64 - 1), from `step` (None: 0, or one int64 on the GPU,
        read when the call runs) and from the place of an element.  The backward pass is the same call on the gradient."""
        torch = _torch()
        xp, code, T, width, stride = self._rows(x, "x")
        rp, rs = self._like(residual, code, T, width, "residual")
        if step is not None and (step.dtype is not torch.int64 or step.numel() != 1 or not step.is_cuda):
            raise ValueError("step must be one int64 on the GPU")
        if not 0 <= seed < 1 << 64:
            raise ValueError("seed must be a whole number from 0 to 2^64 - 1")
        if out is None:
            out, = self._new(x.device, ((self.N, T, width), x.dtype))
        op, os_ = self._like(out, code, T, width, "out")
        self._lend(x, residual, step, out)
        self._check(self._lib.moshpit_dropout(self._h, xp, code, stride, rp, rs, T, width, p, seed, None if step is None else step.data_ptr(), op, os_),
                    "dropout")
        return out

    def _heads(self, q, k, v, heads: int, kv_heads, scale):
        """What attention calls begin with: (q pointer, stride, k .., v ..), type code, query rows, key rows, kv_heads, depth, scale."""
        kv_heads = heads if kv_heads is None else kv_heads
        qp, code, rows, width, qs = self._rows(q, "q")
        if heads < 1 or kv_heads < 1 or width % heads:
            raise ValueError("q must hold `heads` heads in a row")
        depth = width // heads
        kp, kcode, keys, kwidth, ks = self._rows(k, "k")
        vp, vcode, _, vwidth, vs = self._rows(v, "v", keys)
        if kcode != code or vcode != code or kwidth != kv_heads * depth or vwidth != kwidth:
            raise ValueError("k and v must have the type of q and hold `kv_heads` heads of its depth")
        return (qp, qs, kp, ks, vp, vs), code, rows, keys, kv_heads, depth, depth ** -0.5 if scale is None else scale

    def _first(self, first, T: int):
        if first.dtype is not _torch().int32 or first.shape != (self.N, T) or not first.is_cuda or not first.is_contiguous():
            raise ValueError(f"first must be a contiguous int32 GPU tensor {[self.N, T]}")
        return first.data_ptr()

    def attention(self, q, k, v, first, heads: int, kv_heads: int | None = None, scale: float | None = None, out=None):
        """Causal attention for q [N, T, heads * depth], k and v [N, T, kv_heads * depth] over packed sequences: token t sees tokens first[t] .. t
        (int32 [N, T]; -1: no token).  scale: depth ** -0.5 if not given.  Returns (out, lse [N, heads, T])."""
        rows, code, T, keys, kv_heads, depth, scale = self._heads(q, k, v, heads, kv_heads, scale)
        if keys != T:
            raise ValueError("q, k and v must have the same tokens")
        fp, f32 = self._first(first, T), _torch().float32
        if out is None:
            out, lse = self._new(q.device, (q.shape, q.dtype), ((self.N, heads, T), f32))
        else:
            lse, = self._new(q.device, ((self.N, heads, T), f32))
        op, os_ = self._like(out, code, T, heads * depth, "out")
        self._lend(q, k, v, first, out)
        self._check(self._lib.moshpit_attention(self._h, *rows, code, fp, T, heads, kv_heads, depth, scale, op, os_, lse.data_ptr()), "attention")
        return out, lse

    def attention_grad(self, dout, q, k, v, out, lse, first, heads: int, kv_heads: int | None = None, scale: float | None = None, dq=None, dk=None,
                       dv=None):
        """Backward pass of attention for dout [N, T, heads * depth], with the out and lse that it returned: (dq, dk, dv), in the tensors given for
        them or in new ones."""
        rows, code, T, keys, kv_heads, depth, scale = self._heads(q, k, v, heads, kv_heads, scale)
        if keys != T:
            raise ValueError("q, k and v must have the same tokens")
        fp, (lp,) = self._first(first, T), self._per_token((self.N, heads, T), (lse, "lse"))
        width = heads * depth
        yp, ys = self._like(dout, code, T, width, "dout")
        op, os_ = self._like(out, code, T, width, "out")
        missing = [t for t, given in ((q, dq), (k, dk), (v, dv)) if given is None]
        new = self._new(q.device, *((t.shape, t.dtype) for t in missing)) if missing else []
        dq, dk, dv = (new.pop(0) if given is None else given for given in (dq, dk, dv))
        into = [*self._like(dq, code, T, width, "dq"), *self._like(dk, code, T, kv_heads * depth, "dk"), *self._like(dv, code, T, kv_heads * depth, "dv")]
        self._lend(dout, q, k, v, out, lse, first, dq, dk, dv)
        self._check(self._lib.moshpit_attention_grad(self._h, yp, ys, *rows, op, os_, code, lp, fp, T, heads, kv_heads, depth, scale, *into),
                    "attention_grad")
        return dq, dk, dv

    def attention_cached(self, q, k, v, spans, heads: int, kv_heads: int | None = None, scale: float | None = None, out=None):
        """Attention of the new tokens of S sequences a peer, q [N, S * new, heads * depth], over the rows spans[i, s, 0] .. spans[i, s, 1] - 1 (int32
        [N, S, 2]) of the caches k and v [N, keys, kv_heads * depth], whose last ones are the new tokens' own."""
        rows, code, T, keys, kv_heads, depth, scale = self._heads(q, k, v, heads, kv_heads, scale)
        if spans.dtype is not _torch().int32 or spans.dim() != 3 or spans.shape[0] != self.N or spans.shape[2] != 2 or not spans.is_cuda or \
                not spans.is_contiguous():
            raise ValueError("spans must be a contiguous int32 GPU tensor [N, S, 2]")
        seqs = spans.shape[1]
        if (T % seqs if seqs else T) or (seqs and not T):
            raise ValueError("q must hold the same number of new tokens, 1 or more, for every sequence")
        if out is None:
            out, = self._new(q.device, (q.shape, q.dtype))
        op, os_ = self._like(out, code, T, heads * depth, "out")
        self._lend(q, k, v, spans, out)
        self._check(self._lib.moshpit_attention_cached(self._h, *rows, code, spans.data_ptr(), seqs, T // seqs if seqs else 1, keys, heads, kv_heads, depth,
                                                       scale, op, os_), "attention_cached")
        return out

    def sync(self) -> None:
        self._check(self._lib.moshpit_sync(self._h), "sync")


def copy_probe(dst, src, stream=None) -> None:
    """Queue the library's plain copy kernel dst <- src (torch GPU tensors of equal byte size)."""
    import torch
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("size mismatch")
    if stream is None:
        stream = torch.cuda.current_stream(src.device)
    rc = load_library().moshpit_copy_probe(dst.data_ptr(), src.data_ptr(), nbytes, stream.cuda_stream)
    if rc != 0:
        raise MoshpitError(f"copy_probe failed ({rc})")


def check_bf16_rounding(stream=None) -> int:
    """Number of binary32 inputs (of all 2^32) on which the hardware bfloat16 rounding the
    kernels use differs from its integer definition; waits for the result."""
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    out = ctypes.c_uint64(2**64 - 1)
    rc = load_library().moshpit_check_bf16_rounding(stream.cuda_stream, ctypes.byref(out))
    if rc != 0:
        raise MoshpitError(f"check_bf16_rounding failed ({rc})")
    return int(out.value)


def dist_to_mean_static(X, out, stream=None) -> None:
    """Queue the allocation-free distortion of the [N, P] GPU tensor X (float32 or bfloat16,
    unit column stride) into out (GPU tensor holding one float64).  Returns without waiting."""
    import torch
    if X.dim() != 2 or X.stride(1) != 1 or not X.is_cuda or X.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("state tensor has the wrong dtype, shape or device")
    if out.dtype != torch.float64 or out.numel() != 1 or not out.is_cuda:
        raise ValueError("out must be one float64 on the GPU")
    if stream is None:
        stream = torch.cuda.current_stream(X.device)
    lib = load_library()
    rc = lib.moshpit_dist_to_mean_static(X.data_ptr(), X.shape[0], X.shape[1], X.stride(0),
                                         F32 if X.dtype == torch.float32 else BF16, stream.cuda_stream, out.data_ptr())
    if rc != 0:
        raise MoshpitError(f"dist_to_mean_static failed ({rc}): {lib.moshpit_last_error(None).decode()}")
