"""Thin ctypes binding of the C ABI in ``include/dmtd.h``.

Argument marshalling only: every step of the decode path runs in the HIP library.
PyTorch is used for device memory (the weight blob and the workspace) and for the
stream handle.  There is no CPU fallback: if ``libdmtd.so`` has not been built the
import of the library fails with an error.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
import threading

import numpy as np

DMTD_OK, DMTD_EINVAL, DMTD_ESTATE, DMTD_ECAPACITY, DMTD_EHIP = 0, -1, -2, -3, -4
_CODES = {DMTD_EINVAL: "DMTD_EINVAL", DMTD_ESTATE: "DMTD_ESTATE", DMTD_ECAPACITY: "DMTD_ECAPACITY", DMTD_EHIP: "DMTD_EHIP"}

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdmtd.so")


class _Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "intermediate", "vocab")] + [
        ("rms_eps", C.c_float), ("rope_theta", C.c_float),
        ("tied_embeddings", C.c_int32), ("dtype", C.c_int32), ("max_batch", C.c_int32), ("max_seq_len", C.c_int32),
        ("full_pos_add_embed", C.c_int32), ("use_graphs", C.c_int32), ("dry_run", C.c_int32), ("stream", C.c_void_p)]


class _PagePool(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_pages", "page_size", "n_req", "max_pages")] + [
        (n, C.c_void_p) for n in ("block_table", "held", "free_pages", "n_free")]


class _PagedCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("block_table", C.c_void_p)] + [
        (n, C.c_int32) for n in ("n_pages", "page_size", "n_req", "max_pages", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "max_rows")] + [
        ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("scale_stride", C.c_int64)]


class _SharedPlan(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("positions", C.c_int32), ("plan", C.c_void_p), ("plan_bytes", C.c_size_t), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class DmtdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_CODES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def load_library():
    """Load ``libdmtd.so`` and declare the prototypes of every exported call."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it first (python -m paper_2510_11958_amd.build); "
                          "there is no fallback path")
    # PyTorch ships its own HIP runtime: load it first, so that the library binds to the runtime that owns the
    # device memory it is handed (loading the system runtime first leaves the process with two of them)
    import torch  # noqa: F401
    lib = C.CDLL(_LIB_PATH)
    P = C.POINTER
    lib.dmtd_workspace_bytes.restype = C.c_size_t
    lib.dmtd_workspace_bytes.argtypes = [P(_Config)]
    lib.dmtd_create.restype = C.c_int
    lib.dmtd_create.argtypes = [P(_Config), C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, P(C.c_void_p)]
    lib.dmtd_prefill.restype = C.c_int
    lib.dmtd_prefill.argtypes = [C.c_void_p, P(C.c_int32), C.c_int32, C.c_int32, C.c_int32, P(C.c_int32)]
    lib.dmtd_prefill_ragged.restype = C.c_int
    lib.dmtd_prefill_ragged.argtypes = [C.c_void_p, P(C.c_int32), C.c_int32, C.c_int32, P(C.c_int32), C.c_int32, P(C.c_int32)]
    lib.dmtd_decode_cycle.restype = C.c_int
    lib.dmtd_decode_cycle.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, P(C.c_int32), C.c_int32,
                                      P(C.c_int32), C.c_int32, P(C.c_int32)]
    lib.dmtd_decode.restype = C.c_int
    lib.dmtd_decode.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, P(C.c_int32), C.c_int32,
                                P(C.c_int32), C.c_int32, P(C.c_int32)]
    lib.dmtd_decode_per_seq.restype = C.c_int
    lib.dmtd_decode_per_seq.argtypes = [C.c_void_p, P(C.c_int32), C.c_int32, C.c_int32, P(C.c_int32), C.c_int32,
                                        P(C.c_int32), C.c_int32, P(C.c_int32)]
    lib.dmtd_get_seq_state.restype = C.c_int
    lib.dmtd_get_seq_state.argtypes = [C.c_void_p, C.c_int32, P(C.c_int32), P(C.c_int32)]
    lib.dmtd_decode_cycle_noalloc.restype = C.c_int
    lib.dmtd_decode_cycle_noalloc.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int32,
                                              C.c_void_p, C.c_int32, P(C.c_int32)]
    lib.dmtd_logits.restype = C.c_int
    lib.dmtd_logits.argtypes = [C.c_void_p, P(C.c_float), C.c_size_t]
    lib.dmtd_get_state.restype = C.c_int
    lib.dmtd_get_state.argtypes = [C.c_void_p, P(C.c_int32), P(C.c_int32), P(C.c_int32), P(C.c_int64)]
    lib.dmtd_get_trace.restype = C.c_int
    lib.dmtd_get_trace.argtypes = [C.c_void_p, P(C.c_int32), C.c_int32, P(C.c_int32)]
    lib.dmtd_read_kv.restype = C.c_int
    lib.dmtd_read_kv.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, P(C.c_float), C.c_size_t]
    lib.dmtd_time_kernel.restype = C.c_int
    lib.dmtd_time_kernel.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, P(C.c_float)]
    lib.dmtd_wide_plan.restype = C.c_int
    lib.dmtd_wide_plan.argtypes = [P(_Config), C.c_int32, C.c_int32, C.c_int32, P(C.c_int32)]
    lib.dmtd_wide_tile_width.restype = C.c_int
    lib.dmtd_wide_tile_width.argtypes = [P(_Config), C.c_int32, C.c_int32, C.c_int32]
    lib.dmtd_front_plan.restype = C.c_int
    lib.dmtd_front_plan.argtypes = [P(_Config), P(C.c_int32), C.c_int32, P(C.c_int32), P(C.c_int32)]
    lib.dmtd_score_plan.restype = C.c_int
    lib.dmtd_score_plan.argtypes = [P(_Config), C.c_int32, C.c_int32, P(C.c_int32)]
    lib.dmtd_set_n_early.restype = C.c_int
    lib.dmtd_set_n_early.argtypes = [C.c_void_p, C.c_int32]
    lib.dmtd_set_sampling.restype = C.c_int
    lib.dmtd_set_sampling.argtypes = [C.c_void_p, C.c_float, C.c_int32, C.c_uint64]
    lib.dmtd_masked_forward.restype = C.c_int
    lib.dmtd_masked_forward.argtypes = [C.c_void_p, P(C.c_int32), C.c_int32, C.c_int32, P(C.c_uint8), C.c_int32, P(C.c_float),
                                        P(C.c_int32), P(C.c_float), C.c_size_t, P(C.c_float)]
    lib.dmtd_paged_step_bytes.restype = C.c_size_t
    lib.dmtd_paged_step_bytes.argtypes = [P(_Config), C.c_int32]
    lib.dmtd_paged_begin.restype = C.c_int
    lib.dmtd_paged_begin.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t]
    lib.dmtd_paged_step.restype = C.c_int
    lib.dmtd_paged_step.argtypes = [C.c_void_p, C.c_int32, P(C.c_int32), P(C.c_int32), P(C.c_int32), P(C.c_uint8), C.c_int32, P(C.c_int32)]
    lib.dmtd_paged_release.restype = C.c_int
    lib.dmtd_paged_release.argtypes = [C.c_void_p, C.c_int32]
    lib.dmtd_paged_get_state.restype = C.c_int
    lib.dmtd_paged_get_state.argtypes = [C.c_void_p, C.c_int32, P(C.c_int32), P(C.c_int32), P(C.c_int32)]
    lib.dmtd_page_tables.restype = C.c_int
    lib.dmtd_page_tables.argtypes = [P(_PagePool), C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p] * 5
    lib.dmtd_page_tables_shared.restype = C.c_int
    lib.dmtd_page_tables_shared.argtypes = [P(_PagePool), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p] * 5
    lib.dmtd_shared_plan_bytes.restype = C.c_size_t
    lib.dmtd_shared_plan_bytes.argtypes = [P(_PagedCache), C.c_int32]
    lib.dmtd_shared_workspace_bytes.restype = C.c_size_t
    lib.dmtd_shared_workspace_bytes.argtypes = [P(_PagedCache)]
    lib.dmtd_shared_plan_build.restype = C.c_int
    lib.dmtd_shared_plan_build.argtypes = [P(_PagedCache), P(_SharedPlan)] + [C.c_void_p] * 5
    lib.dmtd_paged_attention_shared.restype = C.c_int
    lib.dmtd_paged_attention_shared.argtypes = [P(_PagedCache), P(_SharedPlan), C.c_void_p, C.c_int64, C.c_void_p, C.c_float, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]
    lib.dmtd_paged_append.restype = C.c_int
    lib.dmtd_paged_append.argtypes = [P(_PagedCache), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                      C.c_void_p, C.c_int32, C.c_void_p]
    lib.dmtd_paged_read.restype = C.c_int
    lib.dmtd_paged_read.argtypes = [P(_PagedCache), C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    lib.dmtd_paged_workspace_bytes.restype = C.c_size_t
    lib.dmtd_paged_workspace_bytes.argtypes = [P(_PagedCache)]
    lib.dmtd_paged_attention.restype = C.c_int
    lib.dmtd_paged_attention.argtypes = [P(_PagedCache), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_float,
                                         C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.dmtd_reset.restype = C.c_int
    lib.dmtd_reset.argtypes = [C.c_void_p]
    lib.dmtd_destroy.restype = None
    lib.dmtd_destroy.argtypes = [C.c_void_p]
    lib.dmtd_last_error.restype = C.c_char_p
    lib.dmtd_last_error.argtypes = [C.c_void_p]
    _lib = lib
    return lib


@dataclasses.dataclass
class ModelConfig:
    n_layers: int
    hidden: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    intermediate: int
    vocab: int
    dtype: str = "bf16"
    rms_eps: float = 1e-6
    rope_theta: float = 1e6
    tied_embeddings: bool = True
    max_batch: int = 1
    max_seq_len: int = 2048
    full_pos_add_embed: bool = False
    use_graphs: bool = True
    dry_run: bool = False

    def to_c(self, stream: int = 0) -> _Config:
        return _Config(self.n_layers, self.hidden, self.n_q_heads, self.n_kv_heads, self.head_dim, self.intermediate,
                       self.vocab, self.rms_eps, self.rope_theta, int(self.tied_embeddings),
                       0 if self.dtype == "fp32" else 1, self.max_batch, self.max_seq_len,
                       int(self.full_pos_add_embed), int(self.use_graphs), int(self.dry_run), stream or None)


def _i32p(a: np.ndarray):
    return a.ctypes.data_as(C.POINTER(C.c_int32))


class Engine:
    """One decoding context.  ``weights`` is the flat weight blob (NumPy float32, or uint16 holding
    bfloat16 bits, or a torch uint8/any-dtype CUDA tensor already on the device)."""

    def __init__(self, cfg: ModelConfig, weights=None, stream: int | None = None):
        self.lib = load_library()
        self.cfg = cfg
        self._h = C.c_void_p()
        self._weights = self._workspace = None
        self._stage = None
        self._lock = threading.Lock()
        if cfg.dry_run:
            cc = cfg.to_c(0)
            rc = self.lib.dmtd_create(C.byref(cc), None, 0, None, 0, C.byref(self._h))
            self._check_create(rc)
            return
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the DMTD decode path has no CPU fallback")
        if isinstance(weights, np.ndarray):
            weights = torch.from_numpy(weights.view(np.int16) if weights.dtype == np.uint16 else weights).cuda()
        self._weights = weights.contiguous()
        if stream is None:
            # a stream of its own (default priority): the legacy default stream cannot be captured into a graph
            self._stream = torch.cuda.Stream()
            stream = self._stream.cuda_stream
        torch.cuda.synchronize()   # the weight upload above ran on torch's current stream
        cc = cfg.to_c(stream)
        nbytes = self.lib.dmtd_workspace_bytes(C.byref(cc))
        if nbytes == 0:
            raise DmtdError(DMTD_EINVAL, "invalid configuration")
        self._workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        wbytes = self._weights.numel() * self._weights.element_size()
        rc = self.lib.dmtd_create(C.byref(cc), self._weights.data_ptr(), wbytes, self._workspace.data_ptr(), nbytes,
                                  C.byref(self._h))
        self._check_create(rc)

    _STAGE_LIMIT = 64 << 20

    def _logits_stage(self):
        """Page-locked memory [max_batch, vocab] that the logits' copy from the GPU goes through, the engine's own from the first call to
        ``close``; None where it would be too large."""
        shape = (self.cfg.max_batch, self.cfg.vocab)
        if self._stage is None and not self.cfg.dry_run and 4 * shape[0] * shape[1] <= self._STAGE_LIMIT:
            import torch
            try:
                self._stage = torch.empty(shape, dtype=torch.float32, device="cpu", pin_memory=True).numpy()
            except RuntimeError:    # no page-locked memory to be had
                self._stage = False
        return None if self._stage is None or self._stage is False else self._stage

    def _check_create(self, rc):
        if rc != DMTD_OK:
            raise DmtdError(rc, self.lib.dmtd_last_error(None).decode())

    def _check(self, rc):
        if rc != DMTD_OK:
            raise DmtdError(rc, self.lib.dmtd_last_error(self._h).decode())

    def close(self):
        if self._h:
            self.lib.dmtd_destroy(self._h)
            self._h = C.c_void_p()
        self._stage = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill(self, tokens, n_late: int = 0, lengths=None) -> np.ndarray:
        """``lengths`` (one per sequence): prompts of different lengths, each in the first entries of its row of ``tokens``."""
        t = np.ascontiguousarray(np.atleast_2d(np.asarray(tokens)), dtype=np.int32)
        first = np.empty(t.shape[0], np.int32)
        if lengths is None:
            self._check(self.lib.dmtd_prefill(self._h, _i32p(t), t.shape[0], t.shape[1], n_late, _i32p(first)))
        else:
            ln = np.ascontiguousarray(np.asarray(lengths), dtype=np.int32)
            if ln.shape != (t.shape[0],):
                raise ValueError("one length per sequence")
            self._check(self.lib.dmtd_prefill_ragged(self._h, _i32p(t), t.shape[0], t.shape[1], _i32p(ln), n_late, _i32p(first)))
        self._batch = t.shape[0]
        return first

    def decode_cycle(self, tau: int, n_late: int, max_new: int = 0, forced=None) -> np.ndarray:
        """Returns the argmax tokens of the steps run, ``[batch, n_steps]``."""
        B = getattr(self, "_batch", 1)
        stride = max(1, min(tau, 64))
        out = np.empty((B, stride), np.int32)
        n = C.c_int32(0)
        if forced is not None:
            f = np.ascontiguousarray(np.atleast_2d(np.asarray(forced)), dtype=np.int32)
            fp, nf = _i32p(f), f.shape[1]
        else:
            fp, nf = None, 0
        self._check(self.lib.dmtd_decode_cycle(self._h, tau, n_late, max_new, fp, nf, _i32p(out), stride, C.byref(n)))
        return out[:, :n.value].copy()

    def decode(self, tau: int, n_late: int, n_steps: int, forced=None) -> np.ndarray:
        """``n_steps`` decode steps, cycles back to back, one host synchronisation; ``[batch, n_steps]`` argmax tokens."""
        B = getattr(self, "_batch", 1)
        stride = max(1, min(n_steps, 64))
        out = np.empty((B, stride), np.int32)
        n = C.c_int32(0)
        if forced is not None:
            f = np.ascontiguousarray(np.atleast_2d(np.asarray(forced)), dtype=np.int32)
            fp, nf = _i32p(f), f.shape[1]
        else:
            fp, nf = None, 0
        self._check(self.lib.dmtd_decode(self._h, tau, n_late, n_steps, fp, nf, _i32p(out), stride, C.byref(n)))
        return out[:, :n.value].copy()

    def decode_per_seq(self, taus, n_late: int, n_steps: int, forced=None) -> np.ndarray:
        """``n_steps`` decode steps with one cycle length per sequence (``taus``); ``[batch, n_steps]`` argmax tokens."""
        B = getattr(self, "_batch", 1)
        t = np.ascontiguousarray(np.asarray(taus), dtype=np.int32)
        if t.shape != (B,):
            raise ValueError("one cycle length per sequence")
        stride = max(1, min(n_steps, 64))
        out = np.empty((B, stride), np.int32)
        n = C.c_int32(0)
        if forced is not None:
            f = np.ascontiguousarray(np.atleast_2d(np.asarray(forced)), dtype=np.int32)
            fp, nf = _i32p(f), f.shape[1]
        else:
            fp, nf = None, 0
        self._check(self.lib.dmtd_decode_per_seq(self._h, _i32p(t), n_late, n_steps, fp, nf, _i32p(out), stride, C.byref(n)))
        return out[:, :n.value].copy()

    def seq_state(self, b: int):
        f, ph = C.c_int32(), C.c_int32()
        self._check(self.lib.dmtd_get_seq_state(self._h, b, C.byref(f), C.byref(ph)))
        return {"n_front": f.value, "phase": ph.value}

    def decode_cycle_noalloc(self, tau: int, n_late: int, out_dev, max_new: int = 0, forced_dev=None) -> int:
        """dmtd_decode_cycle without allocation or synchronisation: ``out_dev`` (torch int32 CUDA tensor ``[batch, stride]``)
        receives the steps' tokens once the engine's stream has run the enqueued work, ``forced_dev`` (torch int32 CUDA
        tensor ``[batch, n_forced]`` or None) holds the forced inputs.  Returns the number of steps enqueued."""
        n = C.c_int32(0)
        if forced_dev is not None:
            assert forced_dev.is_cuda and forced_dev.dtype.itemsize == 4 and forced_dev.is_contiguous()
            fp, nf = forced_dev.data_ptr(), forced_dev.shape[1]
        else:
            fp, nf = None, 0
        assert out_dev.is_cuda and out_dev.dtype.itemsize == 4 and out_dev.is_contiguous()
        self._check(self.lib.dmtd_decode_cycle_noalloc(self._h, tau, n_late, max_new, fp, nf, out_dev.data_ptr(),
                                                       out_dev.shape[1], C.byref(n)))
        return n.value

    def synchronize(self):
        """Wait for the engine's stream (after calls that do not synchronise themselves)."""
        if getattr(self, "_stream", None) is not None:
            self._stream.synchronize()
        else:
            import torch
            torch.cuda.synchronize()

    def logits(self) -> np.ndarray:
        """The most recent step's logits, ``[batch, vocab]``, in pageable memory of the caller's own.

        The page-locked staging memory never leaves the engine: an upload of the result that does not wait
        (``torch.from_numpy(...).to("cuda", non_blocking=True)``) would still read it while the next call writes it.  Up to 64 MiB of it stay
        locked from the first call to ``close``.  us per call, straight into pageable memory / staged: 32 x 151936 1088 / 987, 8 x 151936
        268 / 243, 1 x 151936 38 / 38, 1 x 1024 26 / 17.  One thread copies: torch's copy on 16 took 484 for 32 x 151936, but its threads'
        waiting made one in ten passes of a prompt of 8192 5 ms longer (8.8 ms)."""
        B = getattr(self, "_batch", 1)
        out = np.empty((B, self.cfg.vocab), np.float32)
        with self._lock:
            stage = self._logits_stage()
            dst = out if stage is None else stage
            self._check(self.lib.dmtd_logits(self._h, dst.ctypes.data_as(C.POINTER(C.c_float)), out.size))
            if stage is not None:
                np.copyto(out, stage[:B])
        return out

    def state(self):
        a, b, c = C.c_int32(), C.c_int32(), C.c_int32()
        cnt = (C.c_int64 * 4)()
        self._check(self.lib.dmtd_get_state(self._h, C.byref(a), C.byref(b), C.byref(c), cnt))
        return {"n_tok": a.value, "n_front": b.value, "phase": c.value, "gen_layer_visits": cnt[0],
                "refill_layer_visits": cnt[1], "n_emitted": cnt[2], "n_full_steps": cnt[3]}

    def trace(self):
        n = C.c_int32()
        self._check(self.lib.dmtd_get_trace(self._h, None, 0, C.byref(n)))
        buf = np.empty((max(n.value, 1), 4), np.int32)
        self._check(self.lib.dmtd_get_trace(self._h, _i32p(buf), n.value, C.byref(n)))
        names = {0: "front", 1: "late", 2: "enc"}
        return [(int(p), names[int(g)], list(range(int(f), int(f) + int(c)))) for p, g, f, c in buf[:n.value]]

    def read_kv(self, layer: int, b: int, n_pos: int) -> np.ndarray:
        out = np.empty((2, self.cfg.n_kv_heads, n_pos, self.cfg.head_dim), np.float32)
        self._check(self.lib.dmtd_read_kv(self._h, layer, b, n_pos, out.ctypes.data_as(C.POINTER(C.c_float)), out.size))
        return out

    KERNEL_KINDS = {"qkv": 0, "oproj": 1, "gateup": 2, "down": 3, "lmhead": 4, "attn": 5,
                    "read_qkv": 6, "read_oproj": 7, "read_gateup": 8, "read_down": 9}

    def time_kernel(self, kind: str, rows: int = 1, reps: int = 5) -> float:
        """Average duration (microseconds) of one launch of a kernel kind, HIP-event timed on the engine's stream."""
        us = C.c_float()
        self._check(self.lib.dmtd_time_kernel(self._h, self.KERNEL_KINDS[kind], rows, reps, C.byref(us)))
        return us.value

    def set_n_early(self, n_early: int):
        """ExDy variant: in-cycle tokens also pass the first ``n_early`` layers (0 = plain method)."""
        self._check(self.lib.dmtd_set_n_early(self._h, int(n_early)))

    def set_sampling(self, temperature: float, top_k: int = 0, seed: int = 0):
        """Draw tokens from the tempered softmax over the top_k logits (temperature <= 0: greedy, the default)."""
        self._check(self.lib.dmtd_set_sampling(self._h, float(temperature), int(top_k), int(seed)))

    def masked_forward(self, tokens, mask, n_late: int, want_logits: bool = False) -> dict:
        """Whole-sequence masked forward (Eqs. 1-5) with the Eq. 6 loss; returns ``nll`` [batch, n], ``best`` [batch, n],
        ``loss`` [batch] and, if asked for, ``logits`` [batch, n, vocab]."""
        t = np.ascontiguousarray(np.atleast_2d(np.asarray(tokens)), dtype=np.int32)
        m = np.ascontiguousarray(np.asarray(mask), dtype=np.uint8)
        B, n = t.shape
        if m.shape != (n,):
            raise ValueError("mask must have one entry per position")
        nll = np.empty((B, n), np.float32)
        best = np.empty((B, n), np.int32)
        loss = np.empty(B, np.float32)
        logits = np.empty((B, n, self.cfg.vocab), np.float32) if want_logits else None
        fp = C.POINTER(C.c_float)
        self._check(self.lib.dmtd_masked_forward(
            self._h, _i32p(t), B, n, m.ctypes.data_as(C.POINTER(C.c_uint8)), n_late, nll.ctypes.data_as(fp), _i32p(best),
            logits.ctypes.data_as(fp) if want_logits else None, logits.size if want_logits else 0, loss.ctypes.data_as(fp)))
        out = {"nll": nll, "best": best, "loss": loss}
        if want_logits:
            out["logits"] = logits
        return out

    def paged_begin(self, page_size: int = 64):
        """Requests that come and go from here on, until ``reset``: the caches become a pool of pages, steps are :meth:`paged_step`."""
        import torch
        cc = self.cfg.to_c(0)
        nbytes = self.lib.dmtd_paged_step_bytes(C.byref(cc), page_size)
        if nbytes == 0 or self.cfg.dry_run:
            self._check(self.lib.dmtd_paged_begin(self._h, page_size, None, 0))
        memory = torch.empty(nbytes, dtype=torch.uint8, device=self._workspace.device)
        torch.cuda.current_stream(memory.device).synchronize()      # whatever that stream still does with the memory
        self._check(self.lib.dmtd_paged_begin(self._h, page_size, memory.data_ptr(), nbytes))
        self._paged_memory = memory

    def paged_step(self, slots, tokens, full, n_late: int) -> np.ndarray:
        """One step of the requests in ``slots``: ``tokens`` holds one sequence of new tokens per request, ``full`` whether it passes the front layers (a full step, a
        chunk of a prompt) or only the late ones.  Returns the greedy next token of each; ``logits`` then has a row per request."""
        parts = [np.atleast_1d(np.asarray(t, dtype=np.int32)) for t in tokens]
        s, f = np.ascontiguousarray(slots, dtype=np.int32), np.ascontiguousarray(full, dtype=np.uint8)
        if s.shape != (len(parts),) or f.shape != s.shape:
            raise ValueError("one slot, one sequence of tokens and one mark per request")
        counts, flat, out = np.array([p.size for p in parts], np.int32), np.concatenate(parts) if parts else np.empty(0, np.int32), np.empty(len(parts), np.int32)
        self._check(self.lib.dmtd_paged_step(self._h, len(parts), _i32p(s), _i32p(counts), _i32p(flat), f.ctypes.data_as(C.POINTER(C.c_uint8)), n_late, _i32p(out)))
        self._batch = len(parts)
        return out

    def paged_release(self, slot: int):
        """The request in ``slot`` ends; its pages go back to the pool."""
        self._check(self.lib.dmtd_paged_release(self._h, slot))

    def paged_state(self, slot: int) -> dict:
        a, b, f = C.c_int32(), C.c_int32(), C.c_int32()
        self._check(self.lib.dmtd_paged_get_state(self._h, slot, C.byref(a), C.byref(b), C.byref(f)))
        return {"n_tok": a.value, "n_front": b.value, "free_pages": f.value}

    def reset(self):
        self._check(self.lib.dmtd_reset(self._h))
        self._paged_memory = None


# ------------------------------------------------------------------------------- paged key/value cache

def _raise(lib, rc):
    if rc != DMTD_OK:
        raise DmtdError(rc, lib.dmtd_last_error(None).decode())


def _want(t, name, dtype, index, shape):
    """The address of a contiguous GPU tensor of that type and shape on that device."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {index}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


class _OnDevice:
    """What the handles of the paged cache share: the library, a device, and calls on torch's current stream of that device."""

    def _open(self, t):
        import torch
        if not t.is_cuda:
            raise ValueError("the paged cache lives on the GPU")
        self._torch, self._lib, self.device, self._index = torch, load_library(), t.device, t.get_device()
        self._i32, self._i64, self._f32 = torch.int32, torch.int64, torch.float32
        # the stream's handle without the Stream object around it: a microsecond less a call
        self._stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)

    def _call(self, fn, *args):
        stream = self._stream_of(self._index)
        if self._torch.cuda.current_device() == self._index:
            rc = fn(*args, stream)
        else:
            with self._torch.cuda.device(self._index):
                rc = fn(*args, stream)
        if rc != DMTD_OK:
            _raise(self._lib, rc)
        return stream


class PageTables(_OnDevice):
    """Block tables of ``n_req`` requests over a pool of pages (``dmtd_page_tables``), on torch's current stream.

    ``block_table`` int32 ``[n_req, max_pages]``, ``held`` int32 ``[n_req]``, ``free_pages`` int32 ``[n_pages]`` and ``n_free`` int32 ``[1]`` are the
    caller's GPU tensors, changed in place; :meth:`empty` makes those of an empty pool."""

    def __init__(self, block_table, held, free_pages, n_free, page_size: int):
        self._open(block_table)
        n_req, max_pages = block_table.shape
        i32, dev = self._i32, self._index
        self.block_table, self.held, self.free_pages, self.n_free, self.page_size = block_table, held, free_pages, n_free, int(page_size)
        self._c = _PagePool(free_pages.numel(), self.page_size, n_req, max_pages, _want(block_table, "block_table", i32, dev, (n_req, max_pages)),
                            _want(held, "held", i32, dev, (n_req,)), _want(free_pages, "free_pages", i32, dev, (free_pages.numel(),)), _want(n_free, "n_free", i32, dev, (1,)))
        self._p, self._per_req, self._per_end = C.byref(self._c), (n_req,), (n_req + 1,)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_req: int, max_pages: int, device="cuda"):
        """A pool whose pages are all free, handed out from page 0 on."""
        import torch
        free = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        return cls(torch.full((n_req, max_pages), -1, dtype=torch.int32, device=device), torch.zeros(n_req, dtype=torch.int32, device=device), free,
                   torch.full((1,), n_pages, dtype=torch.int32, device=device), page_size)

    def build(self, start, rows, cu_rows, row_pos, slots, status, shared=None):
        """Pages and places for a step: request i has ``start[i]`` tokens and brings ``rows[i]``.  Writes ``cu_rows`` int32 ``[n_req + 1]``, ``row_pos`` int32
        ``[max_rows]``, ``slots`` int64 ``[max_rows]`` and ``status`` int32 ``[2]`` (0, or why the step has no rows: see the header).  ``shared`` int32 ``[n_req]``: the pages at the
        front of each request's table that another one holds (``dmtd_page_tables_shared``): they stay where they are, are not given back, and a step that would bring rows into them is refused by its status."""
        i32, dev = self._i32, self._index
        room = row_pos.shape
        front = None if shared is None else _want(shared, "shared", i32, dev, self._per_req)
        self._call(self._lib.dmtd_page_tables_shared, self._p, _want(start, "start", i32, dev, self._per_req), _want(rows, "rows", i32, dev, self._per_req), front,
                   room[0] if len(room) == 1 else 0, _want(cu_rows, "cu_rows", i32, dev, self._per_end), _want(row_pos, "row_pos", i32, dev, room), _want(slots, "slots", self._i64, dev, room),
                   _want(status, "status", i32, dev, (2,)))


class PagedCache(_OnDevice):
    """One layer's keys and values in pages, ``k`` and ``v`` ``[n_pages, n_kv_heads, page_size, head_dim]`` (bfloat16, float32 or float8_e4m3fn; pages may lie apart,
    a page itself is contiguous), read and filled through ``block_table`` int32 ``[n_req, max_pages]`` (``dmtd_paged_append``, ``dmtd_paged_attention``) on
    torch's current stream.  Steps have up to ``max_rows`` rows.  8-bit caches come with ``k_scale`` and ``v_scale``, uint8 ``[n_pages, n_kv_heads, page_size]``: a value is its code
    times ``2 ** (scale - 127)``; norms' gains, outputs and what :meth:`read` returns are then bfloat16.  The handle holds the attention's workspace: calls of one handle, and of those that
    :meth:`layer` made from it, must not overlap."""

    def __init__(self, k, v, block_table, n_q_heads: int, max_rows: int, k_scale=None, v_scale=None, _workspace_of=None):
        self._open(k)
        torch, dev = self._torch, self._index
        code = {torch.float32: 0, torch.bfloat16: 1, torch.float8_e4m3fn: 3}.get(k.dtype)
        if code is None or v.dtype is not k.dtype:
            raise ValueError("k and v must be bfloat16, float32 or float8_e4m3fn, both alike")
        n_pages, n_kv, page_size, hd = k.shape
        if v.shape != k.shape or v.device != k.device:
            raise ValueError("k and v must have one shape and lie on one GPU")
        stride = (k.stride(0) if n_pages > 1 else n_kv * page_size * hd, page_size * hd, hd, 1)
        for t in (k, v):
            if any(n > 1 and a != b for n, a, b in zip(t.shape, t.stride(), stride)):
                raise ValueError("pages must be contiguous, and k and v laid out alike")
        if stride[0] < n_kv * page_size * hd:      # (0, as of an expanded page, would mean pages behind each other)
            raise ValueError("pages must not overlap")
        n_req, max_pages = block_table.shape
        scales = (None, None, 0)
        if code == 3:
            scales = self._scales(k_scale, v_scale, (n_pages, n_kv, page_size))
        elif k_scale is not None or v_scale is not None:
            raise ValueError("only float8_e4m3fn caches have scales")
        self.k, self.v, self.k_scale, self.v_scale, self.block_table, self.max_rows = k, v, k_scale, v_scale, block_table, int(max_rows)
        self.dtype = torch.bfloat16 if code == 3 else k.dtype      # of gains and outputs
        self._c = _PagedCache(k.data_ptr(), v.data_ptr(), stride[0], _want(block_table, "block_table", self._i32, dev, (n_req, max_pages)), n_pages, page_size, n_req, max_pages,
                              n_q_heads, n_kv, hd, code, max_rows, *scales)
        self._p = C.byref(self._c)
        self._q_heads, self._q_cols, self._cols = (n_q_heads, hd), n_q_heads * hd, (n_q_heads + 2 * n_kv) * hd
        self._per_req, self._per_end, self._per_row, self._gain, self._angles = (n_req,), (n_req + 1,), (self.max_rows,), (hd,), (hd // 2, 2)
        self._kv_heads = (n_kv, hd)
        self._ws_bytes = self._lib.dmtd_paged_workspace_bytes(self._p)
        if self._ws_bytes == 0:
            _raise(self._lib, DMTD_EINVAL)
        if _workspace_of is not None:
            if _workspace_of._ws_bytes < self._ws_bytes or _workspace_of.device != self.device:
                raise ValueError("the workspace is too small for the other layer's caches, or on another GPU")
            self._ws, self._ws_ptr, self._streams = _workspace_of._ws, _workspace_of._ws_ptr, _workspace_of._streams
            return
        self._ws = torch.zeros(self._ws_bytes, dtype=torch.uint8, device=k.device)
        self._ws_ptr = self._ws.data_ptr()
        stream = torch.cuda.current_stream(k.device)
        stream.synchronize()              # zeroed, whichever stream the first call is on
        self._streams = {stream.cuda_stream}

    def _scales(self, k_scale, v_scale, shape):
        """The addresses of an 8-bit cache's scales, and the bytes from page to page."""
        stride = None
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if t is None or t.dtype is not self._torch.uint8 or t.get_device() != self._index or t.shape != shape:
                raise ValueError(f"a float8_e4m3fn cache needs {name}, uint8 {shape} on GPU {self._index}")
            apart = t.stride(0) if shape[0] > 1 else shape[1] * shape[2]
            if any(n > 1 and a != b for n, a, b in zip(shape[1:], t.stride()[1:], (shape[2], 1))) or apart < shape[1] * shape[2] or stride not in (None, apart):
                raise ValueError("a page's scales must be contiguous, not overlap the next one's, and k_scale and v_scale be laid out alike")
            stride = apart
        return k_scale.data_ptr(), v_scale.data_ptr(), stride

    def layer(self, k, v, k_scale=None, v_scale=None) -> "PagedCache":
        """The handle of another layer's pools ``k`` and ``v``, with this one's block table and workspace."""
        return PagedCache(k, v, self.block_table, self._q_heads[0], self.max_rows, k_scale, v_scale, _workspace_of=self)

    def _rows(self, qkv, cols, norm, rope):
        dev, shape = self._index, qkv.shape
        if len(shape) != 2 or qkv.dtype is not self._f32 or qkv.get_device() != dev or shape[0] < self.max_rows or shape[1] < cols or qkv.stride(1) != 1:
            raise ValueError(f"qkv must be float32 [at least {self.max_rows}, at least {cols}] on GPU {dev} with contiguous rows")
        gain = None if norm is None else _want(norm, "the norm's gain", self.dtype, dev, self._gain)
        ld = qkv.stride(0) if shape[0] > 1 else (shape[1] + 3) // 4 * 4
        if rope is None:
            return qkv.data_ptr(), ld, gain, None, 0
        n = rope.shape[0]
        if n < 1:                                  # (its address would be null: no rotation)
            raise ValueError("rope must hold a position")
        return qkv.data_ptr(), ld, gain, _want(rope, "rope", self._f32, dev, (n, *self._angles)), n

    def _out(self, out):
        """The output rows, made if they are not given, and the elements from one to the next."""
        if out is None:
            out = self._torch.empty(self.max_rows, *self._q_heads, dtype=self.dtype, device=self.device)
        shape = out.shape
        if (len(shape) != 3 or shape[1:] != self._q_heads or shape[0] < self.max_rows or out.dtype is not self.dtype or out.get_device() != self._index or
                out.stride(2) != 1 or (shape[1] > 1 and out.stride(1) != shape[2])):
            raise ValueError(f"out must be {self.dtype} [at least {self.max_rows}, {self._q_heads[0]}, {self._q_heads[1]}] on GPU {self._index} with contiguous rows")
        return out, out.stride(0) if shape[0] > 1 else self._q_cols

    def _layout(self):
        """What a plan of shared prefixes depends on."""
        c = self._c
        return (self._index, c.n_req, c.max_pages, c.page_size, c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype == 0, c.max_rows)

    def append(self, qkv, cu_rows, row_pos, slots, k_norm=None, rope=None, eps: float = 1e-6):
        """Keys (normalised with ``k_norm``, rotated by ``rope`` [positions, head_dim / 2, (cos, sin)]) and values of the fused projection's rows
        ``qkv`` into the places that :meth:`PageTables.build` gave them: each its own (of rows with the same place, an 8-bit cache may pair one's codes with another's scale)."""
        x, ld, gain, tab, n_tab = self._rows(qkv, self._cols, k_norm, rope)
        i32, dev = self._i32, self._index
        self._call(self._lib.dmtd_paged_append, self._p, x, ld, _want(cu_rows, "cu_rows", i32, dev, self._per_end), _want(row_pos, "row_pos", i32, dev, self._per_row),
                   _want(slots, "slots", self._i64, dev, self._per_row), gain, eps, tab, n_tab)

    def read(self, slots, k_out=None, v_out=None):
        """Keys and values out of the places ``slots`` (int64 ``[n]``, as :meth:`PageTables.build` numbers them; in any order), into ``k_out`` and ``v_out``
        ``[n, n_kv_heads, head_dim]`` of the cache's type, bfloat16 for 8-bit caches (made if not given).  Rows whose place is outside the pool are not written."""
        n = slots.shape[0] if len(slots.shape) == 1 and slots.shape[0] <= 1 << 27 else -1
        where = _want(slots, "slots", self._i64, self._index, (max(n, 0),))
        shape = (n, *self._kv_heads)
        if k_out is None:
            k_out = self._torch.empty(shape, dtype=self.dtype, device=self.device)
        if v_out is None:
            v_out = self._torch.empty(shape, dtype=self.dtype, device=self.device)
        to_k, to_v = _want(k_out, "k_out", self.dtype, self._index, shape), _want(v_out, "v_out", self.dtype, self._index, shape)
        if n:
            self._call(self._lib.dmtd_paged_read, self._p, where, n, to_k, to_v, shape[1] * shape[2])
        return k_out, v_out

    def attention(self, qkv, start, cu_rows, out=None, q_norm=None, rope=None, eps: float = 1e-6, max_new: int = 0):
        """The rows' queries over their requests' pages, into ``out`` ``[max_rows, n_q_heads, head_dim]`` of the cache's type (made if not given; rows behind
        the last one are not written).  ``max_new``: the most rows one request brings, if known."""
        x, ld, gain, tab, n_tab = self._rows(qkv, self._q_cols, q_norm, rope)
        i32, dev = self._i32, self._index
        out, ldo = self._out(out)
        stream = self._call(self._lib.dmtd_paged_attention, self._p, x, ld, _want(start, "start", i32, dev, self._per_req), _want(cu_rows, "cu_rows", i32, dev, self._per_end),
                            max_new, gain, eps, tab, n_tab, out.data_ptr(), ldo, self._ws_ptr, self._ws_bytes)
        if stream not in self._streams:
            self._streams.add(stream)
            self._ws.record_stream(self._torch.cuda.current_stream(self._index))      # the workspace is not reused before this stream's work has ended
        return out

    def attention_shared(self, plan, qkv, out=None, q_norm=None, rope=None, eps: float = 1e-6):
        """The attention of the step that ``plan`` (:class:`SharedPlan`, of this handle's layout) was built for; ``qkv``, ``out``, ``q_norm``, ``rope`` and ``eps`` as for
        :meth:`attention`."""
        if plan._layout != self._layout():
            raise ValueError("the plan was made for caches of another layout, or on another GPU")
        x, ld, gain, tab, n_tab = self._rows(qkv, self._q_cols, q_norm, rope)
        out, ldo = self._out(out)
        stream = self._call(self._lib.dmtd_paged_attention_shared, self._p, plan._p, x, ld, gain, eps, tab, n_tab, out.data_ptr(), ldo)
        plan._used_on(stream)
        return out


class SharedPlan(_OnDevice):
    """How a step's attention is laid out where groups of requests start with the same pages (``dmtd_shared_plan_build``), for ``cache`` and all handles of its layout (those of the
    other layers; bfloat16 and 8-bit caches are alike).  ``n_groups``: the most groups; ``positions``: how many the rotary table has angles for, if they are fewer than the block
    table's places.  Pays from about 40 thousand keys (requests of the group x shared tokens; 8-bit 60 thousand) on; below that :meth:`PagedCache.attention` over the same tables is faster.
    Holds the memory of the plan and of the attention's partial results: attention calls that use it must not overlap, nor overlap :meth:`build`."""

    def __init__(self, cache: PagedCache, n_groups: int, positions: int = 0):
        self._open(cache.k)
        torch, lib = self._torch, self._lib
        self._layout, self._cache, self.n_groups = cache._layout(), cache, int(n_groups)
        nbytes, room = lib.dmtd_shared_plan_bytes(cache._p, self.n_groups), lib.dmtd_shared_workspace_bytes(cache._p)
        if nbytes == 0 or room == 0:
            _raise(lib, DMTD_EINVAL)
        if positions < 0:
            raise ValueError("positions must not be negative")
        self._memory, self._ws = torch.zeros(nbytes, dtype=torch.uint8, device=self.device), torch.empty(room, dtype=torch.uint8, device=self.device)
        self._c = _SharedPlan(self.n_groups, int(positions), self._memory.data_ptr(), nbytes, self._ws.data_ptr(), room)
        self._p = C.byref(self._c)
        stream = torch.cuda.current_stream(self.device)
        stream.synchronize()              # zeroed, whichever stream the first call is on
        self._streams = {stream.cuda_stream}

    def _used_on(self, stream):
        if stream not in self._streams:
            self._streams.add(stream)
            for t in (self._memory, self._ws):
                t.record_stream(self._torch.cuda.current_stream(self._index))      # not reused before this stream's work has ended

    def build(self, start, cu_rows, group, prefix_pages):
        """A step's plan: ``start`` int32 ``[n_req]`` and ``cu_rows`` int32 ``[n_req + 1]`` as for :meth:`PagedCache.attention`, ``group`` int32 ``[n_req]`` (outside ``[0, n_groups)``: none),
        ``prefix_pages`` int32 ``[n_groups]``, the pages that the tables of a group's requests start with."""
        c, i32, dev = self._cache, self._i32, self._index
        self._used_on(self._call(self._lib.dmtd_shared_plan_build, c._p, self._p, _want(start, "start", i32, dev, c._per_req), _want(cu_rows, "cu_rows", i32, dev, c._per_end),
                                 _want(group, "group", i32, dev, c._per_req), _want(prefix_pages, "prefix_pages", i32, dev, (self.n_groups,))))
