"""Thin ctypes binding to libsdlm.so (include/sdlm.h).  Argument marshalling only.

torch is used for device memory (the workspace, weights, outputs) and for the stream; every step of the
block-decode path runs in the library's own HIP kernels.  There is no fallback: if the library cannot be
loaded, importing the entry points raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsdlm.so")

PHASES = ("rows", "norm", "qkv", "rope", "attn", "oproj", "gateup", "down", "lmhead", "accept", "attn_merge")
OK, EINVAL, ECAPACITY, ESTATE, EHIP = 0, -1, -2, -3, -4

STEP_PLAN = ("chain", "embeds", "qkv_rows", "qkv_rest", "lm_head", "lm_accept", "attn")

EXPORTS = ("sdlm_workspace_bytes", "sdlm_create", "sdlm_init_weights", "sdlm_prefill", "sdlm_decode_step",
           "sdlm_decode_step_static", "sdlm_graph", "sdlm_verify_step", "sdlm_kv_commit", "sdlm_get_lengths", "sdlm_debug_tap", "sdlm_debug_rows", "sdlm_debug_read_kv",
           "sdlm_debug_gemm_plan", "sdlm_debug_step_plan", "sdlm_max_rows", "sdlm_profile", "sdlm_profile_every", "sdlm_profile_read", "sdlm_kernel_info", "sdlm_last_error",
           "sdlm_destroy", "sdlm_op_error", "sdlm_sample_workspace_bytes", "sdlm_sample", "sdlm_tree_attention_workspace_bytes", "sdlm_tree_attention",
           "sdlm_kv_fork_workspace_bytes", "sdlm_kv_fork", "sdlm_kv_compact", "sdlm_sample_step", "sdlm_fork", "sdlm_verify_tree", "sdlm_tree_commit",
           "sdlm_kv_describe")


class ModelCfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("ffn", C.c_int32), ("vocab", C.c_int32),
                ("rope_theta", C.c_float), ("rms_eps", C.c_float), ("logit_scale", C.c_float),
                ("dtype", C.c_int32), ("mask_token_id", C.c_int32), ("has_qkv_bias", C.c_int32),
                ("block_causal", C.c_int32)]


class RunCfg(C.Structure):
    _fields_ = [("max_batch", C.c_int32), ("max_seq_len", C.c_int32), ("block_D", C.c_int32), ("kv_layout", C.c_int32),
                ("page_size", C.c_int32), ("n_pages", C.c_int32), ("tau", C.c_float), ("conf_fn", C.c_int32),
                ("accept_rule", C.c_int32), ("prefill_rows", C.c_int32)]


_PP = C.POINTER(C.c_void_p)
_LAYER_FIELDS = ("attn_norm", "wq", "wk", "wv", "wo", "bq", "bk", "bv", "ffn_norm", "w_gate", "w_up", "w_down")


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("attn_norm", _PP), ("wq", _PP), ("wk", _PP), ("wv", _PP), ("wo", _PP),
                ("bq", _PP), ("bk", _PP), ("bv", _PP), ("ffn_norm", _PP), ("w_gate", _PP), ("w_up", _PP), ("w_down", _PP)]


class SampleArgs(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("row_stride", C.c_int64), ("dtype", C.c_int32), ("rows", C.c_int32), ("vocab", C.c_int32),
                ("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p), ("u", C.c_void_p),
                ("ids", C.c_void_p), ("prob", C.c_void_p)]


class Sampling(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p), ("top_k", C.c_void_p), ("u", C.c_void_p)]


class KvDesc(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("layer_stride", C.c_int64), ("n_layers", C.c_int32), ("n_tiles", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("n_pages", C.c_int32), ("max_seqs", C.c_int32), ("pages_per_seq", C.c_int32),
                ("page_table", C.c_void_p), ("lengths", C.c_void_p), ("backed", C.c_void_p), ("page_refs", C.c_void_p), ("free_pages", C.c_void_p),
                ("free_count", C.c_void_p)]


class TreeArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("q_stride", C.c_int64), ("out_stride", C.c_int64), ("n_rows", C.c_int32), ("n_seqs", C.c_int32),
                ("n_q_heads", C.c_int32), ("max_nodes", C.c_int32), ("max_len", C.c_int32), ("node_offsets", C.c_void_p), ("mask", C.c_void_p),
                ("mask_words", C.c_int32), ("node_pages", C.c_int32), ("node_table", C.c_void_p), ("node_base", C.c_void_p)]


_lib = None


def load():
    """Load libsdlm.so (built by paper_2509_24007_amd/build.py); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python paper_2509_24007_amd/build.py` (no fallback exists)")
    L = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    L.sdlm_workspace_bytes.restype = sz
    L.sdlm_workspace_bytes.argtypes = [vp, vp]
    L.sdlm_create.restype = C.c_int
    L.sdlm_create.argtypes = [vp, vp, vp, sz, vp, C.POINTER(vp)]
    L.sdlm_init_weights.restype = C.c_int
    L.sdlm_init_weights.argtypes = [vp, vp, i32]
    L.sdlm_prefill.restype = C.c_int
    L.sdlm_prefill.argtypes = [vp, i32, vp, vp]
    L.sdlm_decode_step.restype = C.c_int
    L.sdlm_decode_step.argtypes = [vp, vp, vp, vp, vp]
    L.sdlm_decode_step_static.restype = C.c_int
    L.sdlm_decode_step_static.argtypes = [vp, vp, vp, vp, vp]
    L.sdlm_debug_gemm_plan.restype = C.c_int
    L.sdlm_debug_gemm_plan.argtypes = [C.c_int32] * 5 + [vp, vp, vp]
    L.sdlm_debug_step_plan.restype = C.c_int
    L.sdlm_debug_step_plan.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, vp]
    L.sdlm_graph.restype = C.c_int
    L.sdlm_graph.argtypes = [vp, C.c_int32]
    L.sdlm_verify_step.restype = C.c_int
    L.sdlm_verify_step.argtypes = [vp, C.c_int32, vp, vp, vp]
    L.sdlm_kv_commit.restype = C.c_int
    L.sdlm_kv_commit.argtypes = [vp, vp, vp]
    L.sdlm_get_lengths.restype = C.c_int
    L.sdlm_get_lengths.argtypes = [vp, vp, vp]
    L.sdlm_debug_tap.restype = C.c_int
    L.sdlm_debug_tap.argtypes = [vp, i32, i32, vp]
    L.sdlm_debug_rows.restype = C.c_int
    L.sdlm_debug_rows.argtypes = [vp, vp, vp, vp, vp, vp]
    L.sdlm_debug_read_kv.restype = C.c_int
    L.sdlm_debug_read_kv.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp]
    L.sdlm_max_rows.restype = i32
    L.sdlm_max_rows.argtypes = [vp]
    L.sdlm_profile.restype = C.c_int
    L.sdlm_profile.argtypes = [vp, i32]
    L.sdlm_profile_every.restype = C.c_int
    L.sdlm_profile_every.argtypes = [vp, i32]
    L.sdlm_profile_read.restype = C.c_int
    L.sdlm_profile_read.argtypes = [vp, vp, vp]
    L.sdlm_kernel_info.restype = C.c_char_p
    L.sdlm_kernel_info.argtypes = [vp]
    L.sdlm_last_error.restype = C.c_char_p
    L.sdlm_last_error.argtypes = [vp]
    L.sdlm_destroy.restype = None
    L.sdlm_destroy.argtypes = [vp]
    L.sdlm_sample_step.restype = C.c_int
    L.sdlm_sample_step.argtypes = [vp] * 6
    L.sdlm_fork.restype = C.c_int
    L.sdlm_fork.argtypes = [vp, i32, vp]
    L.sdlm_verify_tree.restype = C.c_int
    L.sdlm_verify_tree.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp]
    L.sdlm_tree_commit.restype = C.c_int
    L.sdlm_tree_commit.argtypes = [vp]
    L.sdlm_kv_describe.restype = C.c_int
    L.sdlm_kv_describe.argtypes = [vp, vp]
    L.sdlm_op_error.restype = C.c_char_p
    L.sdlm_op_error.argtypes = []
    L.sdlm_sample_workspace_bytes.restype = sz
    L.sdlm_sample_workspace_bytes.argtypes = [i32, i32]
    L.sdlm_sample.restype = C.c_int
    L.sdlm_sample.argtypes = [vp, vp, sz, vp]
    L.sdlm_tree_attention_workspace_bytes.restype = sz
    L.sdlm_tree_attention_workspace_bytes.argtypes = [vp, i32, i32, i32, i32]
    L.sdlm_tree_attention.restype = C.c_int
    L.sdlm_tree_attention.argtypes = [vp, i32, vp, vp, sz, vp]
    L.sdlm_kv_fork_workspace_bytes.restype = sz
    L.sdlm_kv_fork_workspace_bytes.argtypes = [vp]
    L.sdlm_kv_fork.restype = C.c_int
    L.sdlm_kv_fork.argtypes = [vp, vp, i32, i32, vp, vp, sz, vp]
    L.sdlm_kv_compact.restype = C.c_int
    L.sdlm_kv_compact.argtypes = [vp, i32, vp, i32, vp, i32, vp, i32, vp, vp]
    _lib = L
    return L


class SdlmError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"sdlm error {code}: {msg}")
        self.code = code


def model_cfg(m) -> ModelCfg:
    """From the synthetic-input module's ModelCfg (or any object with the same attributes)."""
    return ModelCfg(m.n_layers, m.hidden, m.n_q_heads, m.n_kv_heads, m.head_dim, m.ffn, m.vocab,
                    m.rope_theta, m.rms_eps, m.logit_scale, 0 if m.dtype == "fp32" else 1, m.mask_token_id,
                    int(bool(m.has_qkv_bias)), int(bool(getattr(m, "block_causal", False))))


def gemm_plan(epilogue: int, rows: int, min_rows: int, n: int, k: int):
    """(tile rows, tile columns, k splits) of the matrix-core GEMM launch for this problem; host logic, no GPU needed."""
    tr, tc, sp = C.c_int32(0), C.c_int32(0), C.c_int32(0)
    rc = load().sdlm_debug_gemm_plan(epilogue, rows, min_rows, n, k, C.byref(tr), C.byref(tc), C.byref(sp))
    if rc != 0:
        raise SdlmError(rc, "bad arguments to sdlm_debug_gemm_plan")
    return tr.value, tc.value, sp.value


def step_plan(mcfg: ModelCfg, batch: int, D: int, *, committed: bool = True, longest: int = 64, max_seq_len: int = 512) -> Dict[str, int]:
    """The forms a decode step takes (see sdlm_debug_step_plan in the header); host logic, no GPU needed."""
    run = RunCfg(batch, max_seq_len, D, 0, 16, 0, 0.5, 0, 0, 0)
    out = (C.c_int32 * len(STEP_PLAN))()
    rc = load().sdlm_debug_step_plan(C.byref(mcfg), C.byref(run), batch, int(committed), longest, out)
    if rc != 0:
        raise SdlmError(rc, "bad arguments to sdlm_debug_step_plan")
    return dict(zip(STEP_PLAN, out))


def _dp(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


class Context:
    """One sdlm_ctx plus the torch allocations it borrows."""

    def __init__(self, mcfg: ModelCfg, *, max_batch: int, max_seq_len: int, block_D: int, tau: float,
                 paged: bool = False, n_pages: int = 0, conf_fn: int = 0, accept_rule: int = 0,
                 prefill_rows: int = 0, device="cuda:0", poison: bool = False):
        L = load()
        self.L = L
        self.m = mcfg
        self.r = RunCfg(max_batch, max_seq_len, block_D, 1 if paged else 0, 16, n_pages, tau, conf_fn, accept_rule,
                        prefill_rows)
        self.device = torch.device(device)
        self.D, self.max_batch = block_D, max_batch
        need = L.sdlm_workspace_bytes(C.byref(self.m), C.byref(self.r))
        if need == 0:
            h = C.c_void_p()
            rc = L.sdlm_create(C.byref(self.m), C.byref(self.r), None, 0, None, C.byref(h))
            msg = L.sdlm_last_error(h).decode() if h else "invalid configuration"
            L.sdlm_destroy(h)
            raise SdlmError(rc, msg)
        self.workspace_bytes = need
        self.workspace = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        if poison:   # tests: every byte 0xFF (NaN as bf16/fp32, -1 as int) so that reliance on fresh memory shows
            self.workspace.fill_(0xFF)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        self.stream = torch.cuda.current_stream(self.device)
        self.h = C.c_void_p()
        rc = L.sdlm_create(C.byref(self.m), C.byref(self.r), C.c_void_p(self._ws_ptr), need,
                           C.c_void_p(self.stream.cuda_stream), C.byref(self.h))
        if rc != 0:
            msg = L.sdlm_last_error(self.h).decode()
            L.sdlm_destroy(self.h)
            self.h = None
            raise SdlmError(rc, msg)
        self.batch = 0
        self._keep: List[object] = []

    # -- helpers
    def _order_inputs(self):
        """The library runs on the stream the context was created on.  When torch's current stream is another one,
        work queued there that produces the tensors being handed over must come first."""
        cur = torch.cuda.current_stream(self.device)
        if cur.cuda_stream != self.stream.cuda_stream:
            self.stream.wait_stream(cur)

    def _check(self, rc: int):
        if rc != 0:
            raise SdlmError(rc, self.L.sdlm_last_error(self.h).decode())

    def close(self):
        if getattr(self, "h", None):
            torch.cuda.synchronize(self.device)
            self.L.sdlm_destroy(self.h)
            self.h = None
            self.workspace = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def kernel_info(self) -> str:
        return self.L.sdlm_kernel_info(self.h).decode()

    @property
    def max_rows(self) -> int:
        return int(self.L.sdlm_max_rows(self.h))

    # -- the four core calls
    def init_weights(self, globals_: Optional[Dict[str, torch.Tensor]] = None,
                     layers: Optional[Dict[int, Dict[str, Optional[torch.Tensor]]]] = None) -> None:
        """globals_: embed / lm_head / final_norm; layers: {layer index: tensors of that layer}.  Either may be
        partial; tensors may live on the device or on the host (all of one call in the same place)."""
        w = Weights()
        nL = self.m.n_layers
        keep = []
        on_dev = None

        def place(t):
            nonlocal on_dev
            assert t.is_contiguous()
            d = t.is_cuda
            assert on_dev is None or on_dev == d, "mixing host and device tensors in one call"
            on_dev = d
            return t.data_ptr()

        for name in ("embed", "lm_head", "final_norm"):
            t = (globals_ or {}).get(name)
            setattr(w, name, place(t) if t is not None else None)
        for name in _LAYER_FIELDS:
            tab = (C.c_void_p * nL)()
            for l in range(nL):
                t = (layers or {}).get(l, {}).get(name)
                tab[l] = place(t) if t is not None else None
            keep.append(tab)
            setattr(w, name, C.cast(tab, _PP))
        self._order_inputs()
        self._check(self.L.sdlm_init_weights(self.h, C.byref(w), 1 if on_dev else 0))

    def prefill(self, prompts: Sequence) -> None:
        ids, offs = [], [0]
        for p in prompts:
            p = [int(v) for v in (p.tolist() if hasattr(p, "tolist") else p)]
            ids.extend(p)
            offs.append(len(ids))
        a = (C.c_int32 * max(1, len(ids)))(*ids)
        o = (C.c_int32 * len(offs))(*offs)
        self._check(self.L.sdlm_prefill(self.h, len(prompts), a, o))
        self.batch = len(prompts)

    def decode_step(self, ids: torch.Tensor, count: torch.Tensor, conf: Optional[torch.Tensor] = None,
                    logits: Optional[torch.Tensor] = None, static_scratch: bool = False) -> None:
        """static_scratch=True calls sdlm_decode_step_static (partial results in the library's static array)."""
        B, D = self.batch, self.D
        assert ids.dtype == torch.int32 and ids.numel() >= B * D and ids.is_cuda and ids.is_contiguous()
        assert count.dtype == torch.int32 and count.numel() >= B and count.is_cuda
        assert conf is None or (conf.dtype == torch.float32 and conf.numel() >= B * D and conf.is_cuda and conf.is_contiguous())
        assert logits is None or (logits.dtype == torch.float32 and logits.numel() >= B * D * self.m.vocab and
                                  logits.is_cuda and logits.is_contiguous())
        fn = self.L.sdlm_decode_step_static if static_scratch else self.L.sdlm_decode_step
        self._check(fn(self.h, _dp(ids), _dp(count), _dp(conf), _dp(logits)))

    def graph(self, enable: bool = True) -> None:
        """Replay decode_step as a HIP graph (the context must have been created on a non-default stream)."""
        self._check(self.L.sdlm_graph(self.h, 1 if enable else 0))

    def verify_step(self, rule: int = 0, ids_tilde: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                    logits: Optional[torch.Tensor] = None) -> None:
        """Self-speculative verification of the last decode_step; ids_tilde [batch, D] int32, count [batch] int32,
        logits [batch, D-1, vocab] fp32 (all optional, on the device)."""
        for t, n in ((ids_tilde, self.batch * self.D), (count, self.batch)):
            if t is not None:
                assert t.dtype == torch.int32 and t.is_cuda and t.is_contiguous() and t.numel() >= n
        if logits is not None:
            assert logits.dtype == torch.float32 and logits.is_cuda and logits.is_contiguous()
            assert logits.numel() >= self.batch * (self.D - 1) * self.m.vocab
        self._check(self.L.sdlm_verify_step(self.h, int(rule), _dp(ids_tilde), _dp(count), _dp(logits)))

    def kv_commit(self, ids_override: Optional[torch.Tensor] = None, count_override: Optional[torch.Tensor] = None) -> None:
        if ids_override is not None:
            assert ids_override.dtype == torch.int32 and ids_override.is_cuda and ids_override.is_contiguous()
            assert count_override is not None and count_override.dtype == torch.int32 and count_override.is_cuda
            assert ids_override.numel() >= self.batch * self.D and count_override.numel() >= self.batch
            self._order_inputs()
        self._check(self.L.sdlm_kv_commit(self.h, _dp(ids_override), _dp(count_override)))

    # -- sampled tokens, forks, token trees
    def sample_step(self, logits: torch.Tensor, u: torch.Tensor, ids: torch.Tensor, count: torch.Tensor, conf: Optional[torch.Tensor] = None, *,
                    temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                    min_p: Optional[torch.Tensor] = None) -> None:
        """Draw the tokens of the last decode_step, whose `logits` it wrote, instead of taking the arg-max ones (sdlm_sample_step); u and the settings: [batch, D]."""
        n, f32 = self.batch * self.D, torch.float32
        how = Sampling(*[_ints(t, n, name, self.device, dt) for t, name, dt in ((temperature, "temperature", f32), (top_p, "top_p", f32), (min_p, "min_p", f32),
                                                                                (top_k, "top_k", torch.int32), (u, "u", f32))])
        self._order_inputs()
        self._check(self.L.sdlm_sample_step(self.h, _ints(logits, n * self.m.vocab, "logits", self.device, f32), C.byref(how), _ints(ids, n, "ids", self.device),
                                            _ints(count, self.batch, "count", self.device), _ints(conf, n, "conf", self.device, f32)))

    def fork(self, parents: Sequence[int]) -> None:
        """The new batch's sequence b continues sequence parents[b]; the others end (sdlm_fork).  Synchronises."""
        p = [int(v) for v in parents]
        if not all(-2 ** 31 <= v < 2 ** 31 for v in p):
            _refuse("parents must be 32-bit integers")
        self._check(self.L.sdlm_fork(self.h, len(p), (C.c_int32 * max(1, len(p)))(*p)))
        self.batch = len(p)

    def verify_tree(self, tokens: torch.Tensor, parents: torch.Tensor, path: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                    next: Optional[torch.Tensor] = None, logits: Optional[torch.Tensor] = None) -> None:
        """Verify a token tree of every sequence behind the last decode_step (sdlm_verify_tree): tokens, parents, path [batch, nodes], count, next [batch], logits [batch, nodes, vocab]."""
        if tokens.dim() != 2 or tokens.shape != parents.shape or tokens.shape[0] != self.batch:
            _refuse("tokens and parents must be [batch, nodes]")
        B, T = tokens.shape
        self._order_inputs()
        self._check(self.L.sdlm_verify_tree(self.h, T, _ints(tokens, B * T, "tokens", self.device), _ints(parents, B * T, "parents", self.device), _ints(path, B * T, "path", self.device),
                                            _ints(count, B, "count", self.device), _ints(next, B, "next", self.device), _ints(logits, B * T * self.m.vocab, "logits", self.device, torch.float32)))

    def tree_commit(self) -> None:
        """Publish the branch that the last verify_tree accepted, and the token behind it (sdlm_tree_commit)."""
        self._check(self.L.sdlm_tree_commit(self.h))

    # -- state and debugging
    def get_lengths(self):
        n = torch.empty(self.batch, dtype=torch.int32, device=self.device)
        c = torch.empty(self.batch, dtype=torch.int32, device=self.device)
        self._check(self.L.sdlm_get_lengths(self.h, _dp(n), _dp(c)))
        return n.cpu(), c.cpu()

    def tap(self, layer: int, which: int, dst: Optional[torch.Tensor]) -> None:
        self._check(self.L.sdlm_debug_tap(self.h, layer, which, _dp(dst)))

    def rows(self):
        mr = self.max_rows
        out = [torch.empty(mr, dtype=torch.int32, device=self.device) for _ in range(4)]
        n = torch.empty(1, dtype=torch.int32, device=self.device)
        self._check(self.L.sdlm_debug_rows(self.h, *[_dp(t) for t in out], _dp(n)))
        torch.cuda.synchronize(self.device)
        R = int(n.item())
        return {k: t[:R].cpu() for k, t in zip(("tok", "pos", "seq", "kind"), out)}

    def read_kv(self, layer: int, seq: int, kv_head: int, pos0: int, count: int):
        d = self.m.head_dim
        k = torch.empty(count, d, dtype=torch.float32, device=self.device)
        v = torch.empty(count, d, dtype=torch.float32, device=self.device)
        self._check(self.L.sdlm_debug_read_kv(self.h, layer, seq, kv_head, pos0, count, _dp(k), _dp(v)))
        torch.cuda.synchronize(self.device)
        return k.cpu(), v.cpu()

    def profile(self, phases=None, every: int = 1) -> None:
        """phases: None/False -> off, True -> all, or an iterable of phase names to bracket with events; every: only
        every n-th launch of a phase is bracketed."""
        self._check(self.L.sdlm_profile_every(self.h, int(every)))
        if phases is None or phases is False:
            mask = 0
        elif phases is True:
            mask = -1
        else:
            mask = 0
            for p in phases:
                mask |= 1 << PHASES.index(p)
        self._check(self.L.sdlm_profile(self.h, mask))

    def profile_read(self):
        ms = (C.c_float * len(PHASES))()
        cnt = (C.c_int32 * len(PHASES))()
        self._check(self.L.sdlm_profile_read(self.h, ms, cnt))
        return {p: (float(ms[i]), int(cnt[i])) for i, p in enumerate(PHASES)}


# ---------------------------------------------------------------- operators on the caller's tensors

PAGE = 16
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _refuse(msg: str) -> None:
    raise SdlmError(EINVAL, msg)


def _ints(t: Optional[torch.Tensor], n: int, name: str, dev, dtype=torch.int32) -> Optional[int]:
    """Address of a contiguous vector of at least n entries on the operator's device."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != dev or not t.is_contiguous() or t.numel() < n:
        _refuse(f"{name} must be {n} or more contiguous {dtype} on {dev}")
    return t.data_ptr()


def _run_op(dev, fn, *args) -> None:
    """Call an entry point on the tensors' device and that device's current stream."""
    if dev.index == torch.cuda.current_device():
        rc = fn(*args, torch.cuda.current_stream(dev).cuda_stream)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, torch.cuda.current_stream(dev).cuda_stream)
    if rc != 0:
        raise SdlmError(rc, load().sdlm_op_error().decode())


def _scratch(need: int, dev) -> torch.Tensor:
    if need == 0:
        raise SdlmError(EINVAL, load().sdlm_op_error().decode() or "sizes outside the operator's limits")
    return torch.empty(need, dtype=torch.uint8, device=dev)


def sample(logits: torch.Tensor, u: torch.Tensor, *, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
           top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None):
    """Draw one token from each row of logits [rows, vocab] (fp32 or bf16, the last dimension contiguous) with the uniform numbers u [rows]; the settings are
    vectors over the rows or None (see sdlm_sample in the header).  Returns ids [rows] int32 and their probabilities [rows] fp32.  Runs on the current stream."""
    L = load()
    if not (logits.is_cuda and logits.dim() == 2 and logits.dtype in _DTYPES and (logits.stride(1) == 1 or logits.shape[1] == 1)):
        _refuse("logits must be [rows, vocab] fp32 or bf16 on a GPU, the last dimension contiguous")
    R, V = logits.shape
    dev, f32 = logits.device, torch.float32
    stride = logits.stride(0) if R > 1 else V
    ids = torch.empty(R, dtype=torch.int32, device=dev)
    prob = torch.empty(R, dtype=f32, device=dev)
    a = SampleArgs(logits.data_ptr(), stride, _DTYPES[logits.dtype], R, V, _ints(temperature, R, "temperature", dev, f32), _ints(top_k, R, "top_k", dev),
                   _ints(top_p, R, "top_p", dev, f32), _ints(min_p, R, "min_p", dev, f32), _ints(u, R, "u", dev, f32), ids.data_ptr(), prob.data_ptr())
    if R:
        need = L.sdlm_sample_workspace_bytes(R, V)
        if not (need > 0):
            _refuse(f"{R} rows of {V} logits are outside the limits")
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        _run_op(dev, L.sdlm_sample, C.byref(a), ws.data_ptr(), need)
    return ids, prob


class KvCache:
    """A paged K/V cache in the caller's tensors (sdlm_kv in the header): pool [layers, tiles, kv heads, 2, 16 * head_dim] fp32 or bf16, page_table [sequences,
    pages a sequence], lengths [sequences].  Forking needs the rest: n_pages, backed [sequences], page_refs [n_pages], free_pages [n_pages] and free_count [1].  All
    int32 on the pool's device.  The operators run on that device's current stream."""

    def __init__(self, pool: torch.Tensor, *, page_table: torch.Tensor, lengths: torch.Tensor, n_pages: int = 0, backed: Optional[torch.Tensor] = None,
                 page_refs: Optional[torch.Tensor] = None, free_pages: Optional[torch.Tensor] = None, free_count: Optional[torch.Tensor] = None):
        if not (pool.is_cuda and pool.dim() == 5 and pool.numel() and pool.dtype in _DTYPES and pool.shape[3] == 2 and pool.shape[4] % PAGE == 0):
            _refuse("pool must be [layers, tiles, kv heads, 2, 16 * head_dim] fp32 or bf16 on a GPU")
        if not (pool[0].is_contiguous()):
            _refuse("a layer of the pool must be contiguous")
        if not (page_table.dim() == 2):
            _refuse("page_table must be [sequences, pages a sequence]")
        self.device = dev = pool.device
        self.dtype, self.head_dim, self.n_kv_heads = pool.dtype, pool.shape[4] // PAGE, pool.shape[2]
        S, pps = page_table.shape
        stride = pool.stride(0) if pool.shape[0] > 1 else pool[0].numel()
        self._keep = (pool, page_table, lengths, backed, page_refs, free_pages, free_count)
        self.max_seqs, self.pages_per_seq = S, pps
        self.desc = KvDesc(pool.data_ptr(), stride, pool.shape[0], pool.shape[1], pool.shape[2], self.head_dim, _DTYPES[pool.dtype], n_pages, S, pps,
                           _ints(page_table, S * pps, "page_table", dev), _ints(lengths, S, "lengths", dev), _ints(backed, S, "backed", dev),
                           _ints(page_refs, n_pages, "page_refs", dev), _ints(free_pages, n_pages, "free_pages", dev), _ints(free_count, 1, "free_count", dev))
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(dev).synchronize()   # a fork may run on any stream

    def fork(self, parent: torch.Tensor, *, share: bool = True) -> None:
        """Sequence b becomes what sequence parent[b] is (-1: empty); see sdlm_kv_fork.  Does not synchronise: check() raises if the last fork was refused."""
        L = load()
        need = L.sdlm_kv_fork_workspace_bytes(C.byref(self.desc))
        ws = _scratch(need, self.device)
        _run_op(self.device, L.sdlm_kv_fork, C.byref(self.desc), _ints(parent, 0, "parent", self.device), parent.numel(), int(share), self.status.data_ptr(), ws.data_ptr(), need)

    def check(self) -> None:
        """Wait for the device, whatever stream the last fork runs on, and raise if it was refused."""
        torch.cuda.synchronize(self.device)
        bad = int(self.status.item())
        if bad & 2:
            raise SdlmError(EINVAL, "a parent or a page of the table is out of range: nothing was changed")
        if bad:
            raise SdlmError(ECAPACITY, "not enough free pages: nothing was changed")

    def compact(self, path: torch.Tensor, path_len: torch.Tensor, *, node_table: torch.Tensor, node_base: Optional[torch.Tensor] = None) -> None:
        """Move the K/V of nodes path[b, :path_len[b]] to the positions from lengths[b] on, in every layer; see sdlm_kv_compact."""
        dev = self.device
        if not (path.dim() == 2 and node_table.dim() == 2 and node_table.shape[0] >= path.shape[0]):
            _refuse("path must be [sequences, most nodes], node_table [sequences, pages]")
        S, P = path.shape
        _run_op(dev, load().sdlm_kv_compact, C.byref(self.desc), S, _ints(path, S * P, "path", dev), P, _ints(path_len, S, "path_len", dev), P,
                _ints(node_table, 1, "node_table", dev), node_table.shape[1], _ints(node_base, S, "node_base", dev))


def tree_attention(kv: KvCache, layer: int, q: torch.Tensor, node_offsets: torch.Tensor, mask: torch.Tensor, *, node_table: torch.Tensor, max_nodes: int,
                   node_base: Optional[torch.Tensor] = None, max_len: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of drafted token trees over one layer of the cache (see sdlm_tree_attention): q [nodes, query heads, head_dim] of the cache's type, rows node_offsets[b] up to
    node_offsets[b + 1] belong to sequence b; mask [nodes, words] int64, bit j of a row: the node sees node j of its sequence.  Returns out, shaped as q; rows outside node_offsets
    are left as they are."""
    L, dev = load(), kv.device
    if not (q.dim() == 3 and q.shape[2] == kv.head_dim and q.dtype == kv.dtype and q.device == dev):
        _refuse("q must be [nodes, query heads, head_dim] of the cache's type and device")
    if not (mask.dim() == 2 and node_table.dim() == 2):
        _refuse("mask must be [nodes, words], node_table [sequences, pages]")
    N, H, d = q.shape
    S = node_offsets.numel() - 1
    if out is None:
        out = torch.empty(N, H, d, dtype=q.dtype, device=dev)
    if not (out.shape == q.shape and out.dtype == q.dtype and out.device == dev):
        _refuse("out must be shaped as q, of its type and device")
    for t in (q, out):
        if not (t.stride(2) == 1 and (t.stride(1) == d or H == 1)):
            _refuse("the heads of a row of q and out must be contiguous")
    if not (S >= 0 and node_table.shape[0] >= S and mask.shape[0] >= N):
        _refuse("node_offsets, node_table and mask must agree with the nodes")
    row = H * d
    a = TreeArgs(q.data_ptr(), out.data_ptr(), q.stride(0) if N > 1 else row, out.stride(0) if N > 1 else row, N, S, H, max_nodes, max_len,
                 _ints(node_offsets, S + 1, "node_offsets", dev), _ints(mask, N, "mask", dev, torch.int64), mask.shape[1], node_table.shape[1],
                 _ints(node_table, 1, "node_table", dev), _ints(node_base, S, "node_base", dev))
    need = L.sdlm_tree_attention_workspace_bytes(C.byref(kv.desc), H, S, max_nodes, max_len)
    ws = _scratch(need, dev)
    _run_op(dev, L.sdlm_tree_attention, C.byref(kv.desc), layer, C.byref(a), ws.data_ptr(), need)
    return out
