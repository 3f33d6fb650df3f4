"""MI355X engine for adaptive self-speculative decoding: thin ctypes binding of libasd.so.

Argument marshalling only: every step of the decoding path runs in the HIP kernels
of the C-ABI library declared in include/asd.h.  PyTorch supplies device memory
(the arena) and the stream.  There is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libasd.so")

OK, E_INVAL, E_STATE, E_NOMEM, E_IO, E_HIP = 0, -1, -2, -3, -4, -5
DT_F32, DT_BF16, DT_FP8 = 0, 1, 2      # DT_FP8: 8-bit pages of a KVCache only
MAX_ROWS = 16
MAX_SEQ = 65536
# development / test switches of Config.debug_flags (none changes what is computed)
DBG_ATT_W4, DBG_ATT_GH1, DBG_RS_POW2, DBG_SAMPLE_MEM = 1, 2, 4, 8
KERNEL_CLASSES = ("embed", "qkv", "attn", "oproj", "gateup", "down", "lmhead", "finish")


class AsdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"asd error {code}: {msg}")
        self.code = code


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab",
                 "max_seq", "page_tokens", "max_rows", "dtype")] + \
               [("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float),
                ("debug_flags", ctypes.c_uint32), ("debug_tune", ctypes.c_char_p)]


class GenParams(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("m", ctypes.c_int32), ("n", ctypes.c_int32), ("use_cs", ctypes.c_int32),
                ("draft_len", ctypes.c_int32), ("mask_mode", ctypes.c_int32), ("fixed_mask", ctypes.c_void_p),
                ("use_graphs", ctypes.c_int32), ("alpha_mlp", ctypes.c_float), ("use_cs_mlp", ctypes.c_int32),
                ("exit_mode", ctypes.c_int32)] + \
               [(n, ctypes.c_double) for n in ("gamma0", "ar0", "ar_target", "eps", "beta1", "beta2")] + \
               [("temperature", ctypes.c_float), ("seed", ctypes.c_uint64), ("sample_index0", ctypes.c_int64)]


class GenStats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("cycles", "drafted", "accepted", "emitted")] + \
               [("ms_prefill", ctypes.c_double), ("ms_decode", ctypes.c_double), ("mask_changes", ctypes.c_int64),
                ("gamma", ctypes.c_double), ("ar", ctypes.c_double)] + \
               [(n, ctypes.c_double) for n in ("ms_draft", "ms_verify", "ms_other", "bytes_draft", "bytes_verify")]


PREFILL_CLASSES = ("rows", "qkv", "attn", "oproj", "gateup", "down", "lmhead")


class PrefillTimes(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * 7), ("launches", ctypes.c_int32 * 7), ("flops", ctypes.c_double * 7),
                ("ms_total", ctypes.c_double)]


class PromptBlock(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_blocks", "row0", "rows", "attn_rows")] + \
               [("tile", ctypes.c_int32 * 4), ("slices", ctypes.c_int32 * 4)]


class KernelTimes(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * 8), ("launches", ctypes.c_int32 * 8), ("bytes", ctypes.c_double * 8),
                ("ms_total", ctypes.c_double)]


class KvShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_heads", "n_kv_heads", "head_dim", "page_tokens", "dtype", "kv_dtype")]


class KvBatch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("pages", "page_table", "row_start", "kv_len", "status")] + \
               [(n, ctypes.c_int32) for n in ("n_pages", "table_stride", "n_seqs", "n_rows", "max_new", "max_len")]


class KvPrep(ctypes.Structure):
    _fields_ = [("q_gain", ctypes.c_void_p), ("k_gain", ctypes.c_void_p), ("eps", ctypes.c_float), ("rope", ctypes.c_void_p)] + \
               [(n, ctypes.c_int32) for n in ("rope_positions", "rot_dim", "interleaved")]


class Rope(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("rot_dim", ctypes.c_int32)] + \
               [(n, ctypes.c_double) for n in ("theta", "factor", "low", "high", "trained", "gain")]


_lib = None
_kv_ready = False


def lib():
    """Load libasd.so (built by paper_2410_01028_amd.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2410_01028_amd.build` first")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        cfgp = ctypes.POINTER(Config)
        L.asd_arena_bytes.restype = sz
        L.asd_arena_bytes.argtypes = [cfgp]
        L.asd_plan_prompt.argtypes = [cfgp, i32, i32, ctypes.POINTER(PromptBlock)]
        L.asd_create.argtypes = [cfgp, vp, sz, vp, ctypes.POINTER(vp)]
        L.asd_destroy.argtypes = [vp]
        L.asd_destroy.restype = None
        L.asd_last_error.restype = ctypes.c_char_p
        L.asd_last_error.argtypes = [vp]
        L.asd_set_weight.argtypes = [vp, i32, i32, vp, sz, i32]
        L.asd_get_weight.argtypes = [vp, i32, i32, vp, sz]
        L.asd_get_kv.argtypes = [vp, i32, i32, i32, vp, vp]
        L.asd_init_synthetic.argtypes = [vp, ctypes.c_uint64]
        L.asd_load_weights_file.argtypes = [vp, ctypes.c_char_p]
        L.asd_set_page_table.argtypes = [vp, vp, i32]
        L.asd_reset.argtypes = [vp]
        L.asd_truncate.argtypes = [vp, i32]
        L.asd_kv_len.argtypes = [vp]
        L.asd_forward.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp, vp, vp]
        L.asd_forward_noalloc.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp, vp]
        L.asd_check.argtypes = [vp]
        L.asd_prefill.argtypes = [vp, vp, i32, vp, vp, vp]
        L.asd_prefill_chunked.argtypes = [vp, vp, i32, vp, vp, vp]
        L.asd_admg2.argtypes = [vp, i32, ctypes.c_float, i32, i32, i32, ctypes.c_float, i32, vp]
        L.asd_admg.argtypes = [vp, i32, ctypes.c_float, i32, i32, i32, vp]
        L.asd_spec_sample.argtypes = [vp, vp, vp, i32, ctypes.c_float, ctypes.c_uint64, ctypes.c_int64, vp, vp, vp]
        L.asd_decode.argtypes = [vp, i32, i32, ctypes.POINTER(GenParams), vp, ctypes.POINTER(GenStats), vp]
        L.asd_generate.argtypes = [vp, vp, i32, i32, ctypes.POINTER(GenParams), vp, ctypes.POINTER(GenStats), vp]
        L.asd_time_pass.argtypes = [vp, i32, vp, i32, i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
        L.asd_profile_forward.argtypes = [vp, i32, vp, ctypes.POINTER(KernelTimes)]
        L.asd_copy_bench.argtypes = [vp, sz, i32, ctypes.POINTER(ctypes.c_double)]
        L.asd_profile_prefill.argtypes = [vp, vp, i32, ctypes.POINTER(PrefillTimes)]
        L.asd_time_step_class.argtypes = [vp, i32, i32, i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
        _lib = L
    return _lib


def _kv_lib():
    """The library with the signatures of the operators over a KVCache."""
    global _kv_ready
    L = lib()
    if not _kv_ready:
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        shape, batch = ctypes.POINTER(KvShape), ctypes.POINTER(KvBatch)
        L.asd_kv_page_bytes.restype = sz
        L.asd_kv_page_bytes.argtypes = [shape]
        # (structures by address: a pointer object per call costs as much as the rest of the marshalling)
        L.asd_kv_append.argtypes = [vp, vp, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp]
        L.asd_kv_attend_workspace.restype = sz
        L.asd_kv_attend_workspace.argtypes = [vp, vp]
        L.asd_kv_attend.argtypes = [vp, vp, vp, i64, vp, i64, ctypes.c_float, vp, sz, vp]
        L.asd_kv_read.argtypes = [vp, vp, vp, i64, vp, i64, vp]
        L.asd_rope_table.argtypes = [ctypes.POINTER(Rope), i32, vp, vp]
        L.asd_kv_view.argtypes = [vp, i32, shape, batch]
        L.asd_set_kv_len.argtypes = [vp, i32]
        _kv_ready = True
    return L


def make_config(shape, max_seq: int, page_tokens: int = 64, max_rows: int = MAX_ROWS, debug_flags: int = 0,
                debug_tune: str | None = None) -> Config:
    """Config from any object with the shape fields (n_layers, d_model, ..., dtype, rms_eps, rope_theta)."""
    return Config(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn,
                  shape.vocab, max_seq, page_tokens, max_rows, shape.dtype, shape.rms_eps, shape.rope_theta,
                  debug_flags, None if debug_tune is None else debug_tune.encode())


def arena_bytes(cfg: Config) -> int:
    return int(lib().asd_arena_bytes(ctypes.byref(cfg)))


PROMPT_GEMMS = ("qkv", "oproj", "gateup", "down")


def plan_prompt(cfg: Config, n: int) -> list[dict]:
    """How Engine.prefill runs a prompt of n tokens: one dict per block (row0, rows, attn_rows, and per contraction of
    PROMPT_GEMMS the ring kernel's tile shape, -1 for the four-wave kernel, and the K slices); [] for a prompt that the
    decode kernels take as one pass."""
    blocks, b = [], PromptBlock()
    while True:
        rc = lib().asd_plan_prompt(ctypes.byref(cfg), n, len(blocks), ctypes.byref(b))
        if rc:
            raise AsdError(rc, "asd_plan_prompt: invalid configuration or prompt length")
        if b.n_blocks == 0:
            return []
        blocks.append({"row0": b.row0, "rows": b.rows, "attn_rows": b.attn_rows, "tile": dict(zip(PROMPT_GEMMS, b.tile)),
                       "slices": dict(zip(PROMPT_GEMMS, b.slices))})
        if len(blocks) == b.n_blocks:
            return blocks


def admg(c_attn, alpha: float, m: int, n: int, use_cs: bool = True) -> np.ndarray:
    """Algorithm 1 on the host: skip mask [2L] from the attention sublayers' ACS."""
    c = np.ascontiguousarray(c_attn, dtype=np.float32)
    mask = np.zeros(2 * c.size, dtype=np.uint8)
    rc = lib().asd_admg(c.ctypes.data, c.size, alpha, m, n, int(use_cs), mask.ctypes.data)
    if rc:
        raise AsdError(rc, "asd_admg: invalid argument")
    return mask


def admg2(c_all, alpha: float, m: int, n: int, use_cs: bool = True, alpha_mlp: float = 0.0, use_cs_mlp: bool = False) -> np.ndarray:
    """Algorithm 1 plus CS thresholding of the MLP sublayers, from all 2L ACS values (attention, MLP interleaved)."""
    c = np.ascontiguousarray(c_all, dtype=np.float32)
    mask = np.zeros(c.size, dtype=np.uint8)
    rc = lib().asd_admg2(c.ctypes.data, c.size // 2, alpha, m, n, int(use_cs), alpha_mlp, int(use_cs_mlp), mask.ctypes.data)
    if rc:
        raise AsdError(rc, "asd_admg2: invalid argument")
    return mask


def _ptr(a):
    return None if a is None else a.ctypes.data


class Engine:
    """One engine on the current CUDA/HIP device; owns a torch uint8 arena it lends to the library."""

    def __init__(self, cfg: Config, device: str = "cuda:0", arena_fill: int | None = None):
        """arena_fill: byte value the arena is filled with before the library sees it (tests: every region the
        library reads must have been written by the library first); None leaves the allocator's bytes."""
        import torch
        self._torch = torch
        self.cfg = cfg
        need = arena_bytes(cfg)
        if need == 0:
            raise AsdError(E_INVAL, "invalid configuration")
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.arena = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        if arena_fill is not None:
            self.arena.fill_(arena_fill)
            torch.cuda.synchronize(self.device)
        base = (self.arena.data_ptr() + 255) // 256 * 256
        # a stream of its own (default priority): graph capture is not allowed on the legacy default stream
        self.stream = torch.cuda.Stream(self.device)
        h = ctypes.c_void_p()
        rc = lib().asd_create(ctypes.byref(cfg), base, need, self.stream.cuda_stream, ctypes.byref(h))
        if rc:
            raise AsdError(rc, lib().asd_last_error(None).decode())
        self._h = h
        self.L2 = 2 * cfg.n_layers

    def close(self):
        if getattr(self, "_h", None):
            lib().asd_destroy(self._h)
            self._h = None
            self.arena = None

    def __del__(self):
        try:
            self.close()
        except Exception:      # interpreter shutdown: module globals may already be gone
            pass

    def _ck(self, rc: int):
        if rc:
            raise AsdError(rc, lib().asd_last_error(self._h).decode())

    # ---- weights
    def set_weight(self, tensor: int, layer: int, arr: np.ndarray):
        a = np.ascontiguousarray(arr)
        self._ck(lib().asd_set_weight(self._h, tensor, layer, a.ctypes.data, a.nbytes, 0))

    def get_weight(self, tensor: int, layer: int, shape, dtype) -> np.ndarray:
        out = np.empty(shape, dtype=dtype)
        self._ck(lib().asd_get_weight(self._h, tensor, layer, out.ctypes.data, out.nbytes))
        return out

    def load(self, tensors):
        for t, l, a in tensors:
            self.set_weight(t, l, a)
        return self

    def init_synthetic(self, seed: int):
        self._ck(lib().asd_init_synthetic(self._h, seed))
        return self

    def load_weights_file(self, path: str):
        self._ck(lib().asd_load_weights_file(self._h, path.encode()))
        return self

    # ---- cache
    def set_page_table(self, table):
        t = np.ascontiguousarray(table, dtype=np.int32)
        self._ck(lib().asd_set_page_table(self._h, t.ctypes.data, t.size))

    def get_kv(self, layer: int, pos0: int, n: int):
        """(K, V) of positions pos0 .. pos0+n-1 of one layer: float32 [n, n_kv_heads, head_dim], the stored values widened."""
        k = np.empty((n, self.cfg.n_kv_heads, self.cfg.head_dim), dtype=np.float32)
        v = np.empty_like(k)
        self._ck(lib().asd_get_kv(self._h, layer, pos0, n, k.ctypes.data, v.ctypes.data))
        return k, v

    def kv_cache(self, layer: int):
        """(KVCache over the engine's own pages of one layer, its page table [1, pages]): asd_kv_view.  Work on them belongs on
        the engine's stream, and they live as long as the engine."""
        s, b = KvShape(), KvBatch()
        self._ck(_kv_lib().asd_kv_view(self._h, layer, s, b))
        each = kv_page_bytes(s.n_heads, s.n_kv_heads, s.head_dim, s.page_tokens, s.dtype, s.kv_dtype)
        part = lambda at, n: self.arena[at - self.arena.data_ptr():][:n]
        table = part(b.page_table, 4 * b.n_pages).view(self._torch.int32).view(1, b.n_pages)
        return KVCache(part(b.pages, each * b.n_pages), s.n_heads, s.n_kv_heads, s.head_dim, s.page_tokens, s.dtype, s.kv_dtype), table

    def park(self, caches, page_table) -> int:
        """Copy the engine's sequence (positions 0 .. kv_len-1) into other pages, one KVCache per layer, 8-bit ones say, with the page table
        [1, pages] of its place there (int32, on the device); returns its length.  Runs on the engine's stream, behind the current one's work,
        and has ended when the call returns."""
        n, target = self.kv_len, self._layers(caches, page_table)
        if n:
            self._move(n, [self.kv_cache(l) for l in range(self.cfg.n_layers)], target)
        return n

    def resume(self, caches, page_table, n: int):
        """Put a sequence of n tokens that park() has copied back into the engine: the next pass starts at position n.  If the copy fails
        (a page or a length out of range), the engine holds no sequence."""
        if n < 0 or n > self.cfg.max_seq:
            raise AsdError(E_INVAL, f"length {n} outside the cache capacity {self.cfg.max_seq}")
        source = self._layers(caches, page_table)
        self._ck(_kv_lib().asd_set_kv_len(self._h, 0))
        if n:
            self._move(n, source, [self.kv_cache(l) for l in range(self.cfg.n_layers)])
        self._ck(_kv_lib().asd_set_kv_len(self._h, n))

    def _layers(self, caches, page_table):
        if len(caches) != self.cfg.n_layers:
            raise AsdError(E_INVAL, f"one cache for each of the {self.cfg.n_layers} layers")
        return [(c, page_table) for c in caches]

    def _move(self, n: int, source, target):
        """Rows 0 .. n-1 of every layer out of `source` into `target`: (KVCache, page table) pairs."""
        torch = self._torch
        self.stream.wait_stream(torch.cuda.current_stream(self.device))
        with torch.cuda.stream(self.stream):
            rows, length = torch.tensor([0, n], dtype=torch.int32, device=self.device), torch.tensor([n], dtype=torch.int32, device=self.device)
            for (a, a_table), (b, b_table) in zip(source, target):
                both = [KVBatch(t, rows, length, n, n, n) for t in (a_table, b_table)]
                k, v = a.read(both[0])
                both[0].check()                          # (what could not be read is not written either)
                b.append(both[1], None, k, v)
                both[1].check()

    def reset(self):
        self._ck(lib().asd_reset(self._h))

    def truncate(self, n: int):
        self._ck(lib().asd_truncate(self._h, n))

    @property
    def kv_len(self) -> int:
        return int(lib().asd_kv_len(self._h))

    # ---- passes
    def forward(self, tokens, pos0: int, skip=None, commit: bool = True, want_logits: bool = True):
        tok = np.ascontiguousarray(tokens, dtype=np.int32)
        n = tok.size
        logits = np.empty((n, self.cfg.vocab), dtype=np.float32) if want_logits else None
        cos = np.empty(self.L2, dtype=np.float32)
        cos_rows = np.empty((n, self.L2), dtype=np.float32)
        am = np.empty(n, dtype=np.int32)
        sk = None if skip is None else np.ascontiguousarray(skip, dtype=np.uint8)
        self._ck(lib().asd_forward(self._h, tok.ctypes.data, n, pos0, _ptr(sk), int(commit), _ptr(logits),
                                   cos.ctypes.data, cos_rows.ctypes.data, am.ctypes.data))
        return {"logits": logits, "cos": cos, "cos_rows": cos_rows, "argmax": am}

    def forward_noalloc(self, d_tokens, pos0: int, skip=None, commit: bool = True, d_logits=None, d_cos=None, d_argmax=None):
        """asd_forward_noalloc: tokens and outputs are device tensors (int32 [n], float32 [n, V], float32 [2L], int32 [n]);
        enqueues on the engine's stream and returns without synchronising."""
        sk = None if skip is None else np.ascontiguousarray(skip, dtype=np.uint8)
        ptr = lambda t: None if t is None else t.data_ptr()
        self._ck(lib().asd_forward_noalloc(self._h, d_tokens.data_ptr(), d_tokens.numel(), pos0, _ptr(sk), int(commit),
                                           ptr(d_logits), ptr(d_cos), ptr(d_argmax)))

    def check(self):
        """Synchronise the engine's stream and raise if a kernel flagged an error since the last pass started."""
        self._ck(lib().asd_check(self._h))

    def prefill(self, tokens, want_logits: bool = False, chunked: bool = False):
        tok = np.ascontiguousarray(tokens, dtype=np.int32)
        first = ctypes.c_int32()
        cos = np.empty(self.L2, dtype=np.float32)
        lg = np.empty(self.cfg.vocab, dtype=np.float32) if want_logits else None
        fn = lib().asd_prefill_chunked if chunked else lib().asd_prefill
        self._ck(fn(self._h, tok.ctypes.data, tok.size, ctypes.byref(first), cos.ctypes.data, _ptr(lg)))
        return int(first.value), cos, lg

    @staticmethod
    def _params(draft_len, alpha=0.985, m=3, n=2, use_cs=True, fixed_mask=None, use_graphs=True, refresh=False,
                alpha_mlp=0.0, use_cs_mlp=False, exit_mode=0, gamma0=0.0, ar0=1.0, ar_target=0.9, eps=0.01, beta1=0.5,
                beta2=0.9, temperature=0.0, seed=0, sample_index0=0):
        fm = None if fixed_mask is None else np.ascontiguousarray(fixed_mask, dtype=np.uint8)
        mode = 1 if fm is not None else (2 if refresh else 0)
        gp = GenParams(alpha, m, n, int(use_cs), draft_len, mode, _ptr(fm), int(use_graphs), alpha_mlp, int(use_cs_mlp),
                       exit_mode, gamma0, ar0, ar_target, eps, beta1, beta2, temperature, seed, sample_index0)
        return gp, fm

    def decode(self, last_token: int, n_more: int, draft_len: int, **kw):
        """Speculative decode from the current cache; kw: alpha, m, n, use_cs, fixed_mask, use_graphs, refresh
        (mask rebuilt from the running ACS), alpha_mlp / use_cs_mlp, exit_mode, gamma0, ar0, ar_target, eps, beta1, beta2,
        temperature (> 0: sampled decoding by speculative sampling), seed, sample_index0."""
        gp, fm = self._params(draft_len, **kw)
        out = np.empty(n_more, dtype=np.int32)
        st = GenStats()
        mask = np.zeros(self.L2, dtype=np.uint8)
        self._ck(lib().asd_decode(self._h, last_token, n_more, ctypes.byref(gp), out.ctypes.data, ctypes.byref(st),
                                  mask.ctypes.data))
        return out, self._stats(st), mask

    def generate(self, prompt, n_new: int, draft_len: int, **kw):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        gp, fm = self._params(draft_len, **kw)
        out = np.empty(n_new, dtype=np.int32)
        st = GenStats()
        mask = np.zeros(self.L2, dtype=np.uint8)
        self._ck(lib().asd_generate(self._h, p.ctypes.data, p.size, n_new, ctypes.byref(gp), out.ctypes.data,
                                    ctypes.byref(st), mask.ctypes.data))
        return out, self._stats(st), mask

    def spec_sample(self, q_logits, p_logits, temperature: float, seed: int, index0: int = 0):
        """The sampling kernels on given logits: q [kk, V] draft, p [kk+1, V] full model; returns (drafts, accepted, next)."""
        p = np.ascontiguousarray(p_logits, dtype=np.float32)
        kk = p.shape[0] - 1
        q = np.ascontiguousarray(q_logits, dtype=np.float32).reshape(kk, p.shape[1]) if kk else None
        drafts = np.zeros(max(kk, 1), dtype=np.int32)
        a, nxt = ctypes.c_int32(), ctypes.c_int32()
        self._ck(lib().asd_spec_sample(self._h, _ptr(q), p.ctypes.data, kk, temperature, seed, index0, drafts.ctypes.data,
                                       ctypes.byref(a), ctypes.byref(nxt)))
        return drafts[:kk], int(a.value), int(nxt.value)

    @staticmethod
    def _stats(st: GenStats) -> dict:
        return {k: getattr(st, k) for k in ("cycles", "drafted", "accepted", "emitted", "ms_prefill", "ms_decode",
                                            "mask_changes", "gamma", "ar", "ms_draft", "ms_verify", "ms_other",
                                            "bytes_draft", "bytes_verify")}

    # ---- measurement
    def time_pass(self, n_rows: int, skip=None, reps: int = 20, use_graph: bool = True):
        sk = None if skip is None else np.ascontiguousarray(skip, dtype=np.uint8)
        ms, by = ctypes.c_double(), ctypes.c_double()
        self._ck(lib().asd_time_pass(self._h, n_rows, _ptr(sk), reps, int(use_graph), ctypes.byref(ms), ctypes.byref(by)))
        return ms.value, by.value

    def profile_forward(self, n_rows: int, skip=None) -> dict:
        sk = None if skip is None else np.ascontiguousarray(skip, dtype=np.uint8)
        kt = KernelTimes()
        self._ck(lib().asd_profile_forward(self._h, n_rows, _ptr(sk), ctypes.byref(kt)))
        out = {name: {"ms": kt.ms[i], "launches": kt.launches[i], "bytes": kt.bytes[i]}
               for i, name in enumerate(KERNEL_CLASSES)}
        out["ms_total"] = kt.ms_total
        return out

    def profile_prefill(self, tokens) -> dict:
        """Per-class GPU time of the prompt pass in blocks (event pair around every launch); resets the cache."""
        tok = np.ascontiguousarray(tokens, dtype=np.int32)
        pt = PrefillTimes()
        self._ck(lib().asd_profile_prefill(self._h, tok.ctypes.data, tok.size, ctypes.byref(pt)))
        out = {name: {"ms": pt.ms[i], "launches": pt.launches[i], "flops": pt.flops[i]} for i, name in enumerate(PREFILL_CLASSES)}
        out["ms_total"] = pt.ms_total
        return out

    def time_step_class(self, name: str, n_rows: int = 1, reps: int = 10):
        """(average microseconds per launch, algorithmic bytes per launch) of one kernel class launched back to back."""
        us, by = ctypes.c_double(), ctypes.c_double()
        self._ck(lib().asd_time_step_class(self._h, KERNEL_CLASSES.index(name), n_rows, reps, ctypes.byref(us), ctypes.byref(by)))
        return us.value, by.value

    def copy_bench(self, nbytes: int, reps: int = 10) -> float:
        ms = ctypes.c_double()
        self._ck(lib().asd_copy_bench(self._h, nbytes, reps, ctypes.byref(ms)))
        return ms.value


# ---------------------------------------------------------------- operators over a paged cache of several sequences
def _kv_ck(rc: int):
    if rc:
        raise AsdError(rc, lib().asd_last_error(None).decode())


def _fits(**numbers):
    """The library takes these in 32 bits (ctypes would keep the low ones and say nothing)."""
    for name, n in numbers.items():
        if not -1 << 31 <= n < 1 << 31:
            raise AsdError(E_INVAL, f"{name} = {n} does not fit 32 bits")


def kv_page_bytes(n_heads: int, n_kv_heads: int, head_dim: int, page_tokens: int, dtype: int = DT_BF16, kv_dtype: int = DT_FP8) -> int:
    """Bytes of one page of a KVCache (asd_kv_page_bytes)."""
    _fits(n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, page_tokens=page_tokens, dtype=dtype, kv_dtype=kv_dtype)
    n = int(_kv_lib().asd_kv_page_bytes(ctypes.byref(KvShape(n_heads, n_kv_heads, head_dim, page_tokens, dtype, kv_dtype))))
    if n == 0:
        raise AsdError(E_INVAL, "invalid cache shape")
    return n


def _on_device(device, call):
    """call(stream) with `device` as the current one and its current stream, as the library's launches expect them."""
    import torch
    index, before = device.index, torch._C._cuda_getDevice()
    if before == index:
        return call(torch._C._cuda_getCurrentRawStream(index))
    torch.cuda.set_device(index)
    try:
        return call(torch._C._cuda_getCurrentRawStream(index))
    finally:
        torch.cuda.set_device(before)


class _Fixed:
    """Attributes are set once: calls pass addresses and bounds that were taken when the object was made."""

    def __setattr__(self, name, value):
        if name in self.__dict__:
            raise AttributeError(f"{name} does not change: make a new {type(self).__name__}")
        self.__dict__[name] = value


class KVBatch(_Fixed):
    """New rows of several sequences (asd_kv_batch): int32 device tensors page_table [n_seqs, pages], row_start [n_seqs + 1],
    kv_len [n_seqs] (tokens with the new ones), and the bounds that hold for them: rows of the row buffers, most new rows
    and most tokens of a sequence.  The tensors are read when a call's kernels run: update them in place between calls.
    status: an int32 word on the device that kernels set bits of where the arrays held something out of range; check() reads it.  The word is cleared, and read, on the
    current stream: calls on another one wait for it, and check() comes after them."""

    def __init__(self, page_table, row_start, kv_len, n_rows: int, max_new: int, max_len: int):
        import torch
        _fits(n_rows=n_rows, max_new=max_new, max_len=max_len)
        for name, t, dims in (("page_table", page_table, 2), ("row_start", row_start, 1), ("kv_len", kv_len, 1)):
            if t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous() or t.device != kv_len.device:
                raise AsdError(E_INVAL, f"{name} must be a contiguous int32 tensor of {dims} dimension(s) on the batch's device")
        if kv_len.device.type != "cuda":
            raise AsdError(E_INVAL, "the batch's tensors must be on the GPU")
        n = kv_len.numel()
        if row_start.numel() != n + 1 or page_table.shape[0] != n:
            raise AsdError(E_INVAL, "page_table, row_start and kv_len must be of n_seqs, n_seqs + 1 and n_seqs sequences")
        self.page_table, self.row_start, self.kv_len, self.device = page_table, row_start, kv_len, kv_len.device
        self.n_rows, self.max_new, self.max_len = n_rows, max_new, max_len
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._c = KvBatch(None, page_table.data_ptr(), row_start.data_ptr(), kv_len.data_ptr(), self.status.data_ptr(), 0,
                          page_table.shape[1], n, n_rows, max_new, max_len)
        self._workspace = {}                            # bytes of an attend call, by cache shape: the bounds do not change

    def check(self):
        """Synchronise and raise if a kernel found the arrays out of range since the last check."""
        bits = int(self.status.item())
        if bits:
            self.status.zero_()
            names = [n for b, n in ((1, "rows or lengths"), (2, "pages"), (4, "positions past the rotary table")) if bits & b]
            raise AsdError(E_INVAL, "batch out of range: " + ", ".join(names))


class KVCache(_Fixed):
    """Pages of a paged cache for several sequences: pages is a uint8 device tensor of n_pages * kv_page_bytes(...) bytes, which the
    caller owns.  The calls enqueue on the current stream of its device and return without synchronising; asd.h has
    the layout and what each call does."""

    def __init__(self, pages, n_heads: int, n_kv_heads: int, head_dim: int, page_tokens: int, dtype: int = DT_BF16, kv_dtype: int = DT_FP8):
        import torch
        each = kv_page_bytes(n_heads, n_kv_heads, head_dim, page_tokens, dtype, kv_dtype)
        if pages.dtype != torch.uint8 or not pages.is_contiguous() or pages.device.type != "cuda" or pages.numel() == 0 or pages.numel() % each:
            raise AsdError(E_INVAL, f"pages must be a contiguous uint8 tensor on the GPU, a multiple of {each} bytes")
        self.pages, self.device, self.n_pages = pages, pages.device, pages.numel() // each
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.torch_dtype = torch.bfloat16 if dtype == DT_BF16 else torch.float32
        self._shape = KvShape(n_heads, n_kv_heads, head_dim, page_tokens, dtype, kv_dtype)
        self._torch, self._lib, self._scale, self._index = torch, _kv_lib(), head_dim ** -0.5, pages.device.index
        self._key, self._s = (n_heads, n_kv_heads, head_dim, page_tokens, dtype, kv_dtype), ctypes.addressof(self._shape)

    def _batch(self, batch: KVBatch):
        """The batch's structure with this cache's pages (each call has its own: calls of several threads may share a batch)."""
        if batch.device != self.device:
            raise AsdError(E_INVAL, "the batch is on another device than the pages")
        b = KvBatch.from_buffer_copy(batch._c)
        b.pages, b.n_pages = self.pages.data_ptr(), self.n_pages
        return b

    def _rows(self, name: str, t, batch: KVBatch, heads: int):
        """(pointer, row stride) of a buffer of rows [>= n_rows, heads, head_dim]; heads packed."""
        if t.dtype is not self.torch_dtype or t.get_device() != self._index:
            raise AsdError(E_INVAL, f"{name} must be {self.torch_dtype} on {self.device}")
        shape, h = t.shape, self.head_dim
        if len(shape) != 3 or shape[0] < batch.n_rows or shape[1] != heads or shape[2] != h:
            raise AsdError(E_INVAL, f"{name} must be [{batch.n_rows}, {heads}, {h}]")
        row, head, one = t.stride()
        if one != 1 or (heads > 1 and head != h):
            raise AsdError(E_INVAL, f"{name}: the heads of a row must lie packed")
        return t.data_ptr(), row if batch.n_rows > 1 else max(row, heads * h)

    def _floats(self, name: str, t, *shape):
        """Pointer of a float32 tensor of `shape` (None first: any number)."""
        if shape[0] is None:
            fits = t.dim() == len(shape) and t.shape[1:] == shape[1:]
        else:
            fits = t.shape == shape
        if not fits or t.dtype is not self._torch.float32 or t.get_device() != self._index or not t.is_contiguous():
            raise AsdError(E_INVAL, f"{name} must be a contiguous float32 tensor [{', '.join('any' if n is None else str(n) for n in shape)}] on {self.device}")
        return t.data_ptr()

    def _call(self, function, *args):
        """function(*args, stream) with the cache's device as the current one and its current stream, as the library's launches expect them."""
        before = self._torch._C._cuda_getDevice()
        if before == self._index:
            rc = function(*args, self._torch._C._cuda_getCurrentRawStream(before))
        else:
            rc = _on_device(self.device, lambda stream: function(*args, stream))
        if rc:
            _kv_ck(rc)

    def append(self, batch: KVBatch, q, k, v, q_out=None, rope=None, rot_dim: int = 0, interleaved: bool = False, q_gain=None, k_gain=None,
               eps: float = 1e-5):
        """Write the batch's new rows into the pages (asd_kv_append): q [n_rows, n_heads, head_dim] or None, k and v
        [n_rows, n_kv_heads, head_dim]; rope [positions, rot_dim / 2, 2] as rope_table makes it, gains [head_dim].  Returns the
        prepared queries (q_out, which may be q; a new tensor if it is not given)."""
        if not 0 <= rot_dim <= self.head_dim:
            raise AsdError(E_INVAL, f"rot_dim {rot_dim} of head_dim {self.head_dim}")
        bound, prep = self._batch(batch), KvPrep(None, None, eps, None, 0, rot_dim, interleaved)
        if q is None and q_out is not None:
            raise AsdError(E_INVAL, "q_out without q")
        if q is not None and q_out is None:
            q_out = self._torch.empty((q.shape[0], self.n_heads, self.head_dim), dtype=self.torch_dtype, device=self.device)
        if rope is not None:
            prep.rope, prep.rope_positions = self._floats("rope", rope, None, rot_dim // 2, 2), rope.shape[0]
        if q_gain is not None:
            prep.q_gain = self._floats("q_gain", q_gain, self.head_dim)
        if k_gain is not None:
            prep.k_gain = self._floats("k_gain", k_gain, self.head_dim)
        qp = self._rows("q", q, batch, self.n_heads) if q is not None else (None, 0)
        op = self._rows("q_out", q_out, batch, self.n_heads) if q is not None else (None, 0)
        kp, vp = self._rows("k", k, batch, self.n_kv_heads), self._rows("v", v, batch, self.n_kv_heads)
        self._call(self._lib.asd_kv_append, self._s, ctypes.addressof(bound), ctypes.addressof(prep), *qp, *kp, *vp, *op)
        return q_out

    def attend(self, batch: KVBatch, q, out=None, scale: float | None = None, workspace=None):
        """Causal attention of the batch's new rows over their sequences' pages (asd_kv_attend); q and out [n_rows, n_heads, head_dim],
        scale 1 / sqrt(head_dim) by default.  workspace: a uint8 tensor of attend_workspace(batch) bytes (by default one of the call's own)."""
        bound = self._batch(batch)
        if out is None:
            out = self._torch.empty((q.shape[0], self.n_heads, self.head_dim), dtype=self.torch_dtype, device=self.device)
        qp, op = self._rows("q", q, batch, self.n_heads), self._rows("out", out, batch, self.n_heads)
        need = batch._workspace.get(self._key)
        if need is None:
            need = batch._workspace[self._key] = self._lib.asd_kv_attend_workspace(self._s, ctypes.addressof(bound))
        if workspace is None:
            wp, wn = None, 0
            if need:
                workspace = self._torch.empty(need, dtype=self._torch.uint8, device=self.device)
                wp, wn = workspace.data_ptr(), need
        elif workspace.device != self.device or workspace.dtype != self._torch.uint8 or not workspace.is_contiguous():
            raise AsdError(E_INVAL, f"workspace must be a contiguous uint8 tensor on {self.device}")
        else:
            wp, wn = workspace.data_ptr(), workspace.numel()
        if scale is None:
            scale = self._scale
        self._call(self._lib.asd_kv_attend, self._s, ctypes.addressof(bound), *qp, *op, scale, wp, wn)
        return out

    def attend_workspace(self, batch: KVBatch) -> int:
        """Bytes of workspace that attend() of a batch with these bounds needs."""
        bound = self._batch(batch)
        return int(self._lib.asd_kv_attend_workspace(self._s, ctypes.addressof(bound)))

    def read(self, batch: KVBatch, k_out=None, v_out=None):
        """The batch's rows out of the pages as values (asd_kv_read): (k, v) [n_rows, n_kv_heads, head_dim]; new tensors where none is given."""
        bound = self._batch(batch)
        if k_out is None:
            k_out = self._torch.empty((batch.n_rows, self.n_kv_heads, self.head_dim), dtype=self.torch_dtype, device=self.device)
        if v_out is None:
            v_out = self._torch.empty_like(k_out, memory_format=self._torch.contiguous_format)
        kp, vp = self._rows("k_out", k_out, batch, self.n_kv_heads), self._rows("v_out", v_out, batch, self.n_kv_heads)
        self._call(self._lib.asd_kv_read, self._s, ctypes.addressof(bound), *kp, *vp)
        return k_out, v_out


ROPE_PLAIN, ROPE_LINEAR, ROPE_BANDS, ROPE_RAMP = 0, 1, 2, 3


def rope_table(rot_dim: int, positions: int, theta: float = 10000.0, kind: int = ROPE_PLAIN, factor: float = 1.0, low: float = 1.0, high: float = 32.0,
               trained: float = 4096.0, gain: float = 1.0, device: str = "cuda:0"):
    """Rotary table [positions, rot_dim / 2, 2] for KVCache.append (asd_rope_table), enqueued on the device's current stream."""
    import torch
    _fits(rot_dim=rot_dim, positions=positions, kind=kind)
    device = torch.device(device)
    if device.type != "cuda":
        raise AsdError(E_INVAL, "the table is made on the GPU")
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    if positions < 1 or rot_dim < 2:
        raise AsdError(E_INVAL, "asd_rope_table: positions and rot_dim must be positive")
    out = torch.empty((positions, rot_dim // 2, 2), dtype=torch.float32, device=device)
    rope = Rope(kind, rot_dim, theta, factor, low, high, trained, gain)
    _kv_ck(_on_device(device, lambda stream: _kv_lib().asd_rope_table(rope, positions, out.data_ptr(), stream)))
    return out
