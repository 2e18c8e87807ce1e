"""ctypes binding of libllmcad (the C ABI in include/llmcad.h).

Argument marshalling only: every step of a pass runs in the library's HIP
kernels.  Device buffers are torch tensors on a ROCm device (torch provides
memory and streams); tree arrays are host int32 arrays.  Importing this module
fails loudly if the library has not been built.
"""

import ctypes
import functools
import os

import numpy as np
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libllmcad.so")

OK = 0
EARG = -1
ETREE = -2
ECAPACITY = -3
ESHAPE = -4
EHIP = -5
EWORKSPACE = -6
MAX_NODES = 128

SYMBOLS = (
    "llmcad_check_config",
    "llmcad_packed_bytes",
    "llmcad_pack_globals",
    "llmcad_pack_layer",
    "llmcad_pack_layer_q4",
    "llmcad_workspace_bytes",
    "llmcad_workspace_init",
    "llmcad_verify_tree",
    "llmcad_verify_tree_noalloc",
    "llmcad_prefill",
    "llmcad_commit_path",
    "llmcad_extend_tree",
    "llmcad_extend_tree_candidates",
    "llmcad_batch_plan_bytes",
    "llmcad_batch_plan_region",
    "llmcad_batch_plan",
    "llmcad_batch_store",
    "llmcad_batch_workspace_bytes",
    "llmcad_batch_attention",
    "llmcad_batch_commit",
    "llmcad_token_scores_workspace_bytes",
    "llmcad_token_scores",
    "llmcad_status_string",
    "llmcad_workspace_region",
    "llmcad_split_plan",
    "llmcad_timing_enable",
    "llmcad_timing_read",
)

KERNEL_PASS = 0  # the whole pass is one persistent launch


class LlmcadConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32),
        ("d_model", ctypes.c_int32),
        ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("d_ffn", ctypes.c_int32),
        ("vocab", ctypes.c_int32),
        ("rms_eps", ctypes.c_float),
        ("rope_theta", ctypes.c_float),
        ("weight_bits", ctypes.c_int32),
    ]


class LlmcadLayerWeights(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in
                ("attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gate_up", "w_down")]


class LlmcadQ4Matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class LlmcadQ4LayerWeights(ctypes.Structure):
    _fields_ = [("attn_norm", ctypes.c_void_p), ("w_qkv", LlmcadQ4Matrix), ("w_o", LlmcadQ4Matrix),
                ("ffn_norm", ctypes.c_void_p), ("w_gate_up", LlmcadQ4Matrix), ("w_down", LlmcadQ4Matrix)]


Q4_GROUP = 128  # inputs per scale group of a 4-bit matrix


class LlmcadError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


# Device pass status (workspace region 5), written by the pass kernel.
PASS_OK = 0
PASS_WAIT_TIMEOUT = 1   # a wait of the single-launch pass ran out of its bounded spin
PASS_BAD_PARAMS = 3     # the kernel did not find its parameter block; it did nothing
_PASS_TEXT = {PASS_WAIT_TIMEOUT: "a grid or join wait ran out of its bounded spin (outputs invalid)",
              PASS_BAD_PARAMS: "the kernel did not find its parameter block (nothing computed)"}


class LlmcadPassError(RuntimeError):
    """A pass ended with a non-zero device status: its outputs are invalid."""

    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: device pass status {status}: {_PASS_TEXT.get(status, 'unknown')}")


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2309_04255_amd.build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(_LIB_PATH)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    CFG = ctypes.POINTER(LlmcadConfig)
    I32P = ctypes.POINTER(ctypes.c_int32)
    sig = {
        "llmcad_check_config": (ctypes.c_int, [CFG]),
        "llmcad_packed_bytes": (SZ, [CFG]),
        "llmcad_pack_globals": (ctypes.c_int, [CFG, P, P, P, P, SZ, P]),
        "llmcad_pack_layer": (ctypes.c_int, [CFG, I32, ctypes.POINTER(LlmcadLayerWeights), P, SZ, P]),
        "llmcad_pack_layer_q4": (ctypes.c_int, [CFG, I32, ctypes.POINTER(LlmcadQ4LayerWeights), P, SZ, P]),
        "llmcad_workspace_bytes": (SZ, [CFG, I32]),
        "llmcad_workspace_init": (ctypes.c_int, [CFG, I32, P, SZ, P]),
        "llmcad_verify_tree": (ctypes.c_int, [CFG, P, P, P, I32, I32, I32P, I32P, I32, P, P, P, P,
                                              P, SZ, P]),
        "llmcad_verify_tree_noalloc": (ctypes.c_int, [CFG, P, P, P, I32, I32, I32P, I32P, I32, P, P, P, P,
                                                      P, P]),
        "llmcad_prefill": (ctypes.c_int, [CFG, P, P, P, I32, I32P, I32, I32, P, P, SZ, P]),
        "llmcad_commit_path": (ctypes.c_int, [CFG, P, P, I32, I32, P, P, I32, P]),
        "llmcad_extend_tree": (ctypes.c_int, [CFG, P, P, P, I32, I32, I32P, I32P, I32, I32, P, P, SZ, P]),
        "llmcad_extend_tree_candidates": (ctypes.c_int, [CFG, P, P, P, I32, I32, I32P, I32P, I32, I32, ctypes.c_float,
                                                         P, P, P, SZ, P]),
        "llmcad_batch_plan_bytes": (SZ, [CFG, I32, I32]),
        "llmcad_batch_plan_region": (ctypes.c_int, [CFG, I32, I32, I32, ctypes.POINTER(SZ), ctypes.POINTER(SZ)]),
        "llmcad_batch_plan": (ctypes.c_int, [CFG, I32, I32, P, P, P, I32, P, I32, P, I32, I32, P, SZ, P]),
        "llmcad_batch_store": (ctypes.c_int, [CFG, I32, I32, P, I64, P, I64, P, I64, P, P, P, I32, P, SZ, I32, I32, P]),
        "llmcad_batch_workspace_bytes": (SZ, [CFG, I32, I32, I32]),
        "llmcad_batch_attention": (ctypes.c_int, [CFG, I32, I32, P, I64, P, P, I32, I32, P, P, I32, P, I32, P, SZ, I32,
                                                  I32, P, P, SZ, P]),
        "llmcad_batch_commit": (ctypes.c_int, [CFG, I32, P, P, I32, P, SZ, I32, I32, P, P, P]),
        "llmcad_token_scores_workspace_bytes": (SZ, [I32, I32, I32]),
        "llmcad_token_scores": (ctypes.c_int, [P, I32, I64, I32, I32, P, P, I32, P, P, P, I32, P, P, P, SZ, P]),
        "llmcad_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "llmcad_workspace_region": (ctypes.c_int, [CFG, I32, I32, ctypes.POINTER(SZ),
                                                   ctypes.POINTER(SZ)]),
        "llmcad_split_plan": (ctypes.c_int, [CFG, I32, I32P]),
        "llmcad_timing_enable": (ctypes.c_int, [I32, I32]),
        "llmcad_timing_read": (ctypes.c_int, [I32, ctypes.POINTER(ctypes.c_double), I32P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()


def lib():
    return _lib


def status_string(status: int) -> str:
    return _lib.llmcad_status_string(int(status)).decode()


def make_config(shape) -> LlmcadConfig:
    """From any object with n_layers, d_model, n_heads, head_dim, d_ffn, vocab, rms_eps, rope_theta
    (and optionally weight_bits: 16, the default, or 4)."""
    return LlmcadConfig(shape.n_layers, shape.d_model, shape.n_heads, shape.head_dim, shape.d_ffn,
                        shape.vocab, float(shape.rms_eps), float(shape.rope_theta),
                        int(getattr(shape, "weight_bits", 16)))


def _ptr(t):
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _i32(a):
    a = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _check(rc, what):
    if rc != OK:
        raise LlmcadError(rc, what)


def check_config(cfg: LlmcadConfig) -> int:
    return _lib.llmcad_check_config(ctypes.byref(cfg))


def packed_bytes(cfg: LlmcadConfig) -> int:
    return _lib.llmcad_packed_bytes(ctypes.byref(cfg))


def workspace_bytes(cfg: LlmcadConfig, max_n: int) -> int:
    return _lib.llmcad_workspace_bytes(ctypes.byref(cfg), int(max_n))


def pack_globals(cfg, tok_embed, final_norm, lm_head, packed, stream=None):
    _check(_lib.llmcad_pack_globals(ctypes.byref(cfg), _ptr(tok_embed), _ptr(final_norm),
                                    _ptr(lm_head), _ptr(packed), packed.numel() * packed.element_size(),
                                    _stream(stream)), "llmcad_pack_globals")


def pack_layer(cfg, layer: int, w: dict, packed, stream=None):
    src = LlmcadLayerWeights(*(w[k].data_ptr() for k in
                               ("attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gate_up", "w_down")))
    _check(_lib.llmcad_pack_layer(ctypes.byref(cfg), int(layer), ctypes.byref(src), _ptr(packed),
                                  packed.numel() * packed.element_size(), _stream(stream)),
           "llmcad_pack_layer")


def pack_layer_q4(cfg, layer: int, w: dict, packed, stream=None):
    """w: attn_norm, ffn_norm (bf16 [d]) and, per matrix m in w_qkv, w_o, w_gate_up,
    w_down, a pair (codes uint8 [out][in/2], scales bf16 [out][in/128]) on the device."""
    def mat(k):
        codes, scales = w[k]
        return LlmcadQ4Matrix(codes.data_ptr(), scales.data_ptr())

    src = LlmcadQ4LayerWeights(w["attn_norm"].data_ptr(), mat("w_qkv"), mat("w_o"), w["ffn_norm"].data_ptr(),
                               mat("w_gate_up"), mat("w_down"))
    _check(_lib.llmcad_pack_layer_q4(ctypes.byref(cfg), int(layer), ctypes.byref(src), _ptr(packed),
                                     packed.numel() * packed.element_size(), _stream(stream)),
           "llmcad_pack_layer_q4")


def workspace_init(cfg, max_n: int, workspace, stream=None):
    _check(_lib.llmcad_workspace_init(ctypes.byref(cfg), int(max_n), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream(stream)),
           "llmcad_workspace_init")


def verify_tree(cfg, packed, k_cache, v_cache, prefix_len: int, tree_tokens, parent, logits, path,
                accept_len, next_token, workspace, stream=None, raise_on_error=True) -> int:
    """Enqueue one verification pass; returns the status (raises on error by default)."""
    tok, tok_p = _i32(tree_tokens)
    par, par_p = _i32(parent)
    n = len(tok)
    if len(par) != n:
        raise ValueError("tree_tokens and parent differ in length")
    cap = k_cache.shape[-2]
    rc = _lib.llmcad_verify_tree(
        ctypes.byref(cfg), _ptr(packed), _ptr(k_cache), _ptr(v_cache), int(cap), int(prefix_len),
        tok_p, par_p, int(n), _ptr(logits), _ptr(path), _ptr(accept_len), _ptr(next_token),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    if raise_on_error:
        _check(rc, "llmcad_verify_tree")
    return rc


SCRATCH_BYTES = 96 << 20  # LLMCAD_SCRATCH_BYTES


def verify_tree_noalloc(cfg, packed, k_cache, v_cache, prefix_len: int, tree_tokens, parent, logits, path,
                        accept_len, next_token, status=None, stream=None, raise_on_error=True) -> int:
    """Enqueue one verification pass on the library's own scratch buffer (no
    workspace argument, no allocation); `status` (device int32 [1] or None)
    receives the pass's device status."""
    tok, tok_p = _i32(tree_tokens)
    par, par_p = _i32(parent)
    n = len(tok)
    if len(par) != n:
        raise ValueError("tree_tokens and parent differ in length")
    cap = k_cache.shape[-2]
    rc = _lib.llmcad_verify_tree_noalloc(
        ctypes.byref(cfg), _ptr(packed), _ptr(k_cache), _ptr(v_cache), int(cap), int(prefix_len),
        tok_p, par_p, int(n), _ptr(logits), _ptr(path), _ptr(accept_len), _ptr(next_token), _ptr(status),
        _stream(stream))
    if raise_on_error:
        _check(rc, "llmcad_verify_tree_noalloc")
    return rc


def prefill(cfg, packed, k_cache, v_cache, tokens, start_pos: int, last_logits, workspace,
            stream=None, raise_on_error=True) -> int:
    tok, tok_p = _i32(tokens)
    cap = k_cache.shape[-2]
    rc = _lib.llmcad_prefill(
        ctypes.byref(cfg), _ptr(packed), _ptr(k_cache), _ptr(v_cache), int(cap), tok_p, int(len(tok)),
        int(start_pos), _ptr(last_logits), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream))
    if raise_on_error:
        _check(rc, "llmcad_prefill")
    return rc


def extend_tree(cfg, packed, k_cache, v_cache, prefix_len: int, tree_tokens, parent, first: int, logits,
                workspace, stream=None, raise_on_error=True) -> int:
    """Tree-decoder step: the forward of nodes [first, n) of the tree (see llmcad_extend_tree)."""
    tok, tok_p = _i32(tree_tokens)
    par, par_p = _i32(parent)
    if len(par) != len(tok):
        raise ValueError("tree_tokens and parent differ in length")
    cap = k_cache.shape[-2]
    rc = _lib.llmcad_extend_tree(
        ctypes.byref(cfg), _ptr(packed), _ptr(k_cache), _ptr(v_cache), int(cap), int(prefix_len), tok_p, par_p,
        int(len(tok)), int(first), _ptr(logits), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream))
    if raise_on_error:
        _check(rc, "llmcad_extend_tree")
    return rc


CAND_MAX = 64  # LLMCAD_CAND_MAX
CAND_WORDS = 4 + 2 * CAND_MAX  # int32 words of one llmcad_candidates record


def extend_tree_candidates(cfg, packed, k_cache, v_cache, prefix_len: int, tree_tokens, parent, first: int,
                           threshold: float, logits, cand, workspace, stream=None, raise_on_error=True) -> int:
    """Tree-decoder step with candidate summaries (see llmcad_extend_tree_candidates):
    cand is a device int32 tensor of at least (n - first) x CAND_WORDS words."""
    tok, tok_p = _i32(tree_tokens)
    par, par_p = _i32(parent)
    if len(par) != len(tok):
        raise ValueError("tree_tokens and parent differ in length")
    if cand.dtype != torch.int32 or cand.numel() < (len(tok) - first) * CAND_WORDS:
        raise ValueError("cand must be an int32 device tensor of (n - first) records")
    cap = k_cache.shape[-2]
    rc = _lib.llmcad_extend_tree_candidates(
        ctypes.byref(cfg), _ptr(packed), _ptr(k_cache), _ptr(v_cache), int(cap), int(prefix_len), tok_p, par_p,
        int(len(tok)), int(first), float(threshold), _ptr(logits), _ptr(cand), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream))
    if raise_on_error:
        _check(rc, "llmcad_extend_tree_candidates")
    return rc


def parse_candidates(words):
    """One llmcad_candidates record (int32 numpy array of CAND_WORDS words) ->
    dict(count, argmax, max_logit, sum_exp, tok (list), prob (list))."""
    w = np.asarray(words, dtype=np.int32)
    f = w.view(np.float32)
    count = int(w[0])
    k = max(count, 0)
    return {"count": count, "argmax": int(w[1]), "max_logit": float(f[2]), "sum_exp": float(f[3]),
            "tok": [int(x) for x in w[4:4 + k]], "prob": [float(x) for x in f[4 + CAND_MAX:4 + CAND_MAX + k]]}


def commit_path(cfg, k_cache, v_cache, prefix_len: int, path, accept_len, n: int, stream=None,
                raise_on_error=True) -> int:
    """Rollback to the verified sequence: path/accept_len are the device outputs of the
    verification pass over n nodes at prefix_len (see llmcad_commit_path)."""
    cap = k_cache.shape[-2]
    rc = _lib.llmcad_commit_path(ctypes.byref(cfg), _ptr(k_cache), _ptr(v_cache), int(cap), int(prefix_len),
                                 _ptr(path), _ptr(accept_len), int(n), _stream(stream))
    if raise_on_error:
        _check(rc, "llmcad_commit_path")
    return rc


# ---- several requests behind one shared prefix (see the header's section)

PAGE = 64  # LLMCAD_PAGE, slots of a page
MAX_REQUESTS = 1024
TOP_MAX = 64  # LLMCAD_TOP_MAX
PLAN_OK = 0
PLAN_BAD_LENGTHS = 1
PLAN_NO_PAGES = 2
PLAN_BAD_TREE = 3
_PLAN_REGIONS = ("slot", "position", "mask", "rope", "status", "taken")


# The current stream's handle: torch.cuda.current_stream() builds an object for it, which takes a
# quarter of a small call's host time (2.7 us; 0.06 us this way).
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _on_device(what, first, *others):
    """The index of the GPU that every tensor of a call lies on (ValueError if they differ or one is on none)."""
    dev = first.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{what}: tensors on {first.device} and {t.device}")
    if dev < 0:
        raise ValueError(f"{what}: the tensors must be on a GPU")
    return dev


def _same_device(dev, stream):
    """A stream's kernels run on its own GPU: it must be the tensors'."""
    if stream is not None and stream.device.index != dev:
        raise ValueError(f"the stream is on {stream.device}, the tensors on cuda:{dev}")


def _enqueue(fn, dev, stream, args):
    """fn(*args, stream) with dev the current device (a launch goes to the current device's kernels)."""
    _same_device(dev, stream)
    if dev == torch.cuda.current_device():
        return fn(*args, _current_stream(dev) if stream is None else stream.cuda_stream)
    with torch.cuda.device(dev):
        return fn(*args, _current_stream(dev) if stream is None else stream.cuda_stream)


def _want(what, name, t, dtype, *shape):
    """t is a contiguous tensor of dtype and shape (None: any size)."""
    got = t.shape
    if t.dtype is dtype and t.is_contiguous() and \
            (got == shape or (len(got) == len(shape) and all(w is None or w == s for w, s in zip(shape, got)))):
        return
    raise ValueError(f"{what}: {name} must be a contiguous {dtype} tensor of shape "
                     f"{tuple('any' if w is None else w for w in shape)}, got {t.dtype} {tuple(got)}")


def _want_rows(what, name, t, n, heads, dh):
    """t is bf16 [n, heads, dh] whose rows are contiguous (any distance between them); returns that distance."""
    if t.dtype != torch.bfloat16 or t.shape != (n, heads, dh) or t.stride(2) != 1 or \
            (heads > 1 and t.stride(1) != dh):
        raise ValueError(f"{what}: {name} must be bfloat16 [{n}, {heads}, {dh}] with contiguous rows, "
                         f"got {t.dtype} {tuple(t.shape)}")
    return t.stride(0) if n > 1 else heads * dh


def batch_plan_bytes(cfg, n_requests: int, n_rows: int) -> int:
    return _lib.llmcad_batch_plan_bytes(ctypes.byref(cfg), int(n_requests), int(n_rows))


@functools.lru_cache(maxsize=64)
def _plan_parts(head_dim, n_requests, n_rows):
    """A plan's int32 words in pieces: (their lengths, the piece of every array)."""
    cfg = LlmcadConfig(1, head_dim, 1, head_dim, 1, 1, 1e-6, 10000.0, 16)  # (the layout depends on head_dim alone)
    off, size, spans = ctypes.c_size_t(), ctypes.c_size_t(), []
    for which in range(len(_PLAN_REGIONS)):
        _check(_lib.llmcad_batch_plan_region(ctypes.byref(cfg), n_requests, n_rows, which, ctypes.byref(off),
                                             ctypes.byref(size)), "llmcad_batch_plan_region")
        spans.append((off.value // 4, off.value // 4 + size.value // 4, which))
    lengths, piece, at = [], {}, 0
    for lo, hi, which in sorted(spans):
        lengths += [lo - at, hi - lo]
        piece[_PLAN_REGIONS[which]] = len(lengths) - 1
        at = hi
    lengths.append(batch_plan_bytes(cfg, n_requests, n_rows) // 4 - at)
    return lengths, piece


def batch_plan_views(cfg, n_requests: int, n_rows: int, plan) -> dict:
    """The arrays of a plan as views of its buffer: slot, position int32 [n_rows], mask int32
    [n_rows, 4], rope float32 [n_rows, Dh/2, 2], status int32 [n_requests], taken int32 [1]."""
    lengths, piece = _plan_parts(cfg.head_dim, n_requests, n_rows)
    words = plan.view(torch.int32)
    if words.shape[0] != sum(lengths):  # (a larger buffer)
        words = words[:sum(lengths)]
    parts = words.split(lengths)
    return {"slot": parts[piece["slot"]], "position": parts[piece["position"]],
            "mask": parts[piece["mask"]].view(n_rows, 4),
            "rope": parts[piece["rope"]].view(torch.float32).view(n_rows, cfg.head_dim // 2, 2),
            "status": parts[piece["status"]], "taken": parts[piece["taken"]]}


def batch_plan(cfg, row_start, held, parent, prefix_len: int, block_table, free_pages, n_pages: int, plan,
               n_rows: int, stream=None):
    """Build a step's plan on the device (see llmcad_batch_plan): row_start [B + 1], held [B], parent
    [n_rows] or None, block_table [B, max_pages] (updated), free_pages [n_free], all int32; plan a uint8
    tensor of batch_plan_bytes."""
    what = "batch_plan"
    dev = _on_device(what, row_start, held, parent, block_table, free_pages, plan)
    B = held.shape[0]
    _want(what, "row_start", row_start, torch.int32, B + 1)
    _want(what, "held", held, torch.int32, B)
    _want(what, "block_table", block_table, torch.int32, B, None)
    _want(what, "free_pages", free_pages, torch.int32, None)
    _want(what, "plan", plan, torch.uint8, None)
    if parent is not None:
        _want(what, "parent", parent, torch.int32, None)
        if parent.shape[0] < n_rows:
            raise ValueError("batch_plan: parent must have an entry for every row")
    _check(_enqueue(_lib.llmcad_batch_plan, dev, stream,
                    (ctypes.byref(cfg), B, int(n_rows), row_start.data_ptr(), held.data_ptr(),
                     parent.data_ptr() if parent is not None else None, int(prefix_len), block_table.data_ptr(),
                     block_table.shape[1], free_pages.data_ptr(), free_pages.shape[0], int(n_pages), plan.data_ptr(),
                     plan.shape[0])), "llmcad_batch_plan")


def _want_pages(what, cfg, n_kv_heads, k_pages, v_pages):
    n_pages = k_pages.shape[1]
    _want(what, "k_pages", k_pages, torch.bfloat16, cfg.n_layers, n_pages, n_kv_heads, PAGE, cfg.head_dim)
    _want(what, "v_pages", v_pages, torch.bfloat16, cfg.n_layers, n_pages, n_kv_heads, cfg.head_dim, PAGE)
    return n_pages


def batch_store(cfg, n_kv_heads: int, layer: int, q, k, v, q_out, k_pages, v_pages, plan, n_requests: int,
                stream=None):
    """Rotary embedding of q [N, H, Dh] (to q_out) and k [N, Hkv, Dh], and the write of k and v into the
    layer's pages at the plan's slots (see llmcad_batch_store).  q, k and v may be slices of one fused
    projection; q_out may be q."""
    what = "batch_store"
    dev = _on_device(what, q, k, v, q_out, k_pages, v_pages, plan)
    N, H, Dh = q.shape[0], cfg.n_heads, cfg.head_dim
    qs = _want_rows(what, "q", q, N, H, Dh)
    ks = _want_rows(what, "k", k, N, n_kv_heads, Dh)
    vs = _want_rows(what, "v", v, N, n_kv_heads, Dh)
    _want(what, "q_out", q_out, torch.bfloat16, N, H, Dh)
    _want(what, "plan", plan, torch.uint8, None)
    n_pages = _want_pages(what, cfg, n_kv_heads, k_pages, v_pages)
    _check(_enqueue(_lib.llmcad_batch_store, dev, stream,
                    (ctypes.byref(cfg), int(n_kv_heads), int(layer), q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
                     q_out.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), n_pages, plan.data_ptr(), plan.shape[0],
                     int(n_requests), N)), "llmcad_batch_store")


def batch_workspace_bytes(cfg, n_kv_heads: int, n_requests: int, n_rows: int) -> int:
    return _lib.llmcad_batch_workspace_bytes(ctypes.byref(cfg), int(n_kv_heads), int(n_requests), int(n_rows))


def batch_attention(cfg, n_kv_heads: int, layer: int, q, k_cache, v_cache, prefix_len: int, k_pages, v_pages,
                    block_table, plan, out, workspace, stream=None):
    """Attention of the rows q [N, H, Dh] (after the rotary embedding) to the shared prefix in slots
    [0, prefix_len) of k_cache [L, Hkv, cap, Dh] / v_cache [L, Hkv, Dh, cap] (None without a prefix), to
    their requests' pages and branches (see llmcad_batch_attention); out [N, H, Dh]."""
    what = "batch_attention"
    dev = _on_device(what, q, k_cache, v_cache, k_pages, v_pages, block_table, plan, out, workspace)
    N, H, Dh = q.shape[0], cfg.n_heads, cfg.head_dim
    qs = _want_rows(what, "q", q, N, H, Dh)
    _want(what, "out", out, torch.bfloat16, N, H, Dh)
    _want(what, "block_table", block_table, torch.int32, None, None)
    _want(what, "plan", plan, torch.uint8, None)
    _want(what, "workspace", workspace, torch.uint8, None)
    n_pages = _want_pages(what, cfg, n_kv_heads, k_pages, v_pages)
    cap = 0
    if k_cache is not None and v_cache is not None:
        cap = k_cache.shape[2] if k_cache.dim() == 4 else 0
        _want(what, "k_cache", k_cache, torch.bfloat16, cfg.n_layers, n_kv_heads, cap, Dh)
        _want(what, "v_cache", v_cache, torch.bfloat16, cfg.n_layers, n_kv_heads, Dh, cap)
    _check(_enqueue(_lib.llmcad_batch_attention, dev, stream,
                    (ctypes.byref(cfg), int(n_kv_heads), int(layer), q.data_ptr(), qs,
                     k_cache.data_ptr() if cap else None, v_cache.data_ptr() if cap else None, cap, int(prefix_len),
                     k_pages.data_ptr(), v_pages.data_ptr(), n_pages, block_table.data_ptr(), block_table.shape[1],
                     plan.data_ptr(), plan.shape[0], block_table.shape[0], N, out.data_ptr(), workspace.data_ptr(),
                     workspace.shape[0])), "llmcad_batch_attention")


def batch_commit(cfg, n_kv_heads: int, k_pages, v_pages, plan, n_requests: int, path, accept_len, stream=None):
    """Rollback of every request to its verified sequence (see llmcad_batch_commit): path int32 [n_rows] (the
    plan's, padding included: with another length nothing moves), accept_len int32 [n_requests], on the device."""
    what = "batch_commit"
    dev = _on_device(what, k_pages, v_pages, plan, path, accept_len)
    _want(what, "path", path, torch.int32, None)
    _want(what, "accept_len", accept_len, torch.int32, n_requests)
    _want(what, "plan", plan, torch.uint8, None)
    n_pages = _want_pages(what, cfg, n_kv_heads, k_pages, v_pages)
    _check(_enqueue(_lib.llmcad_batch_commit, dev, stream,
                    (ctypes.byref(cfg), int(n_kv_heads), k_pages.data_ptr(), v_pages.data_ptr(), n_pages, plan.data_ptr(),
                     plan.shape[0], int(n_requests), path.shape[0], path.data_ptr(), accept_len.data_ptr())),
           "llmcad_batch_commit")


def token_scores_workspace_bytes(n_rows: int, vocab: int, k: int) -> int:
    return _lib.llmcad_token_scores_workspace_bytes(int(n_rows), int(vocab), int(k))


def token_scores(logits, tokens, k: int = 0, row_of=None, workspace=None, stream=None) -> dict:
    """Scores of logits [n, V] (float32 or bfloat16, any distance between rows): {"logprob" of tokens
    (int32; under row row_of[i], or row i), "entropy", "lse", "top_token" [n, k], "top_logprob" [n, k]}
    (see llmcad_token_scores).  tokens may be None.  The outputs are new tensors of `stream`."""
    what = "token_scores"
    dev = _on_device(what, logits, tokens, row_of, workspace)
    fp32 = logits.dtype is torch.float32
    if logits.dim() != 2 or not (fp32 or logits.dtype is torch.bfloat16) or \
            (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("token_scores: logits must be float32 or bfloat16 [n, V] with contiguous rows")
    n, V = logits.shape
    k = int(k)
    if not 0 <= k <= TOP_MAX:
        raise ValueError(f"token_scores: k must be in [0, {TOP_MAX}]")
    m = 0
    if tokens is not None:
        m = tokens.shape[0] if tokens.dim() == 1 else -1
        _want(what, "tokens", tokens, torch.int32, n if row_of is None else m)
        if row_of is not None:
            _want(what, "row_of", row_of, torch.int32, m)
    if max(n, m) >= 1 << 31:  # (ctypes would cut the count)
        raise ValueError(f"token_scores: {n} rows and {m} tokens are too many")
    if stream is not None or dev != torch.cuda.current_device():
        _same_device(dev, stream)
        with torch.cuda.device(dev), torch.cuda.stream(stream):
            return token_scores(logits, tokens, k, row_of, workspace)
    if workspace is None:
        workspace = torch.empty(token_scores_workspace_bytes(n, V, k), dtype=torch.uint8, device=logits.device)
    else:
        _want(what, "workspace", workspace, torch.uint8, None)
    out = torch.empty(m + 2 * n + 2 * n * k, dtype=torch.float32, device=logits.device)
    at = out.data_ptr()
    top = at + 4 * (m + 2 * n)
    _check(_lib.llmcad_token_scores(
        logits.data_ptr(), 32 if fp32 else 16, logits.stride(0) if n > 1 else V, n, V,
        tokens.data_ptr() if m else None, row_of.data_ptr() if m and row_of is not None else None, m, at, at + 4 * m,
        at + 4 * (m + n), k, top, top + 4 * n * k, workspace.data_ptr(), workspace.shape[0],
        _current_stream(dev)), "llmcad_token_scores")
    logprob, entropy, lse, token, value = out.split((m, n, n, n * k, n * k))
    return {"logprob": logprob, "entropy": entropy, "lse": lse, "top_token": token.view(torch.int32).view(n, k),
            "top_logprob": value.view(n, k)}


def workspace_region(cfg, n: int, which: int):
    off, size = ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib.llmcad_workspace_region(ctypes.byref(cfg), int(n), int(which), ctypes.byref(off),
                                        ctypes.byref(size)), "llmcad_workspace_region")
    return off.value, size.value


def split_plan(cfg, n: int):
    """Diagnostics: per layer step, how a pass over n nodes shares it between workgroups
    (see llmcad_split_plan): {step: (workgroups per group, row-split or 4-bit tiles?, blocks of the largest group)}."""
    plan = (ctypes.c_int32 * 12)()
    _check(_lib.llmcad_split_plan(ctypes.byref(cfg), int(n), plan), "llmcad_split_plan")
    return {name: (plan[3 * j], bool(plan[3 * j + 1]), plan[3 * j + 2])
            for j, name in enumerate(("qkv", "o", "gate_up", "down"))}


def timing_enable(kernel_class: int, max_launches: int):
    _check(_lib.llmcad_timing_enable(int(kernel_class), int(max_launches)), "llmcad_timing_enable")


def timing_read(kernel_class: int):
    """(summed milliseconds, launches) of the bracketed launches since the last read."""
    ms, n = ctypes.c_double(), ctypes.c_int32()
    _check(_lib.llmcad_timing_read(int(kernel_class), ctypes.byref(ms), ctypes.byref(n)),
           "llmcad_timing_read")
    return ms.value, n.value


class Session:
    """Owns the device buffers of one target model: packed weights, KV cache,
    workspace and output buffers (all torch tensors), and forwards calls."""

    def __init__(self, shape, capacity: int, max_n: int = MAX_NODES, device="cuda"):
        self.cfg = make_config(shape)
        rc = check_config(self.cfg)
        if rc != OK:
            raise LlmcadError(rc, "config")
        self.shape = shape
        self.device = torch.device(device)
        self.max_n = int(max_n)
        self.capacity = (int(capacity) + 63) // 64 * 64  # (the library takes multiples of 64)
        cap = self.capacity
        L, H, Dh = shape.n_layers, shape.n_heads, shape.head_dim
        self.packed = torch.empty(packed_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        # K [L][H][cap][Dh]; V transposed per head [L][H][Dh][cap].  v_rows is
        # a [L][H][cap][Dh] view of the V cache (slot-major, like k_cache).
        self.k_cache = torch.zeros((L, H, cap, Dh), dtype=torch.bfloat16, device=self.device)
        self.v_cache = torch.zeros((L, H, Dh, cap), dtype=torch.bfloat16, device=self.device)
        self.v_rows = self.v_cache.transpose(2, 3)
        self.workspace = torch.zeros(workspace_bytes(self.cfg, self.max_n), dtype=torch.uint8,
                                     device=self.device)
        self.logits = torch.empty((self.max_n, shape.vocab), dtype=torch.float32, device=self.device)
        self.path = torch.empty(self.max_n, dtype=torch.int32, device=self.device)
        self.accept_len = torch.empty(1, dtype=torch.int32, device=self.device)
        self.next_token = torch.empty(1, dtype=torch.int32, device=self.device)
        self.last_logits = torch.empty(shape.vocab, dtype=torch.float32, device=self.device)
        off, _ = workspace_region(self.cfg, self.max_n, 5)  # (same offset for every pass size)
        self._status = self.workspace[off:off + 4].view(torch.int32)
        self._status_host = torch.zeros(1, dtype=torch.int32, pin_memory=True)

    def pass_status(self) -> int:
        """The device status of the passes enqueued so far (synchronises the stream)."""
        self._status_host.copy_(self._status, non_blocking=True)
        torch.cuda.current_stream().synchronize()
        return int(self._status_host[0])

    def check(self, what="pass"):
        """Raise LlmcadPassError if a pass since the last check failed on the device.
        The workspace's counters and status are cleared first, so the session
        serves the next pass; the failed pass's outputs (and the tree K/V it
        wrote) are invalid."""
        st = self.pass_status()
        if st != PASS_OK:
            workspace_init(self.cfg, self.max_n, self.workspace)
            torch.cuda.current_stream().synchronize()
            raise LlmcadPassError(st, what)

    def load_weights(self, gen, layers=None):
        """Pack weights from a generator with tok_embed(), final_norm(), lm_head(), layer(l)
        returning plain-layout tensors on this device (bf16 matrices, or for a
        4-bit model (codes, scales) pairs as pack_layer_q4 takes them)."""
        pack_globals(self.cfg, gen.tok_embed(), gen.final_norm(), gen.lm_head(), self.packed)
        q4 = self.cfg.weight_bits == 4
        for l in range(self.shape.n_layers) if layers is None else layers:
            (pack_layer_q4 if q4 else pack_layer)(self.cfg, l, gen.layer(l), self.packed)
            torch.cuda.current_stream().synchronize()  # let the plain layer be freed

    def prefill(self, tokens, start_pos=0, want_logits=False):
        prefill(self.cfg, self.packed, self.k_cache, self.v_cache, tokens, start_pos,
                self.last_logits if want_logits else None, self.workspace)
        return self.last_logits if want_logits else None

    def verify_tree(self, prefix_len, tree_tokens, parent, want_logits=True):
        n = len(tree_tokens)
        verify_tree(self.cfg, self.packed, self.k_cache, self.v_cache, prefix_len, tree_tokens,
                    parent, self.logits if want_logits else None, self.path, self.accept_len,
                    self.next_token, self.workspace)
        return n

    def extend(self, prefix_len, tree_tokens, parent, first):
        """Forward of nodes [first, n) of the tree; returns their logits [n - first, V] (device)."""
        n = len(tree_tokens)
        extend_tree(self.cfg, self.packed, self.k_cache, self.v_cache, prefix_len, tree_tokens, parent, first,
                    self.logits, self.workspace)
        return self.logits[: n - first]

    def score_tree(self, tree_tokens, parent, k=0):
        """Scores of the last verify_tree (with logits) over this tree: token_scores of its rows, "logprob"
        being the log probability of every node's token after its parent's branch (the root's entry is 0:
        nothing here predicts it)."""
        n = len(tree_tokens)
        host = np.stack([np.asarray(tree_tokens, dtype=np.int32), np.maximum(np.asarray(parent, dtype=np.int32), 0)])
        host[0, 0] = -1
        given = torch.from_numpy(host).to(self.device)
        return token_scores(self.logits[:n], given[0], k, row_of=given[1])

    def score(self, tokens, start_pos=0, k=0):
        """Takes tokens in as prefill does and scores every position: {"logprob" [n] of the next token of
        `tokens` (the last entry is 0), "entropy", "lse" [n], "top_token", "top_logprob" [n, k]}."""
        tokens = np.asarray(tokens, dtype=np.int32)
        if len(tokens) == 0:
            raise ValueError("score: no tokens")
        following = torch.from_numpy(np.append(tokens[1:], np.int32(-1))).to(self.device)
        parts = []
        for off in range(0, len(tokens), self.max_n):
            chunk = tokens[off:off + self.max_n]
            rows = self.extend(start_pos + off, chunk, np.arange(-1, len(chunk) - 1), 0)
            parts.append(token_scores(rows, following[off:off + len(chunk)], k))
        self.check("scoring pass")
        return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}

    def extend_candidates(self, prefix_len, tree_tokens, parent, first, threshold):
        """Forward of nodes [first, n) with candidate summaries; returns one parsed
        record per computed row (synchronises; checks the device status)."""
        rows = len(tree_tokens) - first
        if not hasattr(self, "_cand"):
            self._cand = torch.zeros((self.max_n, CAND_WORDS), dtype=torch.int32, device=self.device)
            self._cand_host = torch.zeros((self.max_n, CAND_WORDS), dtype=torch.int32, pin_memory=True)
        extend_tree_candidates(self.cfg, self.packed, self.k_cache, self.v_cache, prefix_len, tree_tokens, parent,
                               first, threshold, self.logits, self._cand, self.workspace)
        h = self._cand_host
        h[:rows].copy_(self._cand[:rows], non_blocking=True)
        self.check("tree-decoder step")
        return [parse_candidates(h[i].numpy()) for i in range(rows)]

    def commit(self, prefix_len, n):
        """Roll the cache back to the verified sequence of the last verify_tree over n nodes."""
        commit_path(self.cfg, self.k_cache, self.v_cache, prefix_len, self.path, self.accept_len, n)

    def outcome(self):
        """After verify_tree: synchronise, check the device status, and return
        (path list, accept_len, next_token) -- four small copies, one sync."""
        if not hasattr(self, "_out_host"):
            self._out_host = torch.zeros(self.max_n + 3, dtype=torch.int32, pin_memory=True)
        h = self._out_host
        h[0:1].copy_(self._status, non_blocking=True)
        h[1:2].copy_(self.accept_len, non_blocking=True)
        h[2:3].copy_(self.next_token, non_blocking=True)
        h[3:].copy_(self.path, non_blocking=True)
        torch.cuda.current_stream().synchronize()
        st = int(h[0])
        if st != PASS_OK:
            workspace_init(self.cfg, self.max_n, self.workspace)
            torch.cuda.current_stream().synchronize()
            raise LlmcadPassError(st, "verification pass")
        acc = int(h[1])
        return [int(x) for x in h[3:3 + acc + 1]], acc, int(h[2])

    def results(self, n):
        """Synchronise, check the device status, and return (logits [n, V] fp32 cpu,
        path list, accept_len, next_token)."""
        self.check("verification pass")
        acc = int(self.accept_len.item())
        return (self.logits[:n].cpu(), [int(x) for x in self.path[: acc + 1].cpu()], acc,
                int(self.next_token.item()))


class Batch:
    """Several requests behind one shared prefix: the page pool, block tables and the step's plan and
    workspace for a model of `shape` (device buffers owned here), with the prefix in k_cache / v_cache
    (a Session's, or any of that layout with n_kv_heads heads; None: no prefix).

    A step: plan(row_start, held, parent), advance(), per layer store and attention, then commit with the
    verified paths and trim(held) with the lengths after it.  Lengths are the caller's: after a step request b
    holds held[b] + its accepted rows.  Pages go out in the order of `free_pages`; advance drops the ones a
    plan handed out, trim takes back those of rejected rows, release(b) a finished request's.  (They replace
    `free_pages`: a captured step takes batch_plan with a free list of its own.)

    Until advance, a plan's new pages are in the block tables and on the free list both.  Where it did not
    place every request, advance (which raises), release and trim take them out of the tables, and the step can
    be planned anew; so does another plan, which replaces one that was not advanced.  release and trim after a
    good plan give back the requests' own pages alone, and advance drops those that the tables still hold."""

    def __init__(self, shape, n_requests: int, n_rows: int, n_pages: int, max_pages: int, prefix_len: int = 0,
                 k_cache=None, v_cache=None, n_kv_heads=None, device="cuda"):
        self.cfg = make_config(shape)
        rc = check_config(self.cfg)
        if rc != OK:
            raise LlmcadError(rc, "config")
        dev = torch.device(device)
        self.n_requests, self.n_rows, self.n_pages = int(n_requests), int(n_rows), int(n_pages)
        self.n_kv_heads = int(n_kv_heads or shape.n_heads)
        self.prefix_len, self.k_cache, self.v_cache = int(prefix_len), k_cache, v_cache
        L, Dh = shape.n_layers, shape.head_dim
        size = batch_plan_bytes(self.cfg, self.n_requests, self.n_rows)
        work = batch_workspace_bytes(self.cfg, self.n_kv_heads, self.n_requests, self.n_rows)
        if size == 0 or work == 0:
            raise LlmcadError(EARG, "batch sizes")
        self.k_pages = torch.zeros((L, self.n_pages, self.n_kv_heads, PAGE, Dh), dtype=torch.bfloat16, device=dev)
        self.v_pages = torch.zeros((L, self.n_pages, self.n_kv_heads, Dh, PAGE), dtype=torch.bfloat16, device=dev)
        self.block_table = torch.full((self.n_requests, int(max_pages)), -1, dtype=torch.int32, device=dev)
        self.free_pages = torch.arange(self.n_pages, dtype=torch.int32, device=dev)
        self.plan_buffer = torch.zeros(size, dtype=torch.uint8, device=dev)
        self.workspace = torch.zeros(work, dtype=torch.uint8, device=dev)
        for name, view in batch_plan_views(self.cfg, self.n_requests, self.n_rows, self.plan_buffer).items():
            setattr(self, name, view)  # slot, position, mask, rope, status, taken
        self._planned = False  # the last plan's pages are on the free list still
        self._changed = False  # ... and some of them have left the tables

    def _among(self, ids, others):
        """Which of ids are pages that others hold too (what is no page is not)."""
        index = lambda p: torch.where((p >= 0) & (p < self.n_pages), p, self.n_pages).long()  # noqa: E731
        held = torch.zeros(self.n_pages + 1, dtype=torch.bool, device=ids.device)
        held[index(others)] = True
        held[self.n_pages] = False
        return held[index(ids)]

    def _new_pages(self):
        """Which table entries are pages that are on the free list still (those of a plan before advance)."""
        return self._among(self.block_table, self.free_pages)

    def _undo(self):
        """Takes the pages of a plan that was not advanced out of the tables."""
        self.block_table.masked_fill_(self._new_pages(), -1)
        self._planned = self._changed = False

    def _give_back(self, entries):
        """Takes the table entries marked in `entries` out and those of them that are owned onto the free list
        (returned)."""
        if self._planned and bool(self.status.any()):
            self._undo()
        owned = entries & (self.block_table >= 0)
        if self._planned:
            owned &= ~self._new_pages()
            self._changed = True
        pages = self.block_table[owned]
        self.block_table.masked_fill_(entries, -1)
        return pages

    def plan(self, row_start, held, parent=None):
        if self._planned:
            self._undo()
        self._planned = True
        batch_plan(self.cfg, row_start, held, parent, self.prefix_len, self.block_table, self.free_pages,
                   self.n_pages, self.plan_buffer, self.n_rows)

    def _rows(self, what, **tensors):
        """Every tensor has the plan's n_rows rows (with another number the kernels would leave all as it was)."""
        for name, t in tensors.items():
            if t.dim() == 0 or t.shape[0] != self.n_rows:
                raise ValueError(f"Batch.{what}: {name} must have {self.n_rows} rows, padding included, got {tuple(t.shape)}")

    def store(self, layer, q, k, v, q_out):
        self._rows("store", q=q, k=k, v=v, q_out=q_out)
        batch_store(self.cfg, self.n_kv_heads, layer, q, k, v, q_out, self.k_pages, self.v_pages, self.plan_buffer,
                    self.n_requests)

    def attention(self, layer, q, out):
        self._rows("attention", q=q, out=out)
        batch_attention(self.cfg, self.n_kv_heads, layer, q, self.k_cache, self.v_cache, self.prefix_len, self.k_pages,
                        self.v_pages, self.block_table, self.plan_buffer, out, self.workspace)

    def commit(self, path, accept_len):
        self._rows("commit", path=path)
        batch_commit(self.cfg, self.n_kv_heads, self.k_pages, self.v_pages, self.plan_buffer, self.n_requests, path,
                     accept_len)

    def advance(self, taken=None):
        """Drops the pages that the last plan handed out from the free list (taken: their number if the
        caller has it and every request was placed; both are read from the device otherwise, and a request
        that was not placed raises, with the tables and the free list as they were before the plan)."""
        if taken is None:
            taken, bad = torch.cat([self.taken, self.status.max()[None]]).tolist()
            if bad != PLAN_OK:
                if self._planned:
                    self._undo()
                raise RuntimeError(f"requests {self.status.nonzero()[:, 0].tolist()} were not placed (plan status {bad})")
        taken = int(taken)
        if taken > self.free_pages.shape[0]:
            raise RuntimeError(f"the step needs {taken} pages and {self.free_pages.shape[0]} are free")
        if self._changed:  # (a request of the plan was released or trimmed: what the tables hold is taken)
            self.free_pages = self.free_pages[~self._among(self.free_pages, self.block_table)]
        else:
            self.free_pages = self.free_pages[taken:].clone()
        self._planned = self._changed = False

    def trim(self, held):
        """Takes back the pages past the requests' held tokens (int32 [n_requests], the lengths after a
        rollback; reads how many from the device).  Without it the next plan overwrites their entries."""
        pages = self._give_back(torch.arange(self.block_table.shape[1], device=held.device) * PAGE >= held[:, None])
        self.free_pages = torch.cat([pages, self.free_pages])

    def release(self, request: int):
        """Takes back the pages of a finished request."""
        entries = torch.zeros_like(self.block_table, dtype=torch.bool)
        entries[request] = True
        self.free_pages = torch.cat([self.free_pages, self._give_back(entries)])
