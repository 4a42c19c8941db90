"""Python binding of libditmi (the gfx950 DiT denoising-step library).

Argument marshalling only: torch tensors are checked (device, dtype,
contiguity) and their device pointers, together with the current HIP stream,
are handed to the C ABI declared in include/ditmi.h.  Every step of the
computation runs in the library's HIP kernels; there is no fallback path, and
a missing library raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# DITMI_LIB names another build of the same library (a sanitizer build, or a
# variant being measured); the default is the in-tree build.
LIB_PATH = os.environ.get("DITMI_LIB") or os.path.join(_HERE, "libditmi.so")

DIT_OK, DIT_ERR_INVALID_ARG, DIT_ERR_UNSUPPORTED, DIT_ERR_WORKSPACE, DIT_ERR_HIP = 0, -1, -2, -3, -4
DIT_F32, DIT_BF16, DIT_E4M3 = 0, 1, 2
DIT_WS_BLOCK, DIT_WS_STEP, DIT_WS_COND, DIT_WS_SAMPLE, DIT_WS_SERVE = 0, 1, 2, 3, 4
NOALLOC_SCRATCH_BYTES = 128 << 20  # DIT_NOALLOC_SCRATCH_BYTES of include/ditmi.h
KERNEL_CLASSES = {"gemm_qkv": 0, "attention": 1, "gemm_out": 2, "gemm_fc1": 3, "gemm_fc2": 4,
                  "ln_mod": 5, "adaln": 6, "other": 7}

STREAM_FIELDS = ("w_ada", "b_ada", "w_qkv", "b_qkv", "w_o", "b_o", "w_fc1", "b_fc1", "w_fc2", "b_fc2")
C_API = ("dit_workspace_bytes", "dit_block_forward", "dit_block_forward_noalloc", "dit_step_forward", "dit_sample_euler", "dit_serve", "dit_cond_embed", "dit_pos_embed_2d",
         "dit_attention", "dit_attention_workspace_bytes", "dit_quantize_fp8", "dit_linear_fp8",
         "dit_linear_fp8_workspace_bytes", "dit_norm_residual",
         "dit_timing_enable", "dit_timing_read", "dit_timing_disable", "dit_status_string", "dit_last_error",
         "dit_version")


class DitError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"ditmi status {status}: {msg}")
        self.status = status


class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("text_tokens", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("mlp_hidden", ctypes.c_int32), ("n_blocks", ctypes.c_int32), ("patch_in", ctypes.c_int32),
                ("patch_out", ctypes.c_int32), ("dtype", ctypes.c_int32), ("ln_eps", ctypes.c_float)]


class StreamWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in STREAM_FIELDS]


class BlockWeights(ctypes.Structure):
    _fields_ = [("img", StreamWeights), ("txt", StreamWeights)]


class StepWeights(ctypes.Structure):
    _fields_ = [("w_patch", ctypes.c_void_p), ("b_patch", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("blocks", ctypes.POINTER(BlockWeights)), ("w_ada_final", ctypes.c_void_p),
                ("b_ada_final", ctypes.c_void_p), ("w_final", ctypes.c_void_p), ("b_final", ctypes.c_void_p)]


_LIB: Optional[ctypes.CDLL] = None


class CondWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_t1", "b_t1", "w_t2", "b_t2", "class_table")]


class Request(ctypes.Structure):
    _fields_ = [("z_in", ctypes.c_void_p), ("z_out", ctypes.c_void_p), ("y", ctypes.c_void_p), ("cond", ctypes.c_void_p)]


class AttnShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("docs", "heads", "kv_heads", "head_dim", "q_rows", "k_rows", "max_q",
                                              "max_k", "dtype", "mask")] + \
               [(n, ctypes.c_float) for n in ("scale", "cap")] + \
               [(n, ctypes.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head", "o_row", "o_head")]


class LinearShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "in_features", "out_features", "act", "dtype")]


class NormShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "hidden", "batch", "post", "pre", "y_dtype", "h_dtype")] + \
               [("eps", ctypes.c_float), ("res_scale", ctypes.c_float), ("mod_stride", ctypes.c_int64)]


def lib() -> ctypes.CDLL:
    """Load libditmi.so (raises if it has not been built)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run paper_2605_25550_amd/build.py (or __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    P = ctypes.POINTER
    L.dit_workspace_bytes.argtypes = [P(Shape), ctypes.c_int]
    L.dit_workspace_bytes.restype = sz
    L.dit_block_forward.argtypes = [P(Shape), P(BlockWeights), vp, vp, vp, vp, sz, vp]
    L.dit_block_forward_noalloc.argtypes = [P(Shape), P(BlockWeights), vp, vp, vp, vp]
    L.dit_step_forward.argtypes = [P(Shape), P(StepWeights), vp, vp, vp, vp, vp, sz, vp]
    L.dit_cond_embed.argtypes = [P(Shape), vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dit_sample_euler.argtypes = [P(Shape), P(StepWeights), P(CondWeights), vp, vp, P(ctypes.c_float), i32,
                                   ctypes.c_float, vp, vp, vp, sz, vp]
    L.dit_serve.argtypes = [P(Shape), P(StepWeights), P(CondWeights), P(Request), i32, P(ctypes.c_float), i32,
                            ctypes.c_float, i32, ctypes.c_uint32, ctypes.c_uint32, vp, sz, vp, vp]
    L.dit_pos_embed_2d.argtypes = [i32, i32, i32, vp, vp]
    L.dit_attention_workspace_bytes.argtypes = [P(AttnShape)]
    L.dit_attention.argtypes = [P(AttnShape)] + [vp] * 10 + [sz, vp]
    L.dit_quantize_fp8.argtypes = [i32, i32, i32, i32, vp, ctypes.c_int64, vp, vp, vp]
    L.dit_linear_fp8_workspace_bytes.argtypes = [P(LinearShape)]
    L.dit_linear_fp8.argtypes = [P(LinearShape)] + [vp] * 8 + [sz, vp]
    L.dit_norm_residual.argtypes = [P(NormShape)] + [vp] * 12
    L.dit_attention_workspace_bytes.restype = L.dit_linear_fp8_workspace_bytes.restype = sz
    L.dit_timing_enable.argtypes = [ctypes.c_int, ctypes.c_int]
    L.dit_timing_read.argtypes = [P(ctypes.c_double), P(ctypes.c_int), P(ctypes.c_double), P(ctypes.c_double)]
    L.dit_timing_disable.argtypes = []
    for fn in ("dit_block_forward", "dit_block_forward_noalloc", "dit_step_forward", "dit_cond_embed", "dit_pos_embed_2d", "dit_timing_enable",
               "dit_timing_read", "dit_timing_disable", "dit_attention", "dit_quantize_fp8", "dit_linear_fp8",
               "dit_norm_residual"):
        getattr(L, fn).restype = ctypes.c_int
    L.dit_status_string.argtypes = [ctypes.c_int]
    L.dit_status_string.restype = ctypes.c_char_p
    L.dit_last_error.argtypes = []
    L.dit_last_error.restype = ctypes.c_char_p
    L.dit_version.restype = ctypes.c_int
    _LIB = L
    return L


def _check(st: int) -> None:
    if st != DIT_OK:
        raise DitError(st, lib().dit_last_error().decode())


def last_error() -> str:
    return lib().dit_last_error().decode()


# ---------------------------------------------------------------- marshalling
def make_shape(batch, tokens, hidden, heads, head_dim, mlp_hidden, n_blocks=1, text_tokens=0, patch_in=16,
               patch_out=16, dtype="bf16", ln_eps=1e-6) -> Shape:
    return Shape(batch, tokens, text_tokens, hidden, heads, head_dim, mlp_hidden, n_blocks, patch_in, patch_out,
                 DIT_BF16 if dtype == "bf16" else DIT_F32, ln_eps)


def shape_of(cfg) -> Shape:
    """Shape struct of a workload description with the DiT shape attributes
    (batch, tokens, text_tokens, hidden, heads, head_dim, mlp_hidden, n_blocks,
    patch_in, patch_out, dtype, ln_eps)."""
    return make_shape(cfg.batch, cfg.tokens, cfg.hidden, cfg.heads, cfg.head_dim, cfg.mlp_hidden, cfg.n_blocks,
                      cfg.text_tokens, cfg.patch_in, cfg.patch_out, cfg.dtype, cfg.ln_eps)


def weight_dtype(shape: Shape) -> torch.dtype:
    return torch.bfloat16 if shape.dtype == DIT_BF16 else torch.float32


def _ptr(t: Optional[torch.Tensor], dtype: Optional[torch.dtype] = None, name: str = "tensor"):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:  # cheaper than comparing device.type, and every call checks every tensor
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    return t.data_ptr()


def _stream(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without building a Stream object, which
    # costs 3 us a call: the small calls are bound by the host
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def stream_struct(w: Dict[str, torch.Tensor], dtype: torch.dtype) -> StreamWeights:
    return StreamWeights(*[_ptr(w[n], dtype, n) for n in STREAM_FIELDS])


def block_struct(img: Dict[str, torch.Tensor], txt: Optional[Dict[str, torch.Tensor]], dtype: torch.dtype) -> BlockWeights:
    bw = BlockWeights()
    bw.img = stream_struct(img, dtype)
    if txt is not None:
        bw.txt = stream_struct(txt, dtype)
    return bw


class StepWeightTable:
    """Holds the ctypes step-weight struct and the host array of block structs it points to."""

    def __init__(self, step_w: Dict[str, torch.Tensor], blocks: Sequence[BlockWeights], dtype: torch.dtype,
                 pos: Optional[torch.Tensor] = None):
        self.block_array = (BlockWeights * len(blocks))(*blocks)
        self.struct = StepWeights(
            _ptr(step_w["w_patch"], dtype, "w_patch"), _ptr(step_w["b_patch"], dtype, "b_patch"),
            _ptr(pos, torch.float32, "pos"), ctypes.cast(self.block_array, ctypes.POINTER(BlockWeights)),
            _ptr(step_w["w_ada_final"], dtype, "w_ada_final"), _ptr(step_w["b_ada_final"], dtype, "b_ada_final"),
            _ptr(step_w["w_final"], dtype, "w_final"), _ptr(step_w["b_final"], dtype, "b_final"))
        self._keep = (step_w, blocks, pos)


def _check_pos(shape: Shape, pos: Optional[torch.Tensor]) -> None:
    """The step reads the position table as [tokens, hidden] fp32 rows; the C
    ABI cannot see the size of a device buffer, so a short table is refused
    here rather than read past its end on the device."""
    if pos is None:
        return
    if pos.dim() != 2 or pos.shape[0] < shape.tokens or pos.shape[1] != shape.hidden:
        raise ValueError(f"pos is {tuple(pos.shape)}; the step reads [{shape.tokens}, {shape.hidden}] "
                         "(one row per image token)")


# ---------------------------------------------------------------- entry points
def workspace_bytes(shape: Shape, kind: int = DIT_WS_BLOCK) -> int:
    n = lib().dit_workspace_bytes(ctypes.byref(shape), kind)
    if n == 0:
        raise DitError(DIT_ERR_INVALID_ARG, last_error())
    return n


def alloc_workspace(shape: Shape, kind: int, device="cuda") -> torch.Tensor:
    return torch.empty(workspace_bytes(shape, kind), dtype=torch.uint8, device=device)


def block_forward(shape: Shape, weights: BlockWeights, x: torch.Tensor, cond: torch.Tensor, workspace: torch.Tensor,
                  x_txt: Optional[torch.Tensor] = None, stream=None) -> None:
    """One DiT block in place on x (and x_txt for the joint block)."""
    _check(lib().dit_block_forward(ctypes.byref(shape), ctypes.byref(weights), _ptr(x, torch.float32, "x"),
                                   _ptr(x_txt, torch.float32, "x_txt"), _ptr(cond, torch.float32, "cond"),
                                   _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size(),
                                   _stream(stream)))


def block_forward_noalloc(shape: Shape, weights: BlockWeights, x: torch.Tensor, cond: torch.Tensor,
                          x_txt: Optional[torch.Tensor] = None, stream=None) -> None:
    """One DiT block in place on x, with the library's static per-GPU scratch
    as workspace (no device allocation)."""
    _check(lib().dit_block_forward_noalloc(ctypes.byref(shape), ctypes.byref(weights), _ptr(x, torch.float32, "x"),
                                           _ptr(x_txt, torch.float32, "x_txt"), _ptr(cond, torch.float32, "cond"),
                                           _stream(stream)))


def step_forward(shape: Shape, table: StepWeightTable, patches: torch.Tensor, cond: torch.Tensor, out: torch.Tensor,
                 workspace: torch.Tensor, x_txt: Optional[torch.Tensor] = None, stream=None) -> None:
    """One denoising step (patch embed, blocks, final layer) into out."""
    _check_pos(shape, table._keep[2])
    _check(lib().dit_step_forward(ctypes.byref(shape), ctypes.byref(table.struct),
                                  _ptr(patches, torch.float32, "patches"), _ptr(x_txt, torch.float32, "x_txt"),
                                  _ptr(cond, torch.float32, "cond"), _ptr(out, torch.float32, "out"),
                                  _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size(),
                                  _stream(stream)))


def sample_euler(shape: Shape, table: StepWeightTable, z: torch.Tensor, sigmas, workspace: torch.Tensor,
                 cond_w: Optional[Dict[str, torch.Tensor]] = None, y: Optional[torch.Tensor] = None,
                 cond: Optional[torch.Tensor] = None, t_scale: float = 1000.0,
                 x_txt: Optional[torch.Tensor] = None, stream=None) -> None:
    """Multi-step Euler loop over the step (z updated in place): with cond_w and
    y the conditioning is recomputed per step at t_i = sigmas[i] * t_scale;
    otherwise cond is used for every step.  sigmas: n_steps + 1 floats (host)."""
    _check_pos(shape, table._keep[2])
    sig = [float(v) for v in sigmas]
    if len(sig) < 1:
        raise ValueError("sigmas needs at least one value")
    arr = (ctypes.c_float * len(sig))(*sig)
    cw = None
    if cond_w is not None:
        dt = weight_dtype(shape)
        cw = CondWeights(*[_ptr(cond_w[k], dt, k) for k in ("w_t1", "b_t1", "w_t2", "b_t2", "class_table")])
    _check(lib().dit_sample_euler(ctypes.byref(shape), ctypes.byref(table.struct),
                                  ctypes.byref(cw) if cw is not None else None,
                                  _ptr(y, torch.int32, "y"), _ptr(cond, torch.float32, "cond"), arr, len(sig) - 1,
                                  float(t_scale), _ptr(z, torch.float32, "z"), _ptr(x_txt, torch.float32, "x_txt"),
                                  _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size(),
                                  _stream(stream)))


def _host_ptr(t: Optional[torch.Tensor], dtype: torch.dtype, name: str):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device.type != "cpu" or not t.is_contiguous() or t.dtype != dtype:
        raise ValueError(f"{name} must be a contiguous host {dtype} tensor")
    return t.data_ptr()


def serve(shape: Shape, table: StepWeightTable, requests, sigmas, workspace: torch.Tensor,
          cond_w: Optional[Dict[str, torch.Tensor]] = None, t_scale: float = 1000.0, overlap: bool = True,
          jitter_us: int = 0, jitter_seed: int = 0, stream=None, copy_stream=None) -> None:
    """Run requests through the DiT stage with copy/compute overlap.  requests:
    list of dicts with host tensors z_in, z_out ([B,T,P] fp32, ideally pinned)
    and y ([B] int32, with cond_w) or cond ([B,D] fp32).  Returns after
    enqueueing; synchronise the stream before reading z_out."""
    _check_pos(shape, table._keep[2])
    sig = [float(v) for v in sigmas]
    arr = (ctypes.c_float * len(sig))(*sig)
    reqs = (Request * max(1, len(requests)))()
    for i, r in enumerate(requests):
        reqs[i] = Request(_host_ptr(r["z_in"], torch.float32, "z_in"), _host_ptr(r["z_out"], torch.float32, "z_out"),
                          _host_ptr(r.get("y"), torch.int32, "y"), _host_ptr(r.get("cond"), torch.float32, "cond"))
    cw = None
    if cond_w is not None:
        dt = weight_dtype(shape)
        cw = CondWeights(*[_ptr(cond_w[k], dt, k) for k in ("w_t1", "b_t1", "w_t2", "b_t2", "class_table")])
    cs = copy_stream.cuda_stream if copy_stream is not None else None
    _check(lib().dit_serve(ctypes.byref(shape), ctypes.byref(table.struct), ctypes.byref(cw) if cw is not None else None,
                           reqs, len(requests), arr, len(sig) - 1, float(t_scale), 1 if overlap else 0, int(jitter_us),
                           int(jitter_seed), _ptr(workspace, None, "workspace"),
                           workspace.numel() * workspace.element_size(), _stream(stream), cs))


def cond_embed(shape: Shape, t: torch.Tensor, y: torch.Tensor, w: Dict[str, torch.Tensor], cond: torch.Tensor,
               workspace: torch.Tensor, stream=None) -> None:
    """Timestep + class conditioning into cond [B, D]."""
    dt = weight_dtype(shape)
    _check(lib().dit_cond_embed(ctypes.byref(shape), _ptr(t, torch.float32, "t"), _ptr(y, torch.int32, "y"),
                                _ptr(w["w_t1"], dt, "w_t1"), _ptr(w["b_t1"], dt, "b_t1"), _ptr(w["w_t2"], dt, "w_t2"),
                                _ptr(w["b_t2"], dt, "b_t2"), _ptr(w["class_table"], dt, "class_table"),
                                _ptr(cond, torch.float32, "cond"), _ptr(workspace, None, "workspace"),
                                workspace.numel() * workspace.element_size(), _stream(stream)))


def pos_embed_2d(grid_h: int, grid_w: int, hidden: int, pos: torch.Tensor, stream=None) -> None:
    _check(lib().dit_pos_embed_2d(grid_h, grid_w, hidden, _ptr(pos, torch.float32, "pos"), _stream(stream)))


# ---------------------------------------------------------------- stand-alone operators
_DTYPE_IDS = {torch.float32: DIT_F32, torch.bfloat16: DIT_BF16, torch.float8_e4m3fn: DIT_E4M3}
_TORCH_DTYPES = (torch.float32, torch.bfloat16, torch.float8_e4m3fn)
_DTYPE_NAMES = {"f32": DIT_F32, "bf16": DIT_BF16, "e4m3": DIT_E4M3}
_MASKS = {"full": 0, "causal": 1, "prefix": 2}
_NORMS = {"none": 0, "layer": 1, "rms": 2}
_ACTS = {"none": 0, "gelu": 1}


def _pick(table, key, what):
    if key not in table:
        raise ValueError(f"{what} must be one of {', '.join(table)} (got {key!r})")
    return table[key]


def _refuse(t, dtype, numel: Optional[int], name: str, device: int):
    """The error of a tensor that _arg did not take."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor (got {t.device})")
    if t.get_device() != device:
        raise ValueError(f"tensors on cuda:{device} and {t.device} in one call")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    raise ValueError(f"{name} has {t.numel()} elements, the call reads or writes {numel}")


def _arg(t: Optional[torch.Tensor], dtype, numel: int, name: str, device: int):
    """Pointer of a contiguous tensor of that type, size and device (None stays
    None).  Small calls are bound by the host: one test, and the reasons apart."""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.get_device() == device and t.numel() == numel and t.is_contiguous() and device >= 0:
            return t.data_ptr()
    except AttributeError:
        pass
    return _refuse(t, dtype, numel, name, device)


def _ws_arg(t: Optional[torch.Tensor], device: int):
    if t is None:
        return None, 0
    if device < 0 or t.get_device() != device or not t.is_contiguous():
        _refuse(t, None, None, "workspace", device)
    return t.data_ptr(), t.nbytes


def _launch(device: int, stream, fn, *args) -> None:
    """Calls fn(*args, stream) on the tensors' device, whichever is current,
    and on its current stream unless one is given."""
    if stream is not None:
        if stream.device_index != device:
            raise ValueError(f"the stream is on cuda:{stream.device_index}, the tensors on cuda:{device}")
        raw = stream.cuda_stream
    else:
        raw = torch._C._cuda_getCurrentRawStream(device)
    if device == torch._C._cuda_getDevice():
        st = fn(*args, raw)
    else:
        with torch.cuda.device(device):
            st = fn(*args, raw)
    _check(st)


def _workspace(n: int, device) -> Optional[torch.Tensor]:
    if n == ctypes.c_size_t(-1).value:
        raise DitError(DIT_ERR_INVALID_ARG, last_error())
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _strided_ptr(t: torch.Tensor, dtype, shape, name: str, row: int, head: int, device: int):
    """Pointer of a [rows, heads, head_dim] tensor with the strides its shape struct states."""
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    r, h, d = t.stride() if t.dim() == 3 else (0, 0, 0)
    if t.shape != shape or (t.numel() and (d != 1 or (r != row and shape[0] > 1) or (h != head and shape[1] > 1))):
        raise ValueError(f"{name} is {tuple(t.shape)} with strides {t.stride()}; "
                         f"the shape states {shape} with strides ({row}, {head}, 1)")
    if device < 0 or t.get_device() != device:
        _refuse(t, dtype, None, name, device)
    return t.data_ptr()


def attn_shape(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, docs: int, max_q: int, max_k: int,
               mask: str = "full", scale: Optional[float] = None, cap: float = 0.0) -> AttnShape:
    """Shape struct of attention calls on tensors laid out as these: q, o
    [query rows, heads, head_dim], k, v [key rows, kv_heads, head_dim], the last
    dimension contiguous (views of a fused projection or of a cache).  max_q
    and max_k bound a document's queries and keys (its room, where no q_start
    or k_start is given); scale defaults to 1/sqrt(head_dim)."""
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (o, "o")):
        if t.dim() != 3:
            raise ValueError(f"{name} must be [rows, heads, head_dim] (got {tuple(t.shape)})")
        if t.dtype != q.dtype or t.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"q, k, v and o must all be float32 or all bfloat16 (got {t.dtype} for {name})")
    dh = q.shape[2]
    st = []
    for t in (q, k, v, o):  # a stride over one element is never used, whatever torch states
        st += [t.stride(0) if t.shape[0] > 1 else t.shape[1] * dh, t.stride(1) if t.shape[1] > 1 else dh]
    return AttnShape(docs, q.shape[1], k.shape[1], dh, q.shape[0], k.shape[0], max_q, max_k, _DTYPE_IDS[q.dtype],
                     _pick(_MASKS, mask, "mask"), dh ** -0.5 if scale is None else scale, cap, *st)


def attention_workspace(shape: AttnShape, device="cuda") -> Optional[torch.Tensor]:
    """Workspace of attention calls of this shape (None where none is needed)."""
    return _workspace(lib().dit_attention_workspace_bytes(ctypes.byref(shape)), device)


def attention(shape: AttnShape, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
              workspace: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
              k_start: Optional[torch.Tensor] = None, k_len: Optional[torch.Tensor] = None,
              prefix: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None, stream=None) -> None:
    """Masked attention over documents into o: q_start, k_start [docs + 1], k_len,
    prefix [docs] int32 and slopes [heads] fp32 on the device."""
    s = shape
    dt, i32, dev = _TORCH_DTYPES[s.dtype], torch.int32, q.get_device()
    docs, H, dh = s.docs, s.heads, s.head_dim
    qs, ks = (s.q_rows, H, dh), (s.k_rows, s.kv_heads, dh)
    ws, n = _ws_arg(workspace, dev)
    _launch(dev, stream, lib().dit_attention, ctypes.byref(s), _strided_ptr(q, dt, qs, "q", s.q_row, s.q_head, dev),
            _strided_ptr(k, dt, ks, "k", s.k_row, s.k_head, dev), _strided_ptr(v, dt, ks, "v", s.v_row, s.v_head, dev),
            _strided_ptr(o, dt, qs, "o", s.o_row, s.o_head, dev), _arg(q_start, i32, docs + 1, "q_start", dev),
            _arg(k_start, i32, docs + 1, "k_start", dev), _arg(k_len, i32, docs, "k_len", dev),
            _arg(prefix, i32, docs, "prefix", dev), _arg(slopes, torch.float32, H, "slopes", dev), ws, n)


def quantize_fp8(x: torch.Tensor, codes: torch.Tensor, scale: torch.Tensor, block_rows: int = 1, stream=None) -> None:
    """x [rows, cols] (rows may be strided) to e4m3 codes [rows, cols] and fp32
    scales [ceil(rows / block_rows), ceil(cols / 128)]."""
    if x.dim() != 2 or x.dtype not in (torch.float32, torch.bfloat16) or not x.is_cuda:
        raise ValueError(f"x must be a [rows, cols] float32 or bfloat16 device tensor (got {x.dtype} {tuple(x.shape)})")
    if x.numel() and x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError("x's columns must be contiguous")
    R, C = x.shape
    nr, dev = -(-R // block_rows) if block_rows > 0 else 0, x.get_device()
    _launch(dev, stream, lib().dit_quantize_fp8, R, C, block_rows, _DTYPE_IDS[x.dtype], x.data_ptr(),
            x.stride(0) if R > 1 else C, _arg(codes, torch.float8_e4m3fn, R * C, "codes", dev),
            _arg(scale, torch.float32, nr * -(-C // 128), "scale", dev))


def linear_shape(rows: int, in_features: int, out_features: int, act: str = "none", dtype: str = "bf16") -> LinearShape:
    """Shape struct of linear_fp8: act "none" or "gelu", dtype of the output
    "bf16", "f32" or "e4m3"."""
    return LinearShape(rows, in_features, out_features, _pick(_ACTS, act, "act"), _pick(_DTYPE_NAMES, dtype, "dtype"))


def linear_fp8_workspace(shape: LinearShape, device="cuda") -> Optional[torch.Tensor]:
    """Workspace of linear_fp8 calls of this shape (None where none is needed)."""
    return _workspace(lib().dit_linear_fp8_workspace_bytes(ctypes.byref(shape)), device)


def linear_fp8(shape: LinearShape, a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
               out: torch.Tensor, workspace: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               out_scale: Optional[torch.Tensor] = None, stream=None) -> None:
    """out = act(a w^T + bias) on e4m3 codes a [rows, in], w [out, in] with block
    scales (quantize_fp8 with block_rows 1 and 128); bias fp32 for an fp32
    output, else bf16; out_scale [rows, ceil(out / 128)] for an e4m3 output."""
    s = shape
    M, K, N = s.rows, s.in_features, s.out_features
    kb, nb = -(-K // 128), -(-N // 128)
    f8, f32, dev = torch.float8_e4m3fn, torch.float32, a.get_device()
    ws, n = _ws_arg(workspace, dev)
    _launch(dev, stream, lib().dit_linear_fp8, ctypes.byref(s), _arg(a, f8, M * K, "a", dev),
            _arg(a_scale, f32, M * kb, "a_scale", dev), _arg(w, f8, N * K, "w", dev),
            _arg(w_scale, f32, nb * kb, "w_scale", dev),
            _arg(bias, f32 if s.dtype == DIT_F32 else torch.bfloat16, N, "bias", dev),
            _arg(out, _TORCH_DTYPES[s.dtype], M * N, "out", dev), _arg(out_scale, f32, M * nb, "out_scale", dev), ws, n)


def norm_shape(rows: int, hidden: int, batch: int = 1, post: str = "none", pre: str = "layer", y_dtype: str = "f32",
               h_dtype: str = "bf16", eps: float = 1e-6, res_scale: float = 1.0, mod_stride: int = 0) -> NormShape:
    """Shape struct of norm_residual: norms "none" (post only), "layer" or "rms";
    batch rows of gate, shift and scale, mod_stride elements apart."""
    return NormShape(rows, hidden, batch, _pick(_NORMS, post, "post"), _pick(_NORMS, pre, "pre"),
                     _pick(_DTYPE_NAMES, y_dtype, "y_dtype"), _pick(_DTYPE_NAMES, h_dtype, "h_dtype"), eps, res_scale,
                     mod_stride or hidden)


def _mod_ptr(t: Optional[torch.Tensor], batch: int, hidden: int, stride: int, name: str, device: int):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.shape != (batch, hidden) or t.stride(1) != 1 or \
            (batch > 1 and t.stride(0) != stride):
        raise ValueError(f"{name} must be a float32 [{batch}, {hidden}] tensor whose rows are {stride} apart "
                         f"(got {t.dtype} {tuple(t.shape)}, strides {t.stride()})")
    if device < 0 or t.get_device() != device:
        _refuse(t, torch.float32, None, name, device)
    return t.data_ptr()


def norm_residual(shape: NormShape, x: torch.Tensor, x_out: Optional[torch.Tensor], h: Optional[torch.Tensor],
                  y: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None,
                  shift: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                  row_batch: Optional[torch.Tensor] = None, h_scale: Optional[torch.Tensor] = None, stream=None) -> None:
    """x_out = res_scale x + gate norm_post(y), h = norm_pre(x_out) modulated;
    x_out may be x.  h_scale [rows, ceil(hidden / 128)] for an e4m3 h."""
    s = shape
    R, D, B, st, f32, dev = s.rows, s.hidden, s.batch, s.mod_stride, torch.float32, x.get_device()
    n = R * D
    _launch(dev, stream, lib().dit_norm_residual, ctypes.byref(s), _arg(x, f32, n, "x", dev),
            _arg(x_out, f32, n, "x_out", dev), _arg(y, _TORCH_DTYPES[s.y_dtype], n, "y", dev),
            _arg(w_post, f32, D, "w_post", dev), _mod_ptr(gate, B, D, st, "gate", dev), _arg(w_pre, f32, D, "w_pre", dev),
            _mod_ptr(shift, B, D, st, "shift", dev), _mod_ptr(scale, B, D, st, "scale", dev),
            _arg(row_batch, torch.int32, R, "row_batch", dev), _arg(h, _TORCH_DTYPES[s.h_dtype], n, "h", dev),
            _arg(h_scale, f32, R * -(-D // 128), "h_scale", dev))


def timing_enable(kclass: str, max_launches: int) -> None:
    _check(lib().dit_timing_enable(KERNEL_CLASSES[kclass], max_launches))


def timing_read():
    """(total_ms, launches, flops, bytes) of the launches recorded since timing_enable."""
    ms, n, fl, by = ctypes.c_double(), ctypes.c_int(), ctypes.c_double(), ctypes.c_double()
    _check(lib().dit_timing_read(ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl), ctypes.byref(by)))
    return ms.value, n.value, fl.value, by.value


def timing_disable() -> None:
    _check(lib().dit_timing_disable())
