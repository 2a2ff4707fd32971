"""ctypes binding of libsantapp.so: argument marshalling only.

Every step of the path (team build, routing, sampling, exact attention, split-K
merge) runs in the library's CUDA kernels. PyTorch is used for device memory and
streams. There is no CPU fallback: if the library is missing or cannot be loaded
the first call raises.

The functions keep the names of the C entry points (include/santapp.h, include/santapp_latent.h,
include/santapp_serve.h). With `stream=s` a call runs on s; outputs and workspaces that it makes itself are
that stream's memory, and the current stream may use the outputs once it has waited for s.
"""
import contextlib
import ctypes
import functools
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsantapp.so")

SANTAPP_OK = 0
SANTAPP_ERR_INVALID_ARG = -1
SANTAPP_ERR_UNSUPPORTED = -2
SANTAPP_ERR_WORKSPACE_TOO_SMALL = -3
SANTAPP_ERR_CUDA = -4
SANTAPP_ERR_STATIC_SCRATCH = -5
SANTAPP_STATIC_SCRATCH_BYTES = 2 << 20
SANTAPP_BF16, SANTAPP_FP16 = 0, 1

EXPORTS = [
    "santapp_version", "santapp_strerror", "santapp_last_cuda_error", "santapp_build_teams_sizes",
    "santapp_build_teams", "santapp_decode_workspace_bytes", "santapp_decode_attn",
    "santapp_dense_workspace_bytes", "santapp_dense_decode_attn", "santapp_last_launch_count",
    "santapp_set_stage_mask", "santapp_dense_decode_attn_noalloc", "santapp_build_groups_mean",
    "santapp_kmeans_parent_count", "santapp_assign_parents_workspace_bytes", "santapp_assign_parents",
    "santapp_parent_teams_sizes", "santapp_build_teams_parents", "santapp_build_groups_mean_parents",
    "santapp_kmeans_fit_workspace_bytes", "santapp_kmeans_fit",
    "santapp_latent_sizes", "santapp_latent_build_teams", "santapp_latent_decode_workspace_bytes",
    "santapp_latent_decode_attn", "santapp_latent_dense_workspace_bytes", "santapp_latent_dense_decode_attn",
    "santapp_rope_frequencies", "santapp_rope_append", "santapp_rope_prompt", "santapp_suffix_fork",
    "santapp_prefix_decode_workspace_bytes", "santapp_prefix_decode_attn", "santapp_prompt_attn",
]
LATENT_DIM, LATENT_ROPE_DIM, LATENT_ROW = 512, 64, 576

STAGE_ROUTE, STAGE_SELECT, STAGE_ATTEND, STAGE_MERGE, STAGE_ALL = 1, 2, 4, 8, 15


class SantappError(RuntimeError):
    def __init__(self, status, detail=""):
        self.status = status
        super().__init__(f"santapp status {status}: {detail}")


class CGeom(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("parent_size", ctypes.c_int32),
                ("reps_per_parent", ctypes.c_int32), ("elem_type", ctypes.c_int32)]


class CSizes(ctypes.Structure):
    _fields_ = [("rows_total", ctypes.c_int64), ("teams_total", ctypes.c_int64),
                ("max_teams_per_seq", ctypes.c_int32), ("max_rows_per_seq", ctypes.c_int32),
                ("team_row_start_elems", ctypes.c_int64), ("build_workspace_bytes", ctypes.c_size_t)]


class CTeams(ctypes.Structure):
    _fields_ = [("k_packed", ctypes.c_void_p), ("v_packed", ctypes.c_void_p), ("rep_keys", ctypes.c_void_p),
                ("team_row_start", ctypes.c_void_p), ("row_token", ctypes.c_void_p),
                ("seq_row_off", ctypes.c_void_p), ("seq_team_off", ctypes.c_void_p),
                ("rep_abs_max", ctypes.c_void_p), ("team_count", ctypes.c_void_p),
                ("rows_total", ctypes.c_int64), ("teams_total", ctypes.c_int64),
                ("max_teams_per_seq", ctypes.c_int32), ("max_rows_per_seq", ctypes.c_int32)]


class CKmeansOpts(ctypes.Structure):
    _fields_ = [("batch_size", ctypes.c_int32), ("max_iter", ctypes.c_int32), ("patience", ctypes.c_int32),
                ("no_host_poll", ctypes.c_int32), ("reassignment_ratio", ctypes.c_double), ("seed", ctypes.c_uint64),
                ("stream_base", ctypes.c_uint32), ("reserved2", ctypes.c_uint32)]


class CDebug(ctypes.Structure):
    _fields_ = [("sel_idx", ctypes.c_void_p), ("sel_logc", ctypes.c_void_p), ("tau", ctypes.c_void_p),
                ("union_rows", ctypes.c_void_p), ("status", ctypes.c_void_p), ("trace", ctypes.c_void_p)]


_lib = None


class CLatentGeom(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("parent_size", ctypes.c_int32),
                ("reps_per_parent", ctypes.c_int32)]


class CLatentTeams(ctypes.Structure):
    _fields_ = [("rows_packed", ctypes.c_void_p), ("rep_rows", ctypes.c_void_p), ("team_row_start", ctypes.c_void_p),
                ("row_token", ctypes.c_void_p), ("seq_row_off", ctypes.c_void_p), ("seq_team_off", ctypes.c_void_p),
                ("rep_abs_max", ctypes.c_void_p), ("rows_total", ctypes.c_int64), ("teams_total", ctypes.c_int64),
                ("max_teams_per_seq", ctypes.c_int32), ("max_rows_per_seq", ctypes.c_int32)]


class CRope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("amplitude", ctypes.c_double),
                ("inv_freq", ctypes.c_double * 64)]


class CAttnOpts(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("cap", ctypes.c_float), ("slopes", ctypes.c_void_p),
                ("status", ctypes.c_void_p)]


def load_library(path: Optional[str] = None):
    """Load libsantapp.so and declare its signatures. Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise SantappError(SANTAPP_ERR_CUDA, f"{p} not found: build it with `python -m paper_2609_35629_b200.build` "
                                             "(there is no CPU fallback)")
    L = ctypes.CDLL(p)
    vp, i32, u32, u64, f32, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64,
                                  ctypes.c_float, ctypes.c_size_t)
    L.santapp_version.restype = ctypes.c_int
    L.santapp_strerror.argtypes = [ctypes.c_int]
    L.santapp_strerror.restype = ctypes.c_char_p
    L.santapp_last_cuda_error.restype = ctypes.c_char_p
    L.santapp_last_launch_count.restype = ctypes.c_int
    L.santapp_build_teams_sizes.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(i32), ctypes.POINTER(CSizes)]
    L.santapp_build_teams_sizes.restype = ctypes.c_int
    L.santapp_build_teams.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(i32), vp, vp,
                                      ctypes.POINTER(CTeams), vp, sz, vp]
    L.santapp_build_teams.restype = ctypes.c_int
    L.santapp_build_groups_mean.argtypes = L.santapp_build_teams.argtypes
    L.santapp_build_groups_mean.restype = ctypes.c_int
    L.santapp_kmeans_fit_workspace_bytes.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                                     ctypes.POINTER(CKmeansOpts)]
    L.santapp_kmeans_fit_workspace_bytes.restype = sz
    L.santapp_kmeans_fit.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(i32), ctypes.POINTER(i32), vp,
                                     ctypes.POINTER(CKmeansOpts), vp, vp, vp, sz, vp]
    L.santapp_kmeans_fit.restype = ctypes.c_int
    L.santapp_kmeans_parent_count.argtypes = [i32, i32]
    L.santapp_kmeans_parent_count.restype = i32
    L.santapp_assign_parents_workspace_bytes.argtypes = [ctypes.POINTER(CGeom)]
    L.santapp_assign_parents_workspace_bytes.restype = sz
    L.santapp_assign_parents.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(i32), ctypes.POINTER(i32), vp, vp, vp,
                                         vp, sz, vp]
    L.santapp_assign_parents.restype = ctypes.c_int
    L.santapp_parent_teams_sizes.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                             ctypes.POINTER(CSizes)]
    L.santapp_parent_teams_sizes.restype = ctypes.c_int
    L.santapp_build_teams_parents.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(i32), ctypes.POINTER(i32), vp, vp,
                                              vp, ctypes.POINTER(CTeams), vp, sz, vp]
    L.santapp_build_teams_parents.restype = ctypes.c_int
    L.santapp_build_groups_mean_parents.argtypes = L.santapp_build_teams_parents.argtypes
    L.santapp_build_groups_mean_parents.restype = ctypes.c_int
    L.santapp_decode_workspace_bytes.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(CTeams), i32]
    L.santapp_decode_workspace_bytes.restype = sz
    L.santapp_dense_workspace_bytes.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(CTeams)]
    L.santapp_dense_workspace_bytes.restype = sz
    L.santapp_decode_attn.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(CTeams), vp, vp, vp, vp, i32, i32,
                                      u64, u32, vp, u32, f32, vp, ctypes.POINTER(CDebug), vp, sz, vp]
    L.santapp_set_stage_mask.argtypes = [ctypes.c_int]
    L.santapp_set_stage_mask.restype = None
    L.santapp_decode_attn.restype = ctypes.c_int
    L.santapp_dense_decode_attn.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(CTeams), vp, vp, vp, vp, i32,
                                            f32, vp, vp, sz, vp]
    L.santapp_dense_decode_attn.restype = ctypes.c_int
    L.santapp_dense_decode_attn_noalloc.argtypes = [ctypes.POINTER(CGeom), ctypes.POINTER(CTeams), vp, vp, vp, vp,
                                                    i32, f32, vp, vp]
    L.santapp_dense_decode_attn_noalloc.restype = ctypes.c_int
    LG, LT = ctypes.POINTER(CLatentGeom), ctypes.POINTER(CLatentTeams)
    L.santapp_latent_sizes.argtypes = [LG, ctypes.POINTER(i32), ctypes.POINTER(CSizes)]
    L.santapp_latent_sizes.restype = ctypes.c_int
    L.santapp_latent_build_teams.argtypes = [LG, ctypes.POINTER(i32), vp, LT, vp, sz, vp]
    L.santapp_latent_build_teams.restype = ctypes.c_int
    L.santapp_latent_decode_workspace_bytes.argtypes = [LG, LT, i32, i32]
    L.santapp_latent_decode_workspace_bytes.restype = sz
    L.santapp_latent_dense_workspace_bytes.argtypes = [LG, LT]
    L.santapp_latent_dense_workspace_bytes.restype = sz
    L.santapp_latent_decode_attn.argtypes = [LG, LT, vp, vp, vp, i32, i32, u64, u32, vp, u32, f32, vp,
                                             ctypes.POINTER(CDebug), vp, sz, vp]
    L.santapp_latent_decode_attn.restype = ctypes.c_int
    L.santapp_latent_dense_decode_attn.argtypes = [LG, LT, vp, vp, vp, i32, f32, vp, vp, sz, vp]
    L.santapp_latent_dense_decode_attn.restype = ctypes.c_int
    i64, f64 = ctypes.c_int64, ctypes.c_double
    G, R, O = ctypes.POINTER(CGeom), ctypes.POINTER(CRope), ctypes.POINTER(CAttnOpts)
    L.santapp_rope_frequencies.argtypes = [R, f64, f64, f64, f64, f64]
    L.santapp_rope_frequencies.restype = ctypes.c_int
    L.santapp_rope_append.argtypes = [G, R, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, i32, vp, vp]
    L.santapp_rope_append.restype = ctypes.c_int
    L.santapp_rope_prompt.argtypes = [G, R, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp]
    L.santapp_rope_prompt.restype = ctypes.c_int
    L.santapp_suffix_fork.argtypes = [G, vp, vp, vp, vp, i32, vp, vp]
    L.santapp_suffix_fork.restype = ctypes.c_int
    L.santapp_prefix_decode_workspace_bytes.argtypes = [G, i64, i32]
    L.santapp_prefix_decode_workspace_bytes.restype = sz
    L.santapp_prefix_decode_attn.argtypes = [G, vp, vp, i64, i64, vp, vp, vp, vp, vp, i32, O, vp, vp, sz, vp]
    L.santapp_prefix_decode_attn.restype = ctypes.c_int
    L.santapp_prompt_attn.argtypes = [G, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32), vp, vp, vp, O, vp, vp]
    L.santapp_prompt_attn.restype = ctypes.c_int
    if path is None:
        _lib = L
    return L


def _check(rc):
    if rc != SANTAPP_OK:
        L = load_library()
        detail = L.santapp_strerror(rc).decode()
        if rc in (SANTAPP_ERR_CUDA, SANTAPP_ERR_STATIC_SCRATCH):
            detail += " — " + L.santapp_last_cuda_error().decode()
        raise SantappError(rc, detail)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise SantappError(SANTAPP_ERR_INVALID_ARG, "tensors must be contiguous CUDA tensors")
    return t.data_ptr()


def _stream_ptr(stream):
    # (the raw handle: making torch's Stream object costs more than a kernel launch's share of a call)
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _on(stream):
    """Where a call's buffers are made: on the stream it runs on (None: the current one). Memory that belonged to another stream could
    still be in use there when the call starts, or be given to somebody else on it while the call is under way."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream))


def _handed_out(stream, *tensors):
    """Buffers of a given stream that the caller gets: the current stream may use them too, until they are dropped."""
    if stream is not None:
        for t in tensors:
            if t.is_cuda:
                t.record_stream(torch.cuda.current_stream(t.device))


def _empty(shape, dtype, device, stream, handed_out=True):
    """A buffer made for a call on `stream`: one that the caller gets, or a workspace."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _on(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if handed_out:
        _handed_out(stream, t)
    return t


@functools.lru_cache(maxsize=256)
def _geom_ref(cls, *fields):
    """Reference to a geometry struct (read only, kept for the next call with the same fields)."""
    return ctypes.byref(cls(*fields))


@dataclass
class Geometry:
    n_seqs: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int = 128
    parent_size: int = 512
    reps_per_parent: int = 32
    elem_type: int = 0               # SANTAPP_BF16; 1 = SANTAPP_FP16

    def c(self) -> CGeom:
        return CGeom(self.n_seqs, self.n_q_heads, self.n_kv_heads, self.head_dim, self.parent_size,
                     self.reps_per_parent, self.elem_type)

    def ref(self):
        return _geom_ref(CGeom, self.n_seqs, self.n_q_heads, self.n_kv_heads, self.head_dim, self.parent_size,
                         self.reps_per_parent, self.elem_type)

    @property
    def torch_dtype(self):
        return torch.float16 if self.elem_type == SANTAPP_FP16 else torch.bfloat16


@dataclass
class Sizes:
    rows_total: int
    teams_total: int
    max_teams_per_seq: int
    max_rows_per_seq: int
    team_row_start_elems: int
    build_workspace_bytes: int


class Teams:
    """Team records of one layer: device tensors plus the C struct that points at them."""

    def __init__(self, geom: Geometry, sizes: Sizes, device):
        d = geom.head_dim
        kv = geom.n_kv_heads
        self.geom = geom
        self.sizes = sizes
        self.k_packed = torch.empty((kv, sizes.rows_total, d), dtype=geom.torch_dtype, device=device)
        self.v_packed = torch.empty_like(self.k_packed)
        self.rep_keys = torch.empty((kv, sizes.teams_total, d), dtype=geom.torch_dtype, device=device)
        self.team_row_start = torch.empty((kv, sizes.teams_total + geom.n_seqs), dtype=torch.int32, device=device)
        self.row_token = torch.empty((kv, sizes.rows_total), dtype=torch.int32, device=device)
        self.seq_row_off = torch.empty(geom.n_seqs + 1, dtype=torch.int64, device=device)
        self.seq_team_off = torch.empty(geom.n_seqs + 1, dtype=torch.int64, device=device)
        self.rep_abs_max = torch.empty((kv, geom.n_seqs), dtype=torch.float32, device=device)
        self.team_count = torch.empty((kv, geom.n_seqs), dtype=torch.int32, device=device)
        self.c = CTeams(self.k_packed.data_ptr(), self.v_packed.data_ptr(), self.rep_keys.data_ptr(),
                        self.team_row_start.data_ptr(), self.row_token.data_ptr(),
                        self.seq_row_off.data_ptr(), self.seq_team_off.data_ptr(), self.rep_abs_max.data_ptr(),
                        self.team_count.data_ptr(), sizes.rows_total, sizes.teams_total, sizes.max_teams_per_seq, sizes.max_rows_per_seq)

    def tensors(self):
        return [x for x in vars(self).values() if isinstance(x, torch.Tensor)]


def santapp_version() -> int:
    return load_library().santapp_version()


def santapp_last_launch_count() -> int:
    return load_library().santapp_last_launch_count()


def santapp_set_stage_mask(mask: int) -> None:
    load_library().santapp_set_stage_mask(mask)


def santapp_build_teams_sizes(geom: Geometry, prompt_len) -> Sizes:
    L = load_library()
    n = len(prompt_len)
    arr = (ctypes.c_int32 * n)(*[int(x) for x in prompt_len])
    out = CSizes()
    _check(L.santapp_build_teams_sizes(geom.ref(), arr, ctypes.byref(out)))
    return Sizes(out.rows_total, out.teams_total, out.max_teams_per_seq, out.max_rows_per_seq,
                 out.team_row_start_elems, out.build_workspace_bytes)


def santapp_build_groups_mean(geom: Geometry, prompt_len, k_prompt: torch.Tensor, v_prompt: torch.Tensor,
                              stream=None) -> Teams:
    """Centroid-guided grouping: one group per contiguous parent, routed by its mean key
    (geom.reps_per_parent must be 1). Arguments as for santapp_build_teams."""
    return santapp_build_teams(geom, prompt_len, k_prompt, v_prompt, stream, _entry="santapp_build_groups_mean")


def santapp_build_teams(geom: Geometry, prompt_len, k_prompt: torch.Tensor, v_prompt: torch.Tensor,
                        stream=None, _entry: str = "santapp_build_teams") -> Teams:
    """k_prompt, v_prompt: bf16 CUDA tensors [n_kv_heads, rows_total, d] in token order."""
    L = load_library()
    sizes = santapp_build_teams_sizes(geom, prompt_len)
    with _on(stream):
        teams = Teams(geom, sizes, k_prompt.device)
        ws = torch.empty(max(sizes.build_workspace_bytes, 256), dtype=torch.uint8, device=k_prompt.device)
    _handed_out(stream, *teams.tensors())
    n = len(prompt_len)
    arr = (ctypes.c_int32 * n)(*[int(x) for x in prompt_len])
    _check(getattr(L, _entry)(geom.ref(), arr, _ptr(k_prompt), _ptr(v_prompt), ctypes.byref(teams.c),
                              _ptr(ws), ws.numel(), _stream_ptr(stream)))
    teams._build_ws = ws      # keep alive until the stream has consumed it
    return teams


def _i32_array(values):
    return (ctypes.c_int32 * len(values))(*[int(x) for x in values])


def santapp_kmeans_parent_count(prompt_len: int, parent_size: int) -> int:
    """First line of Algorithm 3: min(N, max(2, N // P)); 0 for N < 2 or P < 1."""
    return int(load_library().santapp_kmeans_parent_count(int(prompt_len), int(parent_size)))


def santapp_kmeans_fit(geom: Geometry, prompt_len, n_centres, k_prompt: torch.Tensor, batch_size: int = 4096,
                       max_iter: int = 100, patience: int = 10, reassignment_ratio: float = 0.01, seed: int = 0,
                       stream_base: int = 0, stream=None, no_host_poll: bool = False):
    """Minibatch k-means fit per (sequence, KV head); the defaults are the paper's settings.
    Returns (centres fp32 [n_kv_heads, sum(n_centres), d], steps int32 [n_kv_heads, n_seqs]; -1: the
    fit's start gave up, see santapp.h)."""
    L = load_library()
    o = CKmeansOpts(batch_size, max_iter, patience, 1 if no_host_poll else 0, reassignment_ratio, seed, stream_base, 0)
    n, c = _i32_array(prompt_len), _i32_array(n_centres)
    need = int(L.santapp_kmeans_fit_workspace_bytes(geom.ref(), n, c, ctypes.byref(o)))
    if need == 0:
        raise SantappError(SANTAPP_ERR_INVALID_ARG, "k-means fit arguments")
    dev = k_prompt.device
    with _on(stream):
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        centres = torch.empty((geom.n_kv_heads, int(sum(n_centres)), geom.head_dim), dtype=torch.float32, device=dev)
        steps = torch.zeros((geom.n_kv_heads, geom.n_seqs), dtype=torch.int32, device=dev)
    _handed_out(stream, centres, steps)
    _check(L.santapp_kmeans_fit(geom.ref(), n, c, _ptr(k_prompt), ctypes.byref(o), _ptr(centres), _ptr(steps),
                                _ptr(ws), ws.numel(), _stream_ptr(stream)))
    centres._ws = ws
    return centres, steps


def santapp_assign_parents(geom: Geometry, prompt_len, n_centres, k_prompt: torch.Tensor, centres: torch.Tensor,
                           stream=None) -> torch.Tensor:
    """Nearest-centre label of every token. centres: fp32 CUDA tensor [n_kv_heads, sum(n_centres), d].
    Returns int32 [n_kv_heads, rows_total]."""
    L = load_library()
    if centres.dtype != torch.float32:
        raise SantappError(SANTAPP_ERR_INVALID_ARG, "centres must be float32")
    with _on(stream):
        parent_of = torch.empty((geom.n_kv_heads, k_prompt.shape[1]), dtype=torch.int32, device=k_prompt.device)
        ws = torch.empty(max(int(L.santapp_assign_parents_workspace_bytes(geom.ref())), 256), dtype=torch.uint8,
                         device=k_prompt.device)
    _handed_out(stream, parent_of)
    _check(L.santapp_assign_parents(geom.ref(), _i32_array(prompt_len), _i32_array(n_centres), _ptr(k_prompt),
                                    _ptr(centres), _ptr(parent_of), _ptr(ws), ws.numel(), _stream_ptr(stream)))
    parent_of._ws = ws
    return parent_of


def santapp_parent_teams_sizes(geom: Geometry, prompt_len, n_parents) -> Sizes:
    L = load_library()
    out = CSizes()
    _check(L.santapp_parent_teams_sizes(geom.ref(), _i32_array(prompt_len), _i32_array(n_parents),
                                        ctypes.byref(out)))
    return Sizes(out.rows_total, out.teams_total, out.max_teams_per_seq, out.max_rows_per_seq,
                 out.team_row_start_elems, out.build_workspace_bytes)


def santapp_build_groups_mean_parents(geom: Geometry, prompt_len, n_parents, k_prompt: torch.Tensor,
                                      v_prompt: torch.Tensor, parent_of: torch.Tensor, stream=None) -> Teams:
    """Centroid-guided groups on a given partition (geom.reps_per_parent must be 1)."""
    return santapp_build_teams_parents(geom, prompt_len, n_parents, k_prompt, v_prompt, parent_of, stream,
                                       _entry="santapp_build_groups_mean_parents")


def santapp_build_teams_parents(geom: Geometry, prompt_len, n_parents, k_prompt: torch.Tensor,
                                v_prompt: torch.Tensor, parent_of: torch.Tensor, stream=None,
                                _entry: str = "santapp_build_teams_parents") -> Teams:
    """Team records from a parent label per token (int32 CUDA tensor [n_kv_heads, rows_total])."""
    L = load_library()
    sizes = santapp_parent_teams_sizes(geom, prompt_len, n_parents)
    with _on(stream):
        teams = Teams(geom, sizes, k_prompt.device)
        ws = torch.empty(max(sizes.build_workspace_bytes, 256), dtype=torch.uint8, device=k_prompt.device)
    _handed_out(stream, *teams.tensors())
    if parent_of.dtype != torch.int32:
        raise SantappError(SANTAPP_ERR_INVALID_ARG, "parent_of must be int32")
    _check(getattr(L, _entry)(geom.ref(), _i32_array(prompt_len), _i32_array(n_parents),
                              _ptr(k_prompt), _ptr(v_prompt), _ptr(parent_of), ctypes.byref(teams.c),
                              _ptr(ws), ws.numel(), _stream_ptr(stream)))
    teams._build_ws = ws      # keep alive until the stream has consumed it
    return teams


def santapp_decode_workspace_bytes(geom: Geometry, teams: Teams, n_sample: int) -> int:
    return int(load_library().santapp_decode_workspace_bytes(geom.ref(), ctypes.byref(teams.c), n_sample))


def santapp_dense_workspace_bytes(geom: Geometry, teams: Teams) -> int:
    return int(load_library().santapp_dense_workspace_bytes(geom.ref(), ctypes.byref(teams.c)))


class DebugBuffers:
    """Optional per-step diagnostics (device tensors)."""

    def __init__(self, geom: Geometry, n_sample: int, device, trace: bool = False):
        B, Hq, Hkv = geom.n_seqs, geom.n_q_heads, geom.n_kv_heads
        self.trace = torch.zeros((5, 256, 16), dtype=torch.int64, device=device) if trace else None
        self.sel_idx = torch.full((B, Hq, n_sample), -1, dtype=torch.int32, device=device)
        self.sel_logc = torch.zeros((B, Hq, n_sample), dtype=torch.float32, device=device)
        self.tau = torch.zeros((B, Hq), dtype=torch.float64, device=device)
        self.union_rows = torch.zeros((B, Hkv), dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.c = CDebug(self.sel_idx.data_ptr(), self.sel_logc.data_ptr(), self.tau.data_ptr(),
                        self.union_rows.data_ptr(), self.status.data_ptr(),
                        self.trace.data_ptr() if trace else None)


def santapp_decode_attn(geom: Geometry, teams: Teams, q: torch.Tensor, k_suffix: Optional[torch.Tensor],
                        v_suffix: Optional[torch.Tensor], suffix_len: Optional[torch.Tensor], n_sample: int,
                        seed: int, step: int, stream_base: int = 0, scale: float = 0.0,
                        out: Optional[torch.Tensor] = None, debug: Optional[DebugBuffers] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None,
                        step_dev: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q bf16 [B, Hq, d]; k_suffix/v_suffix bf16 [B, Hkv, cap, d]; suffix_len int32 [B] (device);
    step_dev optional device int32/uint32 [1] added to `step` on the device."""
    L = load_library()
    if out is None:
        out = _empty((geom.n_seqs, geom.n_q_heads, geom.head_dim), torch.float32, q.device, stream)
    if workspace is None:
        workspace = _empty(santapp_decode_workspace_bytes(geom, teams, n_sample), torch.uint8, q.device, stream, False)
    cap = 0 if k_suffix is None else int(k_suffix.shape[2])
    _check(L.santapp_decode_attn(geom.ref(), ctypes.byref(teams.c), _ptr(q), _ptr(k_suffix), _ptr(v_suffix),
                                 _ptr(suffix_len), cap, n_sample, int(seed), step, _ptr(step_dev),
                                 stream_base, scale, _ptr(out), ctypes.byref(debug.c) if debug is not None else None,
                                 _ptr(workspace), workspace.numel(), _stream_ptr(stream)))
    return out


def santapp_dense_decode_attn(geom: Geometry, teams: Teams, q: torch.Tensor, k_suffix: Optional[torch.Tensor],
                              v_suffix: Optional[torch.Tensor], suffix_len: Optional[torch.Tensor],
                              scale: float = 0.0, out: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    L = load_library()
    if out is None:
        out = _empty((geom.n_seqs, geom.n_q_heads, geom.head_dim), torch.float32, q.device, stream)
    if workspace is None:
        workspace = _empty(santapp_dense_workspace_bytes(geom, teams), torch.uint8, q.device, stream, False)
    cap = 0 if k_suffix is None else int(k_suffix.shape[2])
    _check(L.santapp_dense_decode_attn(geom.ref(), ctypes.byref(teams.c), _ptr(q), _ptr(k_suffix),
                                       _ptr(v_suffix), _ptr(suffix_len), cap, scale, _ptr(out), _ptr(workspace),
                                       workspace.numel(), _stream_ptr(stream)))
    return out


def santapp_dense_decode_attn_noalloc(geom: Geometry, teams: Teams, q: torch.Tensor,
                                      k_suffix: Optional[torch.Tensor], v_suffix: Optional[torch.Tensor],
                                      suffix_len: Optional[torch.Tensor], scale: float = 0.0,
                                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense decode attention that takes no workspace: for callers that cannot allocate device
    memory around the call, the scratch lives in a fixed array inside the library. Pass `out` to
    keep the call itself free of any allocation; if it is omitted this wrapper (not the library)
    creates the output tensor. Same result as santapp_dense_decode_attn. Calls share the array,
    so do not let two of them overlap on the GPU; the first call on a device should come
    before any stream capture."""
    L = load_library()
    if out is None:
        out = _empty((geom.n_seqs, geom.n_q_heads, geom.head_dim), torch.float32, q.device, stream)
    cap = 0 if k_suffix is None else int(k_suffix.shape[2])
    _check(L.santapp_dense_decode_attn_noalloc(geom.ref(), ctypes.byref(teams.c), _ptr(q), _ptr(k_suffix),
                                               _ptr(v_suffix), _ptr(suffix_len), cap, scale, _ptr(out),
                                               _stream_ptr(stream)))
    return out


# ------------------------------------------------------------------------------------------------
# Shared-latent rows (include/santapp_latent.h)
# ------------------------------------------------------------------------------------------------
@dataclass
class LatentGeometry:
    n_seqs: int
    n_heads: int = 16
    parent_size: int = 16
    reps_per_parent: int = 4

    def c(self) -> CLatentGeom:
        return CLatentGeom(self.n_seqs, self.n_heads, self.parent_size, self.reps_per_parent)

    def ref(self):
        return _geom_ref(CLatentGeom, self.n_seqs, self.n_heads, self.parent_size, self.reps_per_parent)


class LatentTeams:
    """Team records of shared-latent rows: device tensors plus the C struct that points at them."""

    def __init__(self, geom: LatentGeometry, sizes: Sizes, device):
        self.geom = geom
        self.sizes = sizes
        self.rows_packed = torch.empty((sizes.rows_total, LATENT_ROW), dtype=torch.bfloat16, device=device)
        self.rep_rows = torch.empty((sizes.teams_total, LATENT_ROW), dtype=torch.bfloat16, device=device)
        self.team_row_start = torch.empty(sizes.teams_total + geom.n_seqs, dtype=torch.int32, device=device)
        self.row_token = torch.empty(sizes.rows_total, dtype=torch.int32, device=device)
        self.seq_row_off = torch.empty(geom.n_seqs + 1, dtype=torch.int64, device=device)
        self.seq_team_off = torch.empty(geom.n_seqs + 1, dtype=torch.int64, device=device)
        self.rep_abs_max = torch.empty(geom.n_seqs, dtype=torch.float32, device=device)
        self.c = CLatentTeams(self.rows_packed.data_ptr(), self.rep_rows.data_ptr(), self.team_row_start.data_ptr(),
                              self.row_token.data_ptr(), self.seq_row_off.data_ptr(), self.seq_team_off.data_ptr(),
                              self.rep_abs_max.data_ptr(), sizes.rows_total, sizes.teams_total,
                              sizes.max_teams_per_seq, sizes.max_rows_per_seq)

    tensors = Teams.tensors


def santapp_latent_sizes(geom: LatentGeometry, prompt_len) -> Sizes:
    L = load_library()
    out = CSizes()
    _check(L.santapp_latent_sizes(geom.ref(), _i32_array(prompt_len), ctypes.byref(out)))
    return Sizes(out.rows_total, out.teams_total, out.max_teams_per_seq, out.max_rows_per_seq,
                 out.team_row_start_elems, out.build_workspace_bytes)


def santapp_latent_build_teams(geom: LatentGeometry, prompt_len, rows_prompt: torch.Tensor, stream=None) -> LatentTeams:
    """rows_prompt: bf16 CUDA tensor [rows_total, 576] in token order (512 latent values, 64 rotary)."""
    L = load_library()
    sizes = santapp_latent_sizes(geom, prompt_len)
    with _on(stream):
        teams = LatentTeams(geom, sizes, rows_prompt.device)
        ws = torch.empty(max(sizes.build_workspace_bytes, 256), dtype=torch.uint8, device=rows_prompt.device)
    _handed_out(stream, *teams.tensors())
    _check(L.santapp_latent_build_teams(geom.ref(), _i32_array(prompt_len), _ptr(rows_prompt), ctypes.byref(teams.c),
                                        _ptr(ws), ws.numel(), _stream_ptr(stream)))
    teams._build_ws = ws
    return teams


def santapp_latent_decode_workspace_bytes(geom: LatentGeometry, teams: LatentTeams, n_sample: int, suffix_cap: int) -> int:
    return int(load_library().santapp_latent_decode_workspace_bytes(geom.ref(), ctypes.byref(teams.c), n_sample,
                                                                    suffix_cap))


def santapp_latent_dense_workspace_bytes(geom: LatentGeometry, teams: LatentTeams) -> int:
    return int(load_library().santapp_latent_dense_workspace_bytes(geom.ref(), ctypes.byref(teams.c)))


class LatentDebugBuffers(DebugBuffers):
    """Diagnostics of a shared-latent step: per (sequence, head) samples, per sequence union rows."""

    def __init__(self, geom: LatentGeometry, n_sample: int, device):
        super().__init__(Geometry(geom.n_seqs, geom.n_heads, 1), n_sample, device)


def santapp_latent_decode_attn(geom: LatentGeometry, teams: LatentTeams, q: torch.Tensor,
                               suffix_rows: Optional[torch.Tensor], suffix_len: Optional[torch.Tensor], n_sample: int,
                               seed: int, step: int, scale: float, stream_base: int = 0,
                               out: Optional[torch.Tensor] = None, debug: Optional[DebugBuffers] = None,
                               workspace: Optional[torch.Tensor] = None, stream=None,
                               step_dev: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q bf16 [B, H, 576]; suffix_rows bf16 [B, cap, 576]; suffix_len int32 [B] (device). Returns fp32 [B, H, 512]."""
    L = load_library()
    cap = 0 if suffix_rows is None else int(suffix_rows.shape[1])
    if out is None:
        out = _empty((geom.n_seqs, geom.n_heads, LATENT_DIM), torch.float32, q.device, stream)
    if workspace is None:
        workspace = _empty(santapp_latent_decode_workspace_bytes(geom, teams, n_sample, cap), torch.uint8, q.device, stream, False)
    _check(L.santapp_latent_decode_attn(geom.ref(), ctypes.byref(teams.c), _ptr(q), _ptr(suffix_rows),
                                        _ptr(suffix_len), cap, n_sample, int(seed), step, _ptr(step_dev),
                                        stream_base, scale, _ptr(out),
                                        ctypes.byref(debug.c) if debug is not None else None, _ptr(workspace),
                                        workspace.numel(), _stream_ptr(stream)))
    return out


def santapp_latent_dense_decode_attn(geom: LatentGeometry, teams: LatentTeams, q: torch.Tensor,
                                     suffix_rows: Optional[torch.Tensor], suffix_len: Optional[torch.Tensor],
                                     scale: float, out: Optional[torch.Tensor] = None,
                                     workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    L = load_library()
    cap = 0 if suffix_rows is None else int(suffix_rows.shape[1])
    if out is None:
        out = _empty((geom.n_seqs, geom.n_heads, LATENT_DIM), torch.float32, q.device, stream)
    if workspace is None:
        workspace = _empty(santapp_latent_dense_workspace_bytes(geom, teams), torch.uint8, q.device, stream, False)
    _check(L.santapp_latent_dense_decode_attn(geom.ref(), ctypes.byref(teams.c), _ptr(q), _ptr(suffix_rows),
                                              _ptr(suffix_len), cap, scale, _ptr(out), _ptr(workspace),
                                              workspace.numel(), _stream_ptr(stream)))
    return out


# ------------------------------------------------------------------------------------------------
# Around the decode step (include/santapp_serve.h)
# ------------------------------------------------------------------------------------------------
def _refuse(why):
    raise SantappError(SANTAPP_ERR_INVALID_ARG, why)


def _device():
    """The current device's index, which no tensor has where there is none."""
    try:
        return torch._C._cuda_getDevice()
    except RuntimeError:
        return -2


def _wrong(name, t, shape, dtype, dense):
    if not t.is_cuda or t.get_device() != _device():
        _refuse(f"{name} must be a CUDA tensor on the current device")
    if t.dtype != dtype:
        _refuse(f"{name} must be {dtype}")
    if t.shape != shape:
        _refuse(f"{name} must have the shape {list(shape)}, not {list(t.shape)}")
    _refuse(f"{name} must be contiguous" + ("" if dense else " behind its first dimension"))


def _expect(name, t, shape, dtype, device):
    """The address of a dense tensor of this shape and type on this device."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _wrong(name, t, shape, dtype, True)
    return t.data_ptr()


def _expect_planes(name, t, shape, dtype, device):
    """The same where the first dimension may have any stride: address and stride (of one plane: what a dense tensor has)."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _wrong(name, t, shape, dtype, False)
    steps, plane = t.stride(), shape[1] * shape[2] if len(shape) == 3 else shape[1]
    if steps[1:] != ((shape[2], 1) if len(shape) == 3 else (1,)) and plane and not t[0].is_contiguous():
        _wrong(name, t, shape, dtype, False)
    return t.data_ptr(), steps[0] if shape[0] > 1 else plane


def _expect_or_none(name, t, shape, dtype, device):
    return None if t is None else _expect(name, t, shape, dtype, device)


class Rope:
    """Rotary positions. factor > 1 scales the frequencies for long contexts: with original_len by their turns over the
    trained length (`low`, `high`), without it all alike (santapp_rope_frequencies). `inv_freq` replaces them all."""

    def __init__(self, rot_dim: int = 128, theta: float = 10000.0, interleaved: bool = False, factor: float = 1.0,
                 low: float = 1.0, high: float = 4.0, original_len: float = 0.0, amplitude: float = 1.0, inv_freq=None):
        self.c = CRope(rot_dim, 1 if interleaved else 0, amplitude)
        if inv_freq is None:
            _check(load_library().santapp_rope_frequencies(ctypes.byref(self.c), theta, factor, low, high, original_len))
        else:
            values = [float(x) for x in inv_freq]
            if len(values) != rot_dim // 2 or rot_dim > 128:
                _refuse("inv_freq holds rot_dim / 2 values")
            self.c.inv_freq[:len(values)] = values
        self.ref = ctypes.byref(self.c)

    @property
    def inv_freq(self):
        return list(self.c.inv_freq[:self.c.rot_dim // 2])


def _rope_rows(geom, n, q, k, v, q_out, device, stream):
    d, kv, dt = geom.head_dim, geom.n_kv_heads, geom.torch_dtype
    heads, keys = (n, geom.n_q_heads, d), (n, kv, d)
    if q_out is None:
        q_out = _empty(heads, dt, q.device, stream)
    return (q_out, *_expect_planes("q", q, heads, dt, device), *_expect_planes("k", k, keys, dt, device),
            *_expect_planes("v", v, keys, dt, device), _expect("q_out", q_out, heads, dt, device))


def santapp_rope_append(geom: Geometry, rope: Rope, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                        base_pos: torch.Tensor, suffix_len: torch.Tensor, k_suffix: torch.Tensor, v_suffix: torch.Tensor,
                        q_out: Optional[torch.Tensor] = None, suffix_len_out: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """q [B, Hq, d], k and v [B, Hkv, d] (any stride between tokens); base_pos, suffix_len int32 [B]; k_suffix, v_suffix
    [B, Hkv, cap, d]. Row suffix_len[b] is written, q_out returned; suffix_len_out (may be suffix_len) gets suffix_len + 1."""
    B, dt, i32, dev = geom.n_seqs, geom.torch_dtype, torch.int32, _device()
    q_out, qp, qs, kp, ks, vp, vs, dst = _rope_rows(geom, B, q, k, v, q_out, dev, stream)
    cap, one = k_suffix.shape[2], (B,)
    shape = (B, geom.n_kv_heads, cap, geom.head_dim)
    _check(load_library().santapp_rope_append(
        geom.ref(), rope.ref, qp, qs, kp, ks, vp, vs, _expect("base_pos", base_pos, one, i32, dev),
        _expect("suffix_len", suffix_len, one, i32, dev), dst, _expect("k_suffix", k_suffix, shape, dt, dev),
        _expect("v_suffix", v_suffix, shape, dt, dev), cap, _expect_or_none("suffix_len_out", suffix_len_out, one, i32, dev),
        _stream_ptr(stream)))
    return q_out


def santapp_rope_prompt(geom: Geometry, rope: Rope, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                        positions: Optional[torch.Tensor], k_prompt: torch.Tensor, v_prompt: torch.Tensor,
                        dst_row: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """q [n, Hq, d], k and v [n, Hkv, d] (any stride between tokens); positions, dst_row int32 [n] or None (the row's
    index); k_prompt, v_prompt [Hkv, rows, d], written at dst_row. Returns q_out [n, Hq, d]."""
    n, dt, i32, dev = q.shape[0], geom.torch_dtype, torch.int32, _device()
    q_out, qp, qs, kp, ks, vp, vs, dst = _rope_rows(geom, n, q, k, v, q_out, dev, stream)
    rows = k_prompt.shape[1]
    shape = (geom.n_kv_heads, rows, geom.head_dim)
    _check(load_library().santapp_rope_prompt(
        geom.ref(), rope.ref, n, qp, qs, kp, ks, vp, vs, _expect_or_none("positions", positions, (n,), i32, dev),
        _expect_or_none("dst_row", dst_row, (n,), i32, dev), dst, _expect("k_prompt", k_prompt, shape, dt, dev),
        _expect("v_prompt", v_prompt, shape, dt, dev), rows, _stream_ptr(stream)))
    return q_out


def santapp_suffix_fork(geom: Geometry, src: torch.Tensor, suffix_len: torch.Tensor, k_suffix: torch.Tensor,
                        v_suffix: torch.Tensor, suffix_len_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Slot b of k_suffix / v_suffix [B, Hkv, cap, d] continues slot src[b] (int32 [B]; outside [0, B): freed), in place;
    suffix_len_out (not suffix_len) gets the new lengths."""
    B, dt, i32, dev = geom.n_seqs, geom.torch_dtype, torch.int32, _device()
    cap, one = k_suffix.shape[2], (B,)
    shape = (B, geom.n_kv_heads, cap, geom.head_dim)
    _check(load_library().santapp_suffix_fork(
        geom.ref(), _expect("src", src, one, i32, dev), _expect("suffix_len", suffix_len, one, i32, dev),
        _expect("k_suffix", k_suffix, shape, dt, dev), _expect("v_suffix", v_suffix, shape, dt, dev), cap,
        _expect_or_none("suffix_len_out", suffix_len_out, one, i32, dev), _stream_ptr(stream)))


def santapp_prefix_decode_workspace_bytes(geom: Geometry, prefix_len: int, suffix_cap: int) -> int:
    return int(load_library().santapp_prefix_decode_workspace_bytes(geom.ref(), prefix_len, suffix_cap))


def _attn_opts(geom, scale, cap, slopes, status, device):
    return CAttnOpts(scale, cap, _expect_or_none("slopes", slopes, (geom.n_q_heads,), torch.float32, device),
                     _expect_or_none("status", status, (1,), torch.int32, device))


def santapp_prefix_decode_attn(geom: Geometry, k_prefix: Optional[torch.Tensor], v_prefix: Optional[torch.Tensor],
                               q: torch.Tensor, k_suffix: Optional[torch.Tensor], v_suffix: Optional[torch.Tensor],
                               suffix_len: Optional[torch.Tensor], scale: float = 0.0, cap: float = 0.0,
                               slopes: Optional[torch.Tensor] = None, prefix_token: Optional[torch.Tensor] = None,
                               out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                               status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One prompt for the whole batch: k_prefix, v_prefix [Hkv, N, d] (the planes may lie further apart; None: no prompt),
    prefix_token int32 of the same planes or None; q [B, Hq, d]; suffix as in santapp_decode_attn. fp32 [B, Hq, d]."""
    B, kv, d, dt, dev = geom.n_seqs, geom.n_kv_heads, geom.head_dim, geom.torch_dtype, _device()
    heads = (B, geom.n_q_heads, d)
    n = plane = suffix_cap = 0
    kp = vp = tok = ks = vs = None
    if k_prefix is not None:
        n = k_prefix.shape[1]
        kp, apart = _expect_planes("k_prefix", k_prefix, (kv, n, d), dt, dev)
        vp, v_apart = _expect_planes("v_prefix", v_prefix, (kv, n, d), dt, dev)
        plane = apart // d
        if apart % d or v_apart != apart:
            _refuse("the planes of k_prefix and v_prefix must lie whole rows and equally far apart")
        if prefix_token is not None:
            tok, t_apart = _expect_planes("prefix_token", prefix_token, (kv, n), torch.int32, dev)
            if t_apart != plane:
                _refuse("the planes of prefix_token must lie as far apart as those of k_prefix")
    if k_suffix is not None:
        suffix_cap = k_suffix.shape[2]
        ks = _expect("k_suffix", k_suffix, (B, kv, suffix_cap, d), dt, dev)
        vs = _expect("v_suffix", v_suffix, (B, kv, suffix_cap, d), dt, dev)
    if out is None:
        out = _empty(heads, torch.float32, q.device, stream)
    if workspace is None:
        workspace = _empty(santapp_prefix_decode_workspace_bytes(geom, n, suffix_cap), torch.uint8, q.device, stream, False)
    size = workspace.numel()
    o = _attn_opts(geom, scale, cap, slopes, status, dev)
    _check(load_library().santapp_prefix_decode_attn(
        geom.ref(), kp, vp, n, plane, tok, _expect("q", q, heads, dt, dev), ks, vs,
        _expect_or_none("suffix_len", suffix_len, (B,), torch.int32, dev), suffix_cap, ctypes.byref(o),
        _expect("out", out, heads, torch.float32, dev), _expect("workspace", workspace, (size,), torch.uint8, dev), size,
        _stream_ptr(stream)))
    return out


def santapp_prompt_attn(geom: Geometry, prompt_len, q: torch.Tensor, k_prompt: torch.Tensor, v_prompt: torch.Tensor,
                        new_len=None, prefix_len=None, scale: float = 0.0, cap: float = 0.0,
                        slopes: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """q [sum(new_len or prompt_len), Hq, d]: the last new_len rows of each sequence; k_prompt, v_prompt
    [Hkv, sum(prompt_len), d]. Returns the element type, shaped like q."""
    if len(prompt_len) != geom.n_seqs or any(x is not None and len(x) != geom.n_seqs for x in (new_len, prefix_len)):
        _refuse("prompt_len, new_len and prefix_len hold a length per sequence")
    dt, dev = geom.torch_dtype, _device()
    heads, keys = (sum(prompt_len if new_len is None else new_len), geom.n_q_heads, geom.head_dim), \
        (geom.n_kv_heads, sum(prompt_len), geom.head_dim)
    if heads[0] < 0 or keys[1] < 0:
        _refuse("prompt_len and new_len hold no negative lengths")
    if out is None:
        out = _empty(heads, dt, q.device, stream)
    o = _attn_opts(geom, scale, cap, slopes, status, dev)
    _check(load_library().santapp_prompt_attn(
        geom.ref(), _i32_array(prompt_len), None if new_len is None else _i32_array(new_len),
        None if prefix_len is None else _i32_array(prefix_len), _expect("q", q, heads, dt, dev),
        _expect("k_prompt", k_prompt, keys, dt, dev), _expect("v_prompt", v_prompt, keys, dt, dev), ctypes.byref(o),
        _expect("out", out, heads, dt, dev), _stream_ptr(stream)))
    return out


def bf16_bits_to_cuda(bits, device="cuda", dtype=torch.bfloat16):
    """numpy uint16 bit patterns -> CUDA tensor of the 16-bit `dtype` (no value conversion)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(dtype)
