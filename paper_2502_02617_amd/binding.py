"""ctypes binding of libpolarquant (argument marshalling only).

Function names mirror the C ABI: ``Context`` wraps ``pq_init_preconditioner`` /
``pq_destroy`` and its methods call ``pq_encode_kv``, ``pq_append_kv``, ``pq_append_kv_pair``,
``pq_decode_kv``, ``pq_export_canonical``, ``pq_attn_decode_polar``, ``pq_attn_decode_hybrid`` and ``pq_decode_step_polar`` with
pointers of torch tensors (torch is used for device memory and streams only).
"""
import ctypes
import os

import numpy as np

from . import _build

PQ_F32, PQ_BF16 = 0, 1
PQ_KEY, PQ_VALUE = 0, 1
TILE_TOKENS = 64
TILE_CODE_BYTES = 2944
TILE_RADII = 512
RECORD_BYTES = 62
D = 128

_lib = None


class PolarQuantError(RuntimeError):
    pass


def library():
    """Loads the in-tree libpolarquant.so (building it first if it is absent)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB_PATH
    if not os.path.exists(path):
        _build.build()
    L = ctypes.CDLL(path)
    vp, i64, i32, u64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint64
    L.pq_status_string.restype = ctypes.c_char_p
    L.pq_status_string.argtypes = [i32]
    L.pq_init_preconditioner.restype = i32
    L.pq_init_preconditioner.argtypes = [ctypes.POINTER(vp), i32, u64, vp]
    L.pq_init_preconditioner_hadamard.restype = i32
    L.pq_init_preconditioner_hadamard.argtypes = [ctypes.POINTER(vp), i32, u64]
    L.pq_set_codebooks.restype = i32
    L.pq_set_codebooks.argtypes = [vp, vp]
    L.pq_fit_codebooks.restype = i32
    L.pq_fit_codebooks.argtypes = [vp, vp, i32, i64, i32, i64, i64, vp, i32, vp, vp, ctypes.c_size_t, vp]
    L.pq_fit_codebooks_deep.restype = i32
    L.pq_fit_codebooks_deep.argtypes = [vp, vp, i32, i64, i32, i64, i64, vp, vp, i32, vp, vp, vp, ctypes.c_size_t, vp]
    L.pq_fit_workspace_bytes.restype = ctypes.c_size_t
    L.pq_fit_workspace_bytes.argtypes = []
    L.pq_fit_count_angles.restype = i32
    L.pq_fit_count_angles.argtypes = [vp, vp, i32, i64, i32, i64, i64, vp, ctypes.c_size_t, vp]
    L.pq_fit_cluster.restype = i32
    L.pq_fit_cluster.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    L.pq_set_recursion_depth.restype = i32
    L.pq_set_recursion_depth.argtypes = [vp, i32, vp]
    L.pq_set_upper_codebooks.restype = i32
    L.pq_set_upper_codebooks.argtypes = [vp, vp]
    L.pq_recursion_depth.restype = i32
    L.pq_recursion_depth.argtypes = [vp]
    L.pq_preconditioner_structure.restype = i32
    L.pq_preconditioner_structure.argtypes = [vp]
    L.pq_radii_halves_per_tile.restype = i32
    L.pq_radii_halves_per_tile.argtypes = [vp]
    L.pq_record_bytes.restype = i32
    L.pq_record_bytes.argtypes = [vp]
    L.pq_get_upper_codebook.restype = i32
    L.pq_get_upper_codebook.argtypes = [vp, i32, vp, vp, vp]
    L.pq_get_preconditioner.restype = i32
    L.pq_get_preconditioner.argtypes = [vp, vp]
    L.pq_get_codebook.restype = i32
    L.pq_get_codebook.argtypes = [vp, i32, vp, vp]
    L.pq_destroy.restype = None
    L.pq_destroy.argtypes = [vp]
    L.pq_encode_kv.restype = i32
    L.pq_encode_kv.argtypes = [vp, vp, i32, i32, i64, i32, i64, i64, vp, vp, i64, i64, vp]
    L.pq_encode_kv_pair.restype = i32
    L.pq_encode_kv_pair.argtypes = [vp, vp, vp, i32, i64, i32, i64, i64, vp, vp, vp, vp, i64, i64, vp]
    L.pq_append_kv.restype = i32
    L.pq_append_kv.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, i64, vp, vp]
    L.pq_append_kv_pair.restype = i32
    L.pq_append_kv_pair.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, i64, vp, vp]
    L.pq_decode_kv.restype = i32
    L.pq_decode_kv.argtypes = [vp, i32, vp, vp, i64, i64, i64, i32, vp, i32, i64, i64, i32, vp]
    L.pq_export_canonical.restype = i32
    L.pq_export_canonical.argtypes = [vp, i32, vp, vp, i64, i64, i64, i32, vp, vp]
    L.pq_attn_decode_polar.restype = i32
    L.pq_attn_decode_polar.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, i64,
                                       ctypes.c_float, vp, ctypes.c_size_t, vp]
    L.pq_decode_step_polar.restype = i32
    L.pq_decode_step_polar.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, i64,
                                       ctypes.c_float, vp, ctypes.c_size_t, vp]
    L.pq_attn_decode_hybrid.restype = i32
    L.pq_attn_decode_hybrid.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, i64, i64,
                                        ctypes.c_float, vp, ctypes.c_size_t, vp]
    L.pq_attn_hybrid_workspace_bytes.restype = ctypes.c_size_t
    L.pq_attn_hybrid_workspace_bytes.argtypes = [i32, i32, i32, i64, i64]
    L.pq_attn_decode_polar_mq.restype = i32
    L.pq_attn_decode_polar_mq.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i64, i64,
                                          ctypes.c_float, vp, ctypes.c_size_t, vp]
    L.pq_attn_mq_workspace_bytes.restype = ctypes.c_size_t
    L.pq_attn_mq_workspace_bytes.argtypes = [i32, i32, i32, i32, i64]
    L.pq_attn_workspace_bytes.restype = ctypes.c_size_t
    L.pq_attn_workspace_bytes.argtypes = [i32, i32, i32, i64]
    L.pq_static_scratch_bytes.restype = ctypes.c_size_t
    L.pq_static_scratch_bytes.argtypes = []
    L.pq_prepare_device.restype = i32
    L.pq_prepare_device.argtypes = [vp]
    L.pq_attn_decode_polar_static.restype = i32
    L.pq_attn_decode_polar_static.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, i64,
                                              ctypes.c_float, vp]
    L.pq_append_paged.restype = i32
    L.pq_append_paged.argtypes = [vp, vp, vp, i32, i64, i32, i64, i64, vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, i32, vp]
    L.pq_decode_paged.restype = i32
    L.pq_decode_paged.argtypes = [vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, i32, i64, i32, vp, vp, i32, i64, i64, vp]
    L.pq_attn_paged.restype = i32
    L.pq_attn_paged.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, i32, i32, i32, i32, i64,
                                ctypes.c_float, vp, ctypes.c_size_t, vp]
    L.pq_attn_paged_workspace_bytes.restype = ctypes.c_size_t
    L.pq_attn_paged_workspace_bytes.argtypes = [i32, i32, i32, i32, i64]
    L.pq_attn_prefix_paged.restype = i32
    L.pq_attn_prefix_paged.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, i32, i32, i32, i32, i64, vp, i64, vp, vp, i32,
                                       i64, ctypes.c_float, vp, ctypes.c_size_t, vp]
    L.pq_attn_prefix_paged_workspace_bytes.restype = ctypes.c_size_t
    L.pq_attn_prefix_paged_workspace_bytes.argtypes = [i32, i32, i32, i32, i64, i32, i64]
    L.pq_general_record_bytes.restype = ctypes.c_size_t
    L.pq_general_record_bytes.argtypes = [vp]
    L.pq_general_codebook_entries.restype = i32
    L.pq_general_codebook_entries.argtypes = [vp]
    L.pq_general_codebooks.restype = i32
    L.pq_general_codebooks.argtypes = [vp, vp]
    L.pq_general_encode.restype = i32
    L.pq_general_encode.argtypes = [vp, vp, vp, vp, i32, i64, i64, vp, vp]
    L.pq_general_decode.restype = i32
    L.pq_general_decode.argtypes = [vp, vp, vp, vp, i64, i32, vp, vp]
    L.pq_general_attn_decode.restype = i32
    L.pq_general_attn_decode.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, ctypes.c_float, vp]
    L.pq_general_attn_workspace_bytes.restype = ctypes.c_size_t
    L.pq_general_attn_workspace_bytes.argtypes = [i32, i32, i32, i64]
    L.pq_general_attn_decode_ws.restype = i32
    L.pq_general_attn_decode_ws.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, ctypes.c_float, vp,
                                            ctypes.c_size_t, vp]
    L.pq_profile_begin.restype = i32
    L.pq_profile_begin.argtypes = [i32]
    L.pq_profile_begin_sampled.restype = i32
    L.pq_profile_begin_sampled.argtypes = [i32, i32]
    L.pq_profile_end.restype = i32
    L.pq_profile_end.argtypes = [vp, vp, vp, vp]
    L.pq_kernel_name_attn.restype = ctypes.c_char_p
    L.pq_kernel_name_encode.restype = ctypes.c_char_p
    _lib = L
    return L


def pq_status_string(code):
    return library().pq_status_string(int(code)).decode()


def profile_begin(max_launches, every=1):
    """Time at most max_launches launches of each of the two dominant kernels, every `every`-th one."""
    _check(library().pq_profile_begin_sampled(int(max_launches), int(every)))


def profile_end():
    """-> dict(attn_ms, attn_launches, encode_ms, encode_launches) of the launches timed since profile_begin."""
    a, e = ctypes.c_double(), ctypes.c_double()
    na, ne = ctypes.c_int(), ctypes.c_int()
    _check(library().pq_profile_end(ctypes.byref(a), ctypes.byref(na), ctypes.byref(e), ctypes.byref(ne)))
    return {"attn_ms": a.value, "attn_launches": na.value, "encode_ms": e.value, "encode_launches": ne.value}


def _check(code):
    if code != 0:
        raise PolarQuantError(pq_status_string(code))


def _stream():
    """The current device's current stream.  The raw handle takes 0.2 us, torch.cuda.current_stream() 2.8 (it builds a Stream):
    a fifth of what the host spends on a decode step."""
    import torch

    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None and torch.cuda.is_initialized():
        return raw(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t):
    global _dtype_codes
    if _dtype_codes is None:
        import torch

        _dtype_codes = {torch.bfloat16: PQ_BF16, torch.float32: PQ_F32}
    code = _dtype_codes.get(t.dtype)
    if code is None:
        raise PolarQuantError("only float32 and bfloat16 tensors are supported")
    return code


_dtype_codes = None


class Rotary(ctypes.Structure):
    """pq_rotary: position rotation by a table cos_sin, float32 device tensor [n_pos, dim], each row dim / 2 cosines, then dim / 2
    sines; pairs (i, i + dim / 2), or (2 i, 2 i + 1) if interleaved.  Keeps the tensor alive."""
    _fields_ = [("cos_sin", ctypes.c_void_p), ("n_pos", ctypes.c_int64), ("dim", ctypes.c_int), ("interleaved", ctypes.c_int)]

    def __init__(self, cos_sin, interleaved=False):
        import torch

        super().__init__()
        if cos_sin.dtype != torch.float32 or cos_sin.dim() != 2 or not cos_sin.is_contiguous() or not cos_sin.is_cuda:
            raise PolarQuantError("cos_sin must be a contiguous float32 device tensor [n_pos, dim]")
        self.tensor = cos_sin
        self.cos_sin, self.n_pos, self.dim, self.interleaved = cos_sin.data_ptr(), cos_sin.shape[0], cos_sin.shape[1], int(bool(interleaved))


def _int32():
    """torch.int32, without an import statement in the path of a call (0.4 us)."""
    global _int32_type
    if _int32_type is None:
        import torch

        _int32_type = torch.int32
    return _int32_type


_int32_type = None


def _ints(name, t, n):
    """Address of an int32 device vector of n entries."""
    if t.dtype is not _int32() or not t.is_cuda or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise PolarQuantError(f"{name} must be a contiguous int32 device tensor of {n} entries")
    return t.data_ptr()


def _pages(t, n_seq):
    """Address and row length of a page table."""
    if t.dtype is not _int32() or not t.is_cuda or t.dim() != 2 or t.shape[0] != n_seq or (t.shape[1] > 1 and t.stride(1) != 1):
        raise PolarQuantError(f"pages must be an int32 device tensor [{n_seq}, pages of a sequence], rows contiguous")
    return t.data_ptr(), t.stride(0) if n_seq > 1 else t.shape[1]


class Context:
    """pq_ctx: the preconditioner S, the codebooks and the device constant tables."""

    _radii_halves = TILE_RADII  # of a tile, in this context's format

    def __init__(self, seed=0, S=None, d=D, hadamard=False):
        """S: explicit d x d orthogonal matrix; hadamard=True: randomised Hadamard matrix from seed
        (pq_init_preconditioner_hadamard); otherwise the QR factor of a seeded Gaussian matrix."""
        L = library()
        h = ctypes.c_void_p()
        if hadamard:
            if S is not None:
                raise PolarQuantError("give either S or hadamard=True")
            _check(L.pq_init_preconditioner_hadamard(ctypes.byref(h), int(d), int(seed)))
            self._h = h
            self.d = d
            return
        if S is not None:
            S = np.ascontiguousarray(S, dtype=np.float64)
            if S.shape != (d, d):
                raise PolarQuantError("S must be d x d")
            sp = S.ctypes.data_as(ctypes.c_void_p)
        else:
            sp = None
        _check(L.pq_init_preconditioner(ctypes.byref(h), int(d), int(seed), sp))
        self._h = h
        self.d = d

    def close(self):
        if getattr(self, "_h", None):
            library().pq_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_codebooks(self, cb):
        """cb: 28 centroids (16 of level 1, then 4 each of levels 2-4); only before the first launch."""
        cb = np.ascontiguousarray(cb, dtype=np.float64).reshape(-1)
        if cb.size != 28:
            raise PolarQuantError("cb must hold 28 centroids")
        _check(library().pq_set_codebooks(self._h, cb.ctypes.data_as(ctypes.c_void_p)))

    def set_recursion_depth(self, depth, upper_bits=None):
        """depth 4 (default) or 7 (full recursion: upper_bits = bits of levels 5, 6, 7); only before the first launch."""
        bits = None
        if upper_bits is not None:
            bits = np.ascontiguousarray(upper_bits, dtype=np.int32).reshape(-1)
            if bits.size != 3:
                raise PolarQuantError("upper_bits must hold 3 widths")
        _check(library().pq_set_recursion_depth(self._h, int(depth), bits.ctypes.data_as(ctypes.c_void_p) if bits is not None else None))
        self._radii_halves = self.radii_halves_per_tile()

    def set_upper_codebooks(self, cbt):
        """Centroids of levels 5, 6, 7 of a depth-7 context, array [3, 8] (2^bits used per row); before the first launch."""
        c = np.ascontiguousarray(cbt, dtype=np.float64)
        if c.shape != (3, 8):
            raise PolarQuantError("cbt must have shape [3, 8]")
        _check(library().pq_set_upper_codebooks(self._h, c.ctypes.data_as(ctypes.c_void_p)))

    def recursion_depth(self):
        return int(library().pq_recursion_depth(self._h))

    def preconditioner_structure(self):
        """0 general S, 1 all entries +-1/sqrt(d), 2 sign diagonal times the Sylvester Hadamard matrix."""
        return int(library().pq_preconditioner_structure(self._h))

    def radii_halves_per_tile(self):
        return int(library().pq_radii_halves_per_tile(self._h))

    def record_bytes(self):
        return int(library().pq_record_bytes(self._h))

    def upper_codebook(self, level):
        """Level 5..7 of a depth-7 context: (bits, centroids, boundaries)."""
        bits = ctypes.c_int(0)
        c = np.zeros(8, dtype=np.float64)
        b = np.zeros(9, dtype=np.float64)
        _check(library().pq_get_upper_codebook(self._h, int(level), ctypes.byref(bits), c.ctypes.data_as(ctypes.c_void_p),
                                               b.ctypes.data_as(ctypes.c_void_p)))
        K = 1 << bits.value
        return bits.value, c[:K].copy(), b[: K + 1].copy()

    def alloc_cache_for(self, n_heads, pool_tokens, device="cuda"):
        """Cache buffers in this context's format (the radius plane depends on the recursion depth)."""
        return Context.alloc_cache(n_heads, pool_tokens, device, self.radii_halves_per_tile())

    def fit_codebooks(self, x, iterations, cb_init=None, workspace=None):
        """Online codebooks from x [n_tokens, n_heads, 128] (strides taken from the tensor, innermost contiguous):
        `iterations` k-means rounds on its angles -> 28 centroids (numpy).  Waits for the stream."""
        import torch

        if x.stride(2) != 1:
            raise PolarQuantError("innermost dimension must be contiguous")
        nbytes = int(library().pq_fit_workspace_bytes())
        if workspace is None:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        init = None
        if cb_init is not None:
            init = np.ascontiguousarray(cb_init, dtype=np.float64).reshape(-1)
            if init.size != 28:
                raise PolarQuantError("cb_init must hold 28 centroids")
        out = np.empty(28, dtype=np.float64)
        _check(library().pq_fit_codebooks(
            self._h, x.data_ptr(), _dtype_code(x), int(x.shape[0]), int(x.shape[1]), int(x.stride(0)), int(x.stride(1)),
            init.ctypes.data if init is not None else None, int(iterations),
            out.ctypes.data, workspace.data_ptr(),
            int(workspace.numel() * workspace.element_size()), _stream()))
        return out

    def fit_count_angles(self, x, workspace):
        """First half of fit_codebooks: counts the angles of x into the histograms in workspace (uint8 device tensor of
        fit_workspace_bytes()); enqueued on the current stream, does not wait."""
        if x.stride(2) != 1:
            raise PolarQuantError("innermost dimension must be contiguous")
        _check(library().pq_fit_count_angles(
            self._h, x.data_ptr(), _dtype_code(x), int(x.shape[0]), int(x.shape[1]), int(x.stride(0)), int(x.stride(1)),
            workspace.data_ptr(), int(workspace.numel() * workspace.element_size()), _stream()))

    def fit_cluster(self, hist, iterations, cb_init=None, cbt_init=None):
        """Second half: hist = host copy (numpy uint32) of the workspace -> 28 centroids, and [3, 8] upper centroids for a
        depth-7 context (None otherwise)."""
        hist = np.ascontiguousarray(hist, dtype=np.uint32)
        if hist.size * 4 != self.fit_workspace_bytes():
            raise PolarQuantError("hist must be a copy of the whole fit workspace")
        init = None if cb_init is None else np.ascontiguousarray(cb_init, dtype=np.float64).reshape(-1)
        init_t = None if cbt_init is None else np.ascontiguousarray(cbt_init, dtype=np.float64)
        out, out_t = np.empty(28, dtype=np.float64), np.empty((3, 8), dtype=np.float64)
        _check(library().pq_fit_cluster(
            self._h, hist.ctypes.data,
            init.ctypes.data if init is not None else None,
            init_t.ctypes.data if init_t is not None else None, int(iterations),
            out.ctypes.data, out_t.ctypes.data))
        return out, (out_t if self.recursion_depth() == 7 else None)

    @staticmethod
    def fit_workspace_bytes():
        return int(library().pq_fit_workspace_bytes())

    def fit_codebooks_deep(self, x, iterations, cb_init=None, cbt_init=None, workspace=None):
        """fit_codebooks for a depth-7 context: also the codebooks of levels 5-7 -> (28 centroids, [3, 8] centroids)."""
        import torch

        if x.stride(2) != 1:
            raise PolarQuantError("innermost dimension must be contiguous")
        nbytes = int(library().pq_fit_workspace_bytes())
        if workspace is None:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        init = init_t = None
        if cb_init is not None:
            init = np.ascontiguousarray(cb_init, dtype=np.float64).reshape(-1)
            if init.size != 28:
                raise PolarQuantError("cb_init must hold 28 centroids")
        if cbt_init is not None:
            init_t = np.ascontiguousarray(cbt_init, dtype=np.float64)
            if init_t.shape != (3, 8):
                raise PolarQuantError("cbt_init must have shape [3, 8]")
        out = np.empty(28, dtype=np.float64)
        out_t = np.empty((3, 8), dtype=np.float64)
        _check(library().pq_fit_codebooks_deep(
            self._h, x.data_ptr(), _dtype_code(x), int(x.shape[0]), int(x.shape[1]), int(x.stride(0)), int(x.stride(1)),
            init.ctypes.data if init is not None else None,
            init_t.ctypes.data if init_t is not None else None, int(iterations),
            out.ctypes.data, out_t.ctypes.data, workspace.data_ptr(),
            int(workspace.numel() * workspace.element_size()), _stream()))
        return out, out_t

    # ---- host-side getters -------------------------------------------------
    def preconditioner(self):
        S = np.empty((self.d, self.d), dtype=np.float64)
        _check(library().pq_get_preconditioner(self._h, S.ctypes.data_as(ctypes.c_void_p)))
        return S

    def codebook(self, level):
        K = 16 if level == 1 else 4
        c = np.empty(K, dtype=np.float64)
        b = np.empty(K + 1, dtype=np.float64)
        _check(library().pq_get_codebook(self._h, int(level), c.ctypes.data_as(ctypes.c_void_p),
                                         b.ctypes.data_as(ctypes.c_void_p)))
        return c, b

    # ---- cache allocation helper (torch owns the memory) --------------------
    @staticmethod
    def alloc_cache(n_heads, pool_tokens, device="cuda", radii_halves=TILE_RADII):
        import torch

        if pool_tokens % TILE_TOKENS:
            raise PolarQuantError("pool_tokens must be a multiple of 64")
        tiles = pool_tokens // TILE_TOKENS
        codes = torch.empty((n_heads, tiles, TILE_CODE_BYTES), dtype=torch.uint8, device=device)
        radii = torch.empty((n_heads, tiles, radii_halves), dtype=torch.int16, device=device)
        return codes, radii

    # ---- kernels -------------------------------------------------------------
    def encode_kv(self, x, kind, codes, radii, dst_token0=0, ld_token=None, ld_head=None, n_tokens=None, n_heads=None):
        """x: [n_tokens, n_heads, 128] (token-major) or any strided view given ld_token / ld_head (elements)."""
        if ld_token is None:
            n_tokens, n_heads = x.shape[0], x.shape[1]
            ld_token, ld_head = x.stride(0), x.stride(1)
            if x.stride(2) != 1:
                raise PolarQuantError("innermost dimension must be contiguous")
        pool_tokens = codes.shape[1] * TILE_TOKENS
        _check(library().pq_encode_kv(self._h, x.data_ptr(), _dtype_code(x), int(kind), int(n_tokens), int(n_heads),
                                      int(ld_token), int(ld_head), codes.data_ptr(), radii.data_ptr(),
                                      int(pool_tokens), int(dst_token0), _stream()))

    def encode_kv_pair(self, xk, xv, k_codes, k_radii, v_codes, v_radii, dst_token0=0, ld_token=None, ld_head=None,
                       n_tokens=None, n_heads=None):
        """Keys and values of the same tokens in one launch; xk, xv as x of encode_kv, same shape, strides, dtype."""
        if ld_token is None:
            n_tokens, n_heads = xk.shape[0], xk.shape[1]
            ld_token, ld_head = xk.stride(0), xk.stride(1)
            if xk.stride(2) != 1 or xv.stride(2) != 1:
                raise PolarQuantError("innermost dimension must be contiguous")
            if xv.shape != xk.shape or xv.stride() != xk.stride():
                raise PolarQuantError("xk and xv must have the same shape and strides")
        if xk.dtype != xv.dtype:
            raise PolarQuantError("xk and xv must have the same dtype")
        if k_codes.shape != v_codes.shape:
            raise PolarQuantError("key and value caches must have the same pool size")
        pool_tokens = k_codes.shape[1] * TILE_TOKENS
        _check(library().pq_encode_kv_pair(self._h, xk.data_ptr(), xv.data_ptr(), _dtype_code(xk), int(n_tokens),
                                           int(n_heads), int(ld_token), int(ld_head), k_codes.data_ptr(),
                                           k_radii.data_ptr(), v_codes.data_ptr(), v_radii.data_ptr(),
                                           int(pool_tokens), int(dst_token0), _stream()))

    def append_kv(self, x, kind, codes, radii, dst_token):
        """x: [n_seq, n_heads, 128] contiguous; dst_token: int64 device tensor [n_seq]."""
        if not x.is_contiguous():
            raise PolarQuantError("x must be contiguous")
        pool_tokens = codes.shape[1] * TILE_TOKENS
        _check(library().pq_append_kv(self._h, x.data_ptr(), _dtype_code(x), int(kind), int(x.shape[0]), int(x.shape[1]),
                                      codes.data_ptr(), radii.data_ptr(), int(pool_tokens), dst_token.data_ptr(),
                                      _stream()))

    def append_kv_pair(self, xk, xv, k_codes, k_radii, v_codes, v_radii, dst_token):
        """xk, xv: [n_seq, n_heads, 128] contiguous, same dtype; dst_token: int64 device tensor [n_seq]."""
        if not (xk.is_contiguous() and xv.is_contiguous()):
            raise PolarQuantError("xk and xv must be contiguous")
        if xk.shape != xv.shape or xk.dtype != xv.dtype:
            raise PolarQuantError("xk and xv must have the same shape and dtype")
        if k_codes.shape != v_codes.shape:
            raise PolarQuantError("key and value caches must have the same pool size")
        pool_tokens = k_codes.shape[1] * TILE_TOKENS
        _check(library().pq_append_kv_pair(self._h, xk.data_ptr(), xv.data_ptr(), _dtype_code(xk), int(xk.shape[0]),
                                           int(xk.shape[1]), k_codes.data_ptr(), k_radii.data_ptr(),
                                           v_codes.data_ptr(), v_radii.data_ptr(), int(pool_tokens),
                                           dst_token.data_ptr(), _stream()))

    def decode_kv(self, kind, codes, radii, token0, n_tokens, out, rotated=False):
        """out: [n_tokens, n_heads, 128] float32 or bfloat16 (strides taken from the tensor)."""
        pool_tokens = codes.shape[1] * TILE_TOKENS
        _check(library().pq_decode_kv(self._h, int(kind), codes.data_ptr(), radii.data_ptr(), int(pool_tokens),
                                      int(token0), int(n_tokens), int(out.shape[1]), out.data_ptr(), _dtype_code(out),
                                      int(out.stride(0)), int(out.stride(1)), 1 if rotated else 0, _stream()))

    def export_canonical(self, kind, codes, radii, token0, n_tokens, rec):
        """rec: uint8 [n_heads, n_tokens, record_bytes()] contiguous (62, or 50 at depth 7)."""
        pool_tokens = codes.shape[1] * TILE_TOKENS
        _check(library().pq_export_canonical(self._h, int(kind), codes.data_ptr(), radii.data_ptr(), int(pool_tokens),
                                             int(token0), int(n_tokens), int(codes.shape[0]), rec.data_ptr(), _stream()))

    @staticmethod
    def attn_workspace_bytes(B, Hq, Hkv, max_ctx):
        return int(library().pq_attn_workspace_bytes(int(B), int(Hq), int(Hkv), int(max_ctx)))

    def attn_decode_polar_mq(self, q, out, k_codes, k_radii, v_codes, v_radii, seq_start, ctx_len, max_ctx,
                             softmax_scale, workspace):
        """M query tokens per sequence: q, out [B, M, Hq, 128]; token m sees ctx_len - (M-1-m) cached tokens."""
        B, M, Hq = q.shape[0], q.shape[1], q.shape[2]
        Hkv = k_codes.shape[0]
        if not (q.is_contiguous() and out.is_contiguous()):
            raise PolarQuantError("q and out must be contiguous")
        pool_tokens = k_codes.shape[1] * TILE_TOKENS
        _check(library().pq_attn_decode_polar_mq(
            self._h, q.data_ptr(), out.data_ptr(), _dtype_code(out), k_codes.data_ptr(), k_radii.data_ptr(),
            v_codes.data_ptr(), v_radii.data_ptr(), seq_start.data_ptr(), ctx_len.data_ptr(), int(B), int(M), int(Hq),
            int(Hkv), int(pool_tokens), int(max_ctx), float(softmax_scale), workspace.data_ptr(),
            int(workspace.numel() * workspace.element_size()), _stream()))

    @staticmethod
    def attn_mq_workspace_bytes(B, M, Hq, Hkv, max_ctx):
        return int(library().pq_attn_mq_workspace_bytes(int(B), int(M), int(Hq), int(Hkv), int(max_ctx)))

    def attn_decode_hybrid(self, q, out, k_codes, k_radii, v_codes, v_radii, seq_start, ctx_len, win_k, win_v, win_len,
                           max_ctx, softmax_scale, workspace):
        """Quantised prefix + bf16 window: win_k, win_v [B, Hkv, win_cap, 128] bf16 contiguous, win_len int32 [B]."""
        if not (win_k.is_contiguous() and win_v.is_contiguous()):
            raise PolarQuantError("win_k and win_v must be contiguous")
        B, Hq = q.shape[0], q.shape[1]
        Hkv = k_codes.shape[0]
        if win_k.shape != win_v.shape or tuple(win_k.shape[:2]) != (B, Hkv) or win_k.shape[3] != 128:
            raise PolarQuantError("win_k and win_v must both be [B, Hkv, win_cap, 128]")
        if _dtype_code(win_k) != PQ_BF16 or _dtype_code(win_v) != PQ_BF16:
            raise PolarQuantError("the window is bfloat16")
        pool_tokens = k_codes.shape[1] * TILE_TOKENS
        _check(library().pq_attn_decode_hybrid(
            self._h, q.data_ptr(), out.data_ptr(), _dtype_code(out), k_codes.data_ptr(), k_radii.data_ptr(),
            v_codes.data_ptr(), v_radii.data_ptr(), seq_start.data_ptr(), ctx_len.data_ptr(), win_k.data_ptr(),
            win_v.data_ptr(), win_len.data_ptr(), int(win_k.shape[2]), int(B), int(Hq), int(Hkv), int(pool_tokens),
            int(max_ctx), float(softmax_scale), workspace.data_ptr(),
            int(workspace.numel() * workspace.element_size()), _stream()))

    # ---- paged caches ----------------------------------------------------------
    def _paged_cache(self, k_codes, k_radii, v_codes, v_radii):
        """Checks the four buffers of a cache in this context's format -> (head planes, slots of a plane)."""
        heads, tiles = k_codes.shape[0], k_codes.shape[1]
        codes, radii = (heads, tiles, TILE_CODE_BYTES), (heads, tiles, self._radii_halves)
        if not (k_codes.shape == codes and v_codes.shape == codes and k_radii.shape == radii and v_radii.shape == radii
                and k_codes.is_contiguous() and v_codes.is_contiguous() and k_radii.is_contiguous() and v_radii.is_contiguous()
                and k_codes.is_cuda and v_codes.is_cuda and k_radii.is_cuda and v_radii.is_cuda
                and k_codes.element_size() == 1 and v_codes.element_size() == 1 and k_radii.element_size() == 2 and v_radii.element_size() == 2):
            raise PolarQuantError("the cache must be device tensors as alloc_cache_for makes them, keys and values of one size")
        return heads, tiles * TILE_TOKENS

    def append_paged(self, xk, xv, row_start, ctx_len, k_codes, k_radii, v_codes, v_radii, pages, rotary=None, positions=None):
        """xk, xv: [rows, n_heads, 128] of one shape, dtype and strides (views of a projection's output, say); row_start int32
        [n_seq + 1], ctx_len int32 [n_seq] (new tokens counted), pages int32 [n_seq, pages]; rotary: Rotary for the keys, positions
        int32 [rows] or None."""
        shape, stride = xk.shape, xk.stride()
        heads, pool_tokens = self._paged_cache(k_codes, k_radii, v_codes, v_radii)
        if len(shape) != 3 or shape != xv.shape or stride != xv.stride() or xk.dtype != xv.dtype or shape[1] != heads or shape[2] != D or stride[2] != 1 \
                or not (xk.is_cuda and xv.is_cuda):
            raise PolarQuantError("xk and xv must be device tensors [rows, n_heads, 128] of one shape, dtype and strides, coordinates contiguous, "
                                  "with the cache's heads")
        n_rows, n_seq = shape[0], ctx_len.shape[0]
        table, ld = _pages(pages, n_seq)
        _check(library().pq_append_paged(
            self._h, xk.data_ptr(), xv.data_ptr(), _dtype_code(xk), n_rows, heads, stride[0], stride[1],
            ctypes.addressof(rotary) if rotary is not None else None, _ints("positions", positions, n_rows) if positions is not None else None,
            k_codes.data_ptr(), k_radii.data_ptr(), v_codes.data_ptr(), v_radii.data_ptr(), pool_tokens, table, ld,
            _ints("row_start", row_start, n_seq + 1), _ints("ctx_len", ctx_len, n_seq), n_seq, _stream()))

    def decode_paged(self, k_codes, k_radii, v_codes, v_radii, pages, row_start, ctx_len, out_k=None, out_v=None):
        """out_k, out_v: [rows, n_heads, 128] float32 or bfloat16, of one shape, dtype and strides, or one of them None."""
        o = out_k if out_k is not None else out_v
        if o is None:
            raise PolarQuantError("give out_k, out_v or both")
        shape, stride = o.shape, o.stride()
        heads, pool_tokens = self._paged_cache(k_codes, k_radii, v_codes, v_radii)
        if len(shape) != 3 or shape[1] != heads or shape[2] != D or stride[2] != 1 or not o.is_cuda or \
                (out_k is not None and out_v is not None
                 and (out_v.shape != shape or out_v.stride() != stride or out_v.dtype != out_k.dtype or not out_v.is_cuda)):
            raise PolarQuantError("out_k and out_v must be device tensors [rows, n_heads, 128] of one shape, dtype and strides, coordinates contiguous, "
                                  "with the cache's heads")
        n_seq = ctx_len.shape[0]
        table, ld = _pages(pages, n_seq)
        _check(library().pq_decode_paged(
            self._h, k_codes.data_ptr(), k_radii.data_ptr(), v_codes.data_ptr(), v_radii.data_ptr(), pool_tokens, table, ld,
            _ints("row_start", row_start, n_seq + 1), _ints("ctx_len", ctx_len, n_seq), n_seq, shape[0], heads,
            out_k.data_ptr() if out_k is not None else None, out_v.data_ptr() if out_v is not None else None, _dtype_code(o),
            stride[0], stride[1], _stream()))

    def attn_paged(self, q, out, k_codes, k_radii, v_codes, v_radii, pages, ctx_len, max_ctx, softmax_scale, workspace, rotary=None,
                   positions=None):
        """M query tokens per sequence on a paged cache: q, out [B, M, Hq, 128] (q bf16); ctx_len int32 [B], pages int32 [B, pages];
        rotary: Rotary for the queries, positions int32 [B, M] or None."""
        B, M, Hq = self._paged_queries(q, out)
        heads, pool_tokens = self._paged_cache(k_codes, k_radii, v_codes, v_radii)
        table, ld = _pages(pages, B)
        _check(library().pq_attn_paged(
            self._h, q.data_ptr(), out.data_ptr(), _dtype_code(out), ctypes.addressof(rotary) if rotary is not None else None,
            self._query_positions(positions, B, M), k_codes.data_ptr(), k_radii.data_ptr(), v_codes.data_ptr(), v_radii.data_ptr(),
            pool_tokens, table, ld, _ints("ctx_len", ctx_len, B), B, M, Hq, heads, int(max_ctx), float(softmax_scale),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream()))

    def attn_prefix_paged(self, q, out, k_codes, k_radii, v_codes, v_radii, pages, ctx_len, max_ctx, prefix_pages, prefix_len, group_start,
                          max_prefix, softmax_scale, workspace, rotary=None, positions=None):
        """attn_paged with common prefixes: prefix_pages int32 [groups, pages], prefix_len int32 [groups], group_start int32 [groups + 1];
        sequences group_start[g] .. group_start[g + 1] - 1 share prefix g, ctx_len and pages are those of their own tokens."""
        B, M, Hq = self._paged_queries(q, out)
        heads, pool_tokens = self._paged_cache(k_codes, k_radii, v_codes, v_radii)
        table, ld = _pages(pages, B)
        n_groups = prefix_len.shape[0]
        pre_table, pre_ld = _pages(prefix_pages, n_groups)
        _check(library().pq_attn_prefix_paged(
            self._h, q.data_ptr(), out.data_ptr(), _dtype_code(out), ctypes.addressof(rotary) if rotary is not None else None,
            self._query_positions(positions, B, M), k_codes.data_ptr(), k_radii.data_ptr(), v_codes.data_ptr(), v_radii.data_ptr(),
            pool_tokens, table, ld, _ints("ctx_len", ctx_len, B), B, M, Hq, heads, int(max_ctx), pre_table, pre_ld,
            _ints("prefix_len", prefix_len, n_groups), _ints("group_start", group_start, n_groups + 1), n_groups, int(max_prefix),
            float(softmax_scale), workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream()))

    @staticmethod
    def attn_prefix_paged_workspace_bytes(B, M, Hq, Hkv, max_ctx, n_groups, max_prefix):
        return int(library().pq_attn_prefix_paged_workspace_bytes(int(B), int(M), int(Hq), int(Hkv), int(max_ctx), int(n_groups), int(max_prefix)))

    @staticmethod
    def _paged_queries(q, out):
        shape = q.shape
        if len(shape) != 4 or shape[3] != D or shape != out.shape or _dtype_code(q) != PQ_BF16 or not (q.is_cuda and out.is_cuda) or \
                not (q.is_contiguous() and out.is_contiguous()):
            raise PolarQuantError("q and out must be contiguous device tensors [B, M, Hq, 128], q bfloat16")
        return shape[0], shape[1], shape[2]

    @staticmethod
    def _query_positions(positions, B, M):
        if positions is None:
            return None
        if positions.shape != (B, M) or not positions.is_contiguous():
            raise PolarQuantError("positions must be contiguous, [B, M]")
        return _ints("positions", positions.view(-1), B * M)

    @staticmethod
    def attn_paged_workspace_bytes(B, M, Hq, Hkv, max_ctx):
        return int(library().pq_attn_paged_workspace_bytes(int(B), int(M), int(Hq), int(Hkv), int(max_ctx)))

    @staticmethod
    def attn_hybrid_workspace_bytes(B, Hq, Hkv, max_ctx, win_cap):
        return int(library().pq_attn_hybrid_workspace_bytes(int(B), int(Hq), int(Hkv), int(max_ctx), int(win_cap)))

    def decode_step_polar(self, xk, xv, dst_token, q, out, k_codes, k_radii, v_codes, v_radii, seq_start, ctx_len,
                          max_ctx, softmax_scale, workspace):
        """append_kv_pair(xk, xv -> dst_token) + attn_decode_polar in one call; xk, xv: [B, Hkv, 128] contiguous."""
        if not (xk.is_contiguous() and xv.is_contiguous()):
            raise PolarQuantError("xk and xv must be contiguous")
        B, Hq = q.shape[0], q.shape[1]
        Hkv = k_codes.shape[0]
        if tuple(xk.shape) != (B, Hkv, 128) or xk.shape != xv.shape or xk.dtype != xv.dtype:
            raise PolarQuantError("xk and xv must both be [B, Hkv, 128] of one dtype")
        pool_tokens = k_codes.shape[1] * TILE_TOKENS
        _check(library().pq_decode_step_polar(
            self._h, xk.data_ptr(), xv.data_ptr(), _dtype_code(xk), dst_token.data_ptr(), q.data_ptr(), out.data_ptr(),
            _dtype_code(out), k_codes.data_ptr(), k_radii.data_ptr(), v_codes.data_ptr(), v_radii.data_ptr(),
            seq_start.data_ptr(), ctx_len.data_ptr(), int(B), int(Hq), int(Hkv), int(pool_tokens), int(max_ctx),
            float(softmax_scale), workspace.data_ptr(), int(workspace.numel() * workspace.element_size()), _stream()))

    @staticmethod
    def static_scratch_bytes():
        return int(library().pq_static_scratch_bytes())

    def prepare_device(self):
        """Uploads the context's constants to the current device (the one call of the static path that allocates)."""
        _check(library().pq_prepare_device(self._h))

    def attn_decode_polar_static(self, q, out, k_codes, k_radii, v_codes, v_radii, seq_start, ctx_len, max_ctx,
                                 softmax_scale):
        """attn_decode_polar with the workspace in the library's static device array; allocates nothing."""
        B, Hq = q.shape[0], q.shape[1]
        Hkv = k_codes.shape[0]
        pool_tokens = k_codes.shape[1] * TILE_TOKENS
        _check(library().pq_attn_decode_polar_static(
            self._h, q.data_ptr(), out.data_ptr(), _dtype_code(out), k_codes.data_ptr(), k_radii.data_ptr(), v_codes.data_ptr(),
            v_radii.data_ptr(), seq_start.data_ptr(), ctx_len.data_ptr(), int(B), int(Hq), int(Hkv), int(pool_tokens),
            int(max_ctx), float(softmax_scale), _stream()))

    def attn_decode_polar(self, q, out, k_codes, k_radii, v_codes, v_radii, seq_start, ctx_len, max_ctx,
                          softmax_scale, workspace):
        """q: [B, Hq, 128] bf16; out: same shape, bf16 or float32; seq_start int64 [B], ctx_len int32 [B] (device)."""
        B, Hq = q.shape[0], q.shape[1]
        Hkv = k_codes.shape[0]
        pool_tokens = k_codes.shape[1] * TILE_TOKENS
        _check(library().pq_attn_decode_polar(
            self._h, q.data_ptr(), out.data_ptr(), _dtype_code(out), k_codes.data_ptr(), k_radii.data_ptr(), v_codes.data_ptr(),
            v_radii.data_ptr(), seq_start.data_ptr(), ctx_len.data_ptr(), int(B), int(Hq), int(Hkv), int(pool_tokens),
            int(max_ctx), float(softmax_scale), workspace.data_ptr(), int(workspace.numel() * workspace.element_size()),
            _stream()))


class GeneralFormat(ctypes.Structure):
    """pq_general_format: recursion depth 4..7 and bits per level (level 1: 3 or 4; 2-4: 2 or 3; 5-7: 1..3)."""
    _fields_ = [("depth", ctypes.c_int), ("bits", ctypes.c_int * 7)]

    def __init__(self, depth, bits):
        super().__init__()
        self.depth = int(depth)
        for l in range(7):
            self.bits[l] = int(bits[l]) if l < len(bits) else 0

    def record_bytes(self):
        n = int(library().pq_general_record_bytes(ctypes.byref(self)))
        if n == 0:
            raise PolarQuantError("general format refused (depth 4..7; bits: level 1 in {3,4}, 2-4 in {2,3}, 5-7 in {1,2,3})")
        return n

    def codebooks(self):
        """Lloyd-Max centroids of levels 1..depth, concatenated (numpy float64)."""
        n = int(library().pq_general_codebook_entries(ctypes.byref(self)))
        if n == 0:
            raise PolarQuantError("general format refused")
        out = np.empty(n, dtype=np.float64)
        _check(library().pq_general_codebooks(ctypes.byref(self), out.ctypes.data_as(ctypes.c_void_p)))
        return out


def _cbg(cbg):
    """The codebooks as contiguous doubles; `.ctypes.data` of the result is what the calls take (data_as costs 2.4 us more)."""
    return np.ascontiguousarray(cbg, dtype=np.float64)


def general_encode(ctx, fmt, cbg, x, records):
    """x [n, 128] (bf16 or fp32 device tensor, rows contiguous) -> records (uint8 device tensor [n, record bytes])."""
    cb = _cbg(cbg)
    _check(library().pq_general_encode(ctx._h, ctypes.byref(fmt), cb.ctypes.data, x.data_ptr(),
                                       _dtype_code(x), int(x.shape[0]), int(x.stride(0)), records.data_ptr(), _stream()))


def general_decode(ctx, fmt, cbg, records, n, out, rotated=False):
    cb = _cbg(cbg)
    _check(library().pq_general_decode(ctx._h, ctypes.byref(fmt), cb.ctypes.data, records.data_ptr(),
                                       int(n), 1 if rotated else 0, out.data_ptr(), _stream()))


def general_attn_decode(ctx, fmt, cbg, q, out, k_records, v_records, seq_start, ctx_len, scale):
    """q bf16 [B, Hq, 128]; records uint8 [Hkv, pool_tokens, record bytes]; out fp32 [B, Hq, 128].  The workspace that lets few
    rows occupy the chip comes from torch's allocator, in the order of the stream; a stream that is being captured gets none (a
    graph outlives it): a captured call is the one without, whose sums are rounded in another order."""
    import torch

    cb = _cbg(cbg)
    B, Hq, _ = q.shape
    Hkv, pool_tokens = k_records.shape[0], k_records.shape[1]
    L = library()
    n = L.pq_general_attn_workspace_bytes(B, Hq, Hkv, pool_tokens)
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n and not torch.cuda.is_current_stream_capturing() else None
    _check(L.pq_general_attn_decode_ws(ctx._h, ctypes.byref(fmt), cb.ctypes.data, q.data_ptr(),
                                       out.data_ptr(), k_records.data_ptr(), v_records.data_ptr(), seq_start.data_ptr(),
                                       ctx_len.data_ptr(), int(B), int(Hq), int(Hkv), int(pool_tokens), float(scale),
                                       ws.data_ptr() if ws is not None else None, n if ws is not None else 0, _stream()))
