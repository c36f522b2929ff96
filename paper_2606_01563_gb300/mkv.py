"""Python binding of the MomentKV C ABI (include/mkv.h, include/mkv_tree.h).

Argument marshalling only: every function forwards to the function of the
same name in libmkv.so, passing device pointers of torch tensors; all work
runs in the library's CUDA kernels.  A non-OK status raises MKVError.  The
library is loaded on first use and a missing build raises immediately --
there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmkv.so")

c_i32 = ctypes.c_int32
c_vp = ctypes.c_void_p


class mkv_geom(ctypes.Structure):
    _fields_ = [("batch", c_i32), ("n_kv_heads", c_i32), ("group", c_i32), ("head_dim", c_i32)]


class mkv_moments(ctypes.Structure):
    _fields_ = [("n", c_vp), ("mu_k", c_vp), ("mu_v", c_vp), ("C", c_vp)]


class mkv_cache(ctypes.Structure):
    _fields_ = [("K", c_vp), ("V", c_vp), ("pos", c_vp), ("len", c_vp), ("seen", c_vp), ("capacity", c_i32),
                ("y", c_vp), ("y_len", c_vp)]


class mkv_compress_params(ctypes.Structure):
    _fields_ = [("budget", c_i32), ("window", c_i32), ("sink", c_i32), ("keep_window", c_i32),
                ("pool", c_i32), ("mi", c_i32), ("causal", c_i32), ("tau", ctypes.c_float), ("adaptive", c_i32)]


class mkv_compress_diag(ctypes.Structure):
    _fields_ = [("scores", c_vp), ("score2", c_vp), ("idx_stage1", c_vp)]


class mkv_decode_params(ctypes.Structure):
    _fields_ = [("correction", c_i32), ("order", c_i32), ("tau", ctypes.c_float), ("C16", c_vp),
                ("early_load", c_i32), ("C_split", c_vp)]


class mkv_tree(ctypes.Structure):
    _fields_ = [("n_nodes", c_i32), ("count", c_vp), ("mask", c_vp), ("q_node", ctypes.c_int64),
                ("q_batch", ctypes.c_int64), ("kv_node", ctypes.c_int64), ("kv_batch", ctypes.c_int64)]


class mkv_tree_layer(ctypes.Structure):
    _fields_ = [("cache", mkv_cache), ("k", c_vp), ("v", c_vp)]


class mkv_rope_params(ctypes.Structure):
    _fields_ = [("rot_dim", c_i32), ("neighbours", c_i32), ("inverse", c_i32), ("n_axes", c_i32),
                ("inv_freq", ctypes.c_float * 64), ("axis", c_i32 * 64)]


class mkv_rope_tensor(ctypes.Structure):
    _fields_ = [("in_", c_vp), ("out", c_vp), ("heads", c_i32)] + [
        (n, ctypes.c_int64) for n in ("in_batch", "in_token", "in_head", "out_batch", "out_token", "out_head")]


STATUS = {0: "MKV_OK", 1: "MKV_ERR_INVALID_ARG", 2: "MKV_ERR_SHAPE", 3: "MKV_ERR_CAPACITY",
          4: "MKV_ERR_CUDA", 5: "MKV_ERR_TIMEOUT", 6: "MKV_ERR_UNSUPPORTED", 7: "MKV_ERR_WORKSPACE"}

EXPORTS = ("mkv_status_str", "mkv_version", "mkv_compress_workspace_size", "mkv_compress",
           "mkv_decode_workspace_size", "mkv_decode_step", "mkv_evict_workspace_size",
           "mkv_evict_append", "mkv_get_device_error", "mkv_decode_step_noalloc", "mkv_moments_pack_bf16",
           "mkv_decode_evict_workspace_size", "mkv_decode_evict_step", "mkv_moments_pack_split")
# declared in include/mkv_tree.h
TREE_EXPORTS = ("mkv_tree_build", "mkv_tree_workspace_size", "mkv_tree_step", "mkv_tree_commit", "mkv_rope")
# test hooks declared in include/mkv_debug.h
DEBUG_EXPORTS = ("mkv_debug_set_poll_limit", "mkv_debug_force_ticket_merge")


class MKVError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)} ({lib().mkv_status_str(code).decode()})")


_lib = None


def lib():
    """The loaded libmkv.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it first "
                              "(python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(LIB_PATH)
        L.mkv_status_str.restype = ctypes.c_char_p
        L.mkv_status_str.argtypes = [c_i32]
        L.mkv_version.restype = c_i32
        L.mkv_compress_workspace_size.restype = ctypes.c_size_t
        L.mkv_compress_workspace_size.argtypes = [mkv_geom, c_i32, ctypes.POINTER(mkv_compress_params)]
        L.mkv_compress.restype = c_i32
        L.mkv_compress.argtypes = [mkv_geom, c_i32, c_vp, c_vp, c_vp, ctypes.POINTER(mkv_compress_params),
                                   ctypes.POINTER(mkv_cache), ctypes.POINTER(mkv_moments),
                                   ctypes.POINTER(mkv_compress_diag), c_vp, ctypes.c_size_t, c_vp]
        L.mkv_decode_workspace_size.restype = ctypes.c_size_t
        L.mkv_decode_workspace_size.argtypes = [mkv_geom, c_i32]
        L.mkv_decode_step.restype = c_i32
        L.mkv_decode_step.argtypes = [mkv_geom, c_vp, c_vp, c_vp, ctypes.POINTER(mkv_cache),
                                      ctypes.POINTER(mkv_moments), ctypes.POINTER(mkv_decode_params),
                                      c_vp, c_vp, c_vp, ctypes.c_size_t, c_vp]
        L.mkv_decode_step_noalloc.restype = c_i32
        L.mkv_decode_step_noalloc.argtypes = [mkv_geom, c_vp, c_vp, c_vp, ctypes.POINTER(mkv_cache),
                                              ctypes.POINTER(mkv_moments), ctypes.POINTER(mkv_decode_params),
                                              c_vp, c_vp, c_vp]
        L.mkv_evict_workspace_size.restype = ctypes.c_size_t
        L.mkv_evict_workspace_size.argtypes = [mkv_geom, c_i32]
        L.mkv_evict_append.restype = c_i32
        L.mkv_evict_append.argtypes = [mkv_geom, c_vp, c_vp, c_vp, c_i32, ctypes.POINTER(mkv_cache),
                                       ctypes.POINTER(mkv_moments), ctypes.c_float, c_vp, ctypes.c_size_t, c_vp]
        L.mkv_decode_evict_workspace_size.restype = ctypes.c_size_t
        L.mkv_decode_evict_workspace_size.argtypes = [mkv_geom, c_i32]
        L.mkv_decode_evict_step.restype = c_i32
        L.mkv_decode_evict_step.argtypes = [mkv_geom, c_vp, c_vp, c_vp, c_i32, ctypes.POINTER(mkv_cache),
                                            ctypes.POINTER(mkv_moments), ctypes.POINTER(mkv_decode_params),
                                            c_vp, c_vp, c_vp, ctypes.c_size_t, c_vp]
        L.mkv_moments_pack_bf16.restype = c_i32
        L.mkv_moments_pack_bf16.argtypes = [mkv_geom, ctypes.POINTER(mkv_moments), c_vp, c_vp]
        L.mkv_moments_pack_split.restype = c_i32
        L.mkv_moments_pack_split.argtypes = [mkv_geom, ctypes.POINTER(mkv_moments), ctypes.c_float, c_vp, c_vp]
        c_i64 = ctypes.c_int64
        L.mkv_tree_build.restype = c_i32
        L.mkv_tree_build.argtypes = [c_i32, c_i32, c_vp, c_vp, c_vp, c_i64, c_vp, c_vp, c_vp, ctypes.c_size_t, c_vp]
        L.mkv_tree_workspace_size.restype = ctypes.c_size_t
        L.mkv_tree_workspace_size.argtypes = [mkv_geom, c_i32, c_i32]
        L.mkv_tree_step.restype = c_i32
        L.mkv_tree_step.argtypes = [mkv_geom, c_vp, c_vp, c_vp, c_vp, ctypes.POINTER(mkv_cache),
                                    ctypes.POINTER(mkv_moments), ctypes.POINTER(mkv_decode_params), c_vp, c_vp, c_vp,
                                    ctypes.c_size_t, c_vp]
        L.mkv_tree_commit.restype = c_i32
        L.mkv_tree_commit.argtypes = [mkv_geom, c_vp, c_i32, ctypes.POINTER(mkv_tree_layer), c_vp,
                                      c_i32, c_vp, c_vp, ctypes.c_size_t, c_vp]
        L.mkv_rope.restype = c_i32
        L.mkv_rope.argtypes = [c_i32, c_i32, c_i32, c_vp, c_i64, c_i64, ctypes.POINTER(mkv_rope_params), c_i32, c_vp, c_vp]
        L.mkv_debug_set_poll_limit.restype = ctypes.c_int64
        L.mkv_debug_set_poll_limit.argtypes = [ctypes.c_int64]
        L.mkv_debug_force_ticket_merge.restype = c_i32
        L.mkv_debug_force_ticket_merge.argtypes = [c_i32]
        L.mkv_get_device_error.restype = c_i32
        L.mkv_get_device_error.argtypes = [c_vp, c_vp, ctypes.POINTER(c_i32)]
        _lib = L
    return _lib


# Addresses go to ctypes as plain integers, and the current stream's handle
# comes from torch without a Stream object around it: the marshalling of a
# decode step took 8 of its 12 us on the host, most of it in those wrappers.
# (A private function of torch: without it, the public one and its object.)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())
    return stream.cuda_stream


def _check(code, where):
    if code != 0:
        raise MKVError(code, where)


_BF16 = torch.bfloat16


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _int32(t, shape, what):
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous int32 {list(shape)}")


def _nodes(t, what):
    """(node, batch) strides in elements of a [b, N, heads, d] bf16 tensor whose heads lie densely."""
    _need(t.dtype is _BF16 and t.dim() == 4 and t.stride(3) == 1 and
          (t.shape[2] == 1 or t.stride(2) == t.shape[3]), f"{what}: bf16 [b, N, heads, d] with dense heads")
    # (a stride over an extent of one is never used: 0, the dense value, stands for it; over a larger
    # extent 0 would be taken for the dense value, past the end of an expanded tensor)
    node, batch = (t.stride(1) if t.shape[1] > 1 else None), (t.stride(0) if t.shape[0] > 1 else None)
    _need(node != 0 and batch != 0, f"{what}: not expanded over nodes or batch items")
    return node or 0, batch or 0


# ----------------------------------------------------------------- state
@dataclass
class Cache:
    """Retained KV cache (mkv_cache): K, V bf16 [b, h_kv, cap, d]; pos [b, h_kv, cap];
    len, seen [b, h_kv] (int32)."""
    K: torch.Tensor
    V: torch.Tensor
    pos: torch.Tensor
    len: torch.Tensor
    seen: torch.Tensor
    y: torch.Tensor | None = None      # optional eviction state: fp32 [b, h_kv, cap, d]
    y_len: torch.Tensor | None = None  # int32 [b, h_kv]

    @property
    def capacity(self):
        return self.K.shape[2]

    def c(self):
        return mkv_cache(self.K.data_ptr(), self.V.data_ptr(), self.pos.data_ptr(), self.len.data_ptr(),
                         self.seen.data_ptr(), self.capacity, None if self.y is None else self.y.data_ptr(),
                         None if self.y_len is None else self.y_len.data_ptr())


@dataclass
class Moments:
    """Evicted-set moments (mkv_moments): n [b, h_kv] int32; mu_k, mu_v [b, h_kv, d]; C [b, h_kv, d, d]."""
    n: torch.Tensor
    mu_k: torch.Tensor
    mu_v: torch.Tensor
    C: torch.Tensor

    def c(self):
        return mkv_moments(self.n.data_ptr(), self.mu_k.data_ptr(), self.mu_v.data_ptr(), self.C.data_ptr())


class Tree:
    """Drafted nodes (mkv_tree): mask int32 [b, N, ceil(N / 32)], the words of mkv_tree_build; count int32 [b],
    the nodes in use (None: all N).  Made once per tree and given to every layer's mkv_tree_step."""
    __slots__ = ("mask", "count", "batch", "n_nodes", "usable")

    def __init__(self, mask, count=None):
        self.mask, self.count = mask, count
        self.batch, self.n_nodes, words = mask.shape
        self.usable = (mask.dtype is torch.int32 and mask.is_contiguous() and words == (self.n_nodes + 31) // 32 and
                       (count is None or (count.dtype is torch.int32 and count.shape == (self.batch,) and
                                          count.is_contiguous())))


@dataclass
class TreeLayers:
    """The layers of a commit (tree_layers): what mkv_tree_commit takes, with the tensors it points into."""
    array: ctypes.Array
    tree: mkv_tree
    batch: int
    held: list


def geom(batch, n_kv_heads, group, head_dim):
    return mkv_geom(batch, n_kv_heads, group, head_dim)


def alloc_cache(g: mkv_geom, capacity, device="cuda", evict_state=False):
    """A zero cache; evict_state adds the y rows and y_len of the eviction state."""
    shp = (g.batch, g.n_kv_heads)
    y = torch.zeros(*shp, capacity, g.head_dim, dtype=torch.float32, device=device) if evict_state else None
    y_len = torch.zeros(*shp, dtype=torch.int32, device=device) if evict_state else None
    return Cache(torch.zeros(*shp, capacity, g.head_dim, dtype=torch.bfloat16, device=device),
                 torch.zeros(*shp, capacity, g.head_dim, dtype=torch.bfloat16, device=device),
                 torch.zeros(*shp, capacity, dtype=torch.int32, device=device),
                 torch.zeros(*shp, dtype=torch.int32, device=device),
                 torch.zeros(*shp, dtype=torch.int32, device=device), y, y_len)


def alloc_moments(g: mkv_geom, device="cuda"):
    shp = (g.batch, g.n_kv_heads)
    d = g.head_dim
    return Moments(torch.zeros(*shp, dtype=torch.int32, device=device),
                   torch.zeros(*shp, d, dtype=torch.float32, device=device),
                   torch.zeros(*shp, d, dtype=torch.float32, device=device),
                   torch.zeros(*shp, d, d, dtype=torch.float32, device=device))


def alloc_workspace(nbytes, device="cuda"):
    """Zero-filled device workspace (torch's allocator returns 512-byte aligned blocks)."""
    return torch.zeros(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ------------------------------------------------------------- functions
def mkv_version():
    return lib().mkv_version()


def mkv_status_str(code):
    return lib().mkv_status_str(code).decode()


def mkv_compress_workspace_size(g, T, p: mkv_compress_params):
    return lib().mkv_compress_workspace_size(g, T, ctypes.byref(p))


def mkv_decode_workspace_size(g, capacity):
    return lib().mkv_decode_workspace_size(g, capacity)


def mkv_evict_workspace_size(g, capacity):
    return lib().mkv_evict_workspace_size(g, capacity)


def mkv_compress(g, T, K, V, Q_obs, p: mkv_compress_params, cache: Cache, mom: Moments, ws, diag=None,
                 stream=None):
    d = mkv_compress_diag(*(None if x is None else x.data_ptr() for x in (diag or (None, None, None))))
    c, m = cache.c(), mom.c()
    code = lib().mkv_compress(g, T, _ptr(K), _ptr(V), _ptr(Q_obs), p, c, m, d, _ptr(ws), ws.numel(), _stream(stream))
    _check(code, "mkv_compress")


def mkv_decode_step(g, q, k_new, v_new, cache: Cache, mom: Moments | None, p: mkv_decode_params, out, lse,
                    ws, stream=None):
    c = cache.c()
    m = mom.c() if mom is not None else None
    code = lib().mkv_decode_step(g, _ptr(q), _ptr(k_new), _ptr(v_new), c, m, p, _ptr(out),
                                 _ptr(lse), _ptr(ws), ws.numel(), _stream(stream))
    _check(code, "mkv_decode_step")


def mkv_decode_step_noalloc(g, q, k_new, v_new, cache: Cache, mom: Moments | None, p: mkv_decode_params, out,
                            lse, stream=None):
    """mkv_decode_step with the library's fixed device scratch instead of a workspace."""
    c = cache.c()
    m = mom.c() if mom is not None else None
    code = lib().mkv_decode_step_noalloc(g, _ptr(q), _ptr(k_new), _ptr(v_new), c, m, p, _ptr(out),
                                         _ptr(lse), _stream(stream))
    _check(code, "mkv_decode_step_noalloc")


def mkv_evict_append(g, q, k_new, v_new, budget, cache: Cache, mom: Moments, tau, ws, stream=None):
    c, m = cache.c(), mom.c()
    code = lib().mkv_evict_append(g, _ptr(q), _ptr(k_new), _ptr(v_new), budget, c, m, tau, _ptr(ws), ws.numel(),
                                  _stream(stream))
    _check(code, "mkv_evict_append")


def mkv_decode_evict_workspace_size(g, capacity):
    return lib().mkv_decode_evict_workspace_size(g, capacity)


def mkv_decode_evict_step(g, q, k_new, v_new, budget, cache: Cache, mom: Moments, p: mkv_decode_params, out, lse,
                          ws, stream=None):
    """Algorithm 1 for one generated token: append, evict down to `budget`, corrected output."""
    c, m = cache.c(), mom.c()
    code = lib().mkv_decode_evict_step(g, _ptr(q), _ptr(k_new), _ptr(v_new), budget, c, m, p, _ptr(out), _ptr(lse),
                                       _ptr(ws), ws.numel(), _stream(stream))
    _check(code, "mkv_decode_evict_step")


def mkv_moments_pack_bf16(g, mom: Moments, C16, stream=None):
    """C16 (bf16 [b, h_kv, d, d]) = bf16(mom.C): the 16-bit copy mkv_decode_params.C16 points at."""
    m = mom.c()
    _check(lib().mkv_moments_pack_bf16(g, m, _ptr(C16), _stream(stream)), "mkv_moments_pack_bf16")


def mkv_moments_pack_split(g, mom: Moments, tau, C_split, stream=None):
    """C_split (int32 [b, h_kv, d, d], as many bytes as C) = the (hi, lo) bf16x2
    operand words of the clamped C': what mkv_decode_params.C_split points at."""
    m = mom.c()
    _check(lib().mkv_moments_pack_split(g, m, float(tau), _ptr(C_split), _stream(stream)),
           "mkv_moments_pack_split")


# -------------------------------------------- speculative decoding, positions
# These calls are made for every layer of every step, and a tensor's attribute
# takes 0.1 us on the host: shapes and strides are read once each, and the small
# structures of whole 64-bit fields go out as integer arrays.
_I64x7, _I64x9 = ctypes.c_int64 * 7, [ctypes.c_int64 * (9 * n) for n in range(5)]


def mkv_tree_build(parents, mask, pos, ws, count=None, base=None, stream=None):
    """Visibility words and positions of drafted trees: parents int32 [b, N] -> mask int32 [b, N, ceil(N / 32)],
    pos int32 [b, N] (or None).  base: int32 [b], any stride (e.g. cache.seen[:, 0])."""
    shape = parents.shape
    b, n = shape
    _int32(parents, shape, "parents")
    _int32(mask, (b, n, (n + 31) // 32), "mask")
    if pos is not None:
        _int32(pos, shape, "pos")
    if count is not None:
        _int32(count, (b,), "count")
    at, step = None, 0
    if base is not None:
        if base.dtype is not torch.int32 or base.shape != (b,):
            raise ValueError("base: int32 [b]")
        at, step = base.data_ptr(), base.stride(0)
    code = lib().mkv_tree_build(b, n, parents.data_ptr(), _ptr(count), at, step, mask.data_ptr(), _ptr(pos),
                                ws.data_ptr(), ws.numel(), _stream(stream))
    if code:
        _check(code, "mkv_tree_build")


def mkv_tree_workspace_size(g, n_nodes, capacity):
    return lib().mkv_tree_workspace_size(g, n_nodes, capacity)


def mkv_tree_step(g, tree: Tree, q, k, v, cache: Cache, mom: Moments | None, p: mkv_decode_params, out, lse, ws,
                  stream=None):
    """Attention of drafted nodes over the cache, the nodes they see and the moments: q bf16 [b, N, g*h_kv, d],
    k and v bf16 [b, N, h_kv, d] (nodes and batch items may be strided), out bf16 [b, N, g*h_kv, d], lse fp32
    [b, N, g*h_kv] or None."""
    b, n, h, d = tree.batch, tree.n_nodes, g.n_kv_heads, g.head_dim
    heads = g.group * h
    if not tree.usable:
        raise ValueError("tree: mask contiguous int32 [b, N, ceil(N / 32)], count contiguous int32 [b]")
    want, want_kv = (b, n, heads, d), (b, n, h, d)
    if g.batch != b or q.shape != want or out.shape != want or k.shape != want_kv or v.shape != want_kv:
        raise ValueError("q, out: [b, N, g*h_kv, d]; k, v: [b, N, h_kv, d], of the tree's b and N")
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    # (strides over an extent of one are never used and may differ)
    if (q.dtype is not _BF16 or k.dtype is not _BF16 or v.dtype is not _BF16 or out.dtype is not _BF16
            or (vs != ks and (vs[3] != 1 or (h > 1 and vs[2] != ks[2]) or (n > 1 and vs[1] != ks[1])
                              or (b > 1 and vs[0] != ks[0])))
            or not out.is_contiguous() or qs[3] != 1 or ks[3] != 1
            or (heads > 1 and qs[2] != d) or (h > 1 and ks[2] != d)):
        raise ValueError("q, k, v, out: bf16 with dense heads, k and v of the same strides, out contiguous")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (b, n, heads) or not lse.is_contiguous()):
        raise ValueError("lse: contiguous float32 [b, N, g*h_kv]")
    # (a stride over an extent of one is never used: 0, the dense value, stands for it; over a larger
    # extent 0 would be taken for the dense value, past the end of an expanded tensor)
    if (n > 1 and (qs[1] == 0 or ks[1] == 0)) or (b > 1 and (qs[0] == 0 or ks[0] == 0)):
        raise ValueError("q, k, v: not expanded over nodes or batch items")
    t = _I64x7(n, 0 if tree.count is None else tree.count.data_ptr(), tree.mask.data_ptr(), qs[1] if n > 1 else 0,
               qs[0] if b > 1 else 0, ks[1] if n > 1 else 0, ks[0] if b > 1 else 0)
    code = lib().mkv_tree_step(g, t, q.data_ptr(), k.data_ptr(), v.data_ptr(), cache.c(),
                               None if mom is None else mom.c(), p, out.data_ptr(), _ptr(lse), ws.data_ptr(),
                               ws.numel(), _stream(stream))
    if code:
        _check(code, "mkv_tree_step")


def tree_layers(layers):
    """(cache, k, v) of every layer, k and v as given to mkv_tree_step.  It holds their addresses: made once and kept
    beside the caches where a program's k and v stay in their buffers, and made again (36 layers: some 0.1 ms on the
    host) where a step has new ones."""
    layers = list(layers)
    _need(len(layers) > 0, "at least one layer")
    k0 = layers[0][1]
    kv, shape, stride = _nodes(k0, "k"), k0.shape, k0.stride()
    b, _, h, d = shape
    for c, k, v in layers:
        for t, what in ((k, "k"), (v, "v")):
            _need(t.shape == shape and ((t.stride() == stride and t.dtype is _BF16) or _nodes(t, what) == kv),
                  "k and v: the same shape and strides in every layer")
        cap = c.K.shape
        _need(cap[0] == b and cap[1] == h and cap[3] == d and c.V.shape == cap, "caches of the batch, heads and dims of k and v")
    array = (mkv_tree_layer * len(layers))(*(mkv_tree_layer(c.c(), k.data_ptr(), v.data_ptr()) for c, k, v in layers))
    return TreeLayers(array, mkv_tree(k0.shape[1], None, None, 0, 0, *kv), k0.shape[0], layers)


def mkv_tree_commit(g, layers: TreeLayers, path, n_path, ws, stream=None):
    """Appends the nodes path[b, :n_path[b]] (int32, root first) to the caches of all layers."""
    _int32(path, (g.batch, path.shape[1]), "path")
    _int32(n_path, (g.batch,), "n_path")
    _need(layers.batch == g.batch and layers.held[0][1].shape[2:] == (g.n_kv_heads, g.head_dim),
          "layers: k and v of this geometry")
    code = lib().mkv_tree_commit(g, ctypes.byref(layers.tree), len(layers.array), layers.array, path.data_ptr(),
                                 path.shape[1], n_path.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream))
    if code:
        _check(code, "mkv_tree_commit")


def rope_params(inv_freq, axis=None, neighbours=False):
    """Rotation parameters from rot_dim / 2 inverse frequencies and the position axis of each (None: axis 0)."""
    inv_freq = [float(x) for x in inv_freq]
    axis = [0] * len(inv_freq) if axis is None else [int(x) for x in axis]
    _need(len(inv_freq) == len(axis) <= 64, "as many axes as frequencies, at most 64")
    return mkv_rope_params(2 * len(inv_freq), int(neighbours), 0, max(axis, default=0) + 1,
                           (ctypes.c_float * 64)(*inv_freq), (c_i32 * 64)(*axis))


def mkv_rope(pos, p: mkv_rope_params, tensors, inverse=False, stream=None):
    """Rotates (in, out) pairs of bf16 [b, tokens, heads, d] tensors (any strides with adjacent dims; out may be in)
    by int32 positions pos [axes, b, tokens] (adjacent tokens; expanded axes and batches are fine).  inverse: by
    the negative angle."""
    axes, b, t = pos.shape
    ps = pos.stride()
    if pos.dtype is not torch.int32 or axes < p.n_axes or (ps[2] != 1 and t > 1):
        raise ValueError("pos: int32 [axes, b, tokens] with adjacent tokens")
    if not 0 < len(tensors) < 5:
        raise ValueError("tensors: one to four (in, out) pairs")
    d = tensors[0][0].shape[3]
    flat = []
    for x, y in tensors:
        shape, xs, ys = x.shape, x.stride(), y.stride()
        h = shape[2]
        if (x.dtype is not _BF16 or y.dtype is not _BF16 or shape != (b, t, h, d) or y.shape != shape or xs[3] != 1
                or ys[3] != 1):
            raise ValueError("tensors: pairs of bf16 [b, tokens, heads, d] with adjacent dims")
        if b == 1 or t == 1 or h == 1:  # (a stride over an extent of one is never used)
            xs, ys = ([s if e > 1 else 0 for s, e in zip(u, shape)] for u in (xs, ys))
        flat += (x.data_ptr(), y.data_ptr(), h, xs[0], xs[1], xs[2], ys[0], ys[1], ys[2])
    if inverse != p.inverse:
        p = mkv_rope_params.from_buffer_copy(p)
        p.inverse = int(inverse)
    code = lib().mkv_rope(b, t, d, pos.data_ptr(), ps[0], ps[1] if b > 1 else 0, p, len(tensors),
                          _I64x9[len(tensors)](*flat), _stream(stream))
    if code:
        _check(code, "mkv_rope")


def mkv_debug_set_poll_limit(polls):
    """Test hook (include/mkv_debug.h): poll limit of the kernels' pipeline
    waits; negative restores the default.  Returns the previous limit."""
    return lib().mkv_debug_set_poll_limit(int(polls))


def mkv_debug_force_ticket_merge(on):
    """Test hook (include/mkv_debug.h): decode merges through global partials."""
    return lib().mkv_debug_force_ticket_merge(1 if on else 0)


def mkv_get_device_error(ws, stream=None):
    """(status, info) recorded by kernels in this workspace; clears it."""
    info = c_i32(0)
    code = lib().mkv_get_device_error(_ptr(ws), _stream(stream), ctypes.byref(info))
    return code, info.value
