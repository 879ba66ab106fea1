"""ctypes binding of include/flatformer.h.  Argument marshalling only."""
import ctypes as C
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(HERE, "libflatformer.so")
_lib = None

FF_F32, FF_BF16, FF_F16 = 0, 1, 2
_TORCH_DTYPE = {FF_F32: torch.float32, FF_BF16: torch.bfloat16, FF_F16: torch.float16}
FF_TAIL_MASK, FF_TAIL_DROP = 0, 1
FF_FLAG_OUT_F32, FF_FLAG_FORCE_GENERIC, FF_FLAG_TAIL_DROP = 1, 2, 4


def FF_FLAG_VARIANT(v):
    return (int(v) & 0xF) << 8


class FlatformerError(RuntimeError):
    pass


class Geometry(C.Structure):
    """ff_geom"""
    _fields_ = [("num_frames", C.c_int32), ("grid_x", C.c_int32), ("grid_y", C.c_int32),
                ("win_x", C.c_int32), ("win_y", C.c_int32)]


class _LayerWeightsC(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o",
                                          "ln2_g", "ln2_b", "w1", "b1", "w2", "b2")] + \
               [("C", C.c_int32), ("F", C.c_int32), ("heads", C.c_int32), ("ln_eps", C.c_float),
                ("packed", C.c_void_p), ("pos_embed", C.c_void_p)]


class Geometry3(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("num_frames", "grid_x", "grid_y", "grid_z", "win_x", "win_y", "win_z")]


class VoxelGrid(C.Structure):
    _fields_ = [("x_min", C.c_float), ("y_min", C.c_float), ("voxel_x", C.c_float), ("voxel_y", C.c_float)]


class _HeadsC(C.Structure):
    """ff_heads"""
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class _GroupListC(C.Structure):
    """ff_group_list"""
    _fields_ = [("perm", C.c_void_p), ("offsets", C.c_void_p), ("n", C.c_int64), ("G", C.c_int32)]


class _AttentionShapeC(C.Structure):
    """ff_attention_shape"""
    _fields_ = [("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("scale", C.c_float),
                ("num_groups", C.c_void_p), ("max_groups", C.c_int32), ("queries", _GroupListC), ("keys", _GroupListC),
                ("key_mask", C.c_void_p)]


class _RotarySpecC(C.Structure):
    """ff_rotary_spec"""
    _fields_ = [("axes", C.c_int32), ("pairs", C.c_int32), ("layout", C.c_int32), ("inverse", C.c_int32),
                ("amplitude", C.c_float), ("freqs", C.c_void_p)]


_PARAMS = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_g", "ln2_b", "w1", "b1", "w2", "b2")


class LayerWeights:
    """Device tensors of one layer plus the ff_layer_weights struct that points at them."""

    def __init__(self, params, dtype, device="cuda"):
        tdt = _TORCH_DTYPE[dtype]
        self.dtype = dtype
        self.tensors = {k: torch.as_tensor(params[k], dtype=torch.float32).to(device=device, dtype=tdt).contiguous()
                        for k in _PARAMS}
        self.C, self.F, self.heads = int(params["C"]), int(params["F"]), int(params["heads"])
        self.ln_eps = float(params["ln_eps"])
        self.packed = None

    def pack(self):
        """Pre-pack the weights once (ff_pack_weights); later calls skip the per-call packing."""
        lib = load_library()
        s = self.struct()
        nbytes = lib.ff_pack_weights_bytes(C.byref(s), self.dtype)
        if nbytes == 0:
            return self
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.tensors["w_o"].device)
        ptr = (buf.data_ptr() + 255) // 256 * 256
        _check(lib.ff_pack_weights(C.byref(s), self.dtype, ptr, _stream()), "ff_pack_weights")
        self._packed_buf, self.packed = buf, ptr
        return self

    def struct(self, pos_embed=None):
        s = _LayerWeightsC()
        for k in _PARAMS:
            setattr(s, k, self.tensors[k].data_ptr())
        s.C, s.F, s.heads, s.ln_eps = self.C, self.F, self.heads, self.ln_eps
        s.packed = self.packed
        s.pos_embed = None if pos_embed is None else pos_embed.data_ptr()
        return s


_SIGS = {
    "ff_flatten_workspace_bytes": (C.c_size_t, [C.c_int64, C.POINTER(Geometry)]),
    "ff_flatten": (C.c_int, [C.c_void_p, C.c_int64, C.POINTER(Geometry), C.c_int, C.c_int, C.c_int, C.c_int,
                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ff_check_coords": (C.c_int, [C.c_void_p, C.c_int64, C.POINTER(Geometry), C.c_void_p, C.c_void_p]),
    "ff_flatten_batch_workspace_bytes": (C.c_size_t, [C.c_int64, C.POINTER(Geometry), C.c_int]),
    "ff_flatten_batch": (C.c_int, [C.c_void_p, C.c_int64, C.POINTER(Geometry), C.c_int, C.POINTER(C.c_int),
                                   C.POINTER(C.c_int), C.c_int, C.c_int, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                   C.POINTER(C.c_void_p), C.c_void_p, C.c_size_t, C.c_void_p]),
    "ff_group_attention_path": (C.c_int, [C.POINTER(_LayerWeightsC), C.c_int, C.c_int, C.c_uint32]),
    "ff_flatten_noalloc": (C.c_int, [C.c_void_p, C.c_int64, C.POINTER(Geometry), C.c_int, C.c_int, C.c_int, C.c_int,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "ff_flatten3d_workspace_bytes": (C.c_size_t, [C.c_int64, C.POINTER(Geometry3)]),
    "ff_flatten3d": (C.c_int, [C.c_void_p, C.c_int64, C.POINTER(Geometry3), C.c_int, C.c_int, C.c_int, C.c_int,
                               C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ff_group_attention_workspace_bytes": (C.c_size_t, [C.c_int64, C.c_int, C.POINTER(_LayerWeightsC), C.c_int]),
    "ff_group_attention": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_int32, C.POINTER(_LayerWeightsC), C.c_int, C.c_int, C.c_uint32,
                                     C.c_void_p, C.c_size_t, C.c_void_p]),
    "ff_pack_weights_bytes": (C.c_size_t, [C.POINTER(_LayerWeightsC), C.c_int]),
    "ff_pack_weights": (C.c_int, [C.POINTER(_LayerWeightsC), C.c_int, C.c_void_p, C.c_void_p]),
    "ff_gather": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_int, C.c_void_p]),
    "ff_scatter": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_int, C.c_void_p]),
    "ff_voxelize_workspace_bytes": (C.c_size_t, [C.c_int64, C.POINTER(Geometry)]),
    "ff_voxelize": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.POINTER(Geometry),
                              C.POINTER(VoxelGrid), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                              C.c_size_t, C.c_void_p]),
    "ff_bev_scatter": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.POINTER(Geometry), C.c_int, C.c_int, C.c_void_p,
                                 C.c_void_p]),
    "ff_fwa_block_workspace_bytes": (C.c_size_t, [C.c_int64, C.POINTER(Geometry), C.c_int,
                                                   C.POINTER(_LayerWeightsC), C.c_int, C.c_int]),
    "ff_fwa_block": (C.c_int, [C.c_void_p, C.c_int64, C.POINTER(Geometry), C.c_int, C.c_int, C.POINTER(_LayerWeightsC),
                               C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ff_fwa_block3d_workspace_bytes": (C.c_size_t, [C.c_int64, C.POINTER(Geometry3), C.c_int,
                                                     C.POINTER(_LayerWeightsC), C.c_int, C.c_int]),
    "ff_fwa_block3d": (C.c_int, [C.c_void_p, C.c_int64, C.POINTER(Geometry3), C.c_int, C.c_int,
                                 C.POINTER(_LayerWeightsC), C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_size_t, C.c_void_p]),
    "ff_attention_workspace_bytes": (C.c_size_t, [C.POINTER(_AttentionShapeC), C.c_int]),
    "ff_attention": (C.c_int, [C.POINTER(_AttentionShapeC)] + [C.POINTER(_HeadsC)] * 4 +
                     [C.c_void_p, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ff_attention_backward_workspace_bytes": (C.c_size_t, [C.POINTER(_AttentionShapeC), C.c_int]),
    "ff_attention_backward": (C.c_int, [C.POINTER(_AttentionShapeC)] + [C.POINTER(_HeadsC)] * 4 + [C.c_void_p] +
                              [C.POINTER(_HeadsC)] * 4 + [C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ff_rotary": (C.c_int, [C.POINTER(_HeadsC), C.POINTER(_HeadsC), C.c_int32, C.POINTER(_HeadsC), C.POINTER(_HeadsC),
                            C.c_int32, C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.c_int64, C.POINTER(_RotarySpecC),
                            C.c_int, C.c_void_p]),
    "ff_rotary_frequencies": (C.c_int, [C.POINTER(C.c_double), C.c_int32] + [C.c_double] * 5),
    "ff_status_string": (C.c_char_p, [C.c_int]),
    "ff_version": (C.c_int, []),
}


def library_path():
    return _LIB_PATH


def exported_symbols():
    return tuple(_SIGS)


def load_library():
    """Load libflatformer.so (built by paper_2301_08739_amd.build).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FlatformerError(f"{_LIB_PATH} not built: run `python -m paper_2301_08739_amd.build`")
        lib = C.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def ff_status_string(status):
    return load_library().ff_status_string(int(status)).decode()


def ff_version():
    return load_library().ff_version()


def _check(st, what):
    if st != 0:
        raise FlatformerError(f"{what}: {ff_status_string(st)} ({st})")


# The number of a device's current stream, 0.3 us; a Stream object on the way to it, where a torch has no shorter one, 3.3
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream():
    """The current stream of the current device as a number."""
    return _raw_stream(torch.cuda.current_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 256) + 256, dtype=torch.uint8, device=device)


def _aligned(ws):
    """The first 256-byte boundary of ws, and the bytes that are there from it on, whatever it is; a smaller tensor has none."""
    p, n = ws.data_ptr(), ws.numel()
    return (p + 255) // 256 * 256, n - 256 if n > 256 else 0


def ff_flatten_workspace_bytes(n, geom):
    return load_library().ff_flatten_workspace_bytes(int(n), C.byref(geom))


def _group_lists(count, cap, device):
    """`count` pairs (group_offsets of capacity cap, -1 throughout, num_groups, which every sort writes).  One fill for all of
    them: it is a launch, 1.3 us in a graph and more in an eager call (a captured call of four sorts of 30,000 pillars: a fill
    for each tensor 25.7 us, one fill 15.2; one sort 15.7 and 14.2)."""
    if count == 1:  # (a view of a filled tensor would cost more than a tensor of its own)
        return [(torch.full((cap,), -1, dtype=torch.int32, device=device), torch.empty(1, dtype=torch.int32, device=device))]
    width = -(-cap // 64) * 64 + 64  # (each tensor on a 256-byte boundary)
    both = torch.full((count, width), -1, dtype=torch.int32, device=device)
    return [(row[:cap], row[width - 64:width - 63]) for row in both.unbind(0)]


def ff_flatten(coords, geom, axis, shift, G, tail=FF_TAIL_MASK, want_keys=False, workspace=None):
    """coords: int32 cuda tensor [n,3].  Returns (perm, group_offsets, num_groups, keys_sorted|None),
    all device tensors; group_offsets has capacity ceil(n/G)+num_frames+1."""
    lib = load_library()
    assert coords.dtype == torch.int32 and coords.is_contiguous() and coords.is_cuda
    n = coords.shape[0]
    dev = coords.device
    cap = -(-n // max(G, 1)) + geom.num_frames + 1
    perm = torch.empty(n, dtype=torch.int32, device=dev)
    (goff, ng), = _group_lists(1, cap, dev)
    keys = torch.empty(n, dtype=torch.int64, device=dev) if want_keys else None
    need = lib.ff_flatten_workspace_bytes(n, C.byref(geom))
    ws = workspace if workspace is not None else _workspace(need, dev)
    st = lib.ff_flatten(_ptr(coords), n, C.byref(geom), axis, shift, G, tail, _ptr(perm), _ptr(goff), _ptr(ng),
                        _ptr(keys), *_aligned(ws), _stream())
    _check(st, "ff_flatten")
    return perm, goff, ng, keys


def ff_check_coords(coords, geom):
    """Device tensor int32 [2]: (rows of coords outside the geometry, index of the first one or n)."""
    lib = load_library()
    assert coords.dtype == torch.int32 and coords.is_contiguous() and coords.is_cuda and coords.shape[1] == 3
    res = torch.empty(2, dtype=torch.int32, device=coords.device)
    _check(lib.ff_check_coords(_ptr(coords), coords.shape[0], C.byref(geom), _ptr(res), _stream()), "ff_check_coords")
    return res


def ff_flatten_batch_workspace_bytes(n, geom, num_sorts):
    return load_library().ff_flatten_batch_workspace_bytes(int(n), C.byref(geom), int(num_sorts))


def ff_flatten_batch(coords, geom, sorts, G, tail=FF_TAIL_MASK, workspace=None, out=None):
    """sorts: up to four (axis, shift) pairs, sorted together.  Returns a list of (perm, group_offsets,
    num_groups) device tensors, one triple per pair (out: such a list to write into instead of new tensors)."""
    lib = load_library()
    assert coords.dtype == torch.int32 and coords.is_contiguous() and coords.is_cuda
    n, dev, S = coords.shape[0], coords.device, len(sorts)
    cap = -(-n // max(G, 1)) + geom.num_frames + 1
    if out is None:
        out = [(torch.empty(n, dtype=torch.int32, device=dev), goff, ng) for goff, ng in _group_lists(S, cap, dev)]
    axis = (C.c_int * S)(*[int(a) for a, _ in sorts])
    shift = (C.c_int * S)(*[int(b) for _, b in sorts])
    ptrs = [(C.c_void_p * S)(*[t[k].data_ptr() for t in out]) for k in range(3)]
    ws = workspace if workspace is not None else _workspace(lib.ff_flatten_batch_workspace_bytes(n, C.byref(geom), S), dev)
    st = lib.ff_flatten_batch(_ptr(coords), n, C.byref(geom), S, axis, shift, G, tail, ptrs[0], ptrs[1], ptrs[2],
                              *_aligned(ws), _stream())
    _check(st, "ff_flatten_batch")
    return out


FF_PATH_PLAIN, FF_PATH_FUSED = 0, 1


def ff_group_attention_path(weights, G, dtype, flags=0):
    """FF_PATH_FUSED (16-bit matrix-core operands) or FF_PATH_PLAIN (fp32 arithmetic, always so for FF_F32): what
    ff_group_attention would run on for these arguments."""
    s = weights.struct()
    st = load_library().ff_group_attention_path(C.byref(s), int(G), int(dtype), int(flags))
    if st < 0:
        _check(st, "ff_group_attention_path")
    return st


FF_NOALLOC_SCRATCH_BYTES = 8 << 20


def ff_flatten_noalloc(coords, geom, axis, shift, G, perm, group_offsets, num_groups, keys=None, tail=FF_TAIL_MASK):
    """ff_flatten on the library's static scratch array: every buffer is the caller's (perm int32 [n],
    group_offsets int32 [ceil(n/G)+num_frames+1], num_groups int32 [1], keys int64 [n] or None) and the call
    allocates nothing."""
    lib = load_library()
    assert coords.dtype == torch.int32 and coords.is_contiguous() and coords.is_cuda
    st = lib.ff_flatten_noalloc(_ptr(coords), coords.shape[0], C.byref(geom), axis, shift, G, tail, _ptr(perm),
                                _ptr(group_offsets), _ptr(num_groups), _ptr(keys), _stream())
    _check(st, "ff_flatten_noalloc")


def ff_flatten3d(coords, geom, axis, shift, G, tail=FF_TAIL_MASK, workspace=None):
    """coords: int32 cuda tensor [n,4] (b,x,y,z).  Returns (perm, group_offsets, num_groups)."""
    lib = load_library()
    assert coords.dtype == torch.int32 and coords.is_contiguous() and coords.is_cuda and coords.shape[1] == 4
    n = coords.shape[0]
    dev = coords.device
    cap = -(-n // max(G, 1)) + geom.num_frames + 1
    perm = torch.empty(n, dtype=torch.int32, device=dev)
    (goff, ng), = _group_lists(1, cap, dev)
    need = lib.ff_flatten3d_workspace_bytes(n, C.byref(geom))
    ws = workspace if workspace is not None else _workspace(need, dev)
    st = lib.ff_flatten3d(_ptr(coords), n, C.byref(geom), axis, shift, G, tail, _ptr(perm), _ptr(goff), _ptr(ng),
                          *_aligned(ws), _stream())
    _check(st, "ff_flatten3d")
    return perm, goff, ng


def ff_group_attention_workspace_bytes(n, G, weights, dtype):
    s = weights.struct()
    return load_library().ff_group_attention_workspace_bytes(int(n), int(G), C.byref(s), dtype)


def ff_group_attention(feats, perm, group_offsets, num_groups, max_groups, weights, G, dtype,
                       flags=0, out=None, workspace=None, pos_embed=None):
    """feats [n,C] (float32, bfloat16 or float16 per dtype) -> out [n,C] in pillar order.  pos_embed: None or a
    tensor like feats (the positional embedding of every pillar)."""
    lib = load_library()
    assert feats.is_cuda and feats.is_contiguous()
    n = feats.shape[0]
    if out is None:
        odt = torch.float32 if (flags & FF_FLAG_OUT_F32) else _TORCH_DTYPE[dtype]
        out = torch.empty((n, weights.C), dtype=odt, device=feats.device)
    if pos_embed is not None:
        assert pos_embed.shape == feats.shape and pos_embed.dtype == feats.dtype and pos_embed.is_contiguous()
    s = weights.struct(pos_embed)
    need = lib.ff_group_attention_workspace_bytes(n, G, C.byref(s), dtype)
    ws = workspace if workspace is not None else _workspace(need, feats.device)
    st = lib.ff_group_attention(_ptr(feats), _ptr(out), n, _ptr(perm), _ptr(group_offsets), _ptr(num_groups),
                                int(max_groups), C.byref(s), G, dtype, flags,
                                *_aligned(ws), _stream())
    _check(st, "ff_group_attention")
    return out


def _rows(fn_name, src, perm, dtype, out):
    lib = load_library()
    n, Cc = src.shape
    if out is None:
        out = torch.empty_like(src)
    st = getattr(lib, fn_name)(_ptr(src), _ptr(out), _ptr(perm), n, Cc, dtype, _stream())
    _check(st, fn_name)
    return out


def ff_gather(src, perm, dtype, out=None):
    return _rows("ff_gather", src, perm, dtype, out)


def ff_scatter(src, perm, dtype, out=None):
    return _rows("ff_scatter", src, perm, dtype, out)


def ff_voxelize(xy, frame, point_feats, geom, grid, want_map=True, workspace=None):
    """xy float32 [m,2], frame int32 [m] or None, point_feats float32 [m,Cp] ->
    (coords int32 [m,3], feats float32 [m,Cp], num_pillars int32 [1], point_to_pillar int32 [m] | None);
    only the first num_pillars rows of coords / feats are meaningful."""
    lib = load_library()
    assert xy.dtype == torch.float32 and xy.is_contiguous() and point_feats.dtype == torch.float32 and point_feats.is_contiguous()
    m, Cp = point_feats.shape
    dev = xy.device
    coords = torch.empty((m, 3), dtype=torch.int32, device=dev)
    feats = torch.empty((m, Cp), dtype=torch.float32, device=dev)
    npil = torch.empty(1, dtype=torch.int32, device=dev)  # (always written)
    p2p = torch.empty(m, dtype=torch.int32, device=dev) if want_map else None
    need = lib.ff_voxelize_workspace_bytes(m, C.byref(geom))
    ws = workspace if workspace is not None else _workspace(need, dev)
    st = lib.ff_voxelize(_ptr(xy), _ptr(frame), _ptr(point_feats), m, Cp, C.byref(geom), C.byref(grid), _ptr(coords),
                         _ptr(feats), _ptr(npil), _ptr(p2p), *_aligned(ws), _stream())
    _check(st, "ff_voxelize")
    return coords, feats, npil, p2p


def ff_voxelize_workspace_bytes(m, geom):
    return load_library().ff_voxelize_workspace_bytes(int(m), C.byref(geom))


def ff_bev_scatter(feats, coords, geom, dtype, out=None):
    """feats [n,C], coords [n,3] -> dense map [num_frames, grid_y, grid_x, C] (channels last)."""
    lib = load_library()
    n, Cc = feats.shape
    if out is None:
        out = torch.empty((geom.num_frames, geom.grid_y, geom.grid_x, Cc), dtype=feats.dtype, device=feats.device)
    st = lib.ff_bev_scatter(_ptr(feats), _ptr(coords), n, C.byref(geom), Cc, dtype, _ptr(out), _stream())
    _check(st, "ff_bev_scatter")
    return out


_ARRAY_CACHE = {}


def _layer_array(layers, pos_embed=None):
    """The ff_layer_weights array of a block's layers.  Built once per (layer objects, packed state, embedding
    buffer) and kept: a serving loop calls the block with the same layers every frame."""
    key = (tuple(id(l) for l in layers), tuple(l.packed for l in layers),
           None if pos_embed is None else pos_embed.data_ptr())
    hit = _ARRAY_CACHE.get(key)
    if hit is not None and all(a is b for a, b in zip(hit[1], layers)):
        return hit[0]
    arr = (_LayerWeightsC * len(layers))()
    for i, l in enumerate(layers):
        arr[i] = l.struct(pos_embed)
    if len(_ARRAY_CACHE) > 64:
        _ARRAY_CACHE.clear()
    _ARRAY_CACHE[key] = (arr, list(layers))
    return arr


def _block_entry(lib, geom):
    if isinstance(geom, Geometry3):
        return lib.ff_fwa_block3d_workspace_bytes, lib.ff_fwa_block3d, "ff_fwa_block3d"
    return lib.ff_fwa_block_workspace_bytes, lib.ff_fwa_block, "ff_fwa_block"


def ff_fwa_block_workspace_bytes(n, geom, G, layers, dtype):
    """geom: Geometry (coords [n,3]) or Geometry3 (coords [n,4]: the ff_fwa_block3d entry points)."""
    arr = _layer_array(layers)
    return _block_entry(load_library(), geom)[0](int(n), C.byref(geom), G, arr, len(layers), dtype)


def ff_fwa_block(coords, geom, G, layers, dtype, feats_in, out=None, workspace=None, tail=FF_TAIL_MASK,
                 pos_embed=None):
    """pos_embed: None or a tensor like feats_in, handed to every layer of the block.  With a Geometry3
    and coords [n,4] this calls ff_fwa_block3d."""
    lib = load_library()
    n = coords.shape[0]
    query, run, name = _block_entry(lib, geom)
    assert coords.shape[1] == (4 if isinstance(geom, Geometry3) else 3)
    if pos_embed is not None:
        assert pos_embed.shape == feats_in.shape and pos_embed.dtype == feats_in.dtype and pos_embed.is_contiguous()
    arr = _layer_array(layers, pos_embed)
    if out is None:
        out = torch.empty_like(feats_in)
    ws = workspace if workspace is not None else _workspace(query(n, C.byref(geom), G, arr, len(layers), dtype),
                                                              coords.device)   # (the call itself checks the size)
    st = run(_ptr(coords), n, C.byref(geom), G, tail, arr, len(layers), dtype, _ptr(feats_in), _ptr(out),
             *_aligned(ws), _stream())
    _check(st, name)
    return out


# ---- attention over rows that the caller holds, and rotary positions ---------------------------------------------------
_FF_DTYPE = {v: k for k, v in _TORCH_DTYPE.items()}
FF_ROTARY_HALF, FF_ROTARY_INTERLEAVED = 0, 1


def _refuse(what, why):
    raise FlatformerError(f"{what}: {why}")


def _heads(what, name, t, shape, dtype, device):
    """ff_heads of a tensor [n, heads, head_dim] of any strides but the last, which is 1.  device: number of the GPU."""
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape:
        _refuse(what, f"{name}: {tuple(t.shape)} of {t.dtype} on {t.device}, wanted {tuple(shape)} of {dtype} on device {device}")
    rs, hs, es = t.stride()
    if es != 1 and shape[2] > 1 and t.numel():
        _refuse(what, f"{name}: the elements of a head have to lie side by side")
    return _HeadsC(t.data_ptr(), rs, hs)


def _array(what, name, t, length, dtype, device):
    """Address of a contiguous tensor of at least `length` elements; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or t.numel() < length or not t.is_contiguous():
        _refuse(what, f"{name}: {tuple(t.shape)} of {t.dtype} on {t.device}, wanted {length} contiguous elements of {dtype} on device {device}")
    return t.data_ptr()


# The number of the current device, 0.1 us; torch.cuda's function takes 0.25
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _off_device(what, device):
    """Is a tensor's device another one than the current?"""
    if device < 0:
        _refuse(what, "the tensors have to be on a GPU")
    return device != _current_device()


def _attention_shape(what, q, k, v, perm, group_offsets, num_groups, max_groups, G, scale, key_mask, key_perm, key_offsets, key_G):
    """(ff_attention_shape, ff_heads of q, of k and of v, dtype code)"""
    dt = _FF_DTYPE.get(q.dtype)
    if dt is None or q.dim() != 3 or k.dim() != 3:
        _refuse(what, "q, k and v are [rows, heads, head_dim] of float32, bfloat16 or float16")
    shape, dtype, dev = q.shape, q.dtype, q.get_device()
    kshape = k.shape
    (nq, H, D), (nk, K, Dk) = shape, kshape
    hq = _heads(what, "q", q, shape, dtype, dev)
    hk = _heads(what, "k", k, kshape if Dk == D else (nk, K, D), dtype, dev)
    hv = _heads(what, "v", v, kshape, dtype, dev)
    if group_offsets is None:
        _refuse(what, "group_offsets is missing")
    i32, mg = torch.int32, int(max_groups)
    lq = (_array(what, "perm", perm, nq, i32, dev), _array(what, "group_offsets", group_offsets, mg + 1, i32, dev), nq, G)
    if key_offsets is None:
        if key_perm is not None or key_G is not None or nk != nq:
            _refuse(what, "keys with a list of their own need key_offsets")
        lk = lq
    else:
        lk = (_array(what, "key_perm", key_perm, nk, i32, dev), _array(what, "key_offsets", key_offsets, mg + 1, i32, dev), nk,
              max(nk, 1) if key_G is None else key_G)
    if key_mask is not None and key_mask.dtype is torch.bool:
        key_mask = key_mask.view(torch.uint8)
    s = _AttentionShapeC(H, K, D, D ** -0.5 if scale is None else scale, _array(what, "num_groups", num_groups, 1, i32, dev), mg,
                         lq, lk, _array(what, "key_mask", key_mask, nk, torch.uint8, dev))
    return s, hq, hk, hv, dt


def ff_attention_workspace_bytes(heads, kv_heads, head_dim, nq, max_groups, G, dtype, nk=None, key_G=None):
    """Bytes that a workspace of ff_attention has to have behind its first 256-byte boundary."""
    s = _plan_shape(heads, kv_heads, head_dim, nq, max_groups, G, nk, key_G)
    return load_library().ff_attention_workspace_bytes(C.byref(s), dtype)


def ff_attention_backward_workspace_bytes(heads, kv_heads, head_dim, nq, max_groups, G, dtype, nk=None, key_G=None):
    s = _plan_shape(heads, kv_heads, head_dim, nq, max_groups, G, nk, key_G)
    return load_library().ff_attention_backward_workspace_bytes(C.byref(s), dtype)


def _plan_shape(heads, kv_heads, head_dim, nq, max_groups, G, nk, key_G):
    nk = nq if nk is None else nk
    return _AttentionShapeC(heads, kv_heads, head_dim, 1.0, None, max_groups, _GroupListC(None, None, nq, G),
                            _GroupListC(None, None, nk, G if key_G is None else key_G), None)


def ff_attention(q, k, v, perm, group_offsets, num_groups, max_groups, G, scale=None, key_mask=None, key_perm=None,
                 key_offsets=None, key_G=None, out=None, lse=None, want_lse=True, workspace=None):
    """Attention inside groups: q [nq, heads, head_dim], k and v [nk, kv_heads, head_dim], any strides with the elements of a
    head side by side.  perm (or None), group_offsets, num_groups (or None) and max_groups are a sort's lists, or any others; keys
    take the same ones unless key_offsets is given (key_perm, key_G: its row numbers and its longest group).  key_mask [nk],
    uint8 or bool: 0 takes a row out.  scale: head_dim ** -0.5 unless given.  Returns (out [nq, heads, head_dim], lse float32
    [nq, heads] or None).  Rows that no group covers are left as they were; new tensors are zero there."""
    what = "ff_attention"
    lib = load_library()
    s, hq, hk, hv, dt = _attention_shape(what, q, k, v, perm, group_offsets, num_groups, max_groups, G, scale, key_mask, key_perm,
                                         key_offsets, key_G)
    shape, dev = q.shape, q.get_device()
    if _off_device(what, dev):
        with torch.cuda.device(dev):
            return ff_attention(q, k, v, perm, group_offsets, num_groups, max_groups, G, scale, key_mask, key_perm, key_offsets, key_G,
                                out, lse, want_lse, workspace)
    if out is None:
        out = torch.zeros(shape, dtype=q.dtype, device=q.device)
    if lse is None and want_lse:
        lse = torch.zeros(shape[:2], dtype=torch.float32, device=q.device)
    ho = _heads(what, "out", out, shape, q.dtype, dev)
    st = lib.ff_attention(s, hq, hk, hv, ho, _array(what, "lse", lse, shape[0] * shape[1], torch.float32, dev), dt,
                          *_room(lib.ff_attention_workspace_bytes, s, dt, workspace, q), _raw_stream(dev))
    _check(st, what)
    return out, lse


def ff_attention_backward(q, k, v, out, lse, dout, perm, group_offsets, num_groups, max_groups, G, scale=None, key_mask=None,
                          key_perm=None, key_offsets=None, key_G=None, dq=None, dk=None, dv=None, workspace=None):
    """The gradient of ff_attention: out and lse as it gave them for the same arguments, dout the gradient of out.  Returns (dq, dk,
    dv), like q, k and v.  Rows that no group covers are left as they were; new tensors are zero there."""
    what = "ff_attention_backward"
    lib = load_library()
    s, hq, hk, hv, dt = _attention_shape(what, q, k, v, perm, group_offsets, num_groups, max_groups, G, scale, key_mask, key_perm,
                                         key_offsets, key_G)
    if lse is None:
        _refuse(what, "lse is missing")
    shape, kshape, dtype, dev = q.shape, k.shape, q.dtype, q.get_device()
    if _off_device(what, dev):
        with torch.cuda.device(dev):
            return ff_attention_backward(q, k, v, out, lse, dout, perm, group_offsets, num_groups, max_groups, G, scale, key_mask,
                                         key_perm, key_offsets, key_G, dq, dk, dv, workspace)
    if dq is None:
        dq = torch.zeros(shape, dtype=dtype, device=q.device)
    if dk is None:
        dk = torch.zeros(kshape, dtype=dtype, device=q.device)
    if dv is None:
        dv = torch.zeros(kshape, dtype=dtype, device=q.device)
    st = lib.ff_attention_backward(
        s, hq, hk, hv, _heads(what, "out", out, shape, dtype, dev), _array(what, "lse", lse, shape[0] * shape[1], torch.float32, dev),
        _heads(what, "dout", dout, shape, dtype, dev), _heads(what, "dq", dq, shape, dtype, dev), _heads(what, "dk", dk, kshape, dtype, dev),
        _heads(what, "dv", dv, kshape, dtype, dev), dt, *_room(lib.ff_attention_backward_workspace_bytes, s, dt, workspace, q),
        _raw_stream(dev))
    _check(st, what)
    return dq, dk, dv


def _room(query, s, dt, workspace, q):
    """Address and size of the workspace: the caller's, or as large a one as the call needs."""
    if workspace is None:
        need = query(s, dt)
        if not need:
            return None, 0
        workspace = _workspace(need, q.device)
    return _aligned(workspace)


def ff_rotary_frequencies(pairs, axes=1, base=10000.0, factor=1.0, original_length=0.0, low_turns=1.0, high_turns=32.0,
                          device="cuda"):
    """float64 [axes, pairs], radians a position, the same for every axis: what ff_rotary takes as freqs."""
    f = (C.c_double * max(int(pairs), 1))()
    _check(load_library().ff_rotary_frequencies(f, int(pairs), float(base), float(factor), float(original_length), float(low_turns),
                                                float(high_turns)), "ff_rotary_frequencies")
    return torch.tensor(list(f), dtype=torch.float64).repeat(axes, 1).to(device)


def ff_rotary(q, k, positions, freqs, layout=FF_ROTARY_HALF, amplitude=1.0, inverse=False, q_out=None, k_out=None):
    """q [n, q_heads, head_dim] and k [n, k_heads, head_dim] (or None) turned by their positions: int32 [n] or [n, axes], such as
    coords[:, 1:], with freqs float64 [axes, pairs].  q_out / k_out may be q / k.  Returns (q_out, k_out)."""
    what = "ff_rotary"
    lib = load_library()
    dt = _FF_DTYPE.get(q.dtype)
    if dt is None or q.dim() != 3 or (k is not None and k.dim() != 3) or freqs.dim() != 2:
        _refuse(what, "q and k are [rows, heads, head_dim] of float32, bfloat16 or float16, freqs is [axes, pairs]")
    shape, dtype, dev, (axes, pairs) = q.shape, q.dtype, q.get_device(), freqs.shape
    n, H, D = shape
    placed = positions.shape
    if positions.dtype is not torch.int32 or positions.get_device() != dev or not (placed == (n, axes) or (axes == 1 and placed == (n,))):
        _refuse(what, f"positions: {tuple(placed)} of {positions.dtype} on {positions.device}, wanted int32 {(n, axes)} on device {dev}")
    spec = _RotarySpecC(axes, pairs, layout, 1 if inverse else 0, amplitude, _array(what, "freqs", freqs, axes * pairs, torch.float64, dev))
    hq = _heads(what, "q", q, shape, dtype, dev)
    if _off_device(what, dev):
        with torch.cuda.device(dev):
            return ff_rotary(q, k, positions, freqs, layout, amplitude, inverse, q_out, k_out)
    if q_out is None:
        q_out = torch.empty(shape, dtype=dtype, device=q.device)
    hqo = _heads(what, "q_out", q_out, shape, dtype, dev)
    hk, hko, K = None, None, 0
    if k is not None:
        kshape = k.shape
        K = kshape[1]
        hk = _heads(what, "k", k, kshape if kshape[0] == n and kshape[2] == D else (n, K, D), dtype, dev)
        if k_out is None:
            k_out = torch.empty(kshape, dtype=dtype, device=q.device)
        hko = _heads(what, "k_out", k_out, kshape, dtype, dev)
    stride = positions.stride()
    st = lib.ff_rotary(hq, hqo, H, hk, hko, K, n, D, positions.data_ptr(), stride[0], stride[-1] if len(stride) > 1 else 1, spec, dt,
                       _raw_stream(dev))
    _check(st, what)
    return q_out, k_out
