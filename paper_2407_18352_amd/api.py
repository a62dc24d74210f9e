"""Python binding of the C ABI, with torch tensors as device memory.

Argument marshalling only: descriptors are filled from plain-data specs and
tensor metadata, and the calls go straight to ``libhpacml.so``.  Specs have the
form ``{"rank", "slices": [(lo, count), ...], "sweep": (start, stop, step),
"bnd": [...]}`` (one right-hand-side slice per entry, Sec. III-B; the sweep is
the concrete slice of a tensor map, Sec. III-C).
"""
from __future__ import annotations

import ctypes as C

from . import _abi
from ._abi import check, lib


def _functor(spec, n_targets, n_features=None):
    R = min(max(int(spec["rank"]), 0), _abi.MAX_RANK)
    slices = spec["slices"]
    arr = (_abi.Slice * max(1, len(slices)))()
    per = 0
    for s, (lo, cnt) in enumerate(slices):
        e = 1
        for d in range(_abi.MAX_RANK):
            arr[s].lo[d] = int(lo[d]) if d < R else 0
            arr[s].count[d] = int(cnt[d]) if d < R else 1
            if d < R:
                e *= int(cnt[d])
        per += e
    f = _abi.Functor()
    f.rank, f.n_slices = int(spec["rank"]), len(slices)
    f.slices = C.cast(arr, C.POINTER(_abi.Slice))
    f.n_features = per * n_targets if n_features is None else int(n_features)
    return f, arr


def _sweep(spec):
    R = min(max(int(spec["rank"]), 0), _abi.MAX_RANK)
    sw = _abi.Sweep()
    start, stop, step = spec["sweep"]
    for d in range(_abi.MAX_RANK):
        sw.start[d] = int(start[d]) if d < R else 0
        sw.stop[d] = int(stop[d]) if d < R else 1
        sw.step[d] = int(step[d]) if d < R else 1
    bl = [int(b) for b in spec.get("bnd", [0] * R)][:R]
    bnd = (C.c_int32 * _abi.MAX_RANK)(*(bl + [0] * (_abi.MAX_RANK - len(bl))))
    return sw, bnd


def array_desc(data_ptr: int, shape, strides, dtype: int = _abi.F32):
    """An ``hpacml_array`` from raw metadata (strides in elements)."""
    a = _abi.Array()
    a.data = C.c_void_p(int(data_ptr))
    a.dtype = dtype
    a.reserved = 0
    for d in range(_abi.MAX_RANK):
        a.extent[d] = int(shape[d]) if d < len(shape) else 1
        a.stride[d] = int(strides[d]) if d < len(strides) else 0
    return a


def _tensor_desc(t):
    import torch
    if t.dtype != torch.float32:
        raise TypeError("map targets must be float32 tensors")
    return array_desc(t.data_ptr(), tuple(t.shape), tuple(t.stride()))


def validate_map(spec, arrays, direction: int, n_features=None):
    """``hpacml_map_validate`` on descriptors (no device access).  ``arrays`` are
    ``hpacml_array`` structures (see ``array_desc``).  Returns
    ``(status, n_points, n_features)``."""
    f, keep = _functor(spec, len(arrays), n_features)
    sw, bnd = _sweep(spec)
    tarr = (_abi.Array * max(1, len(arrays)))(*arrays)
    npts, nfeat = C.c_int64(-1), C.c_int32(-1)
    st = lib().hpacml_map_validate(C.byref(f), direction, tarr, len(arrays), C.byref(sw), bnd,
                                   C.byref(npts), C.byref(nfeat))
    return st, npts.value, nfeat.value


def validate_model(dims, act, compute: int):
    L = len(dims) - 1
    d = (C.c_int32 * len(dims))(*dims)
    a = (C.c_int32 * max(1, len(act)))(*act)
    return lib().hpacml_model_validate(L, d, a, compute)


class Map:
    """A tensor map over torch tensors (device memory is borrowed: keep the
    tensors alive while work that uses the map is in flight)."""

    def __init__(self, spec, targets, direction: int, n_features=None):
        self.targets = list(targets)
        f, keep = _functor(spec, len(self.targets), n_features)
        sw, bnd = _sweep(spec)
        tarr = (_abi.Array * max(1, len(self.targets)))(*[_tensor_desc(t) for t in self.targets])
        h = C.c_void_p()
        check(lib().hpacml_map_create(C.byref(f), direction, tarr, len(self.targets), C.byref(sw), bnd,
                                      C.byref(h)), "hpacml_map_create")
        self.handle = h
        npts, nfeat = C.c_int64(), C.c_int32()
        check(lib().hpacml_map_shape(h, C.byref(npts), C.byref(nfeat)), "hpacml_map_shape")
        self.n_points, self.n_features = npts.value, nfeat.value

    def close(self):
        if getattr(self, "handle", None):
            lib().hpacml_map_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Model:
    """A surrogate MLP; weights are host fp32 arrays [out][in] (numpy or torch
    CPU), copied into library-owned device memory."""

    def __init__(self, spec):
        import numpy as np
        dims = [int(x) for x in spec["dims"]]
        L = len(dims) - 1
        self.W = [np.ascontiguousarray(np.asarray(w, dtype=np.float32)) for w in spec["W"]]
        self.b = [np.ascontiguousarray(np.asarray(b, dtype=np.float32)) for b in spec["b"]]
        # the library reads dims[l+1] x dims[l] weights through a plain pointer:
        # arrays of another size are refused here (invalid dims are left to
        # the library's own status)
        if len(self.W) != L or len(self.b) != L:
            raise ValueError("model spec: %d weight and %d bias arrays for %d layers" % (len(self.W), len(self.b), L))
        if min(dims) > 0:
            for l in range(L):
                if self.W[l].size != dims[l + 1] * dims[l] or self.b[l].size != dims[l + 1]:
                    raise ValueError("layer %d: weights of %d and biases of %d values, expected %d x %d and %d"
                                     % (l, self.W[l].size, self.b[l].size, dims[l + 1], dims[l], dims[l + 1]))
        Wp = (C.POINTER(C.c_float) * L)(*[w.ctypes.data_as(C.POINTER(C.c_float)) for w in self.W])
        bp = (C.POINTER(C.c_float) * L)(*[b.ctypes.data_as(C.POINTER(C.c_float)) for b in self.b])
        d = (C.c_int32 * (L + 1))(*dims)
        a = (C.c_int32 * L)(*[int(x) for x in spec["act"]])
        compute = _abi.BF16 if spec.get("compute", "f32") == "bf16" else _abi.F32
        h = C.c_void_p()
        check(lib().hpacml_model_create(L, d, Wp, bp, a, compute, C.byref(h)), "hpacml_model_create")
        self.handle = h
        self.dims = dims

    def close(self):
        if getattr(self, "handle", None):
            lib().hpacml_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_KIND = {"conv": _abi.LAYER_CONV2D, "pool": _abi.LAYER_MAXPOOL2D, "linear": _abi.LAYER_LINEAR}
_PADDING = {"valid": _abi.PAD_VALID, "same": _abi.PAD_SAME}
_PAD_MODE = {"zeros": _abi.PADMODE_ZEROS, "circular": _abi.PADMODE_CIRCULAR, "replicate": _abi.PADMODE_REPLICATE}


def _layers(spec):
    """``hpacml_layer`` array from a convolutional model spec."""
    Ls = spec["layers"]
    arr = (_abi.Layer * len(Ls))()
    for i, ly in enumerate(Ls):
        a = arr[i]
        a.kind = _KIND[ly["kind"]]
        a.out_channels = int(ly.get("out", 0))
        k = ly.get("kernel", (1, 1))
        st = ly.get("stride", k if ly["kind"] == "pool" else (1, 1))
        a.kernel[0], a.kernel[1] = int(k[0]), int(k[1])
        a.stride[0], a.stride[1] = int(st[0]), int(st[1])
        a.padding = _PADDING[ly.get("padding", "valid")]
        a.pad_mode = _PAD_MODE[ly.get("mode", "zeros")]
        a.act = int(ly.get("act", 0))
    return arr


def validate_cnn(spec):
    """``hpacml_cnn_validate``: (status, output (rows, columns, channels))."""
    H, W = spec["image"]
    arr = _layers(spec)
    shp = (C.c_int32 * 3)()
    st = lib().hpacml_cnn_validate(int(spec["in_channels"]), int(H), int(W), len(spec["layers"]), arr, shp)
    return st, tuple(shp)


class CnnModel:
    """A convolutional surrogate (convolution / max-pool / fully connected
    layers on the composed tensor seen as images); spec as in
    ``workloads.make_cnn``.  Weights are host fp32 arrays, copied into
    library-owned device memory."""

    def __init__(self, spec):
        import numpy as np
        Ls = spec["layers"]
        L = len(Ls)
        arr = _layers(spec)
        self.W = [None if ly["kind"] == "pool" else np.ascontiguousarray(np.asarray(ly["W"], np.float32))
                  for ly in Ls]
        self.b = [None if ly["kind"] == "pool" else np.ascontiguousarray(np.asarray(ly["b"], np.float32))
                  for ly in Ls]
        # weight and bias sizes per layer, as the library reads them (for a
        # description it rejects, its own status reports the error below)
        wc, bc = (C.c_int64 * L)(), (C.c_int64 * L)()
        H, W = spec["image"]
        if lib().hpacml_cnn_param_counts(int(spec["in_channels"]), int(H), int(W), L, arr, wc, bc) == _abi.OK:
            for l in range(L):
                nw = 0 if self.W[l] is None else self.W[l].size
                nb = 0 if self.b[l] is None else self.b[l].size
                if nw != wc[l] or nb != bc[l]:
                    raise ValueError("layer %d: weights of %d and biases of %d values, expected %d and %d"
                                     % (l, nw, nb, wc[l], bc[l]))
        null = C.POINTER(C.c_float)()
        Wp = (C.POINTER(C.c_float) * L)(*[null if w is None else w.ctypes.data_as(C.POINTER(C.c_float))
                                          for w in self.W])
        bp = (C.POINTER(C.c_float) * L)(*[null if b is None else b.ctypes.data_as(C.POINTER(C.c_float))
                                          for b in self.b])
        H, W = spec["image"]
        h = C.c_void_p()
        check(lib().hpacml_cnn_create(int(spec["in_channels"]), int(H), int(W), L, arr, Wp, bp, _abi.F32,
                                      C.byref(h)), "hpacml_cnn_create")
        self.handle = h

    close = Model.close
    __del__ = Model.__del__


def _stream(stream):
    if stream is None:
        import torch
        # the current stream's handle, without the Stream object around it
        return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    if isinstance(stream, int):
        return C.c_void_p(stream)
    return C.c_void_p(stream.cuda_stream)


def infer(model: Model, in_map: Map, out_map: Map, stream=None) -> None:
    """``hpacml_infer``: gather -> MLP -> scatter on ``stream`` (default: torch's
    current stream)."""
    check(lib().hpacml_infer(model.handle, in_map.handle, out_map.handle, _stream(stream)), "hpacml_infer")


def collect(m: Map, dst, ld: int, stream=None) -> None:
    """``hpacml_collect`` into ``dst`` (a float32 device tensor; ``dst`` may be a
    view offset into a larger record, e.g. ``rec[:, 9:]``)."""
    import torch
    if dst.dtype != torch.float32 or not dst.is_cuda:
        raise TypeError("collect destination must be a float32 device tensor")
    check(lib().hpacml_collect(m.handle, C.c_void_p(dst.data_ptr()), int(ld), _stream(stream)),
          "hpacml_collect")


def collect_pair(a: Map, dst_a, ld_a: int, b: Map, dst_b, ld_b: int, stream=None) -> None:
    """``hpacml_collect_pair``: both records of a region in one call (float32
    device tensors or views)."""
    import torch
    for d in (dst_a, dst_b):
        if d.dtype != torch.float32 or not d.is_cuda:
            raise TypeError("collect destinations must be float32 device tensors")
    check(lib().hpacml_collect_pair(a.handle, C.c_void_p(dst_a.data_ptr()), int(ld_a), b.handle,
                                    C.c_void_p(dst_b.data_ptr()), int(ld_b), _stream(stream)),
          "hpacml_collect_pair")


def variant(model: Model, in_map: Map, out_map: Map) -> str:
    r = lib().hpacml_infer_variant(model.handle, in_map.handle, out_map.handle)
    return r.decode() if r else None


class Region:
    """Execution control of one annotated region (``ml(infer | collect |
    predicated)`` and ``if``): ``run`` infers, or records the inputs, calls
    ``accurate(stream_handle)`` (the region's original code, which enqueues its
    work on that stream) and records the outputs and the accurate path's time
    into a sink of ``capacity`` samples."""

    def __init__(self, model, in_map: Map, out_map: Map, mode: int, capacity: int = 0):
        h = C.c_void_p()
        check(lib().hpacml_region_create(model.handle, in_map.handle, out_map.handle, int(mode), int(capacity),
                                         C.byref(h)), "hpacml_region_create")
        self.handle = h
        self.keep = (model, in_map, out_map)
        self.points, self.f_in = in_map.n_points, in_map.n_features
        self.points_out, self.f_out = out_map.n_points, out_map.n_features

    def run(self, accurate=None, cond: bool = True, enabled: bool = True, stream=None) -> None:
        """``accurate(stream_handle)`` gets the stream as an int (0: the null
        stream); an exception it raises is re-raised here once the library
        call has returned."""
        errors = []

        def call(user, st):
            try:
                accurate(st or 0)
            except BaseException as e:   # must not unwind through the C frame
                errors.append(e)
        cb = _abi.ACCURATE_FN(call) if accurate is not None else _abi.ACCURATE_FN()
        check(lib().hpacml_region_run(self.handle, 1 if cond else 0, 1 if enabled else 0, cb, None,
                                      _stream(stream)), "hpacml_region_run")
        if errors:
            raise errors[0]

    @property
    def samples(self) -> int:
        n = C.c_int64()
        check(lib().hpacml_region_samples(self.handle, C.byref(n)), "hpacml_region_samples")
        return n.value

    def read(self):
        """(inputs [n, points, F_in], outputs [n, points_out, F_out], times_ms [n]) as numpy."""
        import numpy as np
        n = self.samples
        ins = np.zeros((n, self.points, self.f_in), np.float32)
        outs = np.zeros((n, self.points_out, self.f_out), np.float32)
        t = np.zeros(n, np.float32)
        check(lib().hpacml_region_read(self.handle, n, ins.ctypes.data, outs.ctypes.data, t.ctypes.data),
              "hpacml_region_read")
        return ins, outs, t

    def save(self, directory: str, name: str) -> None:
        check(lib().hpacml_region_save(self.handle, directory.encode(), name.encode()), "hpacml_region_save")

    def reset(self) -> None:
        check(lib().hpacml_region_reset(self.handle), "hpacml_region_reset")

    def close(self):
        if getattr(self, "handle", None):
            lib().hpacml_region_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- dense layers in 8 bits (include/hpacml8.h) -----------------------------

_kinds8 = {}       # torch's types -> the ABI's, filled by the first call


def _matrix(t, what, rows=None, width=None, kind=None):
    """(pointer, ABI type, row pitch) of a device matrix with contiguous rows."""
    if not _kinds8:
        import torch
        _kinds8.update({torch.float32: _abi.F32, torch.bfloat16: _abi.BF16})
    own = _kinds8.get(t.dtype)
    if own is None or not t.is_cuda or (kind is not None and own != kind):
        raise TypeError("%s must be a %s device tensor" % (what, "float32 or bfloat16" if kind is None else
                                                           "float32" if kind == _abi.F32 else "bfloat16"))
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (width is not None and shape[1] != width):
        raise ValueError("%s: shape %s, expected %s x %s" % (what, tuple(shape), "rows" if rows is None else rows,
                                                             "width" if width is None else width))
    n, m = shape
    ld, step = t.stride()
    if m > 1 and n > 0 and step != 1:
        raise ValueError("%s: the values of a row must be contiguous" % what)
    return t.data_ptr(), own, ld if n > 1 else max(m, 1)


def _scratch8(scratch, need, stream):
    """(the scratch tensor to keep during the call, its address, bytes): the caller's, or, on torch's current stream, whose
    order its allocator follows, one from there."""
    if scratch is None:
        if stream is not None:
            raise ValueError("a call on a stream of its own needs scratch memory")
        import torch
        scratch = torch.empty(need(), dtype=torch.uint8, device="cuda")
    elif not scratch.is_cuda or not scratch.is_contiguous():
        raise TypeError("scratch must be a contiguous device tensor")
    return scratch, scratch.data_ptr(), scratch.numel() * scratch.element_size()


class Linear8:
    """A dense layer's weights in 8-bit integers with a scale per output
    (``hpacml8_linear_create``): ``W`` [out][in] and ``b`` [out] or None,
    float32 (numpy, or torch on the CPU or the device), copied."""

    def __init__(self, W, b=None):
        import numpy as np
        import torch
        W = torch.as_tensor(np.asarray(W) if not isinstance(W, torch.Tensor) else W)
        if W.dim() != 2 or W.numel() == 0:
            raise ValueError("W: shape %s, expected out x in" % (tuple(W.shape),))
        W = W.detach().to(torch.float32).contiguous()
        if b is not None:
            b = torch.as_tensor(np.asarray(b) if not isinstance(b, torch.Tensor) else b).detach().to(torch.float32).contiguous()
            if tuple(b.shape) != (W.shape[0],):
                raise ValueError("b: shape %s, expected %d" % (tuple(b.shape), W.shape[0]))
        self.n_out, self.n_in = int(W.shape[0]), int(W.shape[1])
        h = C.c_void_p()
        check(lib().hpacml8_linear_create(self.n_in, self.n_out, W.data_ptr(), None if b is None else b.data_ptr(),
                                          C.byref(h)), "hpacml8_linear_create")
        self.handle = h

    def scratch_bytes(self, n_rows: int) -> int:
        n = C.c_size_t()
        check(lib().hpacml8_linear_scratch(self.handle, int(n_rows), C.byref(n)), "hpacml8_linear_scratch")
        return n.value

    def close(self):
        if getattr(self, "handle", None):
            lib().hpacml8_linear_destroy(self.handle)
            self.handle = None

    __del__ = Model.__del__


def linear8(layer: Linear8, x, y, act: int = _abi.ACT_IDENTITY, scratch=None, stream=None) -> None:
    """``hpacml8_linear_run``: ``y`` [n][out] = act(``x`` [n][in] W^T + b) with
    8-bit products; float32 or bfloat16 device tensors, rows may lie inside
    wider ones.  ``scratch``: at least ``layer.scratch_bytes(n)`` bytes (None:
    from torch's allocator, on its current stream)."""
    px, tx, ldx = _matrix(x, "x", width=layer.n_in)
    n = x.shape[0]
    py, ty, ldy = _matrix(y, "y", rows=n, width=layer.n_out)
    keep, ps, bytes_ = _scratch8(scratch, lambda: layer.scratch_bytes(n), stream)
    check(lib().hpacml8_linear_run(layer.handle, px, tx, ldx, n, py, ty, ldy, act, ps, bytes_, _stream(stream)),
          "hpacml8_linear_run")


class Checkpoint8:
    """Buffers of an activation [rows][width] kept in 8 bits (``hpacml8_checkpoint``);
    ``act``: what the activation is the output of (ACT_RELU or ACT_IDENTITY).
    ``codes`` and ``exps`` may be given (uint8 device tensors of ``rows`` rows)."""

    def __init__(self, rows: int, width: int, act: int, codes=None, exps=None):
        import torch
        blocks = -(-int(width) // _abi.BLOCK8)
        if codes is None:
            codes = torch.empty((rows, blocks * _abi.BLOCK8), dtype=torch.uint8, device="cuda")
        if exps is None:
            exps = torch.empty((rows, blocks), dtype=torch.uint8, device="cuda")
        for t, what, least in ((codes, "codes", blocks * _abi.BLOCK8), (exps, "exps", blocks)):
            if t.dtype != torch.uint8 or not t.is_cuda:
                raise TypeError("%s must be a uint8 device tensor" % what)
            if t.dim() != 2 or t.shape[0] != rows or t.shape[1] < least or (t.shape[1] > 1 and t.stride(1) != 1):
                raise ValueError("%s: shape %s, expected %d x at least %d, rows contiguous" % (what, tuple(t.shape), rows, least))
        self.rows, self.width, self.act, self.codes, self.exps = int(rows), int(width), int(act), codes, exps
        c = _abi.Checkpoint8()
        c.codes, c.exps = codes.data_ptr(), exps.data_ptr()
        c.rows, c.width, c.act = self.rows, self.width, self.act
        c.ld_codes = codes.stride(0) if rows > 1 else blocks * _abi.BLOCK8
        c.ld_exps = exps.stride(0) if rows > 1 else blocks
        self.desc = c


def checkpoint8_save(kept: Checkpoint8, z, a=None, stream=None) -> None:
    """``hpacml8_checkpoint_save``: keeps act(``z``), and writes it to ``a`` as
    well (which may be ``z``)."""
    pz, tz, ldz = _matrix(z, "z", kept.rows, kept.width)
    pa, ta, lda = (None, 0, 0) if a is None else _matrix(a, "a", kept.rows, kept.width)
    check(lib().hpacml8_checkpoint_save(C.byref(kept.desc), pz, tz, ldz, pa, ta, lda, _stream(stream)),
          "hpacml8_checkpoint_save")


def checkpoint8_load(kept: Checkpoint8, a, stream=None) -> None:
    """``hpacml8_checkpoint_load``: what ``kept`` stands for."""
    pa, ta, lda = _matrix(a, "a", kept.rows, kept.width)
    check(lib().hpacml8_checkpoint_load(C.byref(kept.desc), pa, ta, lda, _stream(stream)), "hpacml8_checkpoint_load")


def _backward8_need(kept, dy, dw, dx):
    """Bytes of scratch; dy: (pointer, type, pitch, width)."""
    n = C.c_size_t()
    check(lib().hpacml8_backward_scratch(kept.desc, *dy, dw, dx, n), "hpacml8_backward_scratch")
    return n.value


def backward8_scratch_bytes(kept: Checkpoint8, dy, W=None, dw: bool = True) -> int:
    """Bytes of scratch ``backward8`` needs (``W``: given when dx is wanted)."""
    p, t, ld = _matrix(dy, "dy", kept.rows)
    return _backward8_need(kept, (p, t, ld, dy.shape[1]), 1 if dw else 0, 0 if W is None else 1)


def backward8(kept: Checkpoint8, dy, dw=None, db=None, W=None, dx=None, accumulate: bool = False, scratch=None,
              stream=None) -> None:
    """``hpacml8_backward``: the gradients of a linear layer whose input is
    ``kept``, from ``dy`` [n][out] (float32 or bfloat16): ``dw`` [out][in] and
    ``db`` [out] in float32, ``dx`` [n][in] in dy's type from ``W`` [out][in]
    (dy's type).  Gradients not given are not computed."""
    py, ty, ldy = _matrix(dy, "dy", kept.rows)
    n_out = dy.shape[1]
    pw = pb = pW = px = None
    lddw = ldW = ldx = 0
    if dw is not None:
        pw, _, lddw = _matrix(dw, "dw", n_out, kept.width, _abi.F32)
    if db is not None:
        if _kinds8.get(db.dtype) != _abi.F32 or not db.is_cuda:
            raise TypeError("db must be a float32 device tensor")
        if db.shape != (n_out,) or not db.is_contiguous():
            raise ValueError("db: shape %s, expected %s contiguous" % (tuple(db.shape), (n_out,)))
        pb = db.data_ptr()
    if dx is not None:
        if W is None:
            raise ValueError("dx needs W")
        pW, _, ldW = _matrix(W, "W", n_out, kept.width, ty)
        px, _, ldx = _matrix(dx, "dx", kept.rows, kept.width, ty)
        if kept.rows == 0 and dw is None and db is None:
            return        # an empty tensor has no address, which would read as "not wanted"
    keep, ps, bytes_ = _scratch8(scratch, lambda: _backward8_need(
        kept, (py, ty, ldy, n_out), 1 if dw is not None or db is not None else 0, 0 if dx is None else 1), stream)
    check(lib().hpacml8_backward(kept.desc, py, ty, ldy, n_out, pW, ldW, pw, lddw, pb, px, ldx,
                                 1 if accumulate else 0, ps, bytes_, _stream(stream)), "hpacml8_backward")
