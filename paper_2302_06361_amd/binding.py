"""ctypes binding of include/dash.h: same names, argument marshalling only.

torch is used for device memory (torch.empty(device="cuda")) and for the current HIP stream; no
arithmetic of the method happens here.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "libdash.so")

MAX_PRIMES = 16
MAX_DIGITS = 16
DENSE, CONV2D, SUMPOOL, RELU, SCALE, SIGN, PROJ, EXPERTS, COMBINE = 1, 2, 3, 4, 5, 6, 7, 8, 9
W8, MX4, F8 = 0, 1, 8
F32, BF16, F16 = 0, 1, 2
SOFTMAX, SIGMOID = 0, 1
GROUP_MAX, GROUP_PAIR = 0, 1
LAMBDA_CEIL, LAMBDA_FLOOR = 0, 1
NOALLOC_SCRATCH_BYTES = 32 << 20

SYMBOLS = ["dash_ctx_create", "dash_ctx_destroy", "dash_lambda", "dash_ctx_offset", "dash_ctx_one", "dash_ctx_digits",
           "dash_layer_sizes", "dash_weights_bytes", "dash_weights_prepare", "dash_expert_weights_bytes", "dash_weights8_prepare",
           "dash_mx4_quantise", "dash_f8_quantise", "dash_f8_prepare", "dash_choose", "dash_route_bytes", "dash_route", "dash_garble_layer", "dash_eval_layer",
           "dash_garble_layers", "dash_eval_layers", "dash_eval_layer_noalloc", "dash_input_labels", "dash_encode", "dash_decode", "dash_labels_pack", "dash_labels_unpack", "dash_tables_packed_bytes", "dash_tables_pack", "dash_tables_unpack", "dash_strerror", "dash_profile_enable", "dash_profile_read", "dash_profile_aes"]


class DashError(RuntimeError):
    pass


class CLabels(C.Structure):
    _fields_ = [("data", C.c_void_p * MAX_PRIMES), ("chunk_stride", C.c_int64 * MAX_PRIMES), ("n_elem", C.c_int64)]


def _shared(*fields):
    """fields of different kinds of layers in one place"""
    return type("CShared", (C.Union,), {"_fields_": list(fields)})


class CLayer(C.Structure):
    _anonymous_ = ("u0", "u1", "u2", "u3")
    _fields_ = [("kind", C.c_int32), ("layer_id", C.c_int32), ("elem_base", C.c_int64), ("n_elem", C.c_int64),
                ("in_h", C.c_int32), ("in_w", C.c_int32), ("in_c", C.c_int32), ("out_c", C.c_int32),
                ("kh", C.c_int32), ("kw", C.c_int32), ("stride", C.c_int32), ("pad", C.c_int32),
                ("weights", C.c_void_p), ("bias", C.c_void_p),
                ("u0", _shared(("repeat", C.c_int32), ("top_k", C.c_int32))),
                ("u1", _shared(("p_index", C.c_int32), ("n_experts", C.c_int32))),
                ("u2", _shared(("q_index", C.c_int32), ("weight_format", C.c_int32))),
                ("u3", _shared(("phi", C.c_void_p), ("routing", C.c_void_p), ("gates", C.c_void_p))),
                ("phi_stride", C.c_int64)]


class CRouting(C.Structure):
    _fields_ = [("data", C.c_void_p), ("ctx", C.c_void_p), ("n", C.c_int64), ("n_experts", C.c_int32)]


class CRouter(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_experts", "top_k", "score", "n_groups", "top_groups", "group_score", "renormalise", "gate_bits")] + \
               [("scale", C.c_float), ("bias", C.c_void_p)]


_lib = None


def lib_path():
    return _SO


def lib():
    """Load libdash.so; fail loudly if it has not been built (python -m paper_2302_06361_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_SO):
            raise DashError("libdash.so is missing: build it with `python -m paper_2302_06361_amd.build` "
                            "(there is no CPU fallback)")
        L = C.CDLL(_SO)
        L.dash_strerror.restype = C.c_char_p
        L.dash_weights_bytes.restype = C.c_size_t
        L.dash_tables_packed_bytes.restype = C.c_size_t
        L.dash_expert_weights_bytes.restype = C.c_size_t
        L.dash_mx4_quantise.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64] + [C.c_int] * 5 + [C.c_void_p] * 3
        L.dash_f8_quantise.argtypes = L.dash_mx4_quantise.argtypes
        L.dash_f8_prepare.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p] + [C.c_int] * 3 + [C.c_void_p] * 2
        L.dash_choose.argtypes = [C.c_void_p] * 3 + [C.c_int, C.c_int64, C.c_int64] + [C.c_void_p] * 5
        L.dash_route_bytes.restype = C.c_size_t
        L.dash_ctx_destroy.restype = None
        _lib = L
    return _lib


def _describe_plain(tensors, address, n_elem):
    """The dash_labels at `address` of a list of tensors, one by one (12 of them: 6 us)."""
    s = CLabels.from_address(address)
    C.memset(address, 0, C.sizeof(s))
    s.n_elem = n_elem
    for i, t in enumerate(tensors):
        if t is not None:
            s.data[i] = t.data_ptr()
            s.chunk_stride[i] = t.stride(0)


def _describe_first(tensors, address, n_elem):
    """The same through the host module built beside the library (0.2 us), where it is there."""
    global _describe
    import torch  # noqa: F401  (the module uses its libraries)
    try:
        from ._bundle import describe
    except ImportError:
        describe = _describe_plain
    _describe = describe
    describe(tensors, address, n_elem)


_describe = _describe_first


def _check(st, what):
    if st != 0:
        raise DashError("%s: %s (%d)" % (what, lib().dash_strerror(st).decode(), st))


_raw_stream = _current_device = None


def _stream():
    """the current stream of the current device"""
    global _raw_stream, _current_device
    if _raw_stream is None:
        import torch
        torch.cuda.current_device()                   # (initialises)
        _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    return C.c_void_p(_raw_stream(_current_device()))


class Labels:
    """One LabelTensor per CRT residue on the GPU: tensors[i] is uint8 [nchunk_i][n_elem][16]."""

    def __init__(self, ctx, n_elem, only=None, zero=False):
        import torch
        self.ctx, self.n_elem = ctx, int(n_elem)
        self.tensors = [None] * ctx.k
        for i, p in enumerate(ctx.primes):
            if only is not None and i not in only:
                continue
            nch = (ctx.lam(p) + 15) // 16
            shape = (nch, max(self.n_elem, 1), 16)
            self.tensors[i] = (torch.zeros if zero else torch.empty)(shape, dtype=torch.uint8, device=ctx.device)

    def c(self):
        s = CLabels()
        t = self.tensors
        _describe(t if type(t) is list else list(t), C.addressof(s), self.n_elem)
        return s

    def slice(self, e0, e1):
        """View of the elements [e0, e1) (same storage)."""
        v = Labels.__new__(Labels)
        v.ctx, v.n_elem = self.ctx, e1 - e0
        v.tensors = [None if t is None else t[:, e0:e1, :] for t in self.tensors]
        return v

    def to_numpy(self, i):
        """Compact host copy [n_elem][lambda] of residue i (layout conversion only)."""
        lam = self.ctx.lam(self.ctx.primes[i])
        t = self.tensors[i][:, :self.n_elem, :].permute(1, 0, 2).reshape(self.n_elem, -1)
        return t[:, :lam].contiguous().cpu().numpy()

    def pad_is_zero(self, i):
        lam = self.ctx.lam(self.ctx.primes[i])
        t = self.tensors[i][:, :self.n_elem, :].permute(1, 0, 2).reshape(self.n_elem, -1)
        return bool((t[:, lam:] == 0).all().item())

    def from_numpy(self, i, arr):
        """Upload compact labels [n_elem][lambda] into residue i (layout conversion only)."""
        import torch
        lam = self.ctx.lam(self.ctx.primes[i])
        nch = (lam + 15) // 16
        a = np.zeros((self.n_elem, nch * 16), np.uint8)
        a[:, :lam] = arr
        t = torch.from_numpy(a).to(self.ctx.device).reshape(self.n_elem, nch, 16).permute(1, 0, 2)
        self.tensors[i][:, :self.n_elem, :].copy_(t)


class ExpertWeights:
    """Prepared weights of an EXPERTS layer: n_experts matrices [out_c][K] in one device buffer, `format` W8, MX4 or F8.  Filled by
    Context.weights8_prepare, Context.mx4_quantise, Context.f8_quantise or Context.f8_prepare."""

    def __init__(self, ctx, format, n_experts, out_c, K):
        import torch
        self.format, self.n_experts, self.out_c, self.K = int(format), int(n_experts), int(out_c), int(K)
        nbytes = ctx.L.dash_expert_weights_bytes(self.format, self.n_experts, self.out_c, self.K)
        if nbytes == 0:
            raise DashError("ExpertWeights: bad format or size")
        self.data = torch.empty(nbytes, dtype=torch.uint8, device=ctx.device)


class Routing:
    """A dash_routing and its device buffer (Context.route)."""

    def __init__(self, ctx, n, n_experts):
        import torch
        self.ctx, self.c = ctx, CRouting()
        self.data = torch.empty(max(ctx.L.dash_route_bytes(ctx.h, C.c_int64(n), int(n_experts)), 16), dtype=torch.uint8, device=ctx.device)

    def address(self):
        return C.addressof(self.c)


class Router:
    """A dash_router: how Context.choose takes top_k of n_experts from a row's logits.  bias: float32 tensor [n_experts] on the device, added to
    the scores for the choice (it may be replaced); groups: equal groups of experts, of which the top_groups best ones (group_score) are chosen from."""

    def __init__(self, n_experts, top_k, score=SOFTMAX, bias=None, groups=1, top_groups=1, group_score=GROUP_MAX, renormalise=True, scale=1.0, gate_bits=8):
        given = dict(n_experts=n_experts, top_k=top_k, score=score, groups=groups, top_groups=top_groups, group_score=group_score, gate_bits=gate_bits)
        for name, v in given.items():
            if v != int(v) or not -2 ** 31 <= v < 2 ** 31:          # (the descriptor would hold another number)
                raise DashError("Router: %s has to be an integer of 32 bits, got %r" % (name, v))
        self.c = CRouter(int(n_experts), int(top_k), int(score), int(groups), int(top_groups), int(group_score), int(bool(renormalise)), int(gate_bits), float(scale))
        self.n_experts, self.top_k, self.bias = int(n_experts), int(top_k), bias

    def __setattr__(self, name, value):
        # (the library reads the descriptor: it follows another bias and keeps its sizes)
        if name == "bias":
            if value is not None:
                import torch
                if value.dtype != torch.float32 or not value.is_contiguous() or value.numel() != self.n_experts:
                    raise DashError("Router: bias has to be a contiguous float32 tensor [n_experts]")
            self.c.bias = None if value is None else value.data_ptr()
        elif name in ("c", "n_experts", "top_k") and hasattr(self, name):
            raise DashError("Router: made for %d of %d experts" % (self.top_k, self.n_experts))
        object.__setattr__(self, name, value)


class Choice:
    """What Context.choose fills for n rows: experts (int32 [n][top_k], -1: none), gates (int32, what COMBINE layers take), weights (float32).  They may be
    replaced by tensors of the same type and size (parts of larger ones)."""

    def __init__(self, ctx, n, top_k):
        import torch
        self.n, self.top_k, self.device = int(n), int(top_k), ctx.device
        self.experts, self.gates = (torch.empty((self.n, self.top_k), dtype=torch.int32, device=ctx.device) for _ in range(2))
        self.weights = torch.empty((self.n, self.top_k), dtype=torch.float32, device=ctx.device)

    def __setattr__(self, name, value):
        # (read by address in every call: looked at here, once)
        if name in ("experts", "gates", "weights"):
            import torch
            dtype = torch.float32 if name == "weights" else torch.int32
            if not torch.is_tensor(value) or value.dtype != dtype or value.numel() != self.n * self.top_k or not value.is_contiguous() or value.device != self.device:
                raise DashError("Choice: %s has to be a contiguous tensor [%d][%d] of %s on %s" % (name, self.n, self.top_k, dtype, self.device))
        elif name in ("n", "top_k", "device") and hasattr(self, name):
            raise DashError("Choice: made for %d rows of %d" % (self.n, self.top_k))
        object.__setattr__(self, name, value)


class Layer:
    """A dash_layer descriptor plus the Python objects that keep its device buffers alive."""

    def __init__(self, kind, layer_id=0, n_elem=0, elem_base=0, **kw):
        self.c = CLayer()
        self.c.kind, self.c.layer_id, self.c.n_elem, self.c.elem_base = kind, layer_id, n_elem, elem_base
        self.keep = []
        for k, v in kw.items():
            if isinstance(v, ExpertWeights):
                if kind != EXPERTS:
                    raise DashError("Layer: ExpertWeights are the weights of EXPERTS layers (one expert, no routing: a dense layer)")
                self.keep.append(v)
                self.c.weights, self.c.weight_format = v.data.data_ptr(), v.format
                self.c.n_experts, self.c.out_c, self.c.in_c = v.n_experts, v.out_c, v.K
            elif k == "routing":
                if v is not None:
                    self.keep.append(v)
                    self.c.routing = v.address()
            elif k in ("weights", "bias", "phi", "gates"):
                if v is not None:
                    if k in ("bias", "gates") and kind in (EXPERTS, COMBINE):
                        # (several numbers a row, read by address)
                        import torch
                        if v.dtype != torch.int32 or not v.is_contiguous():
                            raise DashError("Layer: %s has to be a contiguous int32 tensor" % k)
                    self.keep.append(v)
                    setattr(self.c, k, v.data_ptr())
            else:
                setattr(self.c, k, v)
        weights, bias = kw.get("weights"), kw.get("bias")
        if isinstance(weights, ExpertWeights) and bias is not None and bias.numel() < weights.n_experts * weights.out_c:
            raise DashError("Layer: bias [n_experts][out_c] expected, got %d numbers" % bias.numel())


class Context:
    def __init__(self, primes, seed, digits=None, rule=LAMBDA_CEIL, device=0, lam=None):
        import torch
        if not torch.cuda.is_available():
            raise DashError("no GPU visible: libdash has no CPU path")
        self.L = lib()
        self.primes = [int(p) for p in primes]
        self.k = len(self.primes)
        self.device = torch.device("cuda", device)
        pr = (C.c_uint16 * self.k)(*self.primes)
        sd = (C.c_uint8 * 16)(*bytes(seed))
        h = C.c_void_p()
        la = None if lam is None else (C.c_uint16 * self.k)(*[int(v) for v in lam])
        dg = None if digits is None else (C.c_uint16 * len(digits))(*[int(d) for d in digits])
        st = self.L.dash_ctx_create(C.byref(h), pr, self.k, rule, la, sd, dg, 0 if digits is None else len(digits), device)
        _check(st, "dash_ctx_create")
        self.h = h
        buf = (C.c_uint16 * MAX_DIGITS)()
        n = self.L.dash_ctx_digits(self.h, buf)
        self.digits = [int(buf[j]) for j in range(n)]
        self._lam = {}
        self._types = None

    def close(self):
        if getattr(self, "h", None):
            self.L.dash_ctx_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def lam(self, m):
        if m not in self._lam:
            self._lam[m] = self.L.dash_lambda(self.h, int(m))
        return self._lam[m]

    def pitch(self, m):
        return 4 * ((self.lam(m) + 3) // 4)

    def offset(self, m):
        out = np.zeros(self.lam(m), np.uint8)
        _check(self.L.dash_ctx_offset(self.h, int(m), out.ctypes.data_as(C.c_void_p)), "dash_ctx_offset")
        return out

    def one(self, i, which):
        out = np.zeros(self.lam(self.primes[i]), np.uint8)
        _check(self.L.dash_ctx_one(self.h, int(i), int(which), out.ctypes.data_as(C.c_void_p)), "dash_ctx_one")
        return out

    def profile_enable(self, on):
        _check(self.L.dash_profile_enable(self.h, int(on)), "dash_profile_enable")

    def profile_read(self, kind):
        """-> dict(ms, launches, units, bytes) summed over the launches since the last read"""
        ms, n, u, b = C.c_double(), C.c_int64(), C.c_double(), C.c_double()
        _check(self.L.dash_profile_read(self.h, int(kind), C.byref(ms), C.byref(n), C.byref(u), C.byref(b)), "dash_profile_read")
        return dict(ms=ms.value, launches=n.value, units=u.value, bytes=b.value)

    def profile_aes(self, variant, key, blocks_in, blocks_out, repeat=1):
        """AES-128 alone (variant 0: 4 KB tables, 1: bank-replicated tables T0/T1, 2: bit planes, 3: bank-replicated T0..T3) on device byte tensors
        [n][16]; out = AES_key^repeat(in)"""
        import torch
        key = bytes(key)
        assert len(key) == 16 and blocks_in.dtype == torch.uint8 and blocks_out.dtype == torch.uint8
        assert blocks_in.is_cuda and blocks_out.is_cuda and blocks_in.is_contiguous() and blocks_out.is_contiguous()
        assert blocks_in.numel() % 16 == 0 and blocks_out.numel() == blocks_in.numel()
        kb = (C.c_uint8 * 16).from_buffer_copy(key)
        _check(self.L.dash_profile_aes(self.h, int(variant), kb, C.c_void_p(blocks_in.data_ptr()), C.c_void_p(blocks_out.data_ptr()),
                                       C.c_uint64(blocks_in.numel() // 16), int(repeat), _stream()), "dash_profile_aes")

    # ---- the ABI calls, same names -------------------------------------------------------------
    def layer_sizes(self, layer):
        oe, tb, sb = C.c_int64(), C.c_size_t(), C.c_size_t()
        _check(self.L.dash_layer_sizes(self.h, C.byref(layer.c), C.byref(oe), C.byref(tb), C.byref(sb)), "dash_layer_sizes")
        return oe.value, tb.value, sb.value

    def weights_prepare(self, w):
        """w: int32 array/tensor [out_c][K] -> prepared device buffer (torch uint8)."""
        import torch
        wt = torch.as_tensor(np.ascontiguousarray(w, dtype=np.int32)).to(self.device)
        out_c, K = wt.shape
        nbytes = self.L.dash_weights_bytes(self.h, out_c, K)
        buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        _check(self.L.dash_weights_prepare(self.h, C.c_void_p(wt.data_ptr()), out_c, K, C.c_void_p(buf.data_ptr()), _stream()),
               "dash_weights_prepare")
        torch.cuda.current_stream().synchronize()     # wt may be freed after return
        return buf

    def _expert_matrices(self, w, what, dtypes):
        """w [n_experts][out_c][K] (or [out_c][K]: one expert) on the context's device, rows contiguous -> the same, three-dimensional"""
        if w.dim() == 2:
            w = w[None]
        shape, stride = w.shape, w.stride()
        if len(shape) != 3 or w.dtype not in dtypes or w.device != self.device or (stride[2] != 1 and shape[2] > 1) or 0 in shape:
            raise DashError("%s: weights [n_experts][out_c][K] with contiguous rows on %s expected, got %s %s on %s" %
                            (what, self.device, w.dtype, tuple(shape), w.device))
        return w, shape, stride

    def _expert_out(self, out, format, shape, what):
        if out is None:
            return ExpertWeights(self, format, *shape)
        if out.format != format or (out.n_experts, out.out_c, out.K) != shape:
            raise DashError("%s: `out` was made for another format or size" % what)
        return out

    def weights8_prepare(self, w, out=None):
        """w: int8 tensor [n_experts][out_c][K] on the device -> ExpertWeights in the W8 format"""
        import torch
        w, shape, stride = self._expert_matrices(w, "weights8_prepare", (torch.int8,))
        out = self._expert_out(out, W8, shape, "weights8_prepare")
        _check(self.L.dash_weights8_prepare(self.h, C.c_void_p(w.data_ptr()), C.c_int64(stride[1]), C.c_int64(stride[0]), *shape,
                                            C.c_void_p(out.data.data_ptr()), _stream()), "dash_weights8_prepare")
        return out

    def mx4_quantise(self, w, base, max_shift=255, out=None, values=None):
        """w: float32, bfloat16 or float16 tensor [n_experts][out_c][K] on the device -> ExpertWeights in the MX4 format: integers
        2 * e2m1 * 2^shift in units of 2^(base - 1), shift <= max_shift.  values: contiguous tensor like w that receives the
        weights the codes stand for."""
        return self._quantise(self.L.dash_mx4_quantise, "mx4_quantise", MX4, w, base, max_shift, out, values)

    def _quantise(self, call, what, format, w, base, most, out, values):
        types = self._types or self._float_types()
        w, shape, stride = self._expert_matrices(w, what, types)
        out = self._expert_out(out, format, shape, what)
        dtype, to = w.dtype, None
        if values is not None:
            to = values.data_ptr()
            if values.dtype != dtype or values.numel() != shape[0] * shape[1] * shape[2] or not values.is_contiguous() or values.device != self.device:
                raise DashError("%s: `values` has to be contiguous and of the size and type of the weights" % what)
        st = call(self.h, w.data_ptr(), types[dtype], stride[1], stride[0], *shape, base, most, out.data.data_ptr(), to, _stream())
        if st != 0:
            _check(st, "dash_" + what)
        return out

    def _float_types(self):
        import torch
        self._types = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
        return self._types

    def f8_quantise(self, w, base, max_scale=255, out=None, values=None):
        """w: float32, bfloat16 or float16 tensor [n_experts][out_c][K] on the device -> ExpertWeights in the F8 format: integers
        512 * e4m3 * scale in units of 2^(base - 9), a scale of at most max_scale for every block of 128 x 128.  values: contiguous tensor
        like w that receives the weights the codes stand for."""
        return self._quantise(self.L.dash_f8_quantise, "f8_quantise", F8, w, base, max_scale, out, values)

    def f8_prepare(self, codes, scales, out=None):
        """codes: e4m3 (uint8 or torch.float8_e4m3fn) tensor [n_experts][out_c][K] on the device, scales: contiguous int32 tensor
        [n_experts][ceil(out_c / 128)][ceil(K / 128)] -> ExpertWeights in the F8 format"""
        import torch
        codes, shape, stride = self._expert_matrices(codes, "f8_prepare", (torch.uint8, torch.float8_e4m3fn))
        E, M, K = shape
        blocks = (E, (M + 127) // 128, (K + 127) // 128)
        if scales.dtype != torch.int32 or scales.device != self.device or not scales.is_contiguous() or tuple(scales.shape) not in (blocks, blocks[1:] if E == 1 else blocks):
            raise DashError("f8_prepare: contiguous int32 scales %s on %s expected, got %s %s on %s" % (list(blocks), self.device, scales.dtype, list(scales.shape), scales.device))
        out = self._expert_out(out, F8, shape, "f8_prepare")
        _check(self.L.dash_f8_prepare(self.h, codes.data_ptr(), stride[1], stride[0], scales.data_ptr(), *shape, out.data.data_ptr(), _stream()), "dash_f8_prepare")
        return out

    def choose(self, router, logits, valid=None, out=None):
        """logits: float32, bfloat16 or float16 tensor [n][n_experts] on the device, rows contiguous; valid: bytes or truth values [n], rows of no
        expert false -> Choice"""
        types = self._types or self._float_types()
        shape, stride = logits.shape, logits.stride()
        E = router.n_experts
        if len(shape) != 2 or shape[1] != E or logits.dtype not in types or logits.device != self.device or (stride[1] != 1 and E > 1) or (stride[0] < E and shape[0] > 1):
            raise DashError("choose: logits [n][%d] with contiguous rows on %s expected, got %s %s on %s" % (E, self.device, logits.dtype, tuple(shape), logits.device))
        n = shape[0]
        if router.bias is not None and router.bias.device != self.device:
            raise DashError("choose: the router's bias is on %s" % router.bias.device)
        if valid is not None and (valid.itemsize != 1 or valid.numel() != n or valid.device != self.device or not valid.is_contiguous()):
            raise DashError("choose: `valid` has to be a contiguous tensor of %d bytes or truth values on %s" % (n, self.device))
        if out is None:
            out = Choice(self, n, router.top_k)
        elif out.n != n or out.top_k != router.top_k or out.experts.device != self.device:
            raise DashError("choose: `out` was made for another number of rows or experts")
        st = self.L.dash_choose(self.h, C.addressof(router.c), logits.data_ptr(), types[logits.dtype], max(stride[0], E), n, None if valid is None else valid.data_ptr(),
                                out.experts.data_ptr(), out.gates.data_ptr(), out.weights.data_ptr(), _stream())
        if st != 0:
            _check(st, "dash_choose")
        return out

    def route(self, experts, n_experts, out=None):
        """experts: int32 tensor [n] on the device, the expert of every row (outside [0, n_experts): none) -> Routing"""
        import torch
        if experts.dtype != torch.int32 or experts.device != self.device or not experts.is_contiguous():
            raise DashError("route: a contiguous int32 tensor on %s expected" % self.device)
        r = Routing(self, experts.numel(), n_experts) if out is None else out
        if out is not None and r.data.numel() < self.L.dash_route_bytes(self.h, C.c_int64(experts.numel()), int(n_experts)):
            raise DashError("route: `out` was made for fewer rows or experts")
        _check(self.L.dash_route(self.h, C.c_void_p(experts.data_ptr()), C.c_int64(experts.numel()), int(n_experts),
                                 C.c_void_p(r.data.data_ptr()), C.byref(r.c), _stream()), "dash_route")
        return r

    def input_labels(self, first_wire, zero, n=None):
        """zero labels of the input wires first_wire .. first_wire + n - 1 (n: all elements of `zero` by default)"""
        cz = zero.c()
        n = cz.n_elem if n is None else n
        _check(self.L.dash_input_labels(self.h, C.c_int64(first_wire), C.c_int64(n), C.byref(cz), _stream()), "dash_input_labels")

    def encode(self, values, zero, out):
        cz, co = zero.c(), out.c()
        _check(self.L.dash_encode(self.h, C.c_void_p(values.data_ptr()), C.c_int64(values.numel()), C.byref(cz), C.byref(co),
                                  _stream()), "dash_encode")

    def decode(self, act, zero, values, valid):
        ca, cz = act.c(), zero.c()
        _check(self.L.dash_decode(self.h, C.byref(ca), C.byref(cz), C.c_int64(values.numel()), C.c_void_p(values.data_ptr()),
                                  C.c_void_p(valid.data_ptr()), _stream()), "dash_decode")

    def labels_pack(self, labels, packed):
        """labels -> packed (uint8 tensor [k][n][16]): the 128-bit wire format; floor-rule contexts only"""
        cl = labels.c()
        _check(self.L.dash_labels_pack(self.h, C.byref(cl), C.c_int64(labels.n_elem), C.c_void_p(packed.data_ptr()), _stream()),
               "dash_labels_pack")

    def labels_unpack(self, packed, labels):
        cl = labels.c()
        _check(self.L.dash_labels_unpack(self.h, C.c_void_p(packed.data_ptr()), C.c_int64(labels.n_elem), C.byref(cl), _stream()),
               "dash_labels_unpack")

    def tables_packed_bytes(self, layer):
        """bytes of the layer's tables in the packed storage format (0: not available under this context's label lengths)"""
        return self.L.dash_tables_packed_bytes(self.h, C.byref(layer.c))

    def tables_pack(self, layer, tables, packed):
        _check(self.L.dash_tables_pack(self.h, C.byref(layer.c), C.c_void_p(tables.data_ptr()), C.c_void_p(packed.data_ptr()), _stream()),
               "dash_tables_pack")

    def tables_unpack(self, layer, packed, tables):
        _check(self.L.dash_tables_unpack(self.h, C.byref(layer.c), C.c_void_p(packed.data_ptr()), C.c_void_p(tables.data_ptr()), _stream()),
               "dash_tables_unpack")

    def garble_layer(self, layer, in_zero, out_zero, tables=None, scratch=None):
        ci, co = in_zero.c(), out_zero.c()
        _check(self.L.dash_garble_layer(self.h, C.byref(layer.c), C.byref(ci), C.byref(co),
                                        C.c_void_p(tables.data_ptr() if tables is not None else 0),
                                        C.c_void_p(scratch.data_ptr() if scratch is not None else 0), _stream()),
               "dash_garble_layer")

    def _labels_array(self, n, bundles, residues):
        """n dash_labels; residues: of each bundle the one residue that its call reads or writes (PROJ calls), or None"""
        if residues is None:
            return (CLabels * n)(*[t.c() for t in bundles])
        arr = (CLabels * n)()
        m = len(bundles)
        if m:
            flat = np.frombuffer(arr, np.int64).reshape(n, 2 * MAX_PRIMES + 1)[:m]
            tensors = [b.tensors[i] for b, i in zip(bundles, residues)]
            row, col = np.arange(m), np.array(residues[:m])
            flat[row, col] = [0 if t is None else t.data_ptr() for t in tensors]
            flat[row, MAX_PRIMES + col] = [0 if t is None else t.stride(0) for t in tensors]
            flat[:, 2 * MAX_PRIMES] = [b.n_elem for b in bundles]
        return arr

    def _layer_lists(self, layers, ins, outs, tables, scratch):
        n = len(layers)
        # the library reads n entries of every list: what a shorter one lacks stays null, a longer one is refused here
        ins, outs, tables, scratch = [None if x is None else list(x) for x in (ins, outs, tables, scratch)]
        if max(len(x) for x in (ins, outs, tables, scratch or ())) > n:
            raise IndexError("a list has more entries than there are layers")
        structs = [l.c for l in layers]
        cl = (CLayer * n).from_buffer_copy(b"".join(structs))
        # lists of PROJ calls are long and touch one residue per bundle (144 calls: 270 -> 150 us of host time)
        pi = qi = None
        if n and all(c.kind == PROJ for c in structs):
            pi, qi = [c.p_index for c in structs], [c.q_index for c in structs]
            if min(min(pi), min(qi)) < 0 or max(max(pi), max(qi)) >= self.k:
                pi = qi = None                           # the library refuses the call
        ci = self._labels_array(n, ins, pi)
        co = self._labels_array(n, outs, qi)

        def pointers(tensors):
            arr = (C.c_void_p * n)()
            if tensors:
                np.frombuffer(arr, np.int64)[:len(tensors)] = [0 if t is None else t.data_ptr() for t in tensors]
            return arr
        ct = pointers(tables)
        cs = None if scratch is None else pointers(scratch)
        return n, cl, ci, co, ct, cs

    def garble_layers(self, layers, in_zero, out_zero, tables, scratch=None):
        """n independent layer calls in one ABI call (lists of equal length)"""
        n, cl, ci, co, ct, cs = self._layer_lists(layers, in_zero, out_zero, tables, scratch)
        _check(self.L.dash_garble_layers(self.h, n, cl, ci, co, ct, cs, _stream()), "dash_garble_layers")

    def eval_layers(self, layers, in_act, tables, out_act, scratch=None):
        n, cl, ci, co, ct, cs = self._layer_lists(layers, in_act, out_act, tables, scratch)
        _check(self.L.dash_eval_layers(self.h, n, cl, ci, ct, co, cs, _stream()), "dash_eval_layers")

    def eval_layer_noalloc(self, layer, in_act, tables, out_act):
        """dash_eval_layer with the library's own fixed scratch array (NOALLOC_SCRATCH_BYTES): allocates nothing"""
        ci, co = in_act.c(), out_act.c()
        _check(self.L.dash_eval_layer_noalloc(self.h, C.byref(layer.c), C.byref(ci),
                                              C.c_void_p(tables.data_ptr() if tables is not None else 0), C.byref(co), _stream()),
               "dash_eval_layer_noalloc")

    def eval_layer(self, layer, in_act, tables, out_act, scratch=None):
        ci, co = in_act.c(), out_act.c()
        _check(self.L.dash_eval_layer(self.h, C.byref(layer.c), C.byref(ci),
                                      C.c_void_p(tables.data_ptr() if tables is not None else 0), C.byref(co),
                                      C.c_void_p(scratch.data_ptr() if scratch is not None else 0), _stream()),
               "dash_eval_layer")
