"""ctypes binding of libflround (include/flround.h).

Argument marshalling only: every step of the path runs in the library's
gfx950 kernels.  Tensors are torch CUDA tensors (bf16 buffers may be
torch.bfloat16 or any 2-byte dtype holding bf16 bits); work is enqueued on
the current torch stream unless `stream` is given.  Every non-OK status
raises FlError.  If the library is missing, importing the symbols raises:
there is no fallback.
"""
import array
import ctypes
import functools
import operator
import os

HERE = os.path.dirname(os.path.abspath(__file__))
# FLROUND_LIB names another build of the library to load (the sanitizer
# test's host-instrumented build)
LIB_PATH = os.environ.get("FLROUND_LIB") or os.path.join(HERE, "libflround.so")

FL_OK = 0
FL_ERR_INVALID = -1
FL_ERR_ALIGN = -2
FL_ERR_LAYOUT = -3
FL_ERR_DEVICE = -4
FL_ERR_HIP = -5
FL_ERR_NOMEM = -6
FL_ERR_SCRATCH = -7
FL_NOALLOC_SCRATCH_BYTES = 32 << 20

FL_MAX_PEERS = 64
FL_MAX_GROUPS = 64
FL_MAX_TARGETS = 128
FL_BF16, FL_F32 = 0, 1

# Every symbol include/flround.h declares.
EXPORTS = ("fl_status_string", "fl_version", "fl_layout_create", "fl_layout_destroy",
           "fl_layout_numel", "fl_layout_num_segments", "fl_fingerprint",
           "fl_layout_fingerprint", "fl_shard_reduce", "fl_adamw_step", "fl_local_step",
           "fl_fedavg", "fl_round", "fl_set_blocks_per_cu", "fl_shard_reduce_wire",
           "fl_broadcast_recv", "fl_round_hsdp", "fl_fedopt", "fl_round_outer",
           "fl_lr_cosine", "fl_grad_sumsq", "fl_local_step_clipped", "fl_round_noalloc",
           "fl_noalloc_workspace_bytes", "fl_head_workspace_bytes", "fl_head_loss",
           "fl_head_loss_grad", "fl_head_distill", "fl_head_distill_grad",
           "fl_top_workspace_bytes", "fl_top_logits", "fl_embed", "fl_embed_workspace_bytes",
           "fl_embed_grad", "fl_layer_norm", "fl_layer_norm_workspace_bytes",
           "fl_layer_norm_grad", "fl_tensors_state_numel", "fl_tensors_state_bytes",
           "fl_adamw_tensors", "fl_state_convert")

_P = ctypes.c_void_p


class FlError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s" % (where, status_string(status)))


class AdamwHparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float)]


class RoundCfg(ctypes.Structure):
    _fields_ = [("R", ctypes.c_int), ("G", ctypes.c_int), ("A", ctypes.c_int),
                ("self_group", ctypes.c_int), ("grad_scale", ctypes.c_float),
                ("h", AdamwHparams), ("step0", ctypes.c_int64),
                ("weights", ctypes.POINTER(ctypes.c_float)),
                ("replica_fp", ctypes.POINTER(ctypes.c_uint64)),
                ("phase_events", ctypes.POINTER(ctypes.c_void_p)),
                ("step_lr", ctypes.POINTER(ctypes.c_float)),
                ("max_grad_norm", ctypes.c_float),
                ("grad_scratch", ctypes.c_void_p)]


class OuterHparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("momentum", ctypes.c_float), ("nesterov", ctypes.c_int)]


def outer_hparams(oh):
    if isinstance(oh, OuterHparams):
        return oh
    return OuterHparams(oh["lr"], oh["momentum"], 1 if oh.get("nesterov", True) else 0)


class HsdpCfg(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int), ("replica", ctypes.c_int), ("hsdp_scale", ctypes.c_float),
                ("fedavg_member", ctypes.c_int)]


class HeadShape(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("vocab", ctypes.c_int64), ("width", ctypes.c_int64),
                ("hidden_stride", ctypes.c_int64), ("weight_stride", ctypes.c_int64)]


class EmbedShape(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("vocab", ctypes.c_int64), ("width", ctypes.c_int64),
                ("stride", ctypes.c_int64), ("dtype", ctypes.c_int)]


class NormShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("x_stride", ctypes.c_int64),
                ("dy_stride", ctypes.c_int64), ("dtype", ctypes.c_int), ("rms", ctypes.c_int)]


class FlTensor(ctypes.Structure):
    _fields_ = [("numel", ctypes.c_int64), ("master", ctypes.c_void_p),
                ("working", ctypes.c_void_p), ("decay", ctypes.c_int)]


_lib = None


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libflround.so is not built (%s); run "
                               "`python -m paper_2609_20359_amd.build`" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        L.fl_status_string.argtypes = [ctypes.c_int]
        L.fl_status_string.restype = ctypes.c_char_p
        L.fl_version.restype = ctypes.c_int
        L.fl_layout_create.argtypes = [ctypes.c_int64, ctypes.c_int64, _P, _P,
                                       ctypes.POINTER(_P)]
        L.fl_layout_destroy.argtypes = [_P]
        L.fl_layout_numel.argtypes = [_P]
        L.fl_layout_numel.restype = ctypes.c_int64
        L.fl_layout_num_segments.argtypes = [_P]
        L.fl_layout_num_segments.restype = ctypes.c_int64
        L.fl_fingerprint.argtypes = [ctypes.c_int64, ctypes.c_int64, _P, _P]
        L.fl_fingerprint.restype = ctypes.c_uint64
        L.fl_layout_fingerprint.argtypes = [_P]
        L.fl_layout_fingerprint.restype = ctypes.c_uint64
        L.fl_shard_reduce.argtypes = [_P, ctypes.c_int, _P, ctypes.c_float, _P, _P, _P]
        L.fl_adamw_step.argtypes = [_P, ctypes.POINTER(AdamwHparams), ctypes.c_int64, _P, _P,
                                    _P, _P, _P, _P]
        L.fl_local_step.argtypes = [_P, ctypes.POINTER(AdamwHparams), ctypes.c_int64,
                                    ctypes.c_int, _P, ctypes.c_float, _P, _P, _P, _P, _P, _P]
        L.fl_fedavg.argtypes = [_P, ctypes.c_int, _P, _P, _P, _P, _P, _P]
        L.fl_round.argtypes = [_P, ctypes.POINTER(RoundCfg), _P, _P, _P, _P, _P, _P, _P, _P]
        L.fl_round_noalloc.argtypes = [_P, ctypes.POINTER(RoundCfg), _P, _P, _P, _P, _P, _P, _P,
                                       _P]
        L.fl_noalloc_workspace_bytes.argtypes = [_P]
        L.fl_noalloc_workspace_bytes.restype = ctypes.c_size_t
        L.fl_shard_reduce_wire.argtypes = [_P, ctypes.c_int, _P, ctypes.c_float, _P, _P]
        L.fl_broadcast_recv.argtypes = [_P, _P, _P, _P, _P]
        L.fl_round_hsdp.argtypes = [_P, ctypes.POINTER(RoundCfg), ctypes.POINTER(HsdpCfg), _P, _P,
                                    _P, _P, _P, _P, _P, _P, _P, _P, _P]
        L.fl_fedopt.argtypes = [_P, ctypes.c_int, _P, _P, _P, ctypes.POINTER(OuterHparams), _P, _P,
                                _P, _P, _P]
        L.fl_round_outer.argtypes = [_P, ctypes.POINTER(RoundCfg), ctypes.POINTER(OuterHparams),
                                     _P, _P, _P, _P, _P, _P, _P, _P, _P, _P]
        L.fl_grad_sumsq.argtypes = [_P, ctypes.c_int, _P, ctypes.c_float, _P, _P, _P]
        L.fl_local_step_clipped.argtypes = [_P, ctypes.POINTER(AdamwHparams), ctypes.c_int64,
                                            ctypes.c_int, _P, ctypes.c_float, _P, ctypes.c_float,
                                            _P, _P, _P, _P, _P]
        L.fl_lr_cosine.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_float,
                                   ctypes.c_float]
        L.fl_lr_cosine.restype = ctypes.c_float
        shape = ctypes.POINTER(HeadShape)
        L.fl_head_workspace_bytes.argtypes = [shape, ctypes.c_int, ctypes.c_int]
        L.fl_head_workspace_bytes.restype = ctypes.c_size_t
        L.fl_head_loss.argtypes = [shape] + [_P] * 7 + [ctypes.c_size_t, _P]
        L.fl_head_loss_grad.argtypes = [shape] + [_P] * 9 + [ctypes.c_size_t, _P]
        L.fl_head_distill.argtypes = ([shape, _P, _P, ctypes.c_int, _P, _P, _P, ctypes.c_float]
                                      + [_P] * 4 + [ctypes.c_size_t, _P])
        L.fl_head_distill_grad.argtypes = ([shape, _P, _P, ctypes.c_int, _P, _P, _P,
                                            ctypes.c_float] + [_P] * 6 + [ctypes.c_size_t, _P])
        L.fl_top_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                             ctypes.c_int]
        L.fl_top_workspace_bytes.restype = ctypes.c_size_t
        L.fl_top_logits.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                    _P, ctypes.c_int, ctypes.c_float, _P, _P, _P, _P,
                                    ctypes.c_size_t, _P]
        shape = ctypes.POINTER(EmbedShape)
        L.fl_embed.argtypes = [shape, _P, _P, ctypes.c_float, _P, _P]
        L.fl_embed_workspace_bytes.argtypes = [shape]
        L.fl_embed_workspace_bytes.restype = ctypes.c_size_t
        L.fl_embed_grad.argtypes = [shape, _P, _P, ctypes.c_float, ctypes.c_int, _P, _P,
                                    ctypes.c_size_t, _P]
        shape = ctypes.POINTER(NormShape)
        L.fl_layer_norm.argtypes = [shape, _P, _P, _P, ctypes.c_float, _P, _P, _P, _P]
        L.fl_layer_norm_workspace_bytes.argtypes = [shape]
        L.fl_layer_norm_workspace_bytes.restype = ctypes.c_size_t
        L.fl_layer_norm_grad.argtypes = [shape] + [_P] * 9 + [ctypes.c_size_t, _P]
        L.fl_tensors_state_numel.argtypes = [ctypes.c_int64, _P]
        L.fl_tensors_state_numel.restype = ctypes.c_int64
        L.fl_tensors_state_bytes.argtypes = [ctypes.c_int64, ctypes.c_int]
        L.fl_tensors_state_bytes.restype = ctypes.c_size_t
        L.fl_adamw_tensors.argtypes = [ctypes.c_int64, _P, _P, ctypes.c_int, ctypes.c_float,
                                       ctypes.POINTER(AdamwHparams), ctypes.c_int64,
                                       ctypes.c_int, _P, ctypes.c_uint64, _P]
        L.fl_state_convert.argtypes = [ctypes.c_int64, ctypes.c_int, _P, _P, _P]
        L.fl_set_blocks_per_cu.argtypes = [ctypes.c_int]
        L.fl_set_blocks_per_cu.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status):
    return lib().fl_status_string(status).decode()


def _check(rc, where):
    if rc != FL_OK:
        raise FlError(rc, where)


_MAX_LIST = 1 << 20


def _buf(t, n, esize, what):
    """Device address of a tensor argument, after checking on the host what
    the kernels assume of it: a contiguous CUDA tensor of exactly n elements
    of esize bytes.  None gives NULL (the library decides whether that is
    allowed); an int is taken as a raw device address."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    try:
        if (t.is_cuda and t.is_contiguous() and t.element_size() == esize
                and t.numel() == n):
            return t.data_ptr()
    except AttributeError:
        pass
    # something is wrong with it: say what
    if not getattr(t, "is_cuda", False):
        raise ValueError("%s must be a CUDA tensor" % what)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    if t.element_size() != esize:
        raise ValueError("%s has %d-byte elements; expected %d" % (what, t.element_size(), esize))
    if t.numel() != n:
        raise ValueError("%s has %d elements; expected %d" % (what, t.numel(), n))
    return t.data_ptr()


def _bufs(ts, count, n, esize, what):
    """Host array of the device addresses of `count` tensors (each checked as
    in _buf).  A shorter list is padded with NULL, which the library rejects
    with FL_ERR_INVALID; a longer one is an error.  When `count` is outside
    what any call accepts, the list is passed as given for the library to
    reject the configuration."""
    ts = list(ts)
    if 1 <= count <= _MAX_LIST:
        if len(ts) > count:
            raise ValueError("%s has %d entries; expected %d" % (what, len(ts), count))
        size = count
    else:
        size = max(len(ts), 1)
    ptrs = []
    try:
        for t in ts:
            if t is None:
                ptrs.append(None)
            elif (t.is_cuda and t.is_contiguous() and t.element_size() == esize
                  and t.numel() == n):
                ptrs.append(t.data_ptr())
            else:
                break
        else:
            return (ctypes.c_void_p * size)(*ptrs)
    except AttributeError:
        pass
    # raw addresses among them, or something wrong: one by one
    arr = (ctypes.c_void_p * size)()
    for i, t in enumerate(ts):
        arr[i] = _buf(t, n, esize, "%s[%d]" % (what, i))
    return arr


def _host_list(xs, count, ctype, what):
    xs = list(xs)
    if len(xs) != count:
        raise ValueError("%s has %d entries; expected %d" % (what, len(xs), count))
    return (ctype * max(count, 1))(*xs)


_raw_stream = None   # (current device) -> its current stream's hipStream_t


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream if isinstance(stream, int) else stream.cuda_stream)
    global _raw_stream
    if _raw_stream is None:
        import torch

        # the current stream as a number: 0.3 us, against 2.9 us by way of a
        # torch.cuda.Stream object, which a call of a few us would spend on it
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = torch.cuda.current_device
        if raw is not None:
            _raw_stream = lambda: raw(dev())  # noqa: E731
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    return ctypes.c_void_p(_raw_stream())


def _stream_number(stream):
    """As _stream, as a number (a call of a few us takes it faster)."""
    if stream is None and _raw_stream is not None:
        return _raw_stream()
    return _stream(stream)


def hparams(hp):
    if isinstance(hp, AdamwHparams):
        return hp
    return AdamwHparams(hp["lr"], hp["beta1"], hp["beta2"], hp["eps"], hp["weight_decay"])


def set_blocks_per_cu(n):
    """Cap the streaming kernels' grid at n * CUs (0 = default); returns the
    previous value."""
    return lib().fl_set_blocks_per_cu(int(n))


def fingerprint(seg_offsets, seg_decay=None):
    import numpy as np

    off = np.ascontiguousarray(seg_offsets, dtype=np.int64)
    dec = None if seg_decay is None else np.ascontiguousarray(seg_decay, dtype=np.uint8)
    return lib().fl_fingerprint(int(off[-1]), off.size - 1, off.ctypes.data,
                                None if dec is None else dec.ctypes.data)


class Layout:
    """fl_layout handle: the flat shard's segments and decay flags."""

    def __init__(self, seg_offsets, seg_decay=None):
        import numpy as np

        off = np.ascontiguousarray(seg_offsets, dtype=np.int64)
        dec = None if seg_decay is None else np.ascontiguousarray(seg_decay, dtype=np.uint8)
        h = ctypes.c_void_p()
        rc = lib().fl_layout_create(int(off[-1]), off.size - 1, off.ctypes.data,
                                    None if dec is None else dec.ctypes.data, ctypes.byref(h))
        _check(rc, "fl_layout_create")
        self.handle = h
        self.n = int(off[-1])
        self.n_seg = off.size - 1

    @property
    def fingerprint(self):
        return lib().fl_layout_fingerprint(self.handle)

    def close(self):
        if self.handle:
            lib().fl_layout_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def fl_shard_reduce(layout, peer_grads, grad_scale, grad_out, seg_sumsq=None, stream=None):
    n, R = layout.n, len(peer_grads)
    rc = lib().fl_shard_reduce(layout.handle, R, _bufs(peer_grads, R, n, 2, "peer_grads"),
                               float(grad_scale), _buf(grad_out, n, 4, "grad_out"),
                               _buf(seg_sumsq, layout.n_seg, 4, "seg_sumsq"), _stream(stream))
    _check(rc, "fl_shard_reduce")


def fl_adamw_step(layout, hp, step, grad, master, m, v, working=None, stream=None):
    h = hparams(hp)
    n = layout.n
    rc = lib().fl_adamw_step(layout.handle, ctypes.byref(h), int(step), _buf(grad, n, 4, "grad"),
                             _buf(master, n, 4, "master"), _buf(m, n, 4, "m"),
                             _buf(v, n, 4, "v"), _buf(working, n, 2, "working"), _stream(stream))
    _check(rc, "fl_adamw_step")


def fl_local_step(layout, hp, step, peer_grads, grad_scale, master, m, v, working,
                  seg_sumsq=None, stream=None):
    h = hparams(hp)
    n, R = layout.n, len(peer_grads)
    rc = lib().fl_local_step(layout.handle, ctypes.byref(h), int(step), R,
                             _bufs(peer_grads, R, n, 2, "peer_grads"), float(grad_scale),
                             _buf(master, n, 4, "master"), _buf(m, n, 4, "m"), _buf(v, n, 4, "v"),
                             _buf(working, n, 2, "working"),
                             _buf(seg_sumsq, layout.n_seg, 4, "seg_sumsq"), _stream(stream))
    _check(rc, "fl_local_step")


def fl_fedavg(layout, replicas, weights, master_out, working_out, replica_fp=None, stream=None):
    n, G = layout.n, len(replicas)
    w = _host_list([float(x) for x in weights], G, ctypes.c_float, "weights")
    fp = None if replica_fp is None else _host_list([int(x) for x in replica_fp], G,
                                                    ctypes.c_uint64, "replica_fp")
    rc = lib().fl_fedavg(layout.handle, G, _bufs(replicas, G, n, 2, "replicas"), w, fp,
                         _buf(master_out, n, 4, "master_out"),
                         _buf(working_out, n, 2, "working_out"), _stream(stream))
    _check(rc, "fl_fedavg")


def make_round_cfg(R, G, A, weights, hp, *, self_group=0, grad_scale=None, step0=1,
                   replica_fp=None, phase_events=None, step_lr=None, max_grad_norm=0.0,
                   grad_scratch=None):
    """Build an fl_round_cfg; the returned object keeps its arrays alive.
    weights and replica_fp have G entries, step_lr A, phase_events A + 2;
    grad_scratch is None or a CUDA float32 tensor of the layout's length."""
    w = _host_list([float(x) for x in weights], G, ctypes.c_float, "weights")
    fp = None if replica_fp is None else _host_list([int(x) for x in replica_fp], G,
                                                    ctypes.c_uint64, "replica_fp")
    ev = None if phase_events is None else _host_list(phase_events, A + 2, ctypes.c_void_p,
                                                      "phase_events")
    lrs = None if step_lr is None else _host_list([float(x) for x in step_lr], A, ctypes.c_float,
                                                  "step_lr")
    scratch = None if grad_scratch is None else _buf(grad_scratch, grad_scratch.numel(), 4,
                                                     "grad_scratch")
    cfg = RoundCfg(R, G, A, self_group, float(1.0 / R if grad_scale is None else grad_scale),
                   hparams(hp), int(step0), w, fp, ev, lrs, float(max_grad_norm), scratch)
    cfg._keep = (w, fp, ev, lrs, grad_scratch)
    return cfg


def _check_cfg(layout, cfg):
    """The round configuration's tensor fields against the layout."""
    keep = getattr(cfg, "_keep", None)
    scratch = keep[4] if keep is not None and len(keep) > 4 else None
    if scratch is not None:
        _buf(scratch, layout.n, 4, "grad_scratch")


def lr_cosine(t, total_steps, warmup_steps, lr_max, lr_min=0.0):
    """fl_lr_cosine: the scheduled learning rate of optimiser step t."""
    return lib().fl_lr_cosine(int(t), int(total_steps), int(warmup_steps), float(lr_max),
                              float(lr_min))


def fl_round(layout, cfg, grads, replicas, master, m, v, working, seg_sumsq=None, stream=None):
    """grads: A*R tensors (step-major); replicas: G tensors or None (entry
    self_group is ignored)."""
    n = layout.n
    _check_cfg(layout, cfg)
    rc = lib().fl_round(layout.handle, ctypes.byref(cfg),
                        _bufs(grads, cfg.A * cfg.R, n, 2, "grads"),
                        _bufs(replicas, cfg.G, n, 2, "replicas"), _buf(master, n, 4, "master"),
                        _buf(m, n, 4, "m"), _buf(v, n, 4, "v"), _buf(working, n, 2, "working"),
                        _buf(seg_sumsq, cfg.A * layout.n_seg, 4, "seg_sumsq"), _stream(stream))
    _check(rc, "fl_round")


def fl_round_noalloc(layout, cfg, grads, replicas, master, m, v, working, seg_sumsq=None,
                     stream=None):
    """fl_round with the per-segment workspace in the library's static
    scratch: allocates nothing (see include/flround.h)."""
    n = layout.n
    _check_cfg(layout, cfg)
    rc = lib().fl_round_noalloc(layout.handle, ctypes.byref(cfg),
                                _bufs(grads, cfg.A * cfg.R, n, 2, "grads"),
                                _bufs(replicas, cfg.G, n, 2, "replicas"),
                                _buf(master, n, 4, "master"), _buf(m, n, 4, "m"),
                                _buf(v, n, 4, "v"), _buf(working, n, 2, "working"),
                                _buf(seg_sumsq, cfg.A * layout.n_seg, 4, "seg_sumsq"),
                                _stream(stream))
    _check(rc, "fl_round_noalloc")


def noalloc_workspace_bytes(layout):
    """Bytes of fl_round_noalloc's static scratch the layout's workspace
    needs (FL_NOALLOC_SCRATCH_BYTES is the limit)."""
    return int(lib().fl_noalloc_workspace_bytes(layout.handle))


def fl_shard_reduce_wire(layout, peer_grads, grad_scale, wire_out, stream=None):
    n, R = layout.n, len(peer_grads)
    rc = lib().fl_shard_reduce_wire(layout.handle, R, _bufs(peer_grads, R, n, 2, "peer_grads"),
                                    float(grad_scale), _buf(wire_out, n, 2, "wire_out"),
                                    _stream(stream))
    _check(rc, "fl_shard_reduce_wire")


def fl_broadcast_recv(layout, recv_master, master, working, stream=None):
    n = layout.n
    rc = lib().fl_broadcast_recv(layout.handle, _buf(recv_master, n, 4, "recv_master"),
                                 _buf(master, n, 4, "master"), _buf(working, n, 2, "working"),
                                 _stream(stream))
    _check(rc, "fl_broadcast_recv")


def make_hsdp_cfg(H, replica=0, hsdp_scale=None, fedavg_member=True):
    return HsdpCfg(int(H), int(replica), float(1.0 / H if hsdp_scale is None else hsdp_scale),
                   1 if fedavg_member else 0)


def fl_round_hsdp(layout, cfg, hcfg, grads, replica_wires, wire, replicas, bcast_master, master,
                  m, v, working, seg_sumsq=None, stream=None):
    """grads: A*R tensors; replica_wires: A*H tensors or None (entry
    a*H + replica ignored), or None when H == 1; wire: bf16 scratch (H > 1);
    replicas: G tensors/None (FedAvg member) or None; bcast_master: fp32
    tensor (non-member) or None."""
    n = layout.n
    _check_cfg(layout, cfg)
    rc = lib().fl_round_hsdp(
        layout.handle, ctypes.byref(cfg), ctypes.byref(hcfg),
        _bufs(grads, cfg.A * cfg.R, n, 2, "grads"),
        None if replica_wires is None else _bufs(replica_wires, cfg.A * hcfg.H, n, 2,
                                                 "replica_wires"),
        _buf(wire, n, 2, "wire"),
        None if replicas is None else _bufs(replicas, cfg.G, n, 2, "replicas"),
        _buf(bcast_master, n, 4, "bcast_master"), _buf(master, n, 4, "master"),
        _buf(m, n, 4, "m"), _buf(v, n, 4, "v"), _buf(working, n, 2, "working"),
        _buf(seg_sumsq, cfg.A * layout.n_seg, 4, "seg_sumsq"), _stream(stream))
    _check(rc, "fl_round_hsdp")


def fl_grad_sumsq(layout, peer_grads, grad_scale, total_sumsq, seg_sumsq=None, stream=None):
    """total_sumsq: a CUDA float64 tensor of one element."""
    n, R = layout.n, len(peer_grads)
    rc = lib().fl_grad_sumsq(layout.handle, R, _bufs(peer_grads, R, n, 2, "peer_grads"),
                             float(grad_scale), _buf(total_sumsq, 1, 8, "total_sumsq"),
                             _buf(seg_sumsq, layout.n_seg, 4, "seg_sumsq"), _stream(stream))
    _check(rc, "fl_grad_sumsq")


def fl_local_step_clipped(layout, hp, step, peer_grads, grad_scale, total_sumsq, max_norm, master,
                          m, v, working, stream=None):
    h = hparams(hp)
    n, R = layout.n, len(peer_grads)
    rc = lib().fl_local_step_clipped(layout.handle, ctypes.byref(h), int(step), R,
                                     _bufs(peer_grads, R, n, 2, "peer_grads"), float(grad_scale),
                                     _buf(total_sumsq, 1, 8, "total_sumsq"), float(max_norm),
                                     _buf(master, n, 4, "master"), _buf(m, n, 4, "m"),
                                     _buf(v, n, 4, "v"), _buf(working, n, 2, "working"),
                                     _stream(stream))
    _check(rc, "fl_local_step_clipped")


def fl_fedopt(layout, replicas, weights, outer, prev, buf, master_out, working_out,
              replica_fp=None, stream=None):
    n, G = layout.n, len(replicas)
    w = _host_list([float(x) for x in weights], G, ctypes.c_float, "weights")
    fp = None if replica_fp is None else _host_list([int(x) for x in replica_fp], G,
                                                    ctypes.c_uint64, "replica_fp")
    o = outer_hparams(outer)
    rc = lib().fl_fedopt(layout.handle, G, _bufs(replicas, G, n, 2, "replicas"), w, fp,
                         ctypes.byref(o), _buf(prev, n, 4, "prev"), _buf(buf, n, 4, "buf"),
                         _buf(master_out, n, 4, "master_out"),
                         _buf(working_out, n, 2, "working_out"), _stream(stream))
    _check(rc, "fl_fedopt")


def fl_round_outer(layout, cfg, outer, grads, replicas, prev, buf, master, m, v, working,
                   seg_sumsq=None, stream=None):
    o = outer_hparams(outer)
    n = layout.n
    _check_cfg(layout, cfg)
    rc = lib().fl_round_outer(layout.handle, ctypes.byref(cfg), ctypes.byref(o),
                              _bufs(grads, cfg.A * cfg.R, n, 2, "grads"),
                              _bufs(replicas, cfg.G, n, 2, "replicas"), _buf(prev, n, 4, "prev"),
                              _buf(buf, n, 4, "buf"), _buf(master, n, 4, "master"),
                              _buf(m, n, 4, "m"), _buf(v, n, 4, "v"),
                              _buf(working, n, 2, "working"),
                              _buf(seg_sumsq, cfg.A * layout.n_seg, 4, "seg_sumsq"),
                              _stream(stream))
    _check(rc, "fl_round_outer")


# ---- the output head --------------------------------------------------------


_T = None   # torch and the current device's number, looked up once: a call of a few
_dev = None  # us would spend as long on the module's own way to them


def _torch():
    global _T, _dev
    if _T is None:
        import torch

        _dev = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _T = torch
    return _T


def _array(t, shape, dtype, dev, what):
    """Device address of a contiguous tensor of this shape and dtype on device
    dev."""
    try:
        if (t.dtype is dtype and t.shape == shape and t.get_device() == dev
                and t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        pass
    # something is wrong with it: say what
    _on_device(t, dev, what)
    raise ValueError("%s must be a contiguous %s tensor of shape %s; got %s of shape %s"
                     % (what, dtype, shape, t.dtype, tuple(t.shape)))


def _device_of(t, what):
    """The current device, which has to be t's."""
    if not getattr(t, "is_cuda", False):   # (where there is no GPU, there is no device to ask for)
        raise ValueError("%s must be a CUDA tensor" % what)
    dev = _dev()
    _on_device(t, dev, what)
    return dev


def _on_device(t, dev, what):
    if not getattr(t, "is_cuda", False):
        raise ValueError("%s must be a CUDA tensor" % what)
    if t.get_device() != dev:
        raise ValueError("%s is on device %d; the current device is %d"
                         % (what, t.get_device(), dev))


def _rows(t, dtypes, dev, what):
    """(address, elements between rows) of a 2-D tensor whose rows are
    contiguous and do not overlap."""
    if t.get_device() != dev:
        _on_device(t, dev, what)
    if t.dim() != 2 or t.dtype not in dtypes:
        raise ValueError("%s must be a 2-D tensor of %s" % (what, " or ".join(map(str, dtypes))))
    n, d = t.shape
    between, within = t.stride()
    if d > 1 and within != 1:
        raise ValueError("%s must have contiguous rows" % what)
    if n <= 1:
        between = d
    if between < d:
        raise ValueError("%s has overlapping rows" % what)
    return t.data_ptr(), between


def _workspace(workspace, nbytes, dev, stream):
    """(tensor, bytes) of the workspace: the tensor given, or one from torch's
    allocator, which reuses it in the order of the stream it was taken on."""
    torch = _T
    if workspace is not None:
        _on_device(workspace, dev, "workspace")
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        return workspace, workspace.numel() * workspace.element_size()
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda"), nbytes
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda"), nbytes


@functools.lru_cache(maxsize=256)
def _head_shape(T, V, D, ldh, ldw, k, grad):
    """The shape as the library takes it, and the bytes of workspace for it."""
    s = HeadShape(T, V, D, ldh, ldw)
    return ctypes.byref(s), lib().fl_head_workspace_bytes(ctypes.byref(s), k, grad)


def head_workspace_bytes(tokens, vocab, width, k=0, grad=False, weight_stride=0):
    """Bytes of workspace that fl_head_loss (k = 0) or fl_head_distill and, with
    grad, their gradients need."""
    s = HeadShape(tokens, vocab, width, 0, weight_stride)
    return int(lib().fl_head_workspace_bytes(ctypes.byref(s), k, 1 if grad else 0))


def top_workspace_bytes(rows, vocab, k, dtype=FL_BF16):
    """Bytes of workspace that fl_top_logits needs (0 for many sizes)."""
    return int(lib().fl_top_workspace_bytes(rows, vocab, dtype, k))


def _listed_words(ids):
    """The k of ids (T x k)."""
    if ids.dim() != 2:
        raise ValueError("ids must be a 2-D tensor")
    return ids.shape[1]


class _HeadCall:
    """The arguments that the head's four functions share, checked."""

    def __init__(self, hidden, weight, k, grad, workspace, stream):
        torch = _T or _torch()
        self.dev = dev = _device_of(hidden, "hidden")
        bf16 = (torch.bfloat16,)
        self.h, ldh = _rows(hidden, bf16, dev, "hidden")
        self.w, ldw = _rows(weight, bf16, dev, "weight")
        self.T, self.D = hidden.shape
        self.V, width = weight.shape
        if width != self.D:
            raise ValueError("hidden is %d wide, weight %d" % (self.D, width))
        self.shape, need = _head_shape(self.T, self.V, self.D, ldh, ldw, k, grad)
        self.keep, self.ws_bytes = _workspace(workspace, need, dev, stream)
        self.ws = self.keep.data_ptr()
        self.stream = _stream(stream)

    def floats(self, t, what):
        return _array(t, (self.T,), _T.float32, self.dev, what)

    def listed(self, t, what):
        return _array(t, (self.T, self.k), _T.float32, self.dev, what)

    def labels(self, t):
        return _array(t, (self.T,), _T.int64, self.dev, "labels")

    def teacher(self, ids, teacher, teacher_lse):
        self.k = _listed_words(ids)
        return (_array(ids, (self.T, self.k), _T.int32, self.dev, "ids"),
                self.listed(teacher, "teacher"),
                None if teacher_lse is None else self.floats(teacher_lse, "teacher_lse"))

    def grads(self, dhidden, dweight):
        return (_array(dhidden, (self.T, self.D), _T.bfloat16, self.dev, "dhidden"),
                _array(dweight, (self.V, self.D), _T.bfloat16, self.dev, "dweight"))


def fl_head_loss(hidden, weight, labels, loss, lse, target, workspace=None, stream=None):
    """Cross entropy of hidden (T x D bf16) through weight (V x D bf16) at
    labels (T int64, negative: the token takes no part).  Writes loss, lse and
    target (T float32 each); lse and target go to fl_head_loss_grad."""
    c = _HeadCall(hidden, weight, 0, 0, workspace, stream)
    rc = lib().fl_head_loss(c.shape, c.h, c.w, c.labels(labels), c.floats(loss, "loss"),
                            c.floats(lse, "lse"), c.floats(target, "target"), c.ws, c.ws_bytes,
                            c.stream)
    _check(rc, "fl_head_loss")


def fl_head_loss_grad(hidden, weight, labels, lse, target, dloss, dhidden, dweight,
                      workspace=None, stream=None):
    """Gradient of sum(dloss * loss): writes dhidden (T x D) and dweight
    (V x D), bf16.  lse and target as fl_head_loss wrote them."""
    c = _HeadCall(hidden, weight, 0, 1, workspace, stream)
    dh, dw = c.grads(dhidden, dweight)
    rc = lib().fl_head_loss_grad(c.shape, c.h, c.w, c.labels(labels), c.floats(lse, "lse"),
                                 c.floats(target, "target"), c.floats(dloss, "dloss"), dh, dw,
                                 c.ws, c.ws_bytes, c.stream)
    _check(rc, "fl_head_loss_grad")


def fl_head_distill(hidden, weight, ids, teacher, teacher_lse, tau, loss, lse, target,
                    workspace=None, stream=None):
    """Divergence of the student's distribution from the teacher's over the
    listed words: ids (T x k int32, negative: absent) and teacher (T x k
    float32) as fl_top_logits writes them, teacher_lse (T float32) or None to
    normalise over the listed words.  Writes loss and lse (T float32) and
    target (T x k float32)."""
    c = _HeadCall(hidden, weight, _listed_words(ids), 0, workspace, stream)
    i, a, al = c.teacher(ids, teacher, teacher_lse)
    rc = lib().fl_head_distill(c.shape, c.h, c.w, c.k, i, a, al, float(tau),
                               c.floats(loss, "loss"), c.floats(lse, "lse"),
                               c.listed(target, "target"), c.ws, c.ws_bytes, c.stream)
    _check(rc, "fl_head_distill")


def fl_head_distill_grad(hidden, weight, ids, teacher, teacher_lse, tau, lse, target, dloss,
                         dhidden, dweight, workspace=None, stream=None):
    """Gradient of sum(dloss * loss) of fl_head_distill: writes dhidden and
    dweight, bf16."""
    c = _HeadCall(hidden, weight, _listed_words(ids), 1, workspace, stream)
    i, a, al = c.teacher(ids, teacher, teacher_lse)
    dh, dw = c.grads(dhidden, dweight)
    rc = lib().fl_head_distill_grad(c.shape, c.h, c.w, c.k, i, a, al, float(tau),
                                    c.floats(lse, "lse"), c.listed(target, "target"),
                                    c.floats(dloss, "dloss"), dh, dw, c.ws, c.ws_bytes, c.stream)
    _check(rc, "fl_head_distill_grad")


def fl_top_logits(logits, k, tau, values, ids, lse=None, workspace=None, stream=None):
    """The k largest of each row of logits (rows x vocab, bf16 or float32, rows
    may be longer), largest first, ties to the lowest id: writes values
    (rows x k float32), ids (rows x k int32) and lse (rows float32, or None),
    the log of the sum of exp(logits / tau)."""
    torch = _T or _torch()
    dev = _device_of(logits, "logits")
    p, stride = _rows(logits, (torch.bfloat16, torch.float32), dev, "logits")
    n, v = logits.shape
    dtype = FL_BF16 if logits.dtype == torch.bfloat16 else FL_F32
    args = (_array(values, (n, k), torch.float32, dev, "values"),
            _array(ids, (n, k), torch.int32, dev, "ids"),
            None if lse is None else _array(lse, (n,), torch.float32, dev, "lse"))
    need = lib().fl_top_workspace_bytes(n, v, dtype, k)
    ws, ws_bytes = None, 0
    if need or workspace is not None:
        keep, ws_bytes = _workspace(workspace, need, dev, stream)
        ws = keep.data_ptr()
    rc = lib().fl_top_logits(n, v, stride, dtype, p, k, float(tau), *args, ws, ws_bytes,
                             _stream(stream))
    _check(rc, "fl_top_logits")


# ---- the embedding and the layer norm ----------------------------------------


def _dtype_number(t):
    """FL_BF16 or FL_F32 of a tensor that _rows has seen."""
    return FL_BF16 if t.dtype is _T.bfloat16 else FL_F32


def _row_tensor(t, what):
    """(device, address, elements between rows) of a bf16 or float32 tensor of rows on the
    current device."""
    torch = _T or _torch()
    dev = _device_of(t, what)
    return (dev, *_rows(t, (torch.bfloat16, torch.float32), dev, what))


def _maybe(t, shape, dtype, dev, what):
    return None if t is None else _array(t, shape, dtype, dev, what)


@functools.lru_cache(maxsize=256)
def _embed_shape(T, V, D, stride, dtype):
    """The shape as the library takes it, and the bytes of workspace for its gradient."""
    s = EmbedShape(T, V, D, stride, dtype)
    return ctypes.byref(s), lib().fl_embed_workspace_bytes(ctypes.byref(s))


@functools.lru_cache(maxsize=256)
def _norm_shape(R, D, ldx, ldy, dtype, rms):
    s = NormShape(R, D, ldx, ldy, dtype, rms)
    return ctypes.byref(s), lib().fl_layer_norm_workspace_bytes(ctypes.byref(s))


def embed_workspace_bytes(tokens, vocab, width, dtype=FL_BF16):
    """Bytes of workspace that fl_embed_grad needs."""
    return int(_embed_shape(tokens, vocab, width, 0, dtype)[1])


def layer_norm_workspace_bytes(rows, width, dtype=FL_BF16):
    """Bytes of workspace that fl_layer_norm_grad needs."""
    return int(_norm_shape(rows, width, 0, 0, dtype, 0)[1])


def fl_embed(ids, weight, out, scale=1.0, stream=None):
    """out[t] = scale * weight[ids[t]]: ids (T int64, negative: the row is 0), weight
    (V x D bf16 or float32, rows may be longer), out (T x D of its dtype)."""
    dev, w, ldw = _row_tensor(weight, "weight")
    V, D = weight.shape
    T = ids.numel()
    shape, _ = _embed_shape(T, V, D, ldw, _dtype_number(weight))
    rc = lib().fl_embed(shape, _array(ids, (T,), _T.int64, dev, "ids"), w, scale,
                        _array(out, (T, D), weight.dtype, dev, "out"), _stream_number(stream))
    if rc:
        _check(rc, "fl_embed")


def fl_embed_grad(ids, dout, dweight, scale=1.0, add=False, workspace=None, stream=None):
    """Gradient of sum(dout * out) by the weight: writes dweight (V x D, of dout's
    dtype), or with add adds to the rows of the words that occur.  dout: T x D, rows
    may be longer."""
    dev, d, ldd = _row_tensor(dout, "dout")
    T, D = dout.shape
    if dweight.dim() != 2:
        raise ValueError("dweight must be a 2-D tensor")
    V = dweight.shape[0]
    shape, need = _embed_shape(T, V, D, ldd, _dtype_number(dout))
    keep, nbytes = _workspace(workspace, need, dev, stream)
    rc = lib().fl_embed_grad(shape, _array(ids, (T,), _T.int64, dev, "ids"), d, scale,
                             1 if add else 0, _array(dweight, (V, D), dout.dtype, dev, "dweight"),
                             keep.data_ptr(), nbytes, _stream_number(stream))
    if rc:
        _check(rc, "fl_embed_grad")


def fl_layer_norm(x, weight, bias, eps, y, mean, rstd, rms=False, stream=None):
    """Layer norm of the rows of x (R x D bf16 or float32, rows may be longer) into y;
    weight and bias (D, or None) and y have x's dtype.  Writes mean (or None) and rstd
    (R float32), which the gradient takes.  rms: root mean square norm, without a mean."""
    dev, p, ldx = _row_tensor(x, "x")
    R, D = x.shape
    dt, f32 = x.dtype, _T.float32
    shape, _ = _norm_shape(R, D, ldx, 0, _dtype_number(x), 1 if rms else 0)
    rc = lib().fl_layer_norm(shape, p, _maybe(weight, (D,), dt, dev, "weight"),
                             _maybe(bias, (D,), dt, dev, "bias"), eps,
                             _array(y, (R, D), dt, dev, "y"), _maybe(mean, (R,), f32, dev, "mean"),
                             _array(rstd, (R,), f32, dev, "rstd"), _stream_number(stream))
    if rc:
        _check(rc, "fl_layer_norm")


def fl_layer_norm_grad(x, weight, mean, rstd, dy, dx, dweight, dbias, rms=False, workspace=None,
                       stream=None):
    """Gradient of sum(dy * y) of fl_layer_norm: writes dx (R x D), dweight and dbias (D
    each, or None), all of x's dtype.  mean (None with rms) and rstd as fl_layer_norm
    wrote them; rows of x and dy may be longer."""
    dev, p, ldx = _row_tensor(x, "x")
    R, D = x.shape
    dt, f32 = x.dtype, _T.float32
    g, ldy = _rows(dy, (dt,), dev, "dy")
    if dy.shape != x.shape:
        raise ValueError("dy has shape %s, x %s" % (tuple(dy.shape), tuple(x.shape)))
    shape, need = _norm_shape(R, D, ldx, ldy, _dtype_number(x), 1 if rms else 0)
    keep, nbytes = _workspace(workspace, need, dev, stream)
    rc = lib().fl_layer_norm_grad(
        shape, p, _maybe(weight, (D,), dt, dev, "weight"), _maybe(mean, (R,), f32, dev, "mean"),
        _array(rstd, (R,), f32, dev, "rstd"), g, _array(dx, (R, D), dt, dev, "dx"),
        _maybe(dweight, (D,), dt, dev, "dweight"), _maybe(dbias, (D,), dt, dev, "dbias"),
        keep.data_ptr(), nbytes, _stream_number(stream))
    if rc:
        _check(rc, "fl_layer_norm_grad")


# ---- AdamW over many tensors --------------------------------------------------


_dtype_of = operator.attrgetter("dtype")


def _whole(t, dtype, what):
    """Checks a contiguous CUDA tensor of this dtype."""
    if not getattr(t, "is_cuda", False):
        raise ValueError("%s must be a CUDA tensor" % what)
    if t.dtype is not dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor" % (what, dtype))


class Tensors:
    """Parameters that fl_adamw_tensors steps together: float32 masters and their bf16
    working copies (None, or None for some: not written), all of one device, and which of
    them decay (default: all).  It keeps the tensors, their memory and its addresses: when
    one has moved to other memory, a step raises ValueError, and another Tensors is needed.

    n_state: elements of each moment; state(bits) gives a state before the first step."""

    def __init__(self, masters, workings=None, decays=None):
        torch = _T or _torch()
        self.masters = list(masters)
        count = len(self.masters)
        self.workings = [None] * count if workings is None else list(workings)
        decays = [True] * count if decays is None else list(decays)
        for name, xs in (("workings", self.workings), ("decays", decays)):
            if len(xs) != count:
                raise ValueError("%s has %d entries; expected %d" % (name, len(xs), count))
        self.array = (FlTensor * max(count, 1))()
        self.device = None
        places = []
        held, self._memory = [], []
        for i, (m, w) in enumerate(zip(self.masters, self.workings)):
            for t, dtype, what in ((m, torch.float32, "masters"), (w, torch.bfloat16, "workings")):
                if t is None and what == "workings":
                    continue
                _whole(t, dtype, "%s[%d]" % (what, i))
                if self.device is None:
                    self.device = t.get_device()
                _on_device(t, self.device, "%s[%d]" % (what, i))
                if t.numel() != m.numel():
                    raise ValueError("workings[%d] has %d elements; expected %d"
                                     % (i, t.numel(), m.numel()))
                places.append((t.data_ptr(), t.numel() * t.element_size(), "%s[%d]" % (what, i)))
                held.append(t)
                self._memory.append(t.detach())   # (keeps it where t is given other memory)
            self.array[i] = FlTensor(m.numel(), m.data_ptr(), None if w is None else w.data_ptr(),
                                     1 if decays[i] else 0)
        places = sorted(p for p in places if p[1])
        for a, b in zip(places, places[1:]):
            if a[0] + a[1] > b[0]:
                raise ValueError("%s and %s overlap" % (a[2], b[2]))
        self._held, self._addresses = held, [t.data_ptr() for t in held]
        self.count = count
        self.sizes = [m.numel() for m in self.masters]
        self.n_state = int(lib().fl_tensors_state_numel(count, self.array))

    def _check_places(self):
        """That all masters and working copies are where they were."""
        if list(map(_T.Tensor.data_ptr, self._held)) != self._addresses:
            raise ValueError("a master or a working copy has moved to other memory: Tensors has "
                             "to be made anew")

    def state(self, bits=8):
        """Moments of zero: a uint8 tensor for 8 bits, a float32 one (m, then v) for 32."""
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        nbytes = int(lib().fl_tensors_state_bytes(self.n_state, bits))
        dtype = _T.uint8 if bits == 8 else _T.float32
        device = "cuda" if self.device is None else "cuda:%d" % self.device
        return _T.zeros(nbytes if bits == 8 else nbytes // 4, dtype=dtype, device=device)


@functools.lru_cache(maxsize=64)
def _state_size(n, bits):
    """Elements of the tensor that holds the moments of n elements."""
    return lib().fl_tensors_state_bytes(n, bits) // (1 if bits == 8 else 4)


def _state(t, n, dev, what):
    """(address, bits) of the moments of n elements."""
    torch = _T
    if t.dtype is torch.uint8:
        bits = 8
    elif t.dtype is torch.float32:
        bits = 32
    else:
        raise ValueError("%s must be a uint8 or a float32 tensor" % what)
    return _array(t, (_state_size(n, bits),), t.dtype, dev, what), bits


def _grad_ptrs(grads, sizes, dev):
    """Addresses of the gradients (0 for one that is left out), checked, and their
    dtype."""
    torch = _T
    T = torch.Tensor
    dtype = None
    try:   # all at once: a list of some hundred costs 0.2 us each
        if list(map(T.numel, grads)) == sizes:
            dtypes, devs = set(map(_dtype_of, grads)), set(map(T.get_device, grads))
            if len(dtypes) == 1 and devs == {dev} and all(map(T.is_contiguous, grads)):
                dtype = dtypes.pop()
                if dtype is torch.bfloat16 or dtype is torch.float32:
                    return list(map(T.data_ptr, grads)), dtype
    except (TypeError, AttributeError):
        pass
    # one is left out, or something is wrong: one by one
    ptrs, dtype = [], None
    for i, g in enumerate(grads):
        if g is None:
            ptrs.append(0)
            continue
        what = "grads[%d]" % i
        if dtype is None:
            dtype = getattr(g, "dtype", None)
            if dtype is not torch.bfloat16 and dtype is not torch.float32:
                raise ValueError("%s must be a bf16 or float32 tensor" % what)
        _whole(g, dtype, what)
        _on_device(g, dev, what)
        if g.numel() != sizes[i]:
            raise ValueError("%s has %d elements; expected %d" % (what, g.numel(), sizes[i]))
        ptrs.append(g.data_ptr())
    return ptrs, dtype


def fl_adamw_tensors(tensors, hp, step, grads, state, grad_scale=1.0, seed=0, stream=None):
    """One AdamW step of all `tensors` (a Tensors): grads holds a contiguous bf16 or
    float32 gradient (all of one dtype) for each, or None for one that is left alone;
    state as Tensors.state gives it, updated.  seed: nonzero rounds 8-bit moments by
    random bits of the seed and the step, whose expected value is the moment (captured into
    a graph, the same bits at each replay); 0 to nearest."""
    torch = _T or _torch()
    count, sizes = tensors.count, tensors.sizes
    dev = _dev() if tensors.device is not None else None
    if tensors.device != dev:
        raise ValueError("the tensors are on device %s; the current device is %s"
                         % (tensors.device, dev))
    grads = list(grads)
    if len(grads) != count:
        raise ValueError("grads has %d entries; expected %d" % (len(grads), count))
    tensors._check_places()
    ptrs, dtype = _grad_ptrs(grads, sizes, dev)
    if count == 0:
        return
    if not 0 <= seed < 1 << 64:
        raise ValueError("seed must be between 0 and 2^64 - 1")
    h = hparams(hp)
    p, bits = _state(state, tensors.n_state, dev, "state")
    at = array.array("Q", ptrs)
    rc = lib().fl_adamw_tensors(count, tensors.array, at.buffer_info()[0],
                                FL_F32 if dtype is torch.float32 else FL_BF16, float(grad_scale),
                                ctypes.byref(h), int(step), bits, p, int(seed), _stream(stream))
    _check(rc, "fl_adamw_tensors")


def fl_state_convert(src, dst, stream=None):
    """The moments of an AdamW state in the other form: from 8 bits (uint8) to 32
    (float32: m, then v), exactly, or from 32 to 8, to nearest."""
    torch = _T or _torch()
    dev = _device_of(src, "src")
    if dst.dtype is not (torch.float32 if src.dtype is torch.uint8 else torch.uint8):
        raise ValueError("one of src and dst must be a uint8, the other a float32 tensor")
    wide = dst if src.dtype is torch.uint8 else src
    n = wide.numel() // 2
    p, bits = _state(src, n, dev, "src")
    q, _ = _state(dst, n, dev, "dst")
    rc = lib().fl_state_convert(n, bits, p, q, _stream(stream))
    _check(rc, "fl_state_convert")


# ---- HIP events (for fl_round's per-phase timing) -------------------------

_hip = None


def hip_runtime():
    global _hip
    if _hip is None:
        h = None
        for name in ("libamdhip64.so", "libamdhip64.so.7", "/opt/rocm/lib/libamdhip64.so"):
            try:
                h = ctypes.CDLL(name)
                break
            except OSError:
                continue
        if h is None:
            raise RuntimeError("HIP runtime library not found")
        h.hipMalloc.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_size_t]
        h.hipFree.argtypes = [ctypes.c_void_p]
        h.hipGetDevice.argtypes = [ctypes.POINTER(ctypes.c_int)]
        h.hipSetDevice.argtypes = [ctypes.c_int]
        h.hipEventCreate.argtypes = [ctypes.POINTER(ctypes.c_void_p)]
        h.hipEventCreateWithFlags.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_uint]
        h.hipEventDestroy.argtypes = [ctypes.c_void_p]
        h.hipEventRecord.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        h.hipEventSynchronize.argtypes = [ctypes.c_void_p]
        h.hipEventElapsedTime.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_void_p,
                                          ctypes.c_void_p]
        _hip = h
    return _hip


# hipEventCreateWithFlags flag: no system-scope fence (cache write-back and
# invalidation) when the event is recorded; for events that only time work.
HIP_EVENT_DISABLE_SYSTEM_FENCE = 0x20000000


class HipEvents:
    """k raw hipEvent_t handles, for fl_round's phase_events (created with
    hipEventCreateWithFlags(flags))."""

    def __init__(self, k, flags=0):
        h = hip_runtime()
        self.handles = []
        for _ in range(k):
            e = ctypes.c_void_p()
            if h.hipEventCreateWithFlags(ctypes.byref(e), ctypes.c_uint(flags)) != 0:
                raise RuntimeError("hipEventCreateWithFlags failed")
            self.handles.append(e.value)

    def elapsed_ms(self, i, j):
        h = hip_runtime()
        out = ctypes.c_float()
        if h.hipEventElapsedTime(ctypes.byref(out), self.handles[i], self.handles[j]) != 0:
            raise RuntimeError("hipEventElapsedTime failed")
        return out.value

    def record(self, i, stream):
        if hip_runtime().hipEventRecord(self.handles[i], stream) != 0:
            raise RuntimeError("hipEventRecord failed")

    def synchronize(self, i):
        if hip_runtime().hipEventSynchronize(self.handles[i]) != 0:
            raise RuntimeError("hipEventSynchronize failed")

    def close(self):
        h = hip_runtime()
        for e in self.handles:
            h.hipEventDestroy(e)
        self.handles = []
