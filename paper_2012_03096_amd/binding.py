"""Thin ctypes binding of libpbkd.so (include/pbkd.h): argument marshalling only.

Every step of the distillation path runs inside the library's HIP kernels.  PyTorch appears only as
the owner of device memory (the workspace, inputs, targets are torch tensors whose data_ptr() is
handed over) and of HIP streams.  Loading fails loudly if the library has not been built; there is no
fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct
from itertools import accumulate, chain
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpbkd.so")

OK, EINVAL, ESHAPE, ENOMEM, EHIP, ESTATE, EUNSUPPORTED = 0, -1, -2, -3, -4, -5, -6
CONV3X3, DWSEP3X3 = 0, 1
STUDENT_PARAM, STUDENT_GRAD, STUDENT_MOMENTUM, TEACHER_PARAM, STUDENT_ACT, TEACHER_ACT, STUDENT_BN_RUNNING, TEACHER_BN_RUNNING = range(8)

EXPORTS = [
    "pbkd_arch_validate", "pbkd_block_workspace_bytes", "pbkd_block_create", "pbkd_block_destroy",
    "pbkd_teacher_forward", "pbkd_student_step", "pbkd_distill_step", "pbkd_block_set_aux_stream", "pbkd_block_set_graph_mode", "pbkd_student_forward", "pbkd_block_last_loss",
    "pbkd_schedule_blocks", "pbkd_distill_step_all", "pbkd_run_tasks_work_stealing", "pbkd_network_forward", "pbkd_feature_mse", "pbkd_feature_mse_noalloc", "pbkd_select_blocks", "pbkd_block_flops", "pbkd_arch_flops", "pbkd_arch_conv_kernel",
    "pbkd_block_get_tensor", "pbkd_block_set_tensor", "pbkd_last_error",
    "pbkd_kernel_kinds", "pbkd_kernel_kind_name", "pbkd_block_profile_enable", "pbkd_block_profile_read",
    "pbkd_rmsnorm_forward", "pbkd_rmsnorm_backward", "pbkd_rmsnorm_workspace_bytes", "pbkd_recurrence_forward", "pbkd_recurrence_backward",
    "pbkd_recurrence_step", "pbkd_recurrence_saved_bytes", "pbkd_recurrence_workspace_bytes", "pbkd_adamw_step",
    "pbkd_embed_forward", "pbkd_embed_backward", "pbkd_embed_workspace_bytes", "pbkd_head_loss", "pbkd_head_loss_workspace_bytes", "pbkd_topk_distill",
]


class LayerDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("cin", ctypes.c_int), ("cout", ctypes.c_int), ("stride", ctypes.c_int),
                ("trainable", ctypes.c_int)]


class ArchDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int), ("c", ctypes.c_int), ("h", ctypes.c_int), ("w", ctypes.c_int),
                ("n_layers", ctypes.c_int), ("layers", ctypes.POINTER(LayerDesc)), ("shortcut", ctypes.c_int),
                ("shortcut_stride", ctypes.c_int), ("pool", ctypes.c_int), ("bn_eps", ctypes.c_float)]


class TrainDesc(ctypes.Structure):
    _fields_ = [("momentum", ctypes.c_float), ("loss_reduction", ctypes.c_int), ("bn_decay", ctypes.c_float)]


class PbkdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"pbkd status {status}: {message}")
        self.status = status


_lib = None


def lib():
    """Loads libpbkd.so once; raises if it is missing (build it with __graft_entry__.build())."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
        # PyTorch ships its own copy of the HIP runtime (same soname).  Import it first so that the
        # dynamic loader binds libpbkd.so to that one instance: two HIP runtimes in one process cannot
        # share device memory or streams.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, fp, ip = ctypes.c_void_p, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int)
        ullp = ctypes.POINTER(ctypes.c_ulonglong)
        ap = ctypes.POINTER(ArchDesc)
        L.pbkd_arch_validate.argtypes = [ap, ap]
        L.pbkd_arch_validate.restype = ctypes.c_int
        L.pbkd_block_workspace_bytes.argtypes = [ap, ap]
        L.pbkd_block_workspace_bytes.restype = ctypes.c_size_t
        L.pbkd_block_create.argtypes = [ap, ctypes.POINTER(fp), ap, ctypes.POINTER(fp), ctypes.POINTER(TrainDesc), vp,
                                        ctypes.c_size_t, vp, ctypes.POINTER(vp)]
        L.pbkd_block_create.restype = ctypes.c_int
        L.pbkd_block_destroy.argtypes = [vp]
        L.pbkd_block_destroy.restype = ctypes.c_int
        L.pbkd_teacher_forward.argtypes = [vp, vp, vp, vp]
        L.pbkd_teacher_forward.restype = ctypes.c_int
        L.pbkd_student_step.argtypes = [vp, vp, vp, ctypes.c_float, fp, vp]
        L.pbkd_student_step.restype = ctypes.c_int
        L.pbkd_distill_step.argtypes = [vp, vp, vp, ctypes.c_float, fp, vp, vp]
        L.pbkd_distill_step.restype = ctypes.c_int
        L.pbkd_run_tasks_work_stealing.argtypes = [ctypes.c_int, vp, vp, vp, ctypes.c_float, ctypes.POINTER(ctypes.c_int), ctypes.c_int,
                                                   vp, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int),
                                                   ctypes.POINTER(ctypes.c_int)]
        L.pbkd_run_tasks_work_stealing.restype = ctypes.c_int
        L.pbkd_network_forward.argtypes = [ctypes.c_int, vp, ctypes.POINTER(ctypes.c_int), ctypes.c_int, vp, vp, vp]
        L.pbkd_network_forward.restype = ctypes.c_int
        L.pbkd_select_blocks.argtypes = [ctypes.c_int, vp, ctypes.c_int, vp, vp, vp, ctypes.c_double, ctypes.POINTER(ctypes.c_int),
                                         ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), vp]
        L.pbkd_select_blocks.restype = ctypes.c_int
        L.pbkd_feature_mse.argtypes = [vp, vp, vp, ctypes.c_size_t, ctypes.POINTER(ctypes.c_double), vp]
        L.pbkd_feature_mse.restype = ctypes.c_int
        L.pbkd_feature_mse_noalloc.argtypes = [vp, vp, ctypes.c_size_t, ctypes.POINTER(ctypes.c_double), vp]
        L.pbkd_feature_mse_noalloc.restype = ctypes.c_int
        L.pbkd_block_set_graph_mode.argtypes = [vp, ctypes.c_int]
        L.pbkd_block_set_graph_mode.restype = ctypes.c_int
        L.pbkd_block_set_aux_stream.argtypes = [vp, vp]
        L.pbkd_block_set_aux_stream.restype = ctypes.c_int
        L.pbkd_student_forward.argtypes = [vp, vp, vp, vp]
        L.pbkd_student_forward.restype = ctypes.c_int
        L.pbkd_block_last_loss.argtypes = [vp, fp]
        L.pbkd_block_last_loss.restype = ctypes.c_int
        L.pbkd_schedule_blocks.argtypes = [ctypes.c_int, ullp, ctypes.POINTER(vp), ctypes.c_int, ctypes.c_int, ip, ip, ullp]
        L.pbkd_schedule_blocks.restype = ctypes.c_int
        L.pbkd_distill_step_all.argtypes = [ctypes.c_int, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                            ctypes.c_float, ctypes.c_int, ctypes.POINTER(vp), ip, ip, ctypes.c_int, vp]
        L.pbkd_distill_step_all.restype = ctypes.c_int
        L.pbkd_block_flops.argtypes = [vp, ctypes.c_int]
        L.pbkd_block_flops.restype = ctypes.c_ulonglong
        L.pbkd_arch_flops.argtypes = [ap, ctypes.c_int]
        L.pbkd_arch_flops.restype = ctypes.c_ulonglong
        L.pbkd_arch_conv_kernel.argtypes = [ap, ctypes.c_int, ip]
        L.pbkd_arch_conv_kernel.restype = ctypes.c_char_p
        L.pbkd_block_get_tensor.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, fp, ctypes.c_size_t]
        L.pbkd_block_get_tensor.restype = ctypes.c_int
        L.pbkd_block_set_tensor.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, fp, ctypes.c_size_t]
        L.pbkd_block_set_tensor.restype = ctypes.c_int
        L.pbkd_last_error.argtypes = []
        L.pbkd_last_error.restype = ctypes.c_char_p
        L.pbkd_kernel_kinds.argtypes = []
        L.pbkd_kernel_kinds.restype = ctypes.c_int
        L.pbkd_kernel_kind_name.argtypes = [ctypes.c_int]
        L.pbkd_kernel_kind_name.restype = ctypes.c_char_p
        L.pbkd_block_profile_enable.argtypes = [vp, ctypes.c_uint, ctypes.c_int]
        L.pbkd_block_profile_enable.restype = ctypes.c_int
        L.pbkd_block_profile_read.argtypes = [vp, ctypes.c_int, ctypes.POINTER(ctypes.c_double), ip]
        L.pbkd_block_profile_read.restype = ctypes.c_int
        for f in (L.pbkd_rmsnorm_forward, L.pbkd_rmsnorm_backward, L.pbkd_recurrence_forward, L.pbkd_recurrence_backward, L.pbkd_recurrence_step):
            f.argtypes, f.restype = [vp, vp], ctypes.c_int
        L.pbkd_rmsnorm_workspace_bytes.argtypes = [ctypes.c_longlong, ctypes.c_int]
        L.pbkd_rmsnorm_workspace_bytes.restype = ctypes.c_size_t
        for f in (L.pbkd_recurrence_saved_bytes, L.pbkd_recurrence_workspace_bytes):
            f.argtypes, f.restype = [ctypes.c_int, ctypes.c_longlong, ctypes.c_int], ctypes.c_size_t
        for f in (L.pbkd_embed_forward, L.pbkd_embed_backward, L.pbkd_head_loss, L.pbkd_topk_distill):
            f.argtypes, f.restype = [vp, vp], ctypes.c_int
        L.pbkd_embed_workspace_bytes.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
        L.pbkd_embed_workspace_bytes.restype = ctypes.c_size_t
        L.pbkd_head_loss_workspace_bytes.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.pbkd_head_loss_workspace_bytes.restype = ctypes.c_size_t
        L.pbkd_adamw_step.argtypes = [ctypes.c_int, vp, vp, vp]
        L.pbkd_adamw_step.restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != OK:
        raise PbkdError(status, lib().pbkd_last_error().decode())


def make_arch(arch) -> ArchDesc:
    """Converts a workloads.Arch (or anything with the same attributes) into the C descriptor.
    The returned struct keeps its layer array alive."""
    layers = (LayerDesc * len(arch.layers))(*[LayerDesc(L.kind, L.cin, L.cout, L.stride, L.trainable) for L in arch.layers])
    d = ArchDesc(arch.n, arch.c, arch.h, arch.w, len(arch.layers), layers, arch.shortcut, arch.shortcut_stride, arch.pool,
                 arch.bn_eps)
    d._keep = layers
    return d


def arch_validate(teacher, student) -> int:
    return lib().pbkd_arch_validate(ctypes.byref(make_arch(teacher)), ctypes.byref(make_arch(student)))


def last_error() -> str:
    return lib().pbkd_last_error().decode()


def workspace_bytes(teacher, student) -> int:
    return lib().pbkd_block_workspace_bytes(ctypes.byref(make_arch(teacher)), ctypes.byref(make_arch(student)))


def arch_flops(arch, training_step: bool) -> int:
    return lib().pbkd_arch_flops(ctypes.byref(make_arch(arch)), int(training_step))


def arch_conv_kernel(teacher, layer: int):
    """(name, parts K is split into) of the kernel a teacher's 3x3 convolution runs on; ("", 0) if there is none."""
    parts = ctypes.c_int()
    return lib().pbkd_arch_conv_kernel(ctypes.byref(make_arch(teacher)), layer, ctypes.byref(parts)).decode(), parts.value


def schedule_blocks(weights: Optional[Sequence[int]], n_streams: int, policy: int = 0, blocks: Optional[Sequence["Block"]] = None):
    """Returns (stream_of_block, order, stream_load)."""
    n = len(weights) if weights is not None else len(blocks)
    w = (ctypes.c_ulonglong * n)(*weights) if weights is not None else None
    hb = (ctypes.c_void_p * n)(*[b.handle for b in blocks]) if blocks is not None else None
    sob = (ctypes.c_int * max(n, 1))()
    order = (ctypes.c_int * max(n, 1))()
    load = (ctypes.c_ulonglong * max(n_streams, 1))()
    _check(lib().pbkd_schedule_blocks(n, w, hb, n_streams, policy, sob, order, load))
    return list(sob)[:n], list(order)[:n], list(load)[:n_streams]


def kernel_kind_names() -> List[str]:
    L = lib()
    return [L.pbkd_kernel_kind_name(i).decode() for i in range(L.pbkd_kernel_kinds())]


def _params_array(params: Sequence[Sequence[np.ndarray]]):
    flat = []
    for lp in params:
        for q in lp:
            a = np.ascontiguousarray(q, dtype=np.float32)
            flat.append(a)
    arr = (ctypes.POINTER(ctypes.c_float) * len(flat))(*[a.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) for a in flat])
    return arr, flat


class Block:
    """One distillation task on the GPU.  Owns a torch uint8 workspace tensor and the library handle."""

    def __init__(self, teacher, teacher_params, student, student_params, momentum: float = 0.9, loss_reduction: int = 0,
                 device: str = "cuda:0", stream=None, bn_decay: float = 0.99):
        import torch
        self.teacher, self.student = teacher, student
        self._ta, self._sa = make_arch(teacher), make_arch(student)
        st = lib().pbkd_arch_validate(ctypes.byref(self._ta), ctypes.byref(self._sa))
        _check(st)
        nbytes = lib().pbkd_block_workspace_bytes(ctypes.byref(self._ta), ctypes.byref(self._sa))
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        base = self.workspace.data_ptr()
        aligned = (base + 255) & ~255
        tp, keep_t = _params_array(teacher_params)
        sp, keep_s = _params_array(student_params)
        train = TrainDesc(momentum, loss_reduction, bn_decay)
        handle = ctypes.c_void_p()
        sptr = stream.cuda_stream if stream is not None else torch.cuda.current_stream().cuda_stream
        _check(lib().pbkd_block_create(ctypes.byref(self._ta), tp, ctypes.byref(self._sa), sp, ctypes.byref(train),
                                       ctypes.c_void_p(aligned), nbytes, ctypes.c_void_p(sptr), ctypes.byref(handle)))
        self.handle = handle
        self.workspace_bytes = nbytes

    def close(self):
        if getattr(self, "handle", None):
            lib().pbkd_block_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def _sptr(stream):
        import torch
        return ctypes.c_void_p(stream.cuda_stream if stream is not None else torch.cuda.current_stream().cuda_stream)

    def teacher_forward(self, x, target, stream=None):
        _check(lib().pbkd_teacher_forward(self.handle, ctypes.c_void_p(x.data_ptr()), ctypes.c_void_p(target.data_ptr()),
                                          self._sptr(stream)))

    def student_forward(self, x, out, stream=None):
        _check(lib().pbkd_student_forward(self.handle, ctypes.c_void_p(x.data_ptr()), ctypes.c_void_p(out.data_ptr()),
                                          self._sptr(stream)))

    def set_aux_stream(self, stream) -> None:
        """Second stream for the weight-gradient branch of the backward pass (None: off)."""
        self._aux = stream     # keep it alive
        _check(lib().pbkd_block_set_aux_stream(self.handle, ctypes.c_void_p(stream.cuda_stream if stream is not None else 0)))

    def set_graph_mode(self, on: bool) -> None:
        """Capture each step's launches into a HIP graph once and replay it (pbkd_block_set_graph_mode)."""
        _check(lib().pbkd_block_set_graph_mode(self.handle, int(bool(on))))

    def distill_step(self, x, target, lr: float, want_loss: bool = True, student_stream=None,
                     teacher_stream=None) -> Optional[float]:
        """Teacher forward into `target` on teacher_stream and the student step on student_stream, overlapped."""
        loss = ctypes.c_float()
        _check(lib().pbkd_distill_step(self.handle, ctypes.c_void_p(x.data_ptr()), ctypes.c_void_p(target.data_ptr()), lr,
                                       ctypes.byref(loss) if want_loss else None, self._sptr(student_stream),
                                       self._sptr(teacher_stream)))
        return loss.value if want_loss else None

    def student_step(self, x, target, lr: float, want_loss: bool = True, stream=None) -> Optional[float]:
        loss = ctypes.c_float()
        _check(lib().pbkd_student_step(self.handle, ctypes.c_void_p(x.data_ptr()), ctypes.c_void_p(target.data_ptr()), lr,
                                       ctypes.byref(loss) if want_loss else None, self._sptr(stream)))
        return loss.value if want_loss else None

    def last_loss(self) -> float:
        loss = ctypes.c_float()
        _check(lib().pbkd_block_last_loss(self.handle, ctypes.byref(loss)))
        return loss.value

    def flops(self, which: int) -> int:
        return lib().pbkd_block_flops(self.handle, which)

    def get_tensor(self, which: int, layer: int, slot: int, shape) -> np.ndarray:
        out = np.empty(shape, dtype=np.float32)
        _check(lib().pbkd_block_get_tensor(self.handle, which, layer, slot, out.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                           out.size))
        return out

    def set_tensor(self, which: int, layer: int, slot: int, value: np.ndarray):
        a = np.ascontiguousarray(value, dtype=np.float32)
        _check(lib().pbkd_block_set_tensor(self.handle, which, layer, slot, a.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                           a.size))

    def profile_enable(self, kinds: Optional[Sequence[str]], capacity: int):
        """kinds: kernel-kind names to time (None = all); capacity 0 switches timing off."""
        names = kernel_kind_names()
        mask = 0
        for i, nm in enumerate(names):
            if kinds is None or nm in kinds:
                mask |= 1 << i
        _check(lib().pbkd_block_profile_enable(self.handle, mask, capacity))

    def profile_read(self):
        """{kind name: (summed ms, launches)} of the timed launches since the last read."""
        n = lib().pbkd_kernel_kinds()
        ms = (ctypes.c_double * n)()
        cnt = (ctypes.c_int * n)()
        _check(lib().pbkd_block_profile_read(self.handle, n, ms, cnt))
        return {nm: (ms[i], cnt[i]) for i, nm in enumerate(kernel_kind_names()) if cnt[i]}

    def student_params(self) -> List[List[np.ndarray]]:
        from .workloads import param_shapes
        return [[self.get_tensor(STUDENT_PARAM, l, k, shp) for k, shp in enumerate(lp)]
                for l, lp in enumerate(param_shapes(self.student))]

    def student_grads(self) -> List[List[np.ndarray]]:
        from .workloads import param_shapes
        return [[self.get_tensor(STUDENT_GRAD, l, k, shp) for k, shp in enumerate(lp)]
                for l, lp in enumerate(param_shapes(self.student))]


def distill_step_all(blocks: Sequence[Block], xs, targets, lr: float, streams, stream_of_block, order, chain: bool,
                     teacher_stream=None):
    """One concurrent distillation step of all blocks (pbkd_distill_step_all).  xs / targets: torch tensors;
    streams: torch.cuda.Stream objects."""
    n = len(blocks)
    hb = (ctypes.c_void_p * n)(*[b.handle for b in blocks])
    xp = (ctypes.c_void_p * n)(*[x.data_ptr() for x in xs])
    tp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in targets])
    sp = (ctypes.c_void_p * len(streams))(*[s.cuda_stream for s in streams])
    sob = (ctypes.c_int * n)(*stream_of_block)
    od = (ctypes.c_int * n)(*order)
    ts = ctypes.c_void_p(teacher_stream.cuda_stream) if teacher_stream is not None else ctypes.c_void_p(0)
    _check(lib().pbkd_distill_step_all(n, hb, xp, tp, lr, len(streams), sp, sob, od, int(chain), ts))


def run_tasks_work_stealing(blocks: Sequence[Block], xs, targets, lr: float, steps: Sequence[int], streams,
                            queue_of_task: Sequence[int]):
    """pbkd_run_tasks_work_stealing: whole training tasks over streams with dynamic load balancing.
    Returns (ran_on, n_steals).  Blocks until every task has finished."""
    n = len(blocks)
    hb = (ctypes.c_void_p * n)(*[b.handle for b in blocks])
    xp = (ctypes.c_void_p * n)(*[x.data_ptr() for x in xs])
    tp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in targets])
    sp = (ctypes.c_void_p * len(streams))(*[s.cuda_stream for s in streams])
    st = (ctypes.c_int * n)(*steps)
    qt = (ctypes.c_int * n)(*queue_of_task)
    ran = (ctypes.c_int * n)()
    ns = ctypes.c_int()
    _check(lib().pbkd_run_tasks_work_stealing(n, hb, xp, tp, lr, st, len(streams), sp, qt, ran, ctypes.byref(ns)))
    return list(ran), ns.value


def network_forward(blocks: Sequence[Block], use_student: Sequence[int], x, outs, stream=None, bn_mode: int = 0) -> None:
    """pbkd_network_forward: the chain of blocks on x, block k by its student where use_student[k] is non-zero;
    bn_mode 0 = BatchNorm with batch statistics, 1 = with the running statistics (inference mode)."""
    n = len(blocks)
    hb = (ctypes.c_void_p * n)(*[b.handle for b in blocks])
    us = (ctypes.c_int * n)(*[int(u) for u in use_student])
    op = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
    _check(lib().pbkd_network_forward(n, hb, us, int(bn_mode), ctypes.c_void_p(x.data_ptr()), op, Block._sptr(stream)))


def select_blocks(blocks: Sequence[Block], x, teacher_outs, scratch_outs, threshold: float, stream=None, bn_mode: int = 0):
    """pbkd_select_blocks: returns (use_student, per-block feature error, error of the reassembled network)."""
    n = len(blocks)
    hb = (ctypes.c_void_p * n)(*[b.handle for b in blocks])
    tp = (ctypes.c_void_p * n)(*[o.data_ptr() for o in teacher_outs])
    sp = (ctypes.c_void_p * n)(*[o.data_ptr() for o in scratch_outs])
    use = (ctypes.c_int * n)()
    errs = (ctypes.c_double * n)()
    final = ctypes.c_double()
    _check(lib().pbkd_select_blocks(n, hb, int(bn_mode), ctypes.c_void_p(x.data_ptr()), tp, sp, ctypes.c_double(threshold),
                                    use, errs, ctypes.byref(final), Block._sptr(stream)))
    return list(use), list(errs), final.value


def feature_mse(block: Block, a, b, stream=None) -> float:
    """pbkd_feature_mse: mean squared difference of two device tensors (fp64 accumulation)."""
    out = ctypes.c_double()
    _check(lib().pbkd_feature_mse(block.handle, ctypes.c_void_p(a.data_ptr()), ctypes.c_void_p(b.data_ptr()), a.numel(),
                                  ctypes.byref(out), Block._sptr(stream)))
    return out.value


def feature_mse_noalloc(a, b, stream=None, n: Optional[int] = None) -> float:
    """pbkd_feature_mse_noalloc: the same figure with the library's static scratch array (no block, no allocation)."""
    out = ctypes.c_double()
    _check(lib().pbkd_feature_mse_noalloc(ctypes.c_void_p(a.data_ptr()), ctypes.c_void_p(b.data_ptr()),
                                          a.numel() if n is None else n, ctypes.byref(out), Block._sptr(stream)))
    return out.value


# ------------------------------------------------------------------------------------------------ sequence operators
# Root-mean-square norm, gated recurrence, embedding, vocabulary loss, distillation from top logits and AdamW (include/pbkd.h has the formulas).  All tensors are torch tensors on
# the current GPU, outputs too: nothing is allocated by a call.  A descriptor is packed with struct (native alignment, the C struct's
# field order): a call of a few microseconds on the GPU should not wait for a ctypes structure's.
F32, BF16, F16, E4M3 = range(4)
I32, I64 = 8, 9
_RMSNORM = struct.Struct("@q3if6P4q")
_RMSNORM_GRAD = struct.Struct("@q2if6P4qPN")
_RECURRENCE = struct.Struct("@2iqi8P8qPNPN")
_RECURRENCE_GRAD = struct.Struct("@2iqi12P14qPNPN")
_EMBED = struct.Struct("@q4if3P2q")
_EMBED_GRAD = struct.Struct("@q4ifi3P2qPN")
_HEAD_LOSS = struct.Struct("@q4i8P4qPN")
_TOPK_DISTILL = struct.Struct("@q5if6P2q")
_ADAMW_ARGS = struct.Struct("@5dqiI")
_ADAMW_TENSOR = np.dtype([("n", "i8"), ("first", "i8"), ("param_dtype", "i4"), ("grad_dtype", "i4"), ("weight_decay", "f4"), ("param", "u8"), ("grad", "u8"),
                          ("m", "u8"), ("v", "u8"), ("m_scale", "u8"), ("v_scale", "u8"), ("copy", "u8")], align=True)
_torch = _current_device = None       # set with the types by _types(), at the first call that needs them
_CODES, _INDEX, _FP8, _FP32, _INT32 = {}, {}, None, None, None


def _types():
    """torch and its types by the library's numbers; the library is loaded (and torch with it) on the way."""
    global _torch, _current_device, _CODES, _INDEX, _FP8, _FP32, _INT32
    import torch
    _CODES, _INDEX = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}, {torch.int32: I32, torch.int64: I64}
    _FP8, _FP32, _INT32, _torch, _current_device = torch.float8_e4m3fn, torch.float32, torch.int32, torch, torch.cuda.current_device
    return lib()


def _missing(name: str):
    raise PbkdError(EINVAL, f"{name} is missing")


def _first(t, name: str):
    """(library, type's number, type, shape, GPU) of a call's first tensor, which must lie on the current GPU: the kernels are launched
    there."""
    L = _lib if _torch is not None and _lib is not None else _types()
    if t is None:
        _missing(name)
    dtype, dev = t.dtype, t.get_device()
    code = _CODES.get(dtype)
    if code is None:
        raise PbkdError(EINVAL, f"{name} must be float32, bfloat16 or float16, not {dtype}")
    if dev < 0 or dev != _current_device():
        raise PbkdError(EINVAL, f"{name} must lie on the current GPU, not on {t.device}")
    return L, code, dtype, t.shape, dev


def _stream(stream) -> int:
    return stream.cuda_stream if stream is not None else _torch.cuda.current_stream().cuda_stream


def _same(t, dtype, shape, dev: int, name: str) -> int:
    """Address of t, a tensor of this type and shape on GPU dev."""
    if t is None:
        _missing(name)
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        raise PbkdError(ESHAPE, f"{name} must be a {dtype} tensor of {tuple(shape)} on the same GPU, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _dense(t, shape, dtype, dev: int, name: str) -> int:
    """Address of t, a contiguous tensor of this shape and type on GPU dev; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise PbkdError(ESHAPE, f"{name} must be a contiguous {dtype} tensor of {tuple(shape)} on the same GPU, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _bytes(t, dev: int, name: str):
    """(address, bytes) of a workspace."""
    if t is None:
        return 0, 0
    if t.get_device() != dev or not t.is_contiguous():
        raise PbkdError(EINVAL, f"{name} must be a contiguous tensor on the same GPU")
    return t.data_ptr(), t.nbytes


def _row_stride(t, d: int, name: str) -> int:
    """Elements between the rows of t, whose last dimension are the rows: two dimensions with any stride, or more that are contiguous."""
    s = t.stride()
    if len(s) == 2 and (s[1] == 1 or d == 1):
        return s[0]
    if t.is_contiguous():
        return d
    raise PbkdError(EINVAL, f"{name} must be contiguous, or have two dimensions with contiguous rows")


def rmsnorm_workspace_bytes(rows: int, d: int) -> int:
    return lib().pbkd_rmsnorm_workspace_bytes(rows, d)


def rmsnorm_forward(x, weight, y, residual=None, total=None, scale=None, eps: float = 1e-6, stream=None) -> None:
    """pbkd_rmsnorm_forward: y <- norm(x + residual) * weight over the last dimension, total <- x + residual.
    y: like x, or float8_e4m3fn with scale [rows] float32."""
    L, code, dt, shape, dev = _first(x, "x")
    d = shape[-1] if shape else 0
    if d == 0:
        raise PbkdError(ESHAPE, "x has no elements in a row")
    rows = x.numel() // d
    if y is None:
        _missing("y")
    eight = y.dtype is _FP8
    if eight and (y.shape != shape or y.get_device() != dev):
        raise PbkdError(ESHAPE, f"y must have x's shape {tuple(x.shape)} and lie on its GPU")
    if scale is not None and not eight:
        raise PbkdError(EINVAL, "a scale goes with a float8_e4m3fn y only")
    _check(L.pbkd_rmsnorm_forward(_RMSNORM.pack(
        rows, d, code, E4M3 if eight else code, eps, x.data_ptr(), 0 if residual is None else _same(residual, dt, shape, dev, "residual"),
        _dense(weight, (d,), _FP32, dev, "weight"), 0 if total is None else _same(total, dt, shape, dev, "total"),
        y.data_ptr() if eight else _same(y, dt, shape, dev, "y"), _dense(scale, (rows,), _FP32, dev, "scale"), _row_stride(x, d, "x"),
        0 if residual is None else _row_stride(residual, d, "residual"), 0 if total is None else _row_stride(total, d, "total"), _row_stride(y, d, "y")),
        _stream(stream)))


def rmsnorm_backward(total, weight, dy, dx, dweight, workspace, dtotal=None, eps: float = 1e-6, stream=None) -> None:
    """pbkd_rmsnorm_backward: dx and dweight from the sum as stored by the forward pass, dy and (optionally) the gradient that
    arrives at the sum.  workspace: a tensor of rmsnorm_workspace_bytes(rows, d) bytes."""
    L, code, dt, shape, dev = _first(total, "total")
    d = shape[-1] if shape else 0
    if d == 0:
        raise PbkdError(ESHAPE, "total has no elements in a row")
    wp, wn = _bytes(workspace, dev, "workspace")
    _check(L.pbkd_rmsnorm_backward(_RMSNORM_GRAD.pack(
        total.numel() // d, d, code, eps, total.data_ptr(), _same(dy, dt, shape, dev, "dy"), 0 if dtotal is None else _same(dtotal, dt, shape, dev, "dtotal"),
        _dense(weight, (d,), _FP32, dev, "weight"), _same(dx, dt, shape, dev, "dx"), _dense(dweight, (d,), _FP32, dev, "dweight"),
        _row_stride(total, d, "total"), _row_stride(dy, d, "dy"), 0 if dtotal is None else _row_stride(dtotal, d, "dtotal"), _row_stride(dx, d, "dx"), wp, wn),
        _stream(stream)))


def recurrence_saved_bytes(batch: int, length: int, channels: int) -> int:
    return lib().pbkd_recurrence_saved_bytes(batch, length, channels)


def recurrence_workspace_bytes(batch: int, length: int, channels: int) -> int:
    return lib().pbkd_recurrence_workspace_bytes(batch, length, channels)


def _tokens(t, name: str):
    """(batch stride, token stride) of t [batch, len, channels]."""
    b, s, c = t.stride()
    if c != 1 and t.shape[2] > 1:
        raise PbkdError(EINVAL, f"{name}'s channels must be contiguous")
    return b, s


def _sequence_shape(shape):
    if len(shape) != 3 or shape[2] == 0:
        raise PbkdError(ESHAPE, f"u must be [batch, len, channels], not {tuple(shape)}")
    return shape


def recurrence_forward(u, gate, y, out_gate=None, bias=None, lengths=None, state=None, state_out=None, saved=None, workspace=None, stream=None) -> None:
    """pbkd_recurrence_forward on [batch, len, channels] tensors: y, and the last state in state_out.  saved: a tensor of
    recurrence_saved_bytes() for the backward pass; workspace: one of recurrence_workspace_bytes()."""
    L, code, dt, shape, dev = _first(u, "u")
    b, t, d = _sequence_shape(shape)
    f32 = _FP32
    sp, sn = _bytes(saved, dev, "saved")
    wp, wn = _bytes(workspace, dev, "workspace")
    _check(L.pbkd_recurrence_forward(_RECURRENCE.pack(
        b, d, t, code, u.data_ptr(), _same(gate, dt, shape, dev, "gate"), 0 if out_gate is None else _same(out_gate, dt, shape, dev, "out_gate"),
        _dense(bias, (d,), f32, dev, "bias"), _dense(lengths, (b,), _INT32, dev, "lengths"), _dense(state, (b, d), f32, dev, "state"),
        _dense(state_out, (b, d), f32, dev, "state_out"), _same(y, dt, shape, dev, "y"), *_tokens(u, "u"), *_tokens(gate, "gate"),
        *((0, 0) if out_gate is None else _tokens(out_gate, "out_gate")), *_tokens(y, "y"), sp, sn, wp, wn), _stream(stream)))


def recurrence_backward(u, gate, dy, saved, du, dgate, out_gate=None, dout_gate=None, bias=None, dbias=None, lengths=None, dstate_out=None, dstate=None,
                        workspace=None, stream=None) -> None:
    """pbkd_recurrence_backward: the gradients of recurrence_forward's inputs from dy and what it saved."""
    L, code, dt, shape, dev = _first(u, "u")
    b, t, d = _sequence_shape(shape)
    f32 = _FP32
    sp, sn = _bytes(saved, dev, "saved")
    wp, wn = _bytes(workspace, dev, "workspace")
    none = (0, 0)
    _check(L.pbkd_recurrence_backward(_RECURRENCE_GRAD.pack(
        b, d, t, code, u.data_ptr(), _same(gate, dt, shape, dev, "gate"), 0 if out_gate is None else _same(out_gate, dt, shape, dev, "out_gate"), _same(dy, dt, shape, dev, "dy"),
        _dense(bias, (d,), f32, dev, "bias"), _dense(lengths, (b,), _INT32, dev, "lengths"), _dense(dstate_out, (b, d), f32, dev, "dstate_out"),
        _same(du, dt, shape, dev, "du"), _same(dgate, dt, shape, dev, "dgate"), 0 if dout_gate is None else _same(dout_gate, dt, shape, dev, "dout_gate"),
        _dense(dbias, (d,), f32, dev, "dbias"), _dense(dstate, (b, d), f32, dev, "dstate"), *_tokens(u, "u"), *_tokens(gate, "gate"),
        *(none if out_gate is None else _tokens(out_gate, "out_gate")), *_tokens(dy, "dy"), *_tokens(du, "du"), *_tokens(dgate, "dgate"),
        *(none if dout_gate is None else _tokens(dout_gate, "dout_gate")), sp, sn, wp, wn), _stream(stream)))


def recurrence_step(u, gate, state, y, out_gate=None, bias=None, active=None, state_out=None, stream=None) -> None:
    """pbkd_recurrence_step: one token of each sequence, [batch, channels] rows with any stride; state [batch, channels] float32 is
    updated in place (or goes to state_out).  active: int32 [batch], 0 for idle rows."""
    L, code, dt, shape, dev = _first(u, "u")
    if len(shape) != 2 or shape[1] == 0:
        raise PbkdError(ESHAPE, f"u must be [batch, channels], not {tuple(shape)}")
    f32, (b, d) = _FP32, shape
    sp = _dense(state, (b, d), f32, dev, "state")
    _check(L.pbkd_recurrence_step(_RECURRENCE.pack(
        b, d, 1, code, u.data_ptr(), _same(gate, dt, shape, dev, "gate"), 0 if out_gate is None else _same(out_gate, dt, shape, dev, "out_gate"),
        _dense(bias, (d,), f32, dev, "bias"), _dense(active, (b,), _INT32, dev, "active"), sp, sp if state_out is None else _dense(state_out, (b, d), f32, dev, "state_out"),
        _same(y, dt, shape, dev, "y"), _row_stride(u, d, "u"), 0, _row_stride(gate, d, "gate"), 0, 0 if out_gate is None else _row_stride(out_gate, d, "out_gate"), 0,
        _row_stride(y, d, "y"), 0, 0, 0, 0, 0), _stream(stream)))


def _indices(t, shape, dev: int, name: str):
    """(address, type's number) of t, a contiguous tensor of 32- or 64-bit integers of this shape on GPU dev."""
    if t is None:
        _missing(name)
    code = _INDEX.get(t.dtype)
    if code is None or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise PbkdError(ESHAPE, f"{name} must be a contiguous int32 or int64 tensor of {tuple(shape)} on the same GPU, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr(), code


def _table(shape, name: str):
    """(rows, columns) of a matrix."""
    if len(shape) != 2 or not shape[0] or not shape[1]:
        raise PbkdError(ESHAPE, f"{name} must be a matrix with at least one row and column, not {tuple(shape)}")
    return shape


def embed_workspace_bytes(rows: int, vocab: int, d: int) -> int:
    return lib().pbkd_embed_workspace_bytes(rows, vocab, d)


def embed_forward(tokens, weight, y, scale: float = 1.0, stream=None) -> None:
    """pbkd_embed_forward: y[..., :] <- scale * weight[tokens[...]] for tokens of any shape (int32 or int64), 0 for tokens outside
    0..vocab-1.  weight [vocab, d], y [*tokens.shape, d] of weight's type."""
    L, code, dt, shape, dev = _first(weight, "weight")
    vocab, d = _table(shape, "weight")
    if tokens is None or y is None:
        _missing("tokens" if tokens is None else "y")
    index, at, out = _INDEX.get(tokens.dtype), tokens.shape, y.shape
    if index is None or tokens.get_device() != dev or not tokens.is_contiguous():
        _indices(tokens, at, dev, "tokens")
    # shapes number by number where they are the usual ones: this call is made for one token at a time
    if y.dtype is not dt or y.get_device() != dev or not (len(out) == 2 and len(at) == 1 and out[1] == d and out[0] == at[0] or out == (*at, d)):
        raise PbkdError(ESHAPE, f"y must be a {dt} tensor of {(*at, d)} on the same GPU, not {y.dtype} {tuple(out)} on {y.device}")
    _check(L.pbkd_embed_forward(_EMBED.pack(at[0] if len(at) == 1 else tokens.numel(), vocab, d, code, index, scale, tokens.data_ptr(), weight.data_ptr(), y.data_ptr(),
                                            _row_stride(weight, d, "weight"), _row_stride(y, d, "y")), _stream(stream)))


def embed_backward(tokens, dy, dweight, workspace, scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """pbkd_embed_backward: dweight[v] <- scale * (sum of dy where tokens == v), added to what is there with accumulate (rows whose token
    does not occur then stay as they are).  workspace: a tensor of embed_workspace_bytes(tokens.numel(), vocab, d) bytes."""
    L, code, dt, shape, dev = _first(dweight, "dweight")
    vocab, d = _table(shape, "dweight")
    if tokens is None:
        _missing("tokens")
    tp, index = _indices(tokens, tokens.shape, dev, "tokens")
    wp, wn = _bytes(workspace, dev, "workspace")
    _check(L.pbkd_embed_backward(_EMBED_GRAD.pack(tokens.numel(), vocab, d, code, index, scale, bool(accumulate), tp, _same(dy, dt, (*tokens.shape, d), dev, "dy"),
                                                  dweight.data_ptr(), _row_stride(dy, d, "dy"), _row_stride(dweight, d, "dweight"), wp, wn), _stream(stream)))


def head_loss_workspace_bytes(rows: int, vocab: int, d: int, dtype, gradients: bool) -> int:
    """Bytes of workspace for head_loss on tensors of this torch type; with gradients or for losses only."""
    L = lib() if _torch is not None else _types()
    if dtype not in _CODES:
        raise PbkdError(EINVAL, f"h must be float32, bfloat16 or float16, not {dtype}")
    return L.pbkd_head_loss_workspace_bytes(rows, vocab, d, _CODES[dtype], bool(gradients))


def head_loss(h, weight, labels, loss, workspace, lse=None, row_weight=None, dh=None, dweight=None, stream=None) -> None:
    """pbkd_head_loss: loss [rows] float32 <- softmax cross entropy of h weight^T against labels, without keeping the logits; labels
    outside 0..vocab-1 are ignored.  h [..., d], weight [vocab, d], labels [...] int32 or int64.  lse [rows]: the logits' log-sums.  dh and
    dweight (like h and weight, or these themselves): the gradients of (row_weight * loss).sum().  workspace: a tensor of head_loss_workspace_bytes(...) bytes."""
    L, code, dt, shape, dev = _first(h, "h")
    if weight is None:
        _missing("weight")
    vocab, d = _table(weight.shape, "weight")
    if not shape or shape[-1] != d:
        raise PbkdError(ESHAPE, f"rows of h must have weight's {d} elements, not {tuple(shape)}")
    rows = h.numel() // d
    lp, index = _indices(labels, shape[:-1], dev, "labels")
    wp, wn = _bytes(workspace, dev, "workspace")
    _check(L.pbkd_head_loss(_HEAD_LOSS.pack(
        rows, vocab, d, code, index, h.data_ptr(), _same(weight, dt, weight.shape, dev, "weight"), lp, _dense(row_weight, (rows,), _FP32, dev, "row_weight"),
        _dense(loss, (rows,), _FP32, dev, "loss"), _dense(lse, (rows,), _FP32, dev, "lse"), 0 if dh is None else _same(dh, dt, shape, dev, "dh"),
        0 if dweight is None else _same(dweight, dt, weight.shape, dev, "dweight"), _row_stride(h, d, "h"), _row_stride(weight, d, "weight"),
        0 if dh is None else _row_stride(dh, d, "dh"), 0 if dweight is None else _row_stride(dweight, d, "dweight"), wp, wn), _stream(stream)))


def topk_distill(logits, teacher, at, loss, temperature: float = 1.0, row_weight=None, dlogits=None, stream=None) -> None:
    """pbkd_topk_distill: loss [rows] float32 <- T^2 KL(softmax(teacher / T) || softmax(logits / T)), the teacher known at the places `at` only
    (int32 or int64, like teacher [..., top]; a place outside 0..vocab-1 or a logit of -inf is not known).  logits [..., vocab].  dlogits
    (like logits, or logits itself): the gradient of (row_weight * loss).sum()."""
    L, code, dt, shape, dev = _first(logits, "logits")
    vocab = shape[-1] if shape else 0
    if vocab == 0:
        raise PbkdError(ESHAPE, "logits has no elements in a row")
    if teacher is None:
        _missing("teacher")
    known, flat = teacher.shape, len(shape) == 2
    rows = shape[0] if flat else logits.numel() // vocab
    if not known or not (flat and len(known) == 2 and known[0] == rows or known[:-1] == shape[:-1]) or not known[-1]:
        raise PbkdError(ESHAPE, f"teacher must have logits' shape {tuple(shape)} but for the last dimension, not {tuple(known)}")
    tcode = _CODES.get(teacher.dtype)
    if tcode is None:
        raise PbkdError(EINVAL, f"teacher must be float32, bfloat16 or float16, not {teacher.dtype}")
    ap, index = _indices(at, known, dev, "at")
    each = (rows,)
    _check(L.pbkd_topk_distill(_TOPK_DISTILL.pack(
        rows, vocab, known[-1], code, tcode, index, temperature, logits.data_ptr(), _dense(teacher, known, teacher.dtype, dev, "teacher"), ap,
        0 if row_weight is None else _dense(row_weight, each, _FP32, dev, "row_weight"), _dense(loss, each, _FP32, dev, "loss"), 0 if dlogits is None else _same(dlogits, dt, shape, dev, "dlogits"),
        _row_stride(logits, vocab, "logits"), 0 if dlogits is None else _row_stride(dlogits, vocab, "dlogits")), _stream(stream)))


class AdamW:
    """pbkd_adamw_step over a list of parameters (float32 or bfloat16, contiguous, updated in place), states in 32 or 8 bits.

    states: per parameter (m, v), or (m, v, m_scale, v_scale) for 8 bits, flat tensors as the header describes them; None: zeros,
    allocated here (the constructor then waits for its stream once, so that any stream may step).  copies: bfloat16 tensors
    that receive the new parameters.  weight_decay: one number, or one for each parameter.  steps: how many were made already.

    params, states and copies are lists of this object.  Each step goes to where their tensors lie then, so data or tensors may be
    exchanged between steps; what is no longer of its first type and size is refused."""

    def __init__(self, params, state_bits: int = 32, states=None, copies=None, weight_decay=0.0, betas=(0.9, 0.999), eps: float = 1e-8, steps: int = 0):
        import torch
        if state_bits not in (32, 8):
            raise PbkdError(EINVAL, "state_bits must be 32 or 8")
        self.params, self.copies, self.state_bits, self.betas, self.eps, self.steps = list(params), copies, state_bits, betas, eps, steps
        n = len(self.params)
        decays = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        for name, given in (("states", states), ("copies", copies), ("weight_decay", decays)):
            if given is not None and len(given) != n:
                raise PbkdError(ESHAPE, f"{len(given)} {name} for {n} parameters")
        _types()
        self._dev = _first(self.params[0], "a parameter")[4] if n else -1
        self._table = t = np.zeros(n, _ADAMW_TENSOR)
        self._kind = kind = (torch.float32, torch.float32) if state_bits == 32 else (torch.float8_e4m3fn, torch.float8_e4m3fn, torch.float32, torch.float32)
        self._sizes, self._shapes, self._dtypes, made = [p.numel() for p in self.params], [p.shape for p in self.params], [p.dtype for p in self.params], []
        blocks, codes = [-(-k // 256) for k in self._sizes], [_CODES.get(y) for y in self._dtypes]
        self._state_sizes = [(k, k, m, m)[:len(kind)] for k, m in zip(self._sizes, blocks)]
        for i, p in enumerate(self.params):
            if codes[i] not in (F32, BF16):
                raise PbkdError(EINVAL, f"parameter {i} must be float32 or bfloat16, not {p.dtype}")
            if states is None:
                made.append(tuple(torch.zeros(k, dtype=torch.uint8 if y == torch.float8_e4m3fn else y, device=p.device).view(y) for k, y in zip(self._state_sizes[i], kind)))
        t["first"], t["param_dtype"], t["weight_decay"] = [256 * k for k in accumulate([0, *blocks])][:n], codes, decays
        self.states = made if states is None else list(states)
        self._address = t.ctypes.data
        self._n, self._grad_dtype, self._grad, self._types, self._at = t["n"], t["grad_dtype"], t["grad"], None, None
        self._take_addresses()
        if states is None and n:
            torch.cuda.current_stream().synchronize()

    def _where(self):
        """Addresses of all parameters, states and copies, as one list."""
        at = [*map(_torch.Tensor.data_ptr, chain(self.params, chain.from_iterable(self.states)))]
        return at if self.copies is None else at + [0 if c is None else c.data_ptr() for c in self.copies]

    def _take_addresses(self) -> None:
        """Looks at every tensor, which must be of the type and size it had at first, and writes its address into the table."""
        n, names = len(self._sizes), ("m", "v", "m_scale", "v_scale")
        for name, given in (("parameters", self.params), ("states", self.states), ("copies", self.copies)):
            if given is not None and len(given) != n:
                raise PbkdError(ESHAPE, f"{len(given)} {name}, {n} are needed")
        dev, kind, rows = self._dev, self._kind, []
        for i, (p, s) in enumerate(zip(self.params, self.states)):
            if len(s) != len(kind):
                raise PbkdError(ESHAPE, f"parameter {i}: {len(s)} state tensors, {len(kind)} are needed")
            name = f"state of parameter {i}"
            rows.append((_dense(p, self._shapes[i], self._dtypes[i], dev, f"parameter {i}"), *[_dense(x, (k,), y, dev, name) for x, k, y in zip(s, self._state_sizes[i], kind)],
                         _dense(self.copies[i], self._shapes[i], _torch.bfloat16, dev, f"copy of parameter {i}") if self.copies is not None else 0))
        for k, v in zip(("param", *names[:len(kind)], "copy"), zip(*rows)):
            self._table[k] = v
        self._seen = self._where()

    def step(self, grads, lr: float, grad_scale: float = 1.0, seed: Optional[int] = None, stream=None) -> None:
        """One step with these gradients (one for each parameter, contiguous; None: the parameter and its states stay as they are).
        seed: of the random roundings; None: the number of the step.  Refused while the stream is captured: a graph would repeat this
        very step, its bias corrections and random numbers with it."""
        dev, sizes = self._dev, self._sizes
        if len(grads) != len(sizes):
            raise PbkdError(ESHAPE, f"{len(grads)} gradients for {len(sizes)} parameters")
        if dev >= 0 and dev != _current_device():
            raise PbkdError(EINVAL, "the parameters must lie on the current GPU")
        if self._where() != self._seen:
            self._take_addresses()
        t, live, want = _torch.Tensor, grads, sizes
        try:
            at = [*map(t.data_ptr, grads)]
        except TypeError:                            # some are None
            live, want = [g for g in grads if g is not None], [n for g, n in zip(grads, sizes) if g is not None]
            at = [0 if g is None else g.data_ptr() for g in grads]
        # data of a parameter may be viewed otherwise at the same place (a shorter view: its gradient tells)
        if [*map(t.numel, live)] != want or not all(map(t.is_contiguous, chain(live, self.params))) or set(map(t.get_device, live)) - {dev}:
            raise PbkdError(ESHAPE, "gradients and parameters must be contiguous, a gradient with its parameter's elements, on its GPU")
        types = [*map(t.dtype.__get__, live)]
        if types != self._types or live is not grads:
            if any(y not in _CODES for y in types):
                raise PbkdError(ESHAPE, "a gradient must be float32, bfloat16 or float16")
            codes = iter(types)
            self._grad_dtype[:] = [F32 if g is None else _CODES[next(codes)] for g in grads]
            self._n[:] = [0 if g is None else n for g, n in zip(grads, sizes)]
            self._types = types if live is grads else None
        if at != self._at:
            self._grad[:] = self._at = at
        number = self.steps + 1
        _check(_lib.pbkd_adamw_step(len(sizes), self._address, _ADAMW_ARGS.pack(lr, *self.betas, self.eps, grad_scale, number, self.state_bits,
                                                                               (number if seed is None else seed) & 0xFFFFFFFF), _stream(stream)))
        self.steps = number
