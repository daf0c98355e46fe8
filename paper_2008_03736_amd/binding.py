"""ctypes binding of ``libcrfinside.so`` (C ABI in ``include/crf_inside.h``).

Argument marshalling only: every step of the computation runs in the HIP
library.  PyTorch supplies device memory and the current HIP stream.

The raw entry points keep the C names (``crf_plan_create``, ``crf_inside_fwd``,
``crf_inside_bwd``, ``crf_inside_fwd_bwd``, ``crf_cky_decode``, ...) and take
integer device pointers.  :class:`Plan` wraps them for torch tensors.

There is no fallback: if the library is missing, :func:`load` raises.
"""
import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libcrfinside.so")

CRF_OK, CRF_EINVAL, CRF_ENOMEM, CRF_EHIP, CRF_EUNSUPPORTED = 0, 1, 2, 3, 4
CRF_MAX_LEN = 1023
CRF_MAX_LABELS = 4096
CRF_MAX_TREES = 64
CRF_MAX_ROW = 8192
ROW_BLOCK = 32          # entries of a packed row that share a power of two
CRF_FORCE_SPILL = 0x1
CRF_NO_TEAMS = 0x2

# Every function the C header declares, with its ctypes signature.
_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_F32 = ctypes.c_float
SIGNATURES = {
    "crf_plan_create": (ctypes.c_int, [ctypes.POINTER(_P), _P, _I32, _I32, _I32, ctypes.c_uint32]),
    "crf_plan_destroy": (ctypes.c_int, [_P]),
    "crf_plan_info": (ctypes.c_int, [_P, _P]),
    "crf_inside_fwd": (ctypes.c_int, [_P, _P, _P, _P]),
    "crf_inside_bwd": (ctypes.c_int, [_P, _P, _P, _P, _P]),
    "crf_inside_fwd_bwd": (ctypes.c_int, [_P, _P, _P, _P, _P, _P]),
    "crf_cky_decode": (ctypes.c_int, [_P, _P, _P, _P, _P]),
    "crf_inside_fwd_bwd_cky": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P, _P]),
    "crf_inside_fwd_bwd_cky_noalloc": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P, _P]),
    "crf_mbr_decode": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P]),
    "crf_gold_loss": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P]),
    "crf_cky_decode_labeled": (ctypes.c_int, [_P, _P, _P, _P, _P, _P]),
    "crf_label_spans": (ctypes.c_int, [_P, _P, _I32, _P, _P, _P]),
    "crf_biaffine_scores": (ctypes.c_int, [_P, _P, _P, _P, _I32, _I32, _I32, _P, _P]),
    "crf_tree_workspace": (ctypes.c_int, [_P, ctypes.POINTER(_I64)]),
    "crf_tree_logprobs": (ctypes.c_int, [_P, _P, _P, _I32, _P, _P, _P, _P, _I64, _P]),
    "crf_tree_logprobs_bwd": (ctypes.c_int, [_P, _P, _P, _I32, _P, _P, _P, _P]),
    "crf_policy_loss": (ctypes.c_int, [_P, _P, _P, _I32, _P, _P, _P, _P, _F32, _F32, _F32, _P, _P, _P, _P, _P, _I64,
                                       _P]),
    "crf_pack_rows": (ctypes.c_int, [_P, _P, _I32, _P, _P, _P]),
    "crf_unpack_rows": (ctypes.c_int, [_P, _P, _P, _I32, _P, _P]),
    "crf_biaffine_bwd_workspace": (ctypes.c_int, [_P, _I32, _I32, ctypes.POINTER(_I64)]),
    "crf_biaffine_bwd": (ctypes.c_int, [_P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P, _I64, _P]),
    "crf_biaffine_bwd_packed": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P, _I64, _P]),
    "crf_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "crf_last_error": (ctypes.c_char_p, []),
}


class PlanStats(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n1", ctypes.c_int32),
        ("num_labels", ctypes.c_int32),
        ("max_len", ctypes.c_int32),
        ("lds_count", ctypes.c_int32),
        ("spill_count", ctypes.c_int32),
        ("workspace_bytes", ctypes.c_int64),
        ("lds_bytes_inside", ctypes.c_int32),
        ("lds_bytes_cky", ctypes.c_int32),
        ("cky_spill_count", ctypes.c_int32),
        ("split_ws_count", ctypes.c_int32),
        ("workspace_users", ctypes.c_int32),
        ("fused_queue", ctypes.c_int32),
        ("mbr_fused", ctypes.c_int32),
    ]


class CrfError(RuntimeError):
    def __init__(self, status, where):
        lib = load()
        msg = lib.crf_last_error().decode() or lib.crf_status_string(status).decode()
        super().__init__(f"{where}: status {status} ({lib.crf_status_string(status).decode()}): {msg}")
        self.status = status


_lib = None


def load(path=LIB_PATH):
    """Load the HIP library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with __graft_entry__.build() "
                "(or python paper_2008_03736_amd/build.py); there is no fallback")
        lib = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _check(status, where):
    if status != CRF_OK:
        raise CrfError(status, where)


# --------------------------------------------------------------------------
# Raw entry points (C names, integer pointers).

def crf_plan_create(lengths_ptr, batch, n1, num_labels=1, flags=0):
    plan = _P()
    _check(load().crf_plan_create(ctypes.byref(plan), lengths_ptr, batch, n1, num_labels, flags),
           "crf_plan_create")
    return plan


def crf_plan_destroy(plan):
    _check(load().crf_plan_destroy(plan), "crf_plan_destroy")


def crf_plan_info(plan):
    st = PlanStats()
    _check(load().crf_plan_info(plan, ctypes.byref(st)), "crf_plan_info")
    return {k: getattr(st, k) for k, _ in PlanStats._fields_}


def crf_inside_fwd(plan, scores, logZ, stream):
    _check(load().crf_inside_fwd(plan, scores, logZ, stream), "crf_inside_fwd")


def crf_inside_bwd(plan, scores, grad_logZ, marginals, stream):
    _check(load().crf_inside_bwd(plan, scores, grad_logZ, marginals, stream), "crf_inside_bwd")


def crf_inside_fwd_bwd(plan, scores, grad_logZ, logZ, marginals, stream):
    _check(load().crf_inside_fwd_bwd(plan, scores, grad_logZ, logZ, marginals, stream),
           "crf_inside_fwd_bwd")


def crf_cky_decode(plan, scores, spans, best, stream):
    _check(load().crf_cky_decode(plan, scores, spans, best, stream), "crf_cky_decode")


def crf_inside_fwd_bwd_cky(plan, scores, grad_logZ, logZ, marginals, spans, best, stream):
    _check(load().crf_inside_fwd_bwd_cky(plan, scores, grad_logZ, logZ, marginals, spans, best,
                                         stream), "crf_inside_fwd_bwd_cky")


def crf_inside_fwd_bwd_cky_noalloc(plan, scores, grad_logZ, logZ, marginals, spans, best, stream):
    _check(load().crf_inside_fwd_bwd_cky_noalloc(plan, scores, grad_logZ, logZ, marginals, spans, best,
                                                 stream), "crf_inside_fwd_bwd_cky_noalloc")


def crf_mbr_decode(plan, scores, logZ, marginals, spans, best, stream):
    _check(load().crf_mbr_decode(plan, scores, logZ, marginals, spans, best, stream), "crf_mbr_decode")


def crf_gold_loss(plan, scores, gold_spans, grad_loss, loss, grad_scores, stream):
    _check(load().crf_gold_loss(plan, scores, gold_spans, grad_loss, loss, grad_scores, stream), "crf_gold_loss")


def crf_cky_decode_labeled(plan, scores, spans, labels, best, stream):
    _check(load().crf_cky_decode_labeled(plan, scores, spans, labels, best, stream), "crf_cky_decode_labeled")


def crf_label_spans(plan, label_scores, num_labels, spans, labels, stream):
    _check(load().crf_label_spans(plan, label_scores, num_labels, spans, labels, stream), "crf_label_spans")


def crf_biaffine_scores(plan, rl, rr, w, d, ldw, num_labels, scores, stream):
    _check(load().crf_biaffine_scores(plan, rl, rr, w, d, ldw, num_labels, scores, stream),
           "crf_biaffine_scores")


def crf_tree_workspace(plan):
    n = _I64()
    _check(load().crf_tree_workspace(plan, ctypes.byref(n)), "crf_tree_workspace")
    return n.value


def crf_tree_logprobs(plan, scores, trees, num_trees, counts, logp, logZ, workspace, workspace_bytes, stream):
    _check(load().crf_tree_logprobs(plan, scores, trees, num_trees, counts, logp, logZ, workspace, workspace_bytes,
                                    stream), "crf_tree_logprobs")


def crf_tree_logprobs_bwd(plan, scores, trees, num_trees, counts, grad_logp, grad_scores, stream):
    _check(load().crf_tree_logprobs_bwd(plan, scores, trees, num_trees, counts, grad_logp, grad_scores, stream),
           "crf_tree_logprobs_bwd")


def crf_policy_loss(plan, scores, trees, num_trees, counts, advantages, old_logp, ref_logp, clip_low, clip_high,
                    kl_coef, grad_loss, loss, logp, grad_scores, workspace, workspace_bytes, stream):
    _check(load().crf_policy_loss(plan, scores, trees, num_trees, counts, advantages, old_logp, ref_logp, clip_low,
                                  clip_high, kl_coef, grad_loss, loss, logp, grad_scores, workspace, workspace_bytes,
                                  stream), "crf_policy_loss")


def crf_pack_rows(plan, x, d, codes, scales, stream):
    _check(load().crf_pack_rows(plan, x, d, codes, scales, stream), "crf_pack_rows")


def crf_unpack_rows(plan, codes, scales, d, x, stream):
    _check(load().crf_unpack_rows(plan, codes, scales, d, x, stream), "crf_unpack_rows")


def crf_biaffine_bwd_workspace(plan, d, num_labels):
    n = _I64()
    _check(load().crf_biaffine_bwd_workspace(plan, d, num_labels, ctypes.byref(n)), "crf_biaffine_bwd_workspace")
    return n.value


def crf_biaffine_bwd(plan, rl, rr, w, d, ldw, num_labels, grad_scores, grad_rl, grad_rr, grad_w, workspace,
                     workspace_bytes, stream):
    _check(load().crf_biaffine_bwd(plan, rl, rr, w, d, ldw, num_labels, grad_scores, grad_rl, grad_rr, grad_w, workspace,
                                   workspace_bytes, stream), "crf_biaffine_bwd")


def crf_biaffine_bwd_packed(plan, rl_codes, rl_scales, rr_codes, rr_scales, w, d, ldw, num_labels, grad_scores, grad_rl,
                            grad_rr, grad_w, workspace, workspace_bytes, stream):
    _check(load().crf_biaffine_bwd_packed(plan, rl_codes, rl_scales, rr_codes, rr_scales, w, d, ldw, num_labels,
                                          grad_scores, grad_rl, grad_rr, grad_w, workspace, workspace_bytes, stream),
           "crf_biaffine_bwd_packed")


def crf_status_string(status):
    return load().crf_status_string(status).decode()


def crf_last_error():
    return load().crf_last_error().decode()


# --------------------------------------------------------------------------
# Torch-tensor wrapper.

def _stream_ptr(torch, device):
    return torch.cuda.current_stream(device).cuda_stream


class Plan:
    """A batch shape: sentence lengths, padded side N1, label count.

    Tensors passed to the methods must be contiguous float32 on the plan's
    device with shape ``[B, N1, N1]`` (``[B, N1, N1, L]`` when labelled).
    """

    def __init__(self, lengths, n1=None, num_labels=1, flags=0, device=None):
        import numpy as np
        import torch

        self._torch = torch
        lens = np.ascontiguousarray(np.asarray(lengths, dtype=np.int32))
        if lens.ndim != 1:
            raise ValueError("lengths must be 1-D")
        self.lengths = lens
        self.B = int(lens.shape[0])
        self.n1 = int(lens.max()) + 1 if n1 is None else int(n1)
        self.L = int(num_labels)
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self._handle = None
        with torch.cuda.device(self.device):
            self._handle = crf_plan_create(lens.ctypes.data, self.B, self.n1, self.L, flags)

    def close(self):
        if self._handle is not None:
            with self._torch.cuda.device(self.device):
                crf_plan_destroy(self._handle)
            self._handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def info(self):
        return crf_plan_info(self._handle)

    # shape / dtype checks (host side only)
    def _scores(self, scores):
        t = self._torch
        shape = (self.B, self.n1, self.n1) if self.L == 1 else (self.B, self.n1, self.n1, self.L)
        if tuple(scores.shape) != shape or scores.dtype != t.float32 or not scores.is_contiguous():
            raise ValueError(f"scores must be contiguous float32 {shape}, got "
                             f"{tuple(scores.shape)} {scores.dtype}")
        if scores.device != self.device:
            raise ValueError(f"scores on {scores.device}, plan on {self.device}")
        return scores.data_ptr()

    def _vec(self, v, name):
        """Pointer of a float32 [B] vector.  Outputs and inputs alike must be
        contiguous: a pointer into a temporary copy would let the kernel write
        results that the caller never sees."""
        if v is None:
            return None
        if tuple(v.shape) != (self.B,) or v.dtype != self._torch.float32 or v.device != self.device:
            raise ValueError(f"{name} must be float32 [{self.B}] on {self.device}")
        if not v.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return v.data_ptr()

    def _rewritten(self, x):
        """The library writes a buffer of the caller's: autograd refuses the
        backward pass of what it has kept of it before."""
        if x is not None and not x.is_inference():
            self._torch.autograd.graph.increment_version(x)

    def inside_fwd(self, scores, logZ=None):
        """log Z per sentence (float32 [B])."""
        t = self._torch
        sp = self._scores(scores)
        if logZ is None:
            logZ = t.empty(self.B, dtype=t.float32, device=self.device)
        crf_inside_fwd(self._handle, sp, self._vec(logZ, "logZ"), _stream_ptr(t, self.device))
        return logZ

    def inside_fwd_bwd(self, scores, grad_logZ=None, logZ=None, marginals=None):
        """(log Z, marginals).  Only valid cells of ``marginals`` are written;
        a fresh buffer is zero-filled first."""
        t = self._torch
        sp = self._scores(scores)
        if logZ is None:
            logZ = t.empty(self.B, dtype=t.float32, device=self.device)
        if marginals is None:
            marginals = t.zeros_like(scores)
        elif tuple(marginals.shape) != tuple(scores.shape) or not marginals.is_contiguous():
            raise ValueError("marginals must be a contiguous tensor shaped like scores")
        crf_inside_fwd_bwd(self._handle, sp, self._vec(grad_logZ, "grad_logZ"),
                           self._vec(logZ, "logZ"), marginals.data_ptr(),
                           _stream_ptr(t, self.device))
        return logZ, marginals

    def inside_bwd(self, scores, grad_logZ=None, marginals=None):
        t = self._torch
        sp = self._scores(scores)
        if marginals is None:
            marginals = t.zeros_like(scores)
        elif tuple(marginals.shape) != tuple(scores.shape) or not marginals.is_contiguous():
            raise ValueError("marginals must be a contiguous tensor shaped like scores")
        crf_inside_bwd(self._handle, sp, self._vec(grad_logZ, "grad_logZ"), marginals.data_ptr(),
                       _stream_ptr(t, self.device))
        return marginals

    def parse(self, scores, grad_logZ=None, logZ=None, marginals=None, spans=None, best=None):
        """inside_fwd_bwd and cky_decode in one launch:
        (logZ, marginals, spans, best)."""
        t = self._torch
        sp = self._scores(scores)
        R = 2 * (self.n1 - 1) - 1
        if logZ is None:
            logZ = t.empty(self.B, dtype=t.float32, device=self.device)
        if marginals is None:
            marginals = t.zeros_like(scores)
        elif tuple(marginals.shape) != tuple(scores.shape) or not marginals.is_contiguous():
            raise ValueError("marginals must be a contiguous tensor shaped like scores")
        if spans is None:
            spans = t.empty((self.B, R, 2), dtype=t.int32, device=self.device)
        elif tuple(spans.shape) != (self.B, R, 2) or spans.dtype != t.int32 or not spans.is_contiguous():
            raise ValueError(f"spans must be contiguous int32 [{self.B}, {R}, 2]")
        if best is None:
            best = t.empty(self.B, dtype=t.float32, device=self.device)
        self._rewritten(spans)
        crf_inside_fwd_bwd_cky(self._handle, sp, self._vec(grad_logZ, "grad_logZ"),
                               self._vec(logZ, "logZ"), marginals.data_ptr(), spans.data_ptr(),
                               self._vec(best, "best"), _stream_ptr(t, self.device))
        return logZ, marginals, spans, best

    def _spans_out(self, spans):
        t = self._torch
        R = 2 * (self.n1 - 1) - 1
        if spans is None:
            return t.empty((self.B, R, 2), dtype=t.int32, device=self.device)
        if tuple(spans.shape) != (self.B, R, 2) or spans.dtype != t.int32 or not spans.is_contiguous():
            raise ValueError(f"spans must be contiguous int32 [{self.B}, {R}, 2]")
        if spans.device != self.device:
            raise ValueError(f"spans on {spans.device}, plan on {self.device}")
        return spans

    def _labels_out(self, labels):
        t = self._torch
        R = 2 * (self.n1 - 1) - 1
        if labels is None:
            return t.empty((self.B, R), dtype=t.int32, device=self.device)
        if tuple(labels.shape) != (self.B, R) or labels.dtype != t.int32 or not labels.is_contiguous():
            raise ValueError(f"labels must be contiguous int32 [{self.B}, {R}]")
        if labels.device != self.device:
            raise ValueError(f"labels on {labels.device}, plan on {self.device}")
        return labels

    def mbr_decode(self, scores, logZ=None, marginals=None, spans=None, best=None):
        """MBR decoding (Sec. 3.3): (logZ, marginals, spans, best), the trees
        decoded by CKY over the marginals."""
        t = self._torch
        sp = self._scores(scores)
        if logZ is None:
            logZ = t.empty(self.B, dtype=t.float32, device=self.device)
        if marginals is None:
            marginals = t.zeros_like(scores)
        elif tuple(marginals.shape) != tuple(scores.shape) or not marginals.is_contiguous():
            raise ValueError("marginals must be a contiguous tensor shaped like scores")
        spans = self._spans_out(spans)
        if best is None:
            best = t.empty(self.B, dtype=t.float32, device=self.device)
        self._rewritten(spans)
        crf_mbr_decode(self._handle, sp, self._vec(logZ, "logZ"), marginals.data_ptr(), spans.data_ptr(),
                       self._vec(best, "best"), _stream_ptr(t, self.device))
        return logZ, marginals, spans, best

    def gold_loss(self, scores, gold_spans, grad_loss=None, loss=None, grad_scores=None):
        """Gold-tree CRF loss (Sec. 2.3, Eq. bracket-loss): (loss [B],
        gradient shaped like scores, valid cells only; a fresh buffer is
        zero-filled)."""
        t = self._torch
        sp = self._scores(scores)
        R = 2 * (self.n1 - 1) - 1
        if (tuple(gold_spans.shape) != (self.B, R, 2) or gold_spans.dtype != t.int32
                or not gold_spans.is_contiguous() or gold_spans.device != self.device):
            raise ValueError(f"gold_spans must be contiguous int32 [{self.B}, {R}, 2] on {self.device}")
        if loss is None:
            loss = t.empty(self.B, dtype=t.float32, device=self.device)
        if grad_scores is None:
            grad_scores = t.zeros_like(scores)
        elif tuple(grad_scores.shape) != tuple(scores.shape) or not grad_scores.is_contiguous():
            raise ValueError("grad_scores must be a contiguous tensor shaped like scores")
        crf_gold_loss(self._handle, sp, gold_spans.data_ptr(), self._vec(grad_loss, "grad_loss"),
                      self._vec(loss, "loss"), grad_scores.data_ptr(), _stream_ptr(t, self.device))
        return loss, grad_scores

    def cky_decode_labeled(self, scores, spans=None, labels=None, best=None):
        """One-stage labelled decoding (Sec. 4.2): (spans, labels, best)."""
        t = self._torch
        sp = self._scores(scores)
        spans = self._spans_out(spans)
        labels = self._labels_out(labels)
        if best is None:
            best = t.empty(self.B, dtype=t.float32, device=self.device)
        self._rewritten(spans)
        crf_cky_decode_labeled(self._handle, sp, spans.data_ptr(), labels.data_ptr(), self._vec(best, "best"),
                               _stream_ptr(t, self.device))
        return spans, labels, best

    def label_spans(self, label_scores, spans, labels=None):
        """Labelling stage (Sec. 2.1, Eq. label-argmax) of given trees:
        label_scores [B, N1, N1, L'] float32 (any L'), spans as cky_decode
        writes them; returns int32 [B, 2(N1-1)-1]."""
        t = self._torch
        if (label_scores.dim() != 4 or tuple(label_scores.shape[:3]) != (self.B, self.n1, self.n1)
                or label_scores.dtype != t.float32 or not label_scores.is_contiguous()
                or label_scores.device != self.device):
            raise ValueError(f"label_scores must be contiguous float32 [{self.B}, {self.n1}, {self.n1}, L]")
        spans = self._spans_out(spans)
        labels = self._labels_out(labels)
        crf_label_spans(self._handle, label_scores.data_ptr(), int(label_scores.shape[3]), spans.data_ptr(),
                        labels.data_ptr(), _stream_ptr(t, self.device))
        return labels

    def biaffine_scores(self, rl, rr, w, scores=None):
        """Span (or label) scores from boundary representations (Sec. 2.2,
        Eq. biaffine).  rl, rr: bf16 bit patterns as int16/uint16 tensors
        [B, N1, d]; w: [L, d, ldw] (W transposed, bias at index d).  Returns
        float32 [B, N1, N1] (L = 1) or [B, N1, N1, L]; a fresh buffer is
        NaN-filled, and only valid cells are written."""
        t = self._torch
        if rl.dim() != 3 or tuple(rl.shape[:2]) != (self.B, self.n1) or tuple(rr.shape) != tuple(rl.shape):
            raise ValueError(f"rl and rr must be [{self.B}, {self.n1}, d]")
        d = int(rl.shape[2])
        if w.dim() != 3 or int(w.shape[1]) != d:
            raise ValueError("w must be [L, d, ldw]")
        for x in (rl, rr, w):
            if x.dtype not in (t.int16, t.uint16) or not x.is_contiguous() or x.device != self.device:
                raise ValueError("rl, rr and w must be contiguous 16-bit tensors on the plan's device")
        L = int(w.shape[0])
        shape = (self.B, self.n1, self.n1) if L == 1 else (self.B, self.n1, self.n1, L)
        if scores is None:
            scores = t.full(shape, float("nan"), dtype=t.float32, device=self.device)
        elif tuple(scores.shape) != shape or scores.dtype != t.float32 or not scores.is_contiguous():
            raise ValueError(f"scores must be contiguous float32 {shape}")
        self._rewritten(scores)
        crf_biaffine_scores(self._handle, rl.data_ptr(), rr.data_ptr(), w.data_ptr(), d, int(w.shape[2]), L,
                            scores.data_ptr(), _stream_ptr(t, self.device))
        return scores

    def _tensor(self, x, name, shape, dtypes, optional=False):
        """Pointer of a contiguous tensor of the given shape on the plan's device."""
        if x is None and optional:
            return None
        if tuple(x.shape) != tuple(shape) or x.dtype not in dtypes:
            raise ValueError(f"{name} must be {' or '.join(str(t) for t in dtypes)} {tuple(shape)}, got "
                             f"{x.dtype} {tuple(x.shape)}")
        if x.device != self.device:
            raise ValueError(f"{name} on {x.device}, plan on {self.device}")
        if not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return x.data_ptr()

    def _trees(self, trees, counts):
        """(number of trees, pointers of trees and counts)."""
        t = self._torch
        if trees.dim() != 4:
            raise ValueError("trees must be [B, G, 2 (N1 - 1) - 1, 2]")
        G, R = int(trees.shape[1]), 2 * (self.n1 - 1) - 1
        return (G, self._tensor(trees, "trees", (self.B, G, R, 2), (t.int32,)),
                self._tensor(counts, "counts", (self.B,), (t.int32,), optional=True))

    def _workspace(self, size):
        return self._torch.empty(max(int(size), 1), dtype=self._torch.uint8, device=self.device)

    def _out(self, x, shape, dtype, zero=False):
        if x is not None:
            return x
        make = self._torch.zeros if zero else self._torch.empty
        return make(shape, dtype=dtype, device=self.device)

    def tree_logprobs(self, scores, trees, counts=None, logp=None, logZ=None):
        """Log-probabilities of G trees a sentence (Sec. 2.1, Eq. tree-prob):
        trees int32 [B, G, 2(N1-1)-1, 2] as cky_decode writes them, counts
        int32 [B] (how many of them are there; default all).  Returns
        (logp [B, G], logZ [B]); a fresh logp is 0 where no tree is there."""
        t = self._torch
        sp = self._scores(scores)
        G, tp, cp = self._trees(trees, counts)
        logp = self._out(logp, (self.B, G), t.float32, zero=counts is not None)
        logZ = self._out(logZ, (self.B,), t.float32)
        ws = self._workspace(crf_tree_workspace(self._handle))
        crf_tree_logprobs(self._handle, sp, tp, G, cp, self._tensor(logp, "logp", (self.B, G), (t.float32,)),
                          self._vec(logZ, "logZ"), ws.data_ptr(), ws.numel(), _stream_ptr(t, self.device))
        return logp, logZ

    def tree_logprobs_bwd(self, scores, trees, grad_logp, counts=None, grad_scores=None):
        """Gradient of sum(grad_logp * logp) with respect to the scores (valid
        cells only; a fresh buffer is zero-filled)."""
        t = self._torch
        sp = self._scores(scores)
        G, tp, cp = self._trees(trees, counts)
        up = self._tensor(grad_logp, "grad_logp", (self.B, G), (t.float32,))
        grad_scores = self._out(grad_scores, scores.shape, t.float32, zero=True)
        crf_tree_logprobs_bwd(self._handle, sp, tp, G, cp, up,
                              self._tensor(grad_scores, "grad_scores", scores.shape, (t.float32,)),
                              _stream_ptr(t, self.device))
        return grad_scores

    def policy_loss(self, scores, trees, advantages, old_logp, ref_logp=None, counts=None, clip_low=0.2, clip_high=0.2,
                    kl_coef=0.0, grad_loss=None, loss=None, logp=None, grad_scores=None):
        """Clipped policy loss of G trees a sentence with a KL term: (loss [B],
        logp [B, G], gradient shaped like scores).  advantages, old_logp and
        ref_logp (needed where kl_coef is not 0) are float32 [B, G]; a fresh
        gradient is zero-filled, a fresh logp 0 where no tree is there."""
        t = self._torch
        sp = self._scores(scores)
        G, tp, cp = self._trees(trees, counts)
        each = (self.B, G)
        ins = [self._tensor(x, name, each, (t.float32,), optional=name == "ref_logp")
               for x, name in ((advantages, "advantages"), (old_logp, "old_logp"), (ref_logp, "ref_logp"))]
        loss = self._out(loss, (self.B,), t.float32)
        logp = self._out(logp, each, t.float32, zero=counts is not None)
        grad_scores = self._out(grad_scores, scores.shape, t.float32, zero=True)
        ws = self._workspace(crf_tree_workspace(self._handle))
        crf_policy_loss(self._handle, sp, tp, G, cp, *ins, float(clip_low), float(clip_high), float(kl_coef),
                        self._vec(grad_loss, "grad_loss"), self._vec(loss, "loss"),
                        self._tensor(logp, "logp", each, (t.float32,)),
                        self._tensor(grad_scores, "grad_scores", scores.shape, (t.float32,)), ws.data_ptr(), ws.numel(),
                        _stream_ptr(t, self.device))
        return loss, logp, grad_scores

    def _bf16(self, x, name, shape):
        t = self._torch
        return self._tensor(x, name, shape, (t.bfloat16, t.int16, t.uint16))

    def _packed(self, codes, scales, d):
        wide = (d + ROW_BLOCK - 1) // ROW_BLOCK * ROW_BLOCK
        u8 = (self._torch.uint8,)
        return (self._tensor(codes, "codes", (self.B, self.n1, wide), u8),
                self._tensor(scales, "scales", (self.B, self.n1, wide // ROW_BLOCK), u8))

    def pack_rows(self, x, codes=None, scales=None):
        """Rows of bf16 activations [B, N1, d] in 8 bits: (codes uint8
        [B, N1, dc], e4m3 bit patterns, dc = d rounded up to a multiple of 32;
        scales uint8 [B, N1, dc/32], the exponent plus 127 of the power of two
        that 32 codes share).  Rows past a sentence's last fence post are left
        as they were (zero in fresh buffers)."""
        t = self._torch
        if x.dim() != 3:
            raise ValueError("x must be [B, N1, d]")
        d = int(x.shape[2])
        xp = self._bf16(x, "x", (self.B, self.n1, d))
        wide = (d + ROW_BLOCK - 1) // ROW_BLOCK * ROW_BLOCK
        codes = self._out(codes, (self.B, self.n1, wide), t.uint8, zero=True)
        scales = self._out(scales, (self.B, self.n1, wide // ROW_BLOCK), t.uint8, zero=True)
        crf_pack_rows(self._handle, xp, d, *self._packed(codes, scales, d), _stream_ptr(t, self.device))
        return codes, scales

    def unpack_rows(self, codes, scales, d, out=None):
        """The bf16 rows [B, N1, d] that packed ones stand for."""
        t = self._torch
        d = int(d)
        cp, sc = self._packed(codes, scales, d)
        out = self._out(out, (self.B, self.n1, d), t.bfloat16, zero=True)
        self._rewritten(out)
        crf_unpack_rows(self._handle, cp, sc, d, self._bf16(out, "out", (self.B, self.n1, d)),
                        _stream_ptr(t, self.device))
        return out

    def biaffine_bwd(self, rl, rr, w, grad_scores, grad_rl=None, grad_rr=None, grad_w=None, need=(True, True, True)):
        """Backward pass of biaffine_scores (Sec. 2.2, Eq. biaffine) from the
        gradient of its scores: (grad_rl bf16 [B, N1, d], grad_rr, grad_w
        float32 shaped like w).  rl and rr: bf16 (or its bit patterns)
        [B, N1, d], or both what pack_rows gave for them.  need: which of the
        three to compute (None in the place of the others); rows past a
        sentence and entries of grad_w past the bias are left as they were
        (zero in fresh buffers)."""
        t = self._torch
        if w.dim() != 3:
            raise ValueError("w must be [L, d, ldw]")
        L, d, ldw = (int(x) for x in w.shape)
        wp = self._bf16(w, "w", w.shape)
        rows = (self.B, self.n1, d)
        packed = isinstance(rl, (tuple, list))
        if packed != isinstance(rr, (tuple, list)):
            raise ValueError("rl and rr must both be rows or both be packed")
        ins = (*self._packed(*rl, d), *self._packed(*rr, d)) if packed else (self._bf16(rl, "rl", rows),
                                                                            self._bf16(rr, "rr", rows))
        shape = (self.B, self.n1, self.n1) if L == 1 else (self.B, self.n1, self.n1, L)
        gp = self._tensor(grad_scores, "grad_scores", shape, (t.float32,))
        out = [self._out(x, s, dt, zero=True) if want else None
               for x, s, dt, want in ((grad_rl, rows, t.bfloat16, need[0]), (grad_rr, rows, t.bfloat16, need[1]),
                                      (grad_w, tuple(w.shape), t.float32, need[2]))]
        types = ((t.bfloat16, t.int16, t.uint16),) * 2 + ((t.float32,),)
        ptrs = [self._tensor(x, name, s, dt, optional=True)
                for x, name, s, dt in zip(out, ("grad_rl", "grad_rr", "grad_w"), (rows, rows, w.shape), types)]
        ws = self._workspace(crf_biaffine_bwd_workspace(self._handle, d, L))
        call = crf_biaffine_bwd_packed if packed else crf_biaffine_bwd
        call(self._handle, *ins, wp, d, ldw, L, gp, *ptrs, ws.data_ptr(), ws.numel(), _stream_ptr(t, self.device))
        return tuple(out)

    def cky_decode(self, scores, spans=None, best=None):
        """(spans int32 [B, 2(N1-1)-1, 2] preorder padded with -1, best float32 [B])."""
        t = self._torch
        sp = self._scores(scores)
        R = 2 * (self.n1 - 1) - 1
        if spans is None:
            spans = t.empty((self.B, R, 2), dtype=t.int32, device=self.device)
        elif tuple(spans.shape) != (self.B, R, 2) or spans.dtype != t.int32 or not spans.is_contiguous():
            raise ValueError(f"spans must be contiguous int32 [{self.B}, {R}, 2]")
        if best is None:
            best = t.empty(self.B, dtype=t.float32, device=self.device)
        self._rewritten(spans)
        crf_cky_decode(self._handle, sp, spans.data_ptr(), self._vec(best, "best"),
                       _stream_ptr(t, self.device))
        return spans, best


def log_partition(scores, plan):
    """Differentiable log Z: backward returns the span marginals times the
    upstream gradient (Sec. 3.2, Eq. partial-derivative)."""
    import torch

    class _LogZ(torch.autograd.Function):
        @staticmethod
        def forward(ctx, s):
            ctx.save_for_backward(s)
            return plan.inside_fwd(s)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, g):
            (s,) = ctx.saved_tensors
            g = g.float().contiguous()   # held by this frame until the call has been enqueued
            return plan.inside_bwd(s, grad_logZ=g)

    return _LogZ.apply(scores)


def tree_log_prob(scores, trees, plan, counts=None):
    """Differentiable log-probabilities of given trees (Sec. 2.1,
    Eq. tree-prob), float32 [B, G]: backward returns, per sentence, the trees'
    upstream gradients on their spans less their sum times the marginals.
    scores, trees and counts are kept for it, not copied: after a change in
    place of one of them it raises."""
    import torch

    class _LogP(torch.autograd.Function):
        @staticmethod
        def forward(ctx, s, trees, counts):
            ctx.save_for_backward(s, trees, counts)
            return plan.tree_logprobs(s, trees, counts=counts)[0]

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, g):
            s, trees, counts = ctx.saved_tensors
            g = g.float().contiguous()   # held by this frame until the call has been enqueued
            return plan.tree_logprobs_bwd(s, trees, g, counts=counts), None, None

    return _LogP.apply(scores, trees, counts)


def policy_loss(scores, trees, advantages, old_logp, plan, ref_logp=None, counts=None, clip_low=0.2, clip_high=0.2,
                kl_coef=0.0):
    """Differentiable clipped policy loss, float32 [B] (Plan.policy_loss's
    arguments): the gradient is computed with the loss and kept."""
    import torch

    class _Policy(torch.autograd.Function):
        @staticmethod
        def forward(ctx, s):
            loss, _, grad = plan.policy_loss(s, trees, advantages, old_logp, ref_logp=ref_logp, counts=counts,
                                              clip_low=clip_low, clip_high=clip_high, kl_coef=kl_coef)
            ctx.save_for_backward(grad)
            return loss

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, g):
            (grad,) = ctx.saved_tensors
            return grad * g[:, None, None]

    return _Policy.apply(scores)


def biaffine(rl, rr, w, plan, held="bf16"):
    """Differentiable span (or label) scores from boundary representations
    (Sec. 2.2, Eq. biaffine): rl, rr bfloat16 [B, N1, d], w bfloat16 or float32
    [L, d, ldw]; cells that are no spans are 0.  A float32 w enters the products
    rounded to bfloat16 and gets its gradient in float32, as it is computed; a
    bfloat16 one gets it rounded.  held="8bit": the backward pass keeps the
    representations in 8 bits (Plan.pack_rows) and gives the gradients at the
    values those stand for."""
    import torch

    if held not in ("bf16", "8bit"):
        raise ValueError('held must be "bf16" or "8bit"')
    bf16 = (torch.bfloat16, torch.int16, torch.uint16)
    for x, name, types in ((rl, "rl", bf16), (rr, "rr", bf16), (w, "w", (*bf16, torch.float32))):
        if x.dtype not in types:
            raise ValueError(f"{name} must be bfloat16 (or its bit patterns; w also float32), got {x.dtype}")
    differentiable = torch.is_grad_enabled() and any(x.requires_grad for x in (rl, rr, w))

    class _Biaffine(torch.autograd.Function):
        @staticmethod
        def forward(ctx, rl, rr, w):
            L = w.shape[0]
            ctx.w_type = w.dtype
            if w.dtype == torch.float32:
                w = w.to(torch.bfloat16)
            shape = (plan.B, plan.n1, plan.n1) if L == 1 else (plan.B, plan.n1, plan.n1, L)
            scores = torch.zeros(shape, dtype=torch.float32, device=rl.device)
            plan.biaffine_scores(rl.view(torch.int16), rr.view(torch.int16), w.view(torch.int16), scores=scores)
            if differentiable:
                kept = (*plan.pack_rows(rl), *plan.pack_rows(rr)) if held == "8bit" else (rl, rr)
                ctx.save_for_backward(w, *kept)
            return scores

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, g):
            w, *kept = ctx.saved_tensors
            rl, rr = (kept[:2], kept[2:]) if held == "8bit" else kept
            g = g.float().contiguous()   # held by this frame until the call has been enqueued
            need = ctx.needs_input_grad
            if not any(need):
                return None, None, None
            grad_rl, grad_rr, grad_w = plan.biaffine_bwd(rl, rr, w, g, need=need)
            return grad_rl, grad_rr, None if grad_w is None else grad_w.to(ctx.w_type)

    return _Biaffine.apply(rl, rr, w)
