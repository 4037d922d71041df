"""Thin Python binding of the C ABI in ``include/signsgd.h``.

Argument marshalling only: every function takes torch tensors (device memory
and streams are torch's), checks dtype / device / contiguity, and passes raw
pointers and sizes to the function of the same name in ``libsignsgd_b200.so``.
All arithmetic of Algorithms 1-3 runs inside that library's CUDA kernels.
There is no fallback: if the library is missing or a call fails, an exception
is raised.
"""
from __future__ import annotations

import array
import contextlib
import ctypes
import os
import struct
from typing import NamedTuple, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsignsgd_b200.so")
MAX_WORKERS = 1024

_lib = None


class SignSGDError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: status %d (%s)" % (where, status, status_str(status)))


def lib() -> ctypes.CDLL:
    """Load the CUDA library (built by ``_build.build()``); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "%s not found: build it with `python -m paper_1802_04434_b200._build` "
            "(needs nvcc); there is no CPU fallback" % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    sz, f32, vp, ci = ctypes.c_size_t, ctypes.c_float, ctypes.c_void_p, ctypes.c_int
    i64, u32 = ctypes.c_int64, ctypes.c_uint
    L.ssgd_words.restype = sz
    L.ssgd_words.argtypes = [sz]
    L.ssgd_density_from_sums.restype = ctypes.c_double
    L.ssgd_density_from_sums.argtypes = [ctypes.c_double, ctypes.c_double, sz]
    L.ssgd_count_planes.restype = sz
    L.ssgd_count_planes.argtypes = [sz]
    L.ssgd_warmup_steps.restype = sz
    L.ssgd_warmup_steps.argtypes = [f32]
    L.ssgd_step_is_fused.restype = ci
    L.ssgd_step_is_fused.argtypes = [sz, sz, ci]
    L.ssgd_fp4_row_bytes.restype = sz
    L.ssgd_fp4_row_bytes.argtypes = [sz]
    L.ssgd_fp4_scale_bytes.restype = sz
    L.ssgd_fp4_scale_bytes.argtypes = [ci, sz, sz]
    L.ssgd_status_str.restype = ctypes.c_char_p
    L.ssgd_status_str.argtypes = [ci]
    L.ssgd_orthogonal_ws_bytes.restype = sz
    L.ssgd_orthogonal_ws_bytes.argtypes = [sz, sz, sz]
    sigs = {
        "ssgd_sign_pack": [vp, sz, sz, sz, vp, sz, vp],
        "ssgd_signum_momentum_pack": [vp, vp, sz, sz, sz, f32, vp, sz, vp],
        "ssgd_majority_vote": [vp, sz, sz, sz, vp, vp],
        "ssgd_sign_apply": [vp, vp, sz, f32, vp],
        "ssgd_signsgd_step": [vp, vp, vp, sz, sz, sz, f32, f32, vp, sz, vp, vp],
        "ssgd_signum_warmup_pack": [vp, vp, sz, sz, sz, f32, vp, sz, vp],
        "ssgd_signsgd_warmup_step": [vp, vp, vp, sz, sz, sz, f32, f32, vp, sz, vp, vp],
        "ssgd_vote_counts": [vp, sz, sz, sz, vp, sz, vp],
        "ssgd_sum_apply": [vp, vp, sz, sz, sz, f32, vp],
        "ssgd_ternary_pack": [vp, vp, sz, sz, sz, f32, f32, vp, vp, sz, vp],
        "ssgd_quorum_vote": [vp, vp, sz, sz, sz, sz, vp, vp, vp],
        "ssgd_ternary_apply": [vp, vp, vp, sz, f32, vp],
        "ssgd_welford_update": [vp, sz, vp, vp, sz, vp],
        "ssgd_density_sums": [vp, sz, ci, vp, vp],
        "ssgd_signsgd_step_host": [vp, vp, vp, sz, sz, sz, f32, f32, vp, vp, sz, vp, vp, vp],
        "ssgd_signsgd_step_noalloc": [vp, vp, vp, sz, sz, sz, f32, f32, vp],
        "ssgd_signum_momentum_pack_scatter": [vp, vp, sz, f32, vp, sz, sz, sz, vp],
        "ssgd_majority_vote_staged": [vp, sz, sz, sz, vp, vp, vp],
        "ssgd_majority_vote_staged_wait_selftest": [vp, sz, sz, sz, vp, vp, vp],
        "ssgd_table_size": [vp, sz, sz, vp, vp, vp],
        "ssgd_table_build": [vp, sz, sz, vp, sz],
        "ssgd_tensors_norm": [vp, sz, sz, ci, vp, vp, vp],
        "ssgd_tensors_clip": [vp, sz, sz, ci, f32, ci, vp, vp, vp],
        "ssgd_fp4_matmul_form": [sz, sz, sz, ci, sz, ci, vp],
        "ssgd_fp4_matmul_wait_selftest": [vp, vp, vp, vp, sz, sz, sz, ci, vp, ci, sz, vp, vp],
        "ssgd_tensors_clip_block": [ctypes.c_char_p],
        "ssgd_fp4_quantise_block": [ctypes.c_char_p],
        "ssgd_fp4_dequantise_block": [ctypes.c_char_p],
        "ssgd_fp4_matmul_block": [ctypes.c_char_p],
        "ssgd_fp4_quantise": [vp, ci, sz, sz, sz, ci, vp, vp, vp, vp, vp, vp, vp],
        "ssgd_fp4_dequantise": [vp, vp, vp, ci, sz, sz, vp, ci, sz, vp],
        "ssgd_fp4_matmul": [vp, vp, vp, vp, vp, vp, sz, sz, sz, ci, vp, ci, sz, vp, vp],
        "ssgd_xent_sizes": [sz, sz, sz, vp, vp],
        "ssgd_xent_forward": [vp, sz, vp, sz, ci, sz, sz, sz, vp, i64, vp, vp, vp, vp, vp, vp],
        "ssgd_xent_wait_selftest": [vp, sz, vp, sz, ci, sz, sz, sz, vp, i64, vp, vp, vp, vp, vp, vp],
        "ssgd_xent_backward": [vp, sz, vp, sz, ci, sz, sz, sz, vp, vp, vp, vp, sz, vp, sz, vp, ci, sz, vp, vp, vp],
        "ssgd_orthogonalise": [vp, ci, sz, sz, sz, sz, sz, vp, u32, ci, vp, ci, sz, sz, vp, vp, vp],
        "ssgd_orthogonal_wait_selftest": [vp, ci, sz, sz, vp, ci, vp, ci, vp, vp, vp],
        "ssgd_orthogonal_step": [vp, sz, sz, vp, ci, sz, sz, vp, sz, sz, sz, sz, sz, f32, f32, ci, vp, u32, ci, vp, vp, vp],
        "ssgd_xent_align": [vp, sz, sz, sz, vp, vp, sz, sz, sz, vp, sz, sz, vp],
        "ssgd_xent_align_block": [ctypes.c_char_p],
        "ssgd_xent_forward_block": [ctypes.c_char_p],
        "ssgd_xent_backward_block": [ctypes.c_char_p],
        "ssgd_orthogonalise_block": [ctypes.c_char_p],
        "ssgd_orthogonal_step_block": [ctypes.c_char_p],
    }
    for name, args in sigs.items():
        fn = getattr(L, name)
        fn.restype = ci
        fn.argtypes = args
    _lib = L
    return L


def status_str(status: int) -> str:
    return lib().ssgd_status_str(int(status)).decode()


def words(d: int) -> int:
    """ceil(d / 32)."""
    return int(lib().ssgd_words(d))


def _ptr(t: Optional[torch.Tensor], dtype, name: str, cuda: bool = True) -> Optional[int]:
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise TypeError("%s must be a torch tensor of dtype %s" % (name, dtype))
    if t.is_cuda != cuda:
        raise ValueError("%s must live in %s memory" % (name, "device" if cuda else "host"))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def _need(t: torch.Tensor, n: int, name: str) -> None:
    if t is None:
        raise ValueError("%s must be given" % name)
    if t.numel() < n:
        raise ValueError("%s holds %d elements, the call needs %d" % (name, t.numel(), n))


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_of(index: int) -> int:
    """The current stream of a device.  (torch.cuda.current_stream() makes a stream object; this only asks for its handle,
    2 us less a call.)"""
    return torch._C._cuda_getCurrentRawStream(index)


# torch.cuda.current_device() without its check that CUDA is up, which it is where a device tensor is at hand
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _on(index: int):
    """Makes a device current, where it is not: a launch goes to the current device, whatever stream and pointers it is given."""
    return contextlib.nullcontext() if index == _current_device() else torch.cuda.device(index)


def _need_device(index: int, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and t.get_device() != index:
            raise ValueError("%s must live in the memory of device %d, as the call's other tensors" % (name, index))


def _check(status: int, where: str) -> None:
    if status != 0:
        raise SignSGDError(status, where)


# words are stored in int32 tensors on the torch side (torch has no full uint32 support);
# the library sees the same 32 bits.
WORD_DTYPE = torch.int32


def sign_pack(g: torch.Tensor, M: int, d: int, ld: int, bits: torch.Tensor, ldw: int,
              stream=None) -> None:
    """Algorithm 1 / 3 worker side: bits[w] <- packed sign(g[w])."""
    _need(g, M * ld, "g"); _need(bits, M * ldw, "bits")
    _check(lib().ssgd_sign_pack(_ptr(g, torch.float32, "g"), M, d, ld,
                                _ptr(bits, WORD_DTYPE, "bits"), ldw, _stream(stream)),
           "ssgd_sign_pack")


def signum_momentum_pack(g: torch.Tensor, m: torch.Tensor, M: int, d: int, ld: int, beta: float,
                         bits: torch.Tensor, ldw: int, stream=None) -> None:
    """Algorithm 2 per worker, fused with packing: m updated in place, bits <- sign(m_new)."""
    _need(g, M * ld, "g"); _need(m, M * ld, "m"); _need(bits, M * ldw, "bits")
    _check(lib().ssgd_signum_momentum_pack(
        _ptr(g, torch.float32, "g"), _ptr(m, torch.float32, "m"), M, d, ld, beta,
        _ptr(bits, WORD_DTYPE, "bits"), ldw, _stream(stream)), "ssgd_signum_momentum_pack")


def majority_vote(bits: torch.Tensor, M: int, d: int, ldw: int, vote: torch.Tensor,
                  stream=None) -> None:
    """Algorithm 3 server side: vote <- packed sign of the sum of the workers' signs."""
    _need(bits, M * ldw, "bits"); _need(vote, -(-d // 32), "vote")
    _check(lib().ssgd_majority_vote(_ptr(bits, WORD_DTYPE, "bits"), M, d, ldw,
                                    _ptr(vote, WORD_DTYPE, "vote"), _stream(stream)),
           "ssgd_majority_vote")


def majority_vote_staged(bits: torch.Tensor, M: int, d: int, ldw: int, vote: torch.Tensor, status: torch.Tensor,
                         stream=None) -> None:
    """The majority vote by the kernel that stages the rows through shared memory with bulk copies; same
    output as `majority_vote`.  `status` is a one-element int32 device tensor, zero before the call; it is
    non-zero afterwards only if a bounded wait in the kernel ran out."""
    _need(bits, M * ldw, "bits"); _need(vote, -(-d // 32), "vote"); _need(status, 1, "status")
    _check(lib().ssgd_majority_vote_staged(_ptr(bits, WORD_DTYPE, "bits"), M, d, ldw, _ptr(vote, WORD_DTYPE, "vote"),
                                           _ptr(status, torch.int32, "status"), _stream(stream)),
           "ssgd_majority_vote_staged")


def sign_apply(x: torch.Tensor, vote: torch.Tensor, d: int, delta: float, stream=None) -> None:
    """Algorithm 3 worker side: x <- x - delta * sign(vote), in place."""
    _need(x, d, "x"); _need(vote, -(-d // 32), "vote")
    _check(lib().ssgd_sign_apply(_ptr(x, torch.float32, "x"), _ptr(vote, WORD_DTYPE, "vote"), d,
                                 delta, _stream(stream)), "ssgd_sign_apply")


def signsgd_step(x: torch.Tensor, g: torch.Tensor, m: Optional[torch.Tensor], M: int, d: int,
                 ld: int, beta: float, delta: float, bits_ws: torch.Tensor, ldw: int,
                 vote_ws: torch.Tensor, stream=None) -> None:
    """One step of Algorithm 3 with Signum workers (m=None with beta=0: plain signSGD)."""
    _need(x, d, "x"); _need(g, M * ld, "g"); _need(bits_ws, M * ldw, "bits_ws")
    _need(vote_ws, -(-d // 32), "vote_ws")
    if m is not None:
        _need(m, M * ld, "m")
    _check(lib().ssgd_signsgd_step(
        _ptr(x, torch.float32, "x"), _ptr(g, torch.float32, "g"), _ptr(m, torch.float32, "m"),
        M, d, ld, beta, delta, _ptr(bits_ws, WORD_DTYPE, "bits_ws"), ldw,
        _ptr(vote_ws, WORD_DTYPE, "vote_ws"), _stream(stream)), "ssgd_signsgd_step")


def step_is_fused(M: int, d: int, momentum: bool) -> bool:
    """Whether signsgd_step runs as one kernel for this problem on the current device (else worker,
    vote and apply kernels); a query for measurement tools."""
    return lib().ssgd_step_is_fused(M, d, 1 if momentum else 0) != 0


def step_kernel_name(M: int, d: int, momentum: bool) -> str:
    """Name of the kernel that is the whole step, or '' when the step is three kernels."""
    return ("", "fused_step_kernel", "step_rows_kernel")[lib().ssgd_step_is_fused(M, d, 1 if momentum else 0)]


def warmup_steps(beta: float) -> int:
    """C(beta) of Theorem 3: how many warm-up iterations Signum's analysis asks for (54 at 0.9)."""
    return int(lib().ssgd_warmup_steps(beta))


def signum_warmup_pack(g: torch.Tensor, m: torch.Tensor, M: int, d: int, ld: int, beta: float,
                       bits: torch.Tensor, ldw: int, stream=None) -> None:
    """Warm-up worker step of Theorem 3: m updated as in Algorithm 2, bits <- sign(g)."""
    _need(g, M * ld, "g"); _need(m, M * ld, "m"); _need(bits, M * ldw, "bits")
    _check(lib().ssgd_signum_warmup_pack(
        _ptr(g, torch.float32, "g"), _ptr(m, torch.float32, "m"), M, d, ld, beta,
        _ptr(bits, WORD_DTYPE, "bits"), ldw, _stream(stream)), "ssgd_signum_warmup_pack")


def signsgd_warmup_step(x: torch.Tensor, g: torch.Tensor, m: torch.Tensor, M: int, d: int, ld: int,
                        beta: float, delta: float, bits_ws: torch.Tensor, ldw: int,
                        vote_ws: torch.Tensor, stream=None) -> None:
    """One whole warm-up step (momentum accumulates, the vote is over sign(g))."""
    _need(x, d, "x"); _need(g, M * ld, "g"); _need(m, M * ld, "m")
    _need(bits_ws, M * ldw, "bits_ws"); _need(vote_ws, -(-d // 32), "vote_ws")
    _check(lib().ssgd_signsgd_warmup_step(
        _ptr(x, torch.float32, "x"), _ptr(g, torch.float32, "g"), _ptr(m, torch.float32, "m"),
        M, d, ld, beta, delta, _ptr(bits_ws, WORD_DTYPE, "bits_ws"), ldw,
        _ptr(vote_ws, WORD_DTYPE, "vote_ws"), _stream(stream)), "ssgd_signsgd_warmup_step")


def count_planes(M: int) -> int:
    """Bit planes that hold a vote count 0..M (the bit length of M)."""
    return int(lib().ssgd_count_planes(M))


def vote_counts(bits: torch.Tensor, M: int, d: int, ldw: int, counts: torch.Tensor, ldc: int,
                stream=None) -> None:
    """Server side of the "(good)" scheme of Sec. 4: bit-sliced number of +1 votes per parameter."""
    _need(bits, M * ldw, "bits"); _need(counts, count_planes(M) * ldc, "counts")
    _check(lib().ssgd_vote_counts(_ptr(bits, WORD_DTYPE, "bits"), M, d, ldw,
                                  _ptr(counts, WORD_DTYPE, "counts"), ldc, _stream(stream)),
           "ssgd_vote_counts")


def sum_apply(x: torch.Tensor, counts: torch.Tensor, M: int, d: int, ldc: int, delta: float,
              stream=None) -> None:
    """Worker side of the "(good)" scheme: x <- x - delta * (sum of the M signs), in place."""
    _need(x, d, "x"); _need(counts, count_planes(M) * ldc, "counts")
    _check(lib().ssgd_sum_apply(_ptr(x, torch.float32, "x"), _ptr(counts, WORD_DTYPE, "counts"), M, d,
                                ldc, delta, _stream(stream)), "ssgd_sum_apply")


def ternary_pack(g: torch.Tensor, m: Optional[torch.Tensor], M: int, d: int, ld: int, beta: float,
                 tau: float, sign_bits: torch.Tensor, active_bits: torch.Tensor, ldw: int,
                 stream=None) -> None:
    """Abstaining worker (Discussion): sign plane as in the 1-bit path, active plane = !(|v| < tau)."""
    _need(g, M * ld, "g"); _need(sign_bits, M * ldw, "sign_bits"); _need(active_bits, M * ldw, "active_bits")
    if m is not None:
        _need(m, M * ld, "m")
    _check(lib().ssgd_ternary_pack(
        _ptr(g, torch.float32, "g"), _ptr(m, torch.float32, "m"), M, d, ld, beta, tau,
        _ptr(sign_bits, WORD_DTYPE, "sign_bits"), _ptr(active_bits, WORD_DTYPE, "active_bits"), ldw,
        _stream(stream)), "ssgd_ternary_pack")


def quorum_vote(sign_bits: torch.Tensor, active_bits: torch.Tensor, M: int, d: int, ldw: int, quorum: int,
                vote_sign: torch.Tensor, vote_active: torch.Tensor, stream=None) -> None:
    """Server with quorum: decided where |P - N| >= max(quorum, 1), sign of P - N there."""
    _need(sign_bits, M * ldw, "sign_bits"); _need(active_bits, M * ldw, "active_bits")
    _need(vote_sign, -(-d // 32), "vote_sign"); _need(vote_active, -(-d // 32), "vote_active")
    _check(lib().ssgd_quorum_vote(
        _ptr(sign_bits, WORD_DTYPE, "sign_bits"), _ptr(active_bits, WORD_DTYPE, "active_bits"), M, d, ldw,
        quorum, _ptr(vote_sign, WORD_DTYPE, "vote_sign"), _ptr(vote_active, WORD_DTYPE, "vote_active"),
        _stream(stream)), "ssgd_quorum_vote")


def ternary_apply(x: torch.Tensor, vote_sign: torch.Tensor, vote_active: torch.Tensor, d: int, delta: float,
                  stream=None) -> None:
    """x moves by -/+ delta where the server decided, stays where it answered 0."""
    _need(x, d, "x"); _need(vote_sign, -(-d // 32), "vote_sign"); _need(vote_active, -(-d // 32), "vote_active")
    _check(lib().ssgd_ternary_apply(
        _ptr(x, torch.float32, "x"), _ptr(vote_sign, WORD_DTYPE, "vote_sign"),
        _ptr(vote_active, WORD_DTYPE, "vote_active"), d, delta, _stream(stream)), "ssgd_ternary_apply")


def welford_update(g: torch.Tensor, n: int, mean: torch.Tensor, m2: torch.Tensor, d: int, stream=None) -> None:
    """Fold the n-th gradient sample (n from 1) into the running mean and sum of squared deviations."""
    _need(g, d, "g"); _need(mean, d, "mean"); _need(m2, d, "m2")
    _check(lib().ssgd_welford_update(_ptr(g, torch.float32, "g"), n, _ptr(mean, torch.float32, "mean"),
                                     _ptr(m2, torch.float32, "m2"), d, _stream(stream)), "ssgd_welford_update")


def density(v: torch.Tensor, d: int, root: bool = False, sums: Optional[torch.Tensor] = None, stream=None) -> float:
    """phi(v) = |v|_1^2 / (d |v|_2^2) (Sec. 3); with root=True the density of sqrt(v).

    `sums` is a float64 device tensor of 2 elements used for the two norms (allocated here if not
    given).  Waits for the result: this is a measurement call, not part of the step."""
    _need(v, d, "v")
    if sums is None:
        sums = torch.zeros(2, dtype=torch.float64, device=v.device)
    _check(lib().ssgd_density_sums(_ptr(v, torch.float32, "v"), d, 1 if root else 0,
                                   _ptr(sums, torch.float64, "sums"), _stream(stream)), "ssgd_density_sums")
    l1, l2 = sums.tolist()
    return float(lib().ssgd_density_from_sums(l1, l2, d))


def signsgd_step_host(x: torch.Tensor, g_host: torch.Tensor, m: Optional[torch.Tensor], M: int,
                      d: int, ld: int, beta: float, delta: float, g_stage: torch.Tensor,
                      bits_ws: torch.Tensor, ldw: int, vote_ws: torch.Tensor,
                      vote_host: Optional[torch.Tensor], stream=None) -> None:
    """The whole step with gradients in (pinned) host memory and the vote read back to the host."""
    _need(x, d, "x"); _need(g_host, M * ld, "g_host"); _need(g_stage, M * ld, "g_stage")
    _need(bits_ws, M * ldw, "bits_ws"); _need(vote_ws, -(-d // 32), "vote_ws")
    if m is not None:
        _need(m, M * ld, "m")
    if vote_host is not None:
        _need(vote_host, -(-d // 32), "vote_host")
    _check(lib().ssgd_signsgd_step_host(
        _ptr(x, torch.float32, "x"), _ptr(g_host, torch.float32, "g_host", cuda=False),
        _ptr(m, torch.float32, "m"), M, d, ld, beta, delta,
        _ptr(g_stage, torch.float32, "g_stage"), _ptr(bits_ws, WORD_DTYPE, "bits_ws"), ldw,
        _ptr(vote_ws, WORD_DTYPE, "vote_ws"), _ptr(vote_host, WORD_DTYPE, "vote_host", cuda=False),
        _stream(stream)), "ssgd_signsgd_step_host")


MAX_PEERS = 64


def signum_momentum_pack_scatter(g: torch.Tensor, m: Optional[torch.Tensor], d: int, beta: float, rows, row: int,
                                 ldw: int, stream=None) -> None:
    """One worker's momentum update + sign packing, with its words stored into row `row` of every rank's
    rows buffer.  `rows` is a sequence with one entry per rank: a device tensor of int32 words (this
    GPU's own memory) or a raw device address as int (another GPU's memory this GPU can write)."""
    _need(g, d, "g")
    if m is not None:
        _need(m, d, "m")
    addrs = []
    for i, r in enumerate(rows):
        if isinstance(r, torch.Tensor):
            _need(r, (row + 1) * ldw, "rows[%d]" % i)
            addrs.append(_ptr(r, WORD_DTYPE, "rows[%d]" % i))
        else:
            addrs.append(int(r))
    table = (ctypes.c_void_p * len(addrs))(*addrs)
    _check(lib().ssgd_signum_momentum_pack_scatter(
        _ptr(g, torch.float32, "g"), _ptr(m, torch.float32, "m"), d, beta, table, len(addrs), row, ldw,
        _stream(stream)), "ssgd_signum_momentum_pack_scatter")


NOALLOC_SCRATCH_WORDS = 4 << 20


def signsgd_step_noalloc(x: torch.Tensor, g: torch.Tensor, m: Optional[torch.Tensor], M: int, d: int,
                         ld: int, beta: float, delta: float, stream=None) -> None:
    """The whole step without workspace arguments, for callers that cannot allocate device memory.

    The packed sign rows and the vote go to a fixed 16 MiB array inside the library, so the problem
    must satisfy (M + 1) * round_up(ceil(d / 32), 4) <= NOALLOC_SCRATCH_WORDS; larger ones raise
    (status 6).  Calls on one device share that array: keep them on one stream.  The first call on a
    device does a one-time address look-up and should come before any stream capture.
    """
    _need(x, d, "x"); _need(g, M * ld, "g")
    if m is not None:
        _need(m, M * ld, "m")
    _check(lib().ssgd_signsgd_step_noalloc(
        _ptr(x, torch.float32, "x"), _ptr(g, torch.float32, "g"), _ptr(m, torch.float32, "m"),
        M, d, ld, beta, delta, _stream(stream)), "ssgd_signsgd_step_noalloc")


# --------------------------------------------------------------------------
# gradients that come as many tensors; 4-bit operands

class _Codes(dict):
    """The header's codes of some names; looking up anything else raises what the caller should see."""

    def __init__(self, codes, error, message):
        super().__init__(codes)
        self.error, self.message = error, message

    def __missing__(self, name):
        raise self.error("%s, got %r" % (self.message, name))


DTYPE_CODE = _Codes({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}, TypeError, "the dtype must be float32, bfloat16 or float16")


class _Tensor(ctypes.Structure):                 # ssgd_tensor
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("n", ctypes.c_size_t), ("src_type", ctypes.c_uint),
                ("dst_type", ctypes.c_uint), ("group", ctypes.c_uint), ("reserved", ctypes.c_uint)]


assert ctypes.sizeof(_Tensor) == 40


def _typed_ptr(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor) or t.dtype not in DTYPE_CODE:
        raise TypeError("%s must be a torch tensor of dtype float32, bfloat16 or float16" % name)
    if not t.is_cuda:
        raise ValueError("%s must live in device memory" % name)
    return t.data_ptr()


def _need_first(t: Optional[torch.Tensor], name: str) -> None:
    """A tensor of one value that may be left out must hold it where it is given: an empty one has address 0, as one that is left out."""
    if t is not None:
        _need(t, 1, name)


def _need_rows(t: torch.Tensor, rows: int, cols: int, ld: int, name: str) -> None:
    """t's memory, from its first element on, must hold `rows` rows of `cols` elements at a stride of ld."""
    n = (rows - 1) * ld + cols if rows and cols else 0
    if t.numel() < n and t.untyped_storage().nbytes() // t.element_size() - t.storage_offset() < n:
        raise ValueError("%s is too small for %d x %d elements at a row stride of %d" % (name, rows, cols, ld))


class TensorTable:
    """The tensors of one or more workers' gradients, described once for `tensors_norm` and `tensors_clip`.

    src     device tensors (float32, bfloat16, float16; contiguous), any number, any size
    dst     where the clipped values go, one tensor of the same number of elements for each (None entries, or None
            altogether: norm only); a tensor of `src` itself: in place.  Slices of a worker's flat row are the usual ones
    groups  the worker of each tensor, not descending; None: all belong to worker 0

    The table keeps the tensors alive and holds for as long as they stay where they are; building it takes about a microsecond
    a tensor and a blocking copy, more than a call that uses it, so keep it, and the gradients' buffers, over the steps.  Its
    calls share one workspace: they go to one stream, or wait for one another; for calls that may run at the same time build a
    table each.  Where they run on another stream than the one it was built on, keep it until they are done."""

    def __init__(self, src, dst=None, groups=None, workers: Optional[int] = None):
        src = list(src)
        dst = [None] * len(src) if dst is None else list(dst)
        groups = [0] * len(src) if groups is None else list(groups)
        if len(dst) != len(src) or len(groups) != len(src):
            raise ValueError("src, dst and groups must have one entry per tensor")
        self.workers = (max(groups) + 1 if groups else 1) if workers is None else int(workers)
        codes = DTYPE_CODE
        for t in src + [t for t in dst if t is not None]:
            if not isinstance(t, torch.Tensor) or t.dtype not in codes:
                raise TypeError("src and dst must be torch tensors of dtype float32, bfloat16 or float16")
            if not t.is_contiguous():
                raise ValueError("src and dst must be contiguous")
        places = {t.get_device() for t in src} | {t.get_device() for t in dst if t is not None}
        if len(places) > 1 or -1 in places:
            raise ValueError("all tensors must live in the memory of one device")
        device = src[0].device if src else None
        words = []                            # five 64-bit words an entry: src, dst, n, the two types, group
        for s, t, w in zip(src, dst, groups):
            n = s.numel()
            if t is None:
                words += (s.data_ptr(), 0, n, codes[s.dtype], w)
            elif t.numel() != n:
                raise ValueError("a dst holds %d elements, its src %d" % (t.numel(), n))
            else:
                words += (s.data_ptr(), t.data_ptr(), n, codes[s.dtype] | codes[t.dtype] << 32, w)
        block = array.array("Q", words or [0])
        entries = block.buffer_info()[0]
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        tiles, nbytes, ws = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        _check(lib().ssgd_table_size(entries, len(src), self.workers, ctypes.byref(tiles), ctypes.byref(nbytes), ctypes.byref(ws)),
               "ssgd_table_size")
        host = torch.zeros(nbytes.value, dtype=torch.uint8)
        _check(lib().ssgd_table_build(entries, len(src), self.workers, host.data_ptr(), nbytes.value), "ssgd_table_build")
        self.tiles = tiles.value
        self.table = host.to(self.device)
        self.ws = torch.empty(ws.value, dtype=torch.uint8, device=self.device)      # not filled: nothing is pending when this returns
        self._keep = (src, dst)
        self._index = self.device.index
        self._args = (self.table.data_ptr(), self.tiles, self.workers)
        self._ws = self.ws.data_ptr()


NORM_KIND = _Codes({"two": 0, "max": 1}, ValueError, "kind must be 'two' or 'max'")
_CLIP_ARGS = struct.Struct("=4QdQ3Q")      # the blocks of arguments of the hot calls, see the header
FP4_QUANTISE_ARGS, FP4_DEQUANTISE_ARGS, FP4_MATMUL_ARGS = struct.Struct("=13Q"), struct.Struct("=10Q"), struct.Struct("=15Q")


def tensors_norm(table: TensorTable, norms: torch.Tensor, kind: str = "two", stream=None) -> None:
    """norms[w] <- norm of worker w's gradient over all its tensors ("two": sqrt of the sum of squares, "max").  Runs on the
    table's device, whichever is current, by default on its current stream."""
    _need(norms, table.workers, "norms"); _need_device(table._index, norms=norms)
    if table._index != _current_device():
        with _on(table._index):
            return tensors_norm(table, norms, kind, stream)
    status = lib().ssgd_tensors_norm(*table._args, NORM_KIND[kind], table._ws, _ptr(norms, torch.float32, "norms"),
                                     _stream_of(table._index) if stream is None else _stream(stream))
    if status:
        _check(status, "ssgd_tensors_norm")


def tensors_clip(table: TensorTable, max_norm: float, norms: torch.Tensor, kind: str = "two", zero_nonfinite: bool = False,
                 stream=None) -> None:
    """norms as `tensors_norm`; every dst <- src * (max_norm / norm where norm > max_norm, else 1).  With zero_nonfinite a
    worker whose norm is not finite gets zeros."""
    if norms.numel() < table.workers or norms.get_device() != table._index:       # one of the two raises
        _need(norms, table.workers, "norms"); _need_device(table._index, norms=norms)
    if table._index != _current_device():
        with _on(table._index):
            return tensors_clip(table, max_norm, norms, kind, zero_nonfinite, stream)
    status = lib().ssgd_tensors_clip_block(_CLIP_ARGS.pack(
        *table._args, NORM_KIND[kind], max_norm, 1 if zero_nonfinite else 0, table._ws, _ptr(norms, torch.float32, "norms"),
        _stream_of(table._index) if stream is None else _stream(stream)))
    if status:
        _check(status, "ssgd_tensors_clip")


FP4_FORMAT = _Codes({"mx": 0, "nv": 1}, ValueError, "fmt must be 'mx' or 'nv'")
FP4_SMALL, FP4_SCALE_FLOATS = 32768, 1026


def fp4_row_bytes(cols: int) -> int:
    """Bytes of one row of codes."""
    return int(lib().ssgd_fp4_row_bytes(cols))


def fp4_scale_bytes(fmt: str, rows: int, cols: int) -> int:
    """Bytes of the scales of a packed operand."""
    return int(lib().ssgd_fp4_scale_bytes(FP4_FORMAT[fmt], rows, cols))


class ProductForm(NamedTuple):
    """How a product is computed, see ssgd_fp4_matmul_form."""
    ctas: int
    rows: int
    splits: int
    wide: bool
    rounds: int


def fp4_matmul_form(M: int, N: int, K: int, dtype: torch.dtype = torch.bfloat16, ldo: Optional[int] = None, sms: int = 148) -> ProductForm:
    """The form of a product M x N x K into rows of stride ldo (None: N)."""
    form = (ctypes.c_uint * 5)()
    _check(lib().ssgd_fp4_matmul_form(M, N, K, DTYPE_CODE[dtype], N if ldo is None else ldo, sms, form), "ssgd_fp4_matmul_form")
    return ProductForm(form[0], form[1], form[2], bool(form[3]), form[4])


def fp4_quantise(x: torch.Tensor, rows: int, cols: int, ldx: int, fmt: str, amax: Optional[torch.Tensor],
                 tensor_scale: Optional[torch.Tensor], codes: Optional[torch.Tensor], scales: Optional[torch.Tensor],
                 codes_t: Optional[torch.Tensor], scales_t: Optional[torch.Tensor], stream=None) -> None:
    """Packs x (its first element at x, rows of stride ldx) by rows, by columns, or both, into uint8 buffers."""
    _need_rows(x, rows, cols, ldx, "x")
    _need_first(amax, "amax")
    for name, c, s, r, k in (("codes", codes, scales, rows, cols), ("codes_t", codes_t, scales_t, cols, rows)):
        if c is not None:
            _need(c, r * ((k + 31) // 32 * 16), name); _need(s, fp4_scale_bytes(fmt, r, k), "scales of " + name)
    if fmt == "nv":
        _need(tensor_scale, FP4_SCALE_FLOATS if amax is None and rows * cols > FP4_SMALL else 2, "tensor_scale")
    at, index, u8, f32 = _typed_ptr(x, "x"), x.get_device(), torch.uint8, torch.float32
    _need_device(index, amax=amax, tensor_scale=tensor_scale, codes=codes, scales=scales, codes_t=codes_t, scales_t=scales_t)
    with _on(index):
        _check(lib().ssgd_fp4_quantise(
            at, DTYPE_CODE[x.dtype], rows, cols, ldx, FP4_FORMAT[fmt], _ptr(amax, f32, "amax"),
            _ptr(tensor_scale, f32, "tensor_scale"), _ptr(codes, u8, "codes"), _ptr(scales, u8, "scales"),
            _ptr(codes_t, u8, "codes_t"), _ptr(scales_t, u8, "scales_t"), _stream(stream)), "ssgd_fp4_quantise")


def fp4_dequantise(codes: torch.Tensor, scales: torch.Tensor, tensor_scale: Optional[torch.Tensor], fmt: str, rows: int,
                   cols: int, out: torch.Tensor, ldo: int, stream=None) -> None:
    """out <- the values of a packed operand (rows of stride ldo)."""
    _need(codes, rows * ((cols + 31) // 32 * 16), "codes"); _need(scales, fp4_scale_bytes(fmt, rows, cols), "scales")
    _need_first(tensor_scale, "tensor_scale")
    _need_rows(out, rows, cols, ldo, "out")
    at, index, u8 = _typed_ptr(out, "out"), out.get_device(), torch.uint8
    _need_device(index, codes=codes, scales=scales, tensor_scale=tensor_scale)
    with _on(index):
        _check(lib().ssgd_fp4_dequantise(
            _ptr(codes, u8, "codes"), _ptr(scales, u8, "scales"), _ptr(tensor_scale, torch.float32, "tensor_scale"),
            FP4_FORMAT[fmt], rows, cols, at, DTYPE_CODE[out.dtype], ldo, _stream(stream)), "ssgd_fp4_dequantise")


def fp4_matmul(a_codes: torch.Tensor, a_scales: torch.Tensor, a_tensor_scale: Optional[torch.Tensor], b_codes: torch.Tensor,
               b_scales: torch.Tensor, b_tensor_scale: Optional[torch.Tensor], M: int, N: int, K: int, fmt: str,
               out: torch.Tensor, ldo: int, status: torch.Tensor, stream=None) -> None:
    """out[i][j] <- sum_k A[i][k] B[j][k] of two packed operands (rows of out of stride ldo).  `status` is a one-element
    int32 device tensor, zero at first, non-zero afterwards only if a bounded wait in the kernel ran out."""
    row = (K + 31) // 32 * 16
    _need(a_codes, M * row, "a_codes"); _need(b_codes, N * row, "b_codes"); _need(status, 1, "status")
    _need(a_scales, fp4_scale_bytes(fmt, M, K), "a_scales"); _need(b_scales, fp4_scale_bytes(fmt, N, K), "b_scales")
    _need_first(a_tensor_scale, "a_tensor_scale"); _need_first(b_tensor_scale, "b_tensor_scale")
    _need_rows(out, M, N, ldo, "out")
    at, index, u8, f32 = _typed_ptr(out, "out"), out.get_device(), torch.uint8, torch.float32
    _need_device(index, a_codes=a_codes, a_scales=a_scales, a_tensor_scale=a_tensor_scale, b_codes=b_codes, b_scales=b_scales,
                 b_tensor_scale=b_tensor_scale, status=status)
    with _on(index):
        _check(lib().ssgd_fp4_matmul(
            _ptr(a_codes, u8, "a_codes"), _ptr(a_scales, u8, "a_scales"), _ptr(a_tensor_scale, f32, "a_tensor_scale"),
            _ptr(b_codes, u8, "b_codes"), _ptr(b_scales, u8, "b_scales"), _ptr(b_tensor_scale, f32, "b_tensor_scale"), M, N, K,
            FP4_FORMAT[fmt], at, DTYPE_CODE[out.dtype], ldo, _ptr(status, torch.int32, "status"), _stream(stream)), "ssgd_fp4_matmul")


# --------------------------------------------------------------------------
# the loss over a large vocabulary; orthogonalised updates (``loss`` and ``orthogonal`` call these with torch tensors)

XENT_ALIGN_ARGS = struct.Struct("=13Q")
XENT_FORWARD_ARGS, XENT_BACKWARD_ARGS = struct.Struct("=9Qq6Q"), struct.Struct("=21Q")
ORTHOGONALISE_ARGS, ORTHOGONAL_STEP_ARGS = struct.Struct("=7Q3d9Q"), struct.Struct("=13Q2dQ3d5Q")


def xent_sizes(tokens: int, vocab: int, width: int):
    """Workspace bytes of ssgd_xent_forward and ssgd_xent_backward on the current device."""
    forward, backward = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().ssgd_xent_sizes(tokens, vocab, width, ctypes.byref(forward), ctypes.byref(backward)), "ssgd_xent_sizes")
    return forward.value, backward.value


def orthogonal_ws_bytes(n: int, rows: int, cols: int) -> int:
    """Workspace bytes of ssgd_orthogonalise and ssgd_orthogonal_step."""
    size = lib().ssgd_orthogonal_ws_bytes(n, rows, cols)
    if not size:
        raise ValueError("%d matrices of %d x %d: at most 65535, sides up to 32768" % (n, rows, cols))
    return int(size)
