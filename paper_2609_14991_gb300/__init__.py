"""Fused streaming Transducer decode with n-gram shallow fusion and phrase
boosting on one GB300 (sm_103a).

A thin ctypes binding over the C ABI in ``include/tsd.h`` (``libtsd.so``):
the functions below only marshal arguments.  Every step of the decode path
runs in the library's CUDA kernels; PyTorch is used for device memory and
streams.  There is no CPU fallback: if the library is not built, importing
the binding's entry points raises.

Typical use::

    lm = NGram(V, tokens_per_order, logp_per_order, bow_per_order)
    boost = Boost(V, offsets, tokens, bonus)
    dec = Decoder(V, H, W_out, E, lm=lm, boost=boost, max_streams=B, max_T=13)
    slots = [dec.open() for _ in range(B)]
    out = dec.decode_chunk(slots, enc, lam=0.5, beta=1.5)   # enc: cuda bf16 [B, T, H]
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# TSD_LIBRARY selects another build of the library (the range-checked
# libtsd_checks.so); by default the in-tree libtsd.so
LIB_PATH = os.environ.get("TSD_LIBRARY") or os.path.join(_HERE, "libtsd.so")

TSD_OK, TSD_EINVAL, TSD_ENOMEM, TSD_ECUDA, TSD_ESTATE, TSD_EDEVICE = 0, -1, -2, -3, -4, -5
_STATUS = {-1: "EINVAL", -2: "ENOMEM", -3: "ECUDA", -4: "ESTATE", -5: "EDEVICE"}

# every entry point declared in include/tsd.h: name -> (argtypes, restype)
_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_P = ctypes.POINTER


class PredWeightsC(ctypes.Structure):
    _fields_ = [("D", _i32), ("H_enc", _i32), ("emb", _vp), ("W_gates", _vp), ("b_gates", _vp), ("W_pred", _vp),
                ("b_pred", _vp), ("W_enc", _vp), ("b_enc", _vp)]


class DecoderCfg(ctypes.Structure):
    _fields_ = [("V", _i32), ("H", _i32), ("max_symbols", _i32), ("beam_k", _i32), ("max_streams", _i32),
                ("max_T", _i32), ("prune_k", _i32)]


class EncoderCfgC(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("d", "layers", "heads", "ff", "kernel", "left", "max_chunk", "feat", "stack",
                                    "max_streams")]


# field order of tsd_encoder_layer
_ENC_LAYER_FIELDS = ["ln_ff1_g", "ln_ff1_b", "ff1_w1", "ff1_b1", "ff1_w2", "ff1_b2", "ln_att_g", "ln_att_b", "qkv_w",
                     "qkv_b", "pos_w", "pos_u", "pos_v", "out_w", "out_b", "ln_conv_g", "ln_conv_b", "pw1_w", "pw1_b",
                     "dw_w", "dw_b", "bn_scale", "bn_shift", "pw2_w", "pw2_b", "ln_ff2_g", "ln_ff2_b", "ff2_w1",
                     "ff2_b1", "ff2_w2", "ff2_b2", "ln_out_g", "ln_out_b"]


class EncoderLayerC(ctypes.Structure):
    _fields_ = [(n, _vp) for n in _ENC_LAYER_FIELDS]


class KV8C(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("k_tail", _vp), ("v_tail", _vp),
                ("dtype", _i32), ("n_blocks", _i32), ("kv_heads", _i32), ("block", _i32), ("dim", _i32),
                ("n_slots", _i32)]


class KV8BatchC(ctypes.Structure):
    _fields_ = [("n", _i32), ("slots", _vp), ("lens", _vp), ("table", _vp), ("table_width", _i32), ("starts", _vp),
                ("rows", _i32), ("max_new", _i32), ("max_len", _i32)]


SIGNATURES = {
    "tsd_last_error": ([], ctypes.c_char_p),
    "tsd_version": ([], ctypes.c_char_p),
    "tsd_ngram_build": ([_i32, _i32, _vp, _vp, _vp, _vp, _P(_vp)], _i32),
    "tsd_ngram_free": ([_vp], None),
    "tsd_ngram_info": ([_vp, _P(_i64), _P(_i64), _P(_i64)], _i32),
    "tsd_ngram_state_tuple": ([_vp, _i32, _vp, _i32, _P(_i32)], _i32),
    "tsd_boost_build": ([_i32, _i32, _vp, _vp, _f32, _P(_vp)], _i32),
    "tsd_boost_free": ([_vp], None),
    "tsd_boost_info": ([_vp, _P(_i32), _P(_i32), _P(_i64)], _i32),
    "tsd_boost_node_tuple": ([_vp, _i32, _vp, _i32, _P(_i32)], _i32),
    "tsd_decoder_create": ([_P(DecoderCfg), _vp, _vp, _vp, _vp, _vp, _P(_vp)], _i32),
    "tsd_decoder_create_multi": ([_P(DecoderCfg), _vp, _vp, _vp, _vp, _i32, _vp, _vp, _P(_vp)], _i32),
    "tsd_stream_lm_state": ([_vp, _i32, _i32, _P(_i32)], _i32),
    "tsd_decoder_create_pred": ([_P(DecoderCfg), _P(PredWeightsC), _vp, _vp, _vp, _vp, _P(_vp)], _i32),
    "tsd_stream_pred_state": ([_vp, _i32, _vp, _vp], _i32),
    "tsd_stream_export": ([_vp, _i32, _vp, _i64, _P(_i64)], _i32),
    "tsd_stream_import": ([_vp, _i32, _vp, _i64], _i32),
    "tsd_decoder_free": ([_vp], None),
    "tsd_stream_open": ([_vp, _P(_i32)], _i32),
    "tsd_stream_close": ([_vp, _i32], _i32),
    "tsd_decode_chunk": ([_vp, _i32, _vp, _vp, _i32, _f32, _f32, _vp, _vp, _vp, _vp, _vp], _i32),
    "tsd_stream_state": ([_vp, _i32, _P(_i32), _P(_i32), _P(_i32)], _i32),
    "tsd_stream_result": ([_vp, _i32, _vp, _i32, _P(_i32), _P(_f32)], _i32),
    "tsd_stream_hyps": ([_vp, _i32, _vp, _i32, _vp, _vp, _i32, _P(_i32)], _i32),
    "tsd_decoder_set_graphs": ([_vp, _i32], _i32),
    "tsd_decoder_set_timing": ([_vp, _i32], _i32),
    "tsd_decoder_timing": ([_vp, _vp, _vp, _i32, _i32], _i32),
    "tsd_decoder_launches_per_chunk": ([_vp, _i32, _i32, _P(_i64)], _i32),
    "tsd_arpa_parse": ([ctypes.c_char_p, _i64, _i32, _vp, _P(_vp)], _i32),
    "tsd_arpa_info": ([_vp, _P(_i32), _vp, _i32, _P(_i64)], _i32),
    "tsd_arpa_arrays": ([_vp, _i32, _P(_vp), _P(_vp), _P(_vp)], _i32),
    "tsd_arpa_free": ([_vp], None),
    "tsd_ngram_build_arpa": ([ctypes.c_char_p, _i64, _i32, _vp, _P(_vp)], _i32),
    "tsd_decoder_timed_bytes": ([_vp, _P(_i64), _i32], _i32),
    "tsd_decoder_debug_capture": ([_vp, _vp, _vp, _i32], _i32),
    "tsd_decoder_set_joint_kernel": ([_vp, _i32], _i32),
    "tsd_decoder_check": ([_vp], _i32),
    "tsd_decoder_set_option": ([_vp, ctypes.c_char_p, _i64], _i32),
    "tsd_decoder_replay": ([_vp, _i32, _i32, _vp, _P(_i64)], _i32),
    "tsd_joint_select_noalloc": ([_i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp], _i32),
    "tsd_debug_fail_alloc": ([_i32], _i32),
    "tsd_encoder_create": ([_P(EncoderCfgC), _vp, _vp, _vp, _vp, _P(_vp)], _i32),
    "tsd_encoder_free": ([_vp], None),
    "tsd_encoder_open": ([_vp, _P(_i32)], _i32),
    "tsd_encoder_close": ([_vp, _i32], _i32),
    "tsd_encode_chunk": ([_vp, _i32, _vp, _vp, _i32, _vp, _vp], _i32),
    "tsd_encoder_check": ([_vp], _i32),
    "tsd_encoder_set_timing": ([_vp, _i32], _i32),
    "tsd_encoder_timing": ([_vp, _vp, _vp, _i32, _i32], _i32),
    "tsd_encoder_gemm_flops": ([_vp, _i32, _i32, _P(ctypes.c_double)], _i32),
    "tsd_encoder_launches_per_chunk": ([_vp, _i32, _i32, _P(_i64)], _i32),
    "tsd_label_scores": ([_i32, _i32, _vp, _i32, _i64, _f32, _i32, _vp, _i32, _vp, _vp, _vp, _vp, _vp], _i32),
    "tsd_joint_label_scores_workspace": ([_i32, _i32, _i32, _i32, _i32, _P(_i64)], _i32),
    "tsd_joint_label_scores": ([_i32, _i32, _i32, _vp, _i64, _vp, _i64, _f32, _i32, _vp, _i32, _vp, _vp, _vp, _vp, _vp,
                                _i64, _vp], _i32),
    "tsd_kv8_append": ([_P(KV8C), _P(KV8BatchC), _vp, _i64, _i64, _vp, _i64, _i64, _vp], _i32),
    "tsd_kv8_read": ([_P(KV8C), _P(KV8BatchC), _vp, _vp, _vp], _i32),
    "tsd_kv8_attend_workspace": ([_P(KV8C), _P(KV8BatchC), _i32, _i32, _i32, _P(_i64)], _i32),
    "tsd_kv8_attend": ([_P(KV8C), _P(KV8BatchC), _i32, _vp, _i64, _i64, _f32, _i32, _i32, _vp, _i64, _i64, _vp, _i64,
                        _vp], _i32),
}

_lib = None


class TsdError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"tsd {_STATUS.get(status, status)}: {msg}")
        self.status = status


def lib() -> ctypes.CDLL:
    """The loaded library.  Raises if it has not been built: there is no
    fallback implementation."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; "
                               "g.build()')")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in SIGNATURES.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


def _check(st: int):
    if st != TSD_OK:
        raise TsdError(st, lib().tsd_last_error().decode())


def version() -> str:
    return lib().tsd_version().decode()


def _i32arr(x) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(x, dtype=np.int32))


def _ptr(t) -> int:
    """Device or host address of a torch tensor / numpy array."""
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream) -> int:
    import torch

    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


class NGram:
    """Backoff n-gram tables on the device (``tsd_ngram_build``)."""

    def __init__(self, V: int, tokens: Sequence[np.ndarray], logp: Sequence[np.ndarray],
                 bow: Optional[Sequence[np.ndarray]] = None):
        order = len(tokens)
        toks = [np.ascontiguousarray(t, dtype=np.int32) for t in tokens]
        lps = [np.ascontiguousarray(x, dtype=np.float32) for x in logp]
        bws = [np.ascontiguousarray(x, dtype=np.float32) for x in bow] if bow is not None else None
        cnt = np.array([len(x) for x in lps], dtype=np.int64)
        tp = (_vp * order)(*[t.ctypes.data for t in toks])
        lp = (_vp * order)(*[t.ctypes.data for t in lps])
        bp = (_vp * order)(*[t.ctypes.data for t in bws]) if bws is not None else None
        h = _vp()
        _check(lib().tsd_ngram_build(V, order, cnt.ctypes.data, tp, lp, bp, ctypes.byref(h)))
        self.h, self.V, self.order = h, V, order

    @classmethod
    def from_arrays(cls, a) -> "NGram":
        return cls(a.V, a.tokens, a.logp, a.bow)

    @classmethod
    def from_arpa(cls, text, V: int, vocab: Optional[Sequence[str]] = None) -> "NGram":
        """Tables from ARPA text (``tsd_ngram_build_arpa``)."""
        data = text.encode() if isinstance(text, str) else bytes(text)
        keep, vp = _vocab(vocab, V)
        h = _vp()
        _check(lib().tsd_ngram_build_arpa(data, len(data), V, vp, ctypes.byref(h)))
        obj = cls.__new__(cls)
        obj.h, obj.V = h, V
        obj.order = 0
        return obj

    def info(self) -> Tuple[int, int, int]:
        s, a, b = _i64(), _i64(), _i64()
        _check(lib().tsd_ngram_info(self.h, ctypes.byref(s), ctypes.byref(a), ctypes.byref(b)))
        return s.value, a.value, b.value

    def state_tuple(self, state: int) -> Tuple[int, ...]:
        buf = np.zeros(16, dtype=np.int32)
        n = _i32()
        _check(lib().tsd_ngram_state_tuple(self.h, int(state), buf.ctypes.data, 16, ctypes.byref(n)))
        return tuple(int(x) for x in buf[: n.value])

    def __del__(self):
        if getattr(self, "h", None):
            lib().tsd_ngram_free(self.h)
            self.h = None


class Boost:
    """Phrase-boosting trie on the device (``tsd_boost_build``)."""

    def __init__(self, V: int, offsets, tokens, bonus: float):
        off = _i32arr(offsets)
        tok = _i32arr(tokens) if len(tokens) else np.zeros(1, dtype=np.int32)
        h = _vp()
        _check(lib().tsd_boost_build(V, len(off) - 1, off.ctypes.data, tok.ctypes.data, float(bonus),
                                     ctypes.byref(h)))
        self.h, self.V = h, V

    @classmethod
    def from_phrases(cls, V: int, p, bonus: float) -> "Boost":
        return cls(V, p.offsets, p.tokens, bonus)

    def info(self) -> Tuple[int, int, int]:
        q, d, b = _i32(), _i32(), _i64()
        _check(lib().tsd_boost_info(self.h, ctypes.byref(q), ctypes.byref(d), ctypes.byref(b)))
        return q.value, d.value, b.value

    def node_tuple(self, node: int) -> Tuple[int, ...]:
        buf = np.zeros(32, dtype=np.int32)
        n = _i32()
        _check(lib().tsd_boost_node_tuple(self.h, int(node), buf.ctypes.data, 32, ctypes.byref(n)))
        return tuple(int(x) for x in buf[: n.value])

    def __del__(self):
        if getattr(self, "h", None):
            lib().tsd_boost_free(self.h)
            self.h = None


def debug_fail_alloc(n: int):
    """Test hook: the n-th device allocation from now on fails (0: off)."""
    _check(lib().tsd_debug_fail_alloc(int(n)))


def joint_select_noalloc(A, Wt, bias, out_label, out_score, stream=None):
    """Allocation-free joint selection (tsd_joint_select_noalloc): for callers
    that cannot allocate device memory.  A: cuda bf16 [n, H]; Wt: cuda bf16
    [V+1, H]; bias: cuda fp32 [n, V] or None; out_label: cuda int32 [n];
    out_score: cuda fp32 [n].  Nothing is allocated by this call."""
    import torch

    named = {"A": A, "Wt": Wt, "out_label": out_label, "out_score": out_score}
    if bias is not None:
        named["bias"] = bias
    for name, t in named.items():
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"joint_select_noalloc: {name} must be a torch tensor")
    if A.dim() != 2 or A.dtype != torch.bfloat16:
        raise ValueError("joint_select_noalloc: A must be bf16 [n, H]")
    n, H = A.shape
    if Wt.dim() != 2 or Wt.element_size() != 2 or Wt.shape[1] != H:
        raise ValueError(f"joint_select_noalloc: Wt must be 2-byte [V+1, H] with H = {H}")
    V = Wt.shape[0] - 1
    if bias is not None and (bias.dtype != torch.float32 or tuple(bias.shape) != (n, V)):
        raise ValueError(f"joint_select_noalloc: bias must be float32 [{n}, {V}]")
    if out_label.dtype != torch.int32 or out_label.numel() < n:
        raise ValueError(f"joint_select_noalloc: out_label must be int32 with at least {n} elements")
    if out_score.dtype != torch.float32 or out_score.numel() < n:
        raise ValueError(f"joint_select_noalloc: out_score must be float32 with at least {n} elements")
    dev = torch.cuda.current_device() if torch.cuda.is_available() else None
    for name, t in named.items():
        if not t.is_cuda or t.device.index != dev:
            raise ValueError(f"joint_select_noalloc: {name} must be a CUDA tensor on the current device")
        if not t.is_contiguous():
            raise ValueError(f"joint_select_noalloc: {name} must be contiguous")
    _check(lib().tsd_joint_select_noalloc(n, H, V, _ptr(A), _ptr(Wt), _ptr(bias) if bias is not None else None,
                                          _ptr(out_label), _ptr(out_score), _stream(stream)))


class ChunkOut:
    """Device outputs of one decode_chunk call (torch tensors)."""

    def __init__(self, tokens, frames, scores, counts):
        self.tokens, self.frames, self.scores, self.counts = tokens, frames, scores, counts


class Decoder:
    """A decoder on the current CUDA device (``tsd_decoder_create``)."""

    def __init__(self, V: int, H: int, W_out, E, lm: Optional[NGram] = None, boost: Optional[Boost] = None,
                 max_symbols: int = 5, beam_k: int = 1, max_streams: int = 64, max_T: int = 64, stream=None,
                 lms: Optional[Sequence[Tuple[NGram, float]]] = None, prune_k: int = 0, pred=None):
        """lms: several LMs as (NGram, w) pairs instead of lm (LM i enters Eq. 1
        with weight lambda * w; ``tsd_decoder_create_multi``).  prune_k > 0:
        pruned fusion over the acoustic model's prune_k best outputs.  pred:
        the stateful form's weights (fields D, Henc, Ep, Wg, bg, Wp, bp, We, be
        as numpy arrays, bf16 bit patterns and fp32 biases;
        ``tsd_decoder_create_pred``); E is then ignored."""
        import torch

        assert W_out.is_cuda and E.is_cuda and W_out.element_size() == 2 and E.element_size() == 2
        assert tuple(W_out.shape) == (H, V + 1) and tuple(E.shape) == (V + 1, H)
        self.cfg = DecoderCfg(V, H, max_symbols, beam_k, max_streams, max_T, prune_k)
        self.V, self.H, self.max_symbols, self.beam_k = V, H, max_symbols, beam_k
        self.lm, self.boost = lm, boost  # kept alive: the decoder borrows them
        W_out = W_out.contiguous()
        E = E.contiguous()
        h = _vp()
        if pred is not None:
            dev = W_out.device
            up16 = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(dev)
            up32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev)
            t = dict(emb=up16(pred.Ep), Wg=up16(pred.Wg), bg=up32(pred.bg), Wp=up16(pred.Wp), bp=up32(pred.bp),
                     We=up16(pred.We), be=up32(pred.be))
            self._pred_keep = t
            self.pred_D = pred.D
            self.pred_Henc = pred.Henc
            pw = PredWeightsC(pred.D, pred.Henc, _ptr(t["emb"]), _ptr(t["Wg"]), _ptr(t["bg"]), _ptr(t["Wp"]),
                              _ptr(t["bp"]), _ptr(t["We"]), _ptr(t["be"]))
            _check(lib().tsd_decoder_create_pred(ctypes.byref(self.cfg), ctypes.byref(pw), _ptr(W_out),
                                                 lm.h if lm else None, boost.h if boost else None, _stream(stream),
                                                 ctypes.byref(h)))
        elif lms is not None:
            assert lm is None, "give lm or lms, not both"
            self.lm = [m for m, _ in lms]
            hs = (_vp * max(1, len(lms)))(*[m.h for m, _ in lms])
            ws = np.array([w for _, w in lms] or [0.0], dtype=np.float32)
            _check(lib().tsd_decoder_create_multi(ctypes.byref(self.cfg), _ptr(W_out), _ptr(E), hs, ws.ctypes.data,
                                                  len(lms), boost.h if boost else None, _stream(stream),
                                                  ctypes.byref(h)))
        else:
            _check(lib().tsd_decoder_create(ctypes.byref(self.cfg), _ptr(W_out), _ptr(E), lm.h if lm else None,
                                            boost.h if boost else None, _stream(stream), ctypes.byref(h)))
        self.h = h
        self._keep = []

    def __del__(self):
        if getattr(self, "h", None):
            lib().tsd_decoder_free(self.h)
            self.h = None

    def open(self) -> int:
        s = _i32()
        _check(lib().tsd_stream_open(self.h, ctypes.byref(s)))
        return s.value

    def close(self, slot: int):
        _check(lib().tsd_stream_close(self.h, int(slot)))

    def alloc_out(self, n: int, T: int) -> ChunkOut:
        import torch

        cap = T * self.max_symbols
        dev = torch.device("cuda", torch.cuda.current_device())
        return ChunkOut(torch.empty((n, cap), dtype=torch.int32, device=dev),
                        torch.empty((n, cap), dtype=torch.int32, device=dev),
                        torch.empty((n, cap), dtype=torch.float32, device=dev),
                        torch.empty((n,), dtype=torch.int32, device=dev))

    def decode_chunk(self, slots: Sequence[int], enc, lam: float, beta: float, out: Optional[ChunkOut] = None,
                     stream=None) -> ChunkOut:
        """enc: cuda bf16 (or int16/uint16 bit patterns) [n, T, H]."""
        n, T, H = enc.shape
        assert n == len(slots) and H == getattr(self, "pred_Henc", self.H) and enc.is_cuda and enc.is_contiguous()
        if out is None:
            out = self.alloc_out(n, T)
        sl = _i32arr(slots)
        _check(lib().tsd_decode_chunk(self.h, n, sl.ctypes.data, _ptr(enc), T, float(lam), float(beta),
                                      _ptr(out.tokens), _ptr(out.frames), _ptr(out.scores), _ptr(out.counts),
                                      _stream(stream)))
        return out

    def decode_chunk_raw(self, slots_np: np.ndarray, enc_ptr: int, T: int, lam: float, beta: float,
                         out_ptrs: Tuple[int, int, int, int], stream_handle: int):
        """Pointer-level call (for timing loops)."""
        _check(lib().tsd_decode_chunk(self.h, len(slots_np), slots_np.ctypes.data, enc_ptr, T, float(lam),
                                      float(beta), out_ptrs[0], out_ptrs[1], out_ptrs[2], out_ptrs[3],
                                      stream_handle))

    def state(self, slot: int) -> Tuple[int, int, int]:
        a, b, c = _i32(), _i32(), _i32()
        _check(lib().tsd_stream_state(self.h, int(slot), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
        return a.value, b.value, c.value

    def export_state(self, slot: int) -> bytes:
        """The slot's decoding state as bytes (``tsd_stream_export``)."""
        n = _i64()
        _check(lib().tsd_stream_export(self.h, int(slot), None, 0, ctypes.byref(n)))
        buf = ctypes.create_string_buffer(max(1, n.value))
        _check(lib().tsd_stream_export(self.h, int(slot), buf, n.value, ctypes.byref(n)))
        return buf.raw[: n.value]

    def import_state(self, slot: int, blob: bytes):
        """Continues an exported stream in an open slot (``tsd_stream_import``)."""
        buf = ctypes.create_string_buffer(bytes(blob), len(blob))
        _check(lib().tsd_stream_import(self.h, int(slot), buf, len(blob)))

    def pred_state(self, slot: int):
        """(h as bf16 bits [D], c [D]) of a stateful-form stream."""
        h = np.zeros(self.pred_D, dtype=np.uint16)
        c = np.zeros(self.pred_D, dtype=np.float32)
        _check(lib().tsd_stream_pred_state(self.h, int(slot), h.ctypes.data, c.ctypes.data))
        return h, c

    def lm_state(self, slot: int, lm_index: int) -> int:
        """State id of LM lm_index for a slot (``tsd_stream_lm_state``)."""
        x = _i32()
        _check(lib().tsd_stream_lm_state(self.h, int(slot), int(lm_index), ctypes.byref(x)))
        return x.value

    def result(self, slot: int, cap: int = 1 << 16) -> Tuple[List[int], float]:
        buf = np.zeros(cap, dtype=np.int32)
        n, sc = _i32(), _f32()
        _check(lib().tsd_stream_result(self.h, int(slot), buf.ctypes.data, cap, ctypes.byref(n), ctypes.byref(sc)))
        return [int(x) for x in buf[: min(n.value, cap)]], sc.value

    def hyps(self, slot: int, cap_len: int = 4096) -> List[Tuple[List[int], float]]:
        K = self.beam_k
        buf = np.zeros(K * cap_len, dtype=np.int32)
        lens = np.zeros(K, dtype=np.int32)
        scs = np.zeros(K, dtype=np.float32)
        nh = _i32()
        _check(lib().tsd_stream_hyps(self.h, int(slot), buf.ctypes.data, cap_len, lens.ctypes.data,
                                     scs.ctypes.data, K, ctypes.byref(nh)))
        return [([int(x) for x in buf[i * cap_len: i * cap_len + min(lens[i], cap_len)]], float(scs[i]))
                for i in range(nh.value)]

    def set_graphs(self, enable: bool):
        _check(lib().tsd_decoder_set_graphs(self.h, 1 if enable else 0))

    def set_joint_kernel(self, kind: int):
        """0 = tcgen05 tensor-core GEMM (default), 1 = CUDA-core cross-check kernel."""
        _check(lib().tsd_decoder_set_joint_kernel(self.h, int(kind)))

    def set_option(self, name: str, value: int):
        _check(lib().tsd_decoder_set_option(self.h, name.encode(), int(value)))

    def replay(self, kernel: int, reps: int, stream=None, count_bytes: bool = False) -> int:
        """Re-launch one kernel (0 row pass, 1 joint) of the last chunk's final
        step reps times, for timing; with count_bytes, returns the algorithmic
        bytes of one launch (and waits for the stream)."""
        b = _i64(0)
        _check(lib().tsd_decoder_replay(self.h, int(kernel), int(reps), _stream(stream),
                                        ctypes.byref(b) if count_bytes else None))
        return b.value

    def check(self):
        """Raises TsdError(EDEVICE) if a bounded device wait expired."""
        _check(lib().tsd_decoder_check(self.h))

    def set_timing(self, enable: bool):
        _check(lib().tsd_decoder_set_timing(self.h, 1 if enable else 0))

    def timing(self, reset: bool = False):
        """({'row': ms, 'joint': ms, 'pred': ms}, {... launches}): device time
        of timed chunks per kernel class; 'pred' is the stateful form's
        prediction network and projections."""
        ms = np.zeros(3, dtype=np.float64)
        ln = np.zeros(3, dtype=np.int64)
        _check(lib().tsd_decoder_timing(self.h, ms.ctypes.data, ln.ctypes.data, 3, 1 if reset else 0))
        keys = ("row", "joint", "pred")
        return {k: float(ms[i]) for i, k in enumerate(keys)}, {k: int(ln[i]) for i, k in enumerate(keys)}

    def timed_bytes(self, reset: bool = False) -> int:
        """Algorithmic bytes counted by the row passes of timed chunks."""
        x = _i64()
        _check(lib().tsd_decoder_timed_bytes(self.h, ctypes.byref(x), 1 if reset else 0))
        return x.value

    def launches_per_chunk(self, n: int, T: int) -> int:
        x = _i64()
        _check(lib().tsd_decoder_launches_per_chunk(self.h, n, T, ctypes.byref(x)))
        return x.value

    def debug_capture(self, logits=None, rows=None, max_steps: int = 0):
        self._keep = [logits, rows]
        _check(lib().tsd_decoder_debug_capture(self.h, _ptr(logits) if logits is not None else None,
                                               _ptr(rows) if rows is not None else None, int(max_steps)))


def _vocab(vocab, V):
    if vocab is None:
        return None, None
    if len(vocab) != V:
        raise ValueError("vocabulary has %d words, V=%d" % (len(vocab), V))
    keep = [w.encode() if isinstance(w, str) else bytes(w) for w in vocab]
    arr = (ctypes.c_char_p * V)(*keep)
    return (keep, arr), ctypes.cast(arr, ctypes.c_void_p)


def parse_arpa(text, V: int, vocab: Optional[Sequence[str]] = None):
    """(tokens per order, logp per order, bow per order, dropped lines) of
    ARPA text, read by the library's host parser (``tsd_arpa_parse``)."""
    data = text.encode() if isinstance(text, str) else bytes(text)
    keep, vp = _vocab(vocab, V)
    h = _vp()
    _check(lib().tsd_arpa_parse(data, len(data), V, vp, ctypes.byref(h)))
    try:
        order = _i32()
        skipped = _i64()
        counts = np.zeros(16, dtype=np.int64)
        _check(lib().tsd_arpa_info(h, ctypes.byref(order), counts.ctypes.data, 16, ctypes.byref(skipped)))
        toks, lps, bws = [], [], []
        for k in range(1, order.value + 1):
            tp, lp, bp = _vp(), _vp(), _vp()
            _check(lib().tsd_arpa_arrays(h, k, ctypes.byref(tp), ctypes.byref(lp), ctypes.byref(bp)))
            n = int(counts[k - 1])
            if n:
                toks.append(np.ctypeslib.as_array(ctypes.cast(tp, ctypes.POINTER(ctypes.c_int32)), (n * k,))
                            .reshape(n, k).copy())
                lps.append(np.ctypeslib.as_array(ctypes.cast(lp, ctypes.POINTER(ctypes.c_float)), (n,)).copy())
                bws.append(np.ctypeslib.as_array(ctypes.cast(bp, ctypes.POINTER(ctypes.c_float)), (n,)).copy())
            else:
                toks.append(np.zeros((0, k), dtype=np.int32))
                lps.append(np.zeros(0, dtype=np.float32))
                bws.append(np.zeros(0, dtype=np.float32))
        return toks, lps, bws, int(skipped.value)
    finally:
        lib().tsd_arpa_free(h)


class Encoder:
    """The cache-aware encoder chunk step on the current CUDA device
    (``tsd_encoder_create``).  weights: an object with fields cfg (d, layers,
    heads, ff, kernel, left, chunk, feat, stack), sub_w, sub_b and layers (each
    with the fields of ``tsd_encoder_layer``; a layer norm as a (gamma, beta)
    pair named ln_ff1, ln_att, ln_conv, ln_ff2, ln_out), numpy arrays of bf16
    bit patterns (matrices) and float32 (vectors)."""

    def __init__(self, weights, max_streams: int = 64, max_chunk: Optional[int] = None, stream=None):
        import torch

        c = weights.cfg
        self.d, self.stack, self.feat = c.d, c.stack, c.feat
        self.max_chunk = max_chunk or c.chunk
        self.cfg = EncoderCfgC(c.d, len(weights.layers), c.heads, c.ff, c.kernel, c.left, self.max_chunk, c.feat,
                               c.stack, max_streams)
        dev = torch.device("cuda", torch.cuda.current_device())

        def up(a):
            a = np.ascontiguousarray(a)
            if a.dtype == np.uint16:
                return torch.from_numpy(a.view(np.int16)).to(dev)
            return torch.from_numpy(a.astype(np.float32)).to(dev)

        keep = [up(weights.sub_w), up(weights.sub_b)]
        layers = (EncoderLayerC * len(weights.layers))()
        for i, L in enumerate(weights.layers):
            vals = {}
            for name in ("ln_ff1", "ln_att", "ln_conv", "ln_ff2", "ln_out"):
                g, b = getattr(L, name)
                vals[name + "_g"], vals[name + "_b"] = up(g), up(b)
            for name in _ENC_LAYER_FIELDS:
                if name not in vals:
                    vals[name] = up(getattr(L, name))
            keep.extend(vals.values())
            for name in _ENC_LAYER_FIELDS:
                setattr(layers[i], name, _ptr(vals[name]))
        h = _vp()
        _check(lib().tsd_encoder_create(ctypes.byref(self.cfg), _ptr(keep[0]), _ptr(keep[1]), ctypes.cast(layers, _vp),
                                        _stream(stream), ctypes.byref(h)))
        self.h = h  # the encoder copied every weight; the uploads can go

    def __del__(self):
        if getattr(self, "h", None):
            lib().tsd_encoder_free(self.h)
            self.h = None

    def open(self) -> int:
        s = _i32()
        _check(lib().tsd_encoder_open(self.h, ctypes.byref(s)))
        return s.value

    def close(self, slot: int):
        _check(lib().tsd_encoder_close(self.h, int(slot)))

    def encode_chunk(self, slots: Sequence[int], feats, out=None, stream=None):
        """feats: cuda bf16 (or int16 bit patterns) [n, C*stack, feat] ->
        out: cuda int16 (bf16 bit patterns) [n, C, d]."""
        import torch

        n = len(slots)
        assert feats.is_cuda and feats.element_size() == 2 and feats.shape[0] == n
        assert feats.shape[2] == self.feat and feats.shape[1] % self.stack == 0
        C = feats.shape[1] // self.stack
        feats = feats.contiguous()
        if out is None:
            out = torch.empty((n, C, self.d), dtype=torch.int16, device=feats.device)
        sl = _i32arr(slots)
        _check(lib().tsd_encode_chunk(self.h, n, sl.ctypes.data, _ptr(feats), C, _ptr(out), _stream(stream)))
        return out

    def encode_chunk_raw(self, slots_np: np.ndarray, feats_ptr: int, C: int, out_ptr: int, stream_handle: int):
        _check(lib().tsd_encode_chunk(self.h, len(slots_np), slots_np.ctypes.data, feats_ptr, C, out_ptr,
                                      stream_handle))

    def check(self):
        _check(lib().tsd_encoder_check(self.h))

    def set_timing(self, on: bool):
        _check(lib().tsd_encoder_set_timing(self.h, 1 if on else 0))

    def timing(self, reset: bool = False):
        """({'gemm': ms, 'attention': ms, 'other': ms}, {... launches})"""
        ms = np.zeros(3, dtype=np.float64)
        ln = np.zeros(3, dtype=np.int64)
        _check(lib().tsd_encoder_timing(self.h, ms.ctypes.data, ln.ctypes.data, 3, 1 if reset else 0))
        keys = ("gemm", "attention", "other")
        return {k: float(ms[i]) for i, k in enumerate(keys)}, {k: int(ln[i]) for i, k in enumerate(keys)}

    def gemm_flops(self, n: int, C: int) -> float:
        x = ctypes.c_double()
        _check(lib().tsd_encoder_gemm_flops(self.h, n, C, ctypes.byref(x)))
        return x.value

    def launches_per_chunk(self, n: int, C: int) -> int:
        """Kernel launches of one encode_chunk(n, C) with timing off."""
        x = _i64()
        _check(lib().tsd_encoder_launches_per_chunk(self.h, int(n), int(C), ctypes.byref(x)))
        return x.value


# ---------------------------------------------------------------- scores of labels

# What a short call spends on the host is mostly attribute look-ups and small
# tensors: the calls below fetch each attribute once, allocate each output by
# itself (four views of one buffer take twice as long: 11.6 and 5.9 us) and
# remember a shape's workspace size.

_DTYPE = None  # element type -> the library's number


def _dtype_code(t) -> int:
    """The library's number of a tensor's element type; -1 for others."""
    global _DTYPE
    if _DTYPE is None:
        import torch

        _DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return _DTYPE.get(t.dtype, -1)


def _on_current(who, name, t):
    """The current device's index, which t has to be on."""
    import torch

    dev = t.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{who}: {name} must be a CUDA tensor on the current device")
    return dev


def _raw_stream(stream, dev) -> int:
    import torch

    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _empty(n, dtype, dev, stream):
    """n elements that the caching allocator gives out for the call's stream."""
    import torch

    if stream is None:
        return torch.empty(n, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(n, dtype=dtype, device=dev)


_sizes = {}  # workspace bytes by call shape
_MAX32 = 2 ** 31 - 1


def _remember(key, bytes_):
    if len(_sizes) > 4096:
        _sizes.clear()
    _sizes[key] = bytes_
    return bytes_


class LabelScores:
    """Results of one call: logp [n, m] (or [n]), entropy [n], alt_logp [n, k]
    (float32) and alt_labels [n, k] (int32)."""

    __slots__ = ("logp", "entropy", "alt_labels", "alt_logp")

    def __init__(self, logp, entropy, alt_labels, alt_logp):
        self.logp, self.entropy, self.alt_labels, self.alt_logp = logp, entropy, alt_labels, alt_logp


def _label_args(who, n, labels, k, out, dev, stream):
    """(m, LabelScores, addresses of labels, logp, entropy, alt_labels,
    alt_logp): the given labels checked, the outputs checked or allocated."""
    import torch

    m, shape, lp = 0, (n, 0), None
    if labels is not None:
        shape = tuple(labels.shape)
        if labels.dtype != torch.int32 or len(shape) not in (1, 2) or shape[0] != n:
            raise ValueError(f"{who}: labels must be int32 [{n}] or [{n}, m]")
        if labels.get_device() != dev:
            raise ValueError(f"{who}: labels must be a CUDA tensor on the current device")
        if not labels.is_contiguous():
            raise ValueError(f"{who}: labels must be contiguous")
        m = shape[1] if len(shape) == 2 else 1
        lp = labels.data_ptr() if m else None
    if not 0 <= k <= 8 or m > 8:
        raise ValueError(f"{who}: at most 8 given labels and 8 alternatives")
    if out is None:
        f32 = torch.float32
        res = LabelScores(_empty(shape, f32, dev, stream), _empty(n, f32, dev, stream),
                          _empty((n, k), torch.int32, dev, stream), _empty((n, k), f32, dev, stream))
        return (m, res, lp, res.logp.data_ptr() if m else None, res.entropy.data_ptr(),
                res.alt_labels.data_ptr() if k else None, res.alt_logp.data_ptr() if k else None)
    for name, t, dt, want in (("logp", out.logp, torch.float32, shape), ("entropy", out.entropy, torch.float32, (n,)),
                              ("alt_labels", out.alt_labels, torch.int32, (n, k)),
                              ("alt_logp", out.alt_logp, torch.float32, (n, k))):
        if t.dtype != dt or tuple(t.shape) != want or not t.is_contiguous():
            raise ValueError(f"{who}: out.{name} must be contiguous {dt} {list(want)}")
        if t.get_device() != dev:
            raise ValueError(f"{who}: out.{name} must be a CUDA tensor on the current device")
    return (m, out, lp, out.logp.data_ptr() if m else None, out.entropy.data_ptr(),
            out.alt_labels.data_ptr() if k else None, out.alt_logp.data_ptr() if k else None)


def _row_stride(who, name, t, shape):
    """The distance of a matrix's rows, each of which is adjacent."""
    s0, s1 = t.stride()
    if (s1 != 1 and shape[1] > 1) or (s0 < shape[1] and shape[0] > 1):
        raise ValueError(f"{who}: a row of {name} must be adjacent and rows must not overlap")
    return s0


def label_scores(logits, labels=None, k: int = 0, temperature: float = 1.0, out: Optional[LabelScores] = None,
                 stream=None) -> LabelScores:
    """Log probabilities of given labels, entropy and the k most likely labels
    of rows of logits (``tsd_label_scores``).  logits: cuda float32, bfloat16 or
    float16 [n, C], any row stride; -inf masks a label.  labels: cuda int32 [n]
    or [n, m], -1 for none."""
    who = "label_scores"
    shape = logits.shape
    if len(shape) != 2 or not (1 <= shape[0] <= 1 << 27 and 1 <= shape[1] <= 262144):
        raise ValueError(f"{who}: logits must be [n, C] with 1 <= n <= 2^27 and 1 <= C <= 262144")
    code = _dtype_code(logits)
    if code < 0:
        raise ValueError(f"{who}: logits must be float32, bfloat16 or float16")
    dev = _on_current(who, "logits", logits)
    ld = _row_stride(who, "logits", logits, shape)
    m, res, lab, logp, ent, alt, altp = _label_args(who, shape[0], labels, k, out, dev, stream)
    st = lib().tsd_label_scores(shape[0], shape[1], logits.data_ptr(), code, ld, temperature, m, lab, k, logp, ent, alt,
                                altp, _raw_stream(stream, dev))
    if st:
        _check(st)
    return res


def joint_label_scores(A, Wt, labels=None, k: int = 0, temperature: float = 1.0, out: Optional[LabelScores] = None,
                       stream=None) -> LabelScores:
    """The same of the logits A . Wt^T, which are not kept
    (``tsd_joint_label_scores``): A cuda bf16 [n, H], the joint network's input
    rows; Wt cuda bf16 (or int16 bit patterns) [C, H], W_out label-major.  Row
    strides a multiple of 8, H of 64."""
    import torch

    who = "joint_label_scores"
    sa, sw = A.shape, Wt.shape
    if len(sa) != 2 or A.dtype != torch.bfloat16 or not 1 <= sa[0] <= 1 << 24:
        raise ValueError(f"{who}: A must be bf16 [n, H] with 1 <= n <= 2^24")
    n, H = sa
    if len(sw) != 2 or Wt.dtype not in (torch.bfloat16, torch.int16) or sw[1] != H or not 1 <= sw[0] <= 262144:
        raise ValueError(f"{who}: Wt must be bf16 [C, H] with 1 <= C <= 262144 and H = {H}")
    C = sw[0]
    dev = _on_current(who, "A", A)
    if Wt.get_device() != dev:
        raise ValueError(f"{who}: Wt must be a CUDA tensor on the current device")
    lda, ldw = _row_stride(who, "A", A, sa), _row_stride(who, "Wt", Wt, sw)
    m, res, lab, logp, ent, alt, altp = _label_args(who, n, labels, k, out, dev, stream)
    L = lib()
    key = (dev, n, H, C, m, k)
    need = _sizes.get(key)
    if need is None:
        b = _i64()
        _check(L.tsd_joint_label_scores_workspace(n, H, C, m, k, ctypes.byref(b)))
        need = _remember(key, b.value)
    ws = _empty(need, torch.uint8, dev, stream)
    st = L.tsd_joint_label_scores(n, H, C, A.data_ptr(), lda, Wt.data_ptr(), ldw, temperature, m, lab, k, logp, ent, alt,
                                  altp, ws.data_ptr(), need, _raw_stream(stream, dev))
    if st:
        _check(st)
    return res


# ---------------------------------------------------------------- the 8-bit cache

class KV8Cache:
    """One layer's paged cache of keys and values in 8 bits (``tsd_kv8``), over
    tensors of the caller's (``KV8Cache.empty`` makes them):

      k, v              int8 [n_blocks, kv_heads, block, dim]
      k_scale, v_scale  float32 [n_blocks, kv_heads]
      k_tail, v_tail    bf16 or fp16 [n_slots, 2, kv_heads, block, dim]: the
                        unrounded tokens of each slot's last two blocks

    The calls take the same arrays: table int32 [n_slots, width] (block ids),
    lens int32 [n_slots] (tokens, the call's own included), slots int32 [n] (the
    sequences; None: slots 0 .. n-1) and starts int32 [n + 1] (their rows; None:
    one row each).  max_new and max_len bound a sequence's rows and tokens; they
    size launches only.  Everything is read on the device, so a call captured
    into a graph can be replayed with other lengths, tables and rows.

    Tokens are taken back by lowering a length: to a multiple of block, or into
    a block b while no append since its tokens' has reached block b + 2."""

    def __init__(self, k, v, k_scale, v_scale, k_tail, v_tail):
        import torch

        if k.dim() != 4 or k.dtype != torch.int8:
            raise ValueError("KV8Cache: k must be int8 [n_blocks, kv_heads, block, dim]")
        n_blocks, heads, block, dim = k.shape
        code = _dtype_code(k_tail)
        if code not in (1, 2) or k_tail.dim() != 5 or k_tail.shape[1:] != (2, heads, block, dim):
            raise ValueError(f"KV8Cache: k_tail must be bf16 or fp16 [n_slots, 2, {heads}, {block}, {dim}]")
        if block not in (16, 32, 64) or dim not in (64, 128):
            raise ValueError("KV8Cache: block is 16, 32 or 64 and dim 64 or 128")
        n_slots = k_tail.shape[0]
        named = {"k": (k, k), "v": (v, k), "k_scale": (k_scale, None), "v_scale": (v_scale, None),
                 "k_tail": (k_tail, k_tail), "v_tail": (v_tail, k_tail)}
        for name, (t, like) in named.items():
            if like is not None and (t.shape != like.shape or t.dtype != like.dtype):
                raise ValueError(f"KV8Cache: {name} must be {like.dtype} {list(like.shape)}")
            if like is None and (t.dtype != torch.float32 or tuple(t.shape) != (n_blocks, heads)):
                raise ValueError(f"KV8Cache: {name} must be float32 [{n_blocks}, {heads}]")
            if not t.is_cuda or t.device != k.device:
                raise ValueError(f"KV8Cache: {name} must be a CUDA tensor on k's device")
            if not t.is_contiguous():
                raise ValueError(f"KV8Cache: {name} must be contiguous")
        self.k, self.v, self.k_scale, self.v_scale, self.k_tail, self.v_tail = k, v, k_scale, v_scale, k_tail, v_tail
        self.dtype, self.device = k_tail.dtype, k.device
        self.n_blocks, self.kv_heads, self.block, self.dim, self.n_slots = n_blocks, heads, block, dim, n_slots
        self._dev = k.get_device()
        self._c = KV8C(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), k_tail.data_ptr(),
                       v_tail.data_ptr(), code, n_blocks, heads, block, dim, n_slots)
        self._pc = ctypes.byref(self._c)

    @classmethod
    def empty(cls, n_blocks: int, n_slots: int, kv_heads: int, dim: int, block: int = 32, dtype=None, device=None):
        """A cache over new tensors (zeros, scales 1) on the current device."""
        import torch

        dtype = dtype or torch.bfloat16
        device = device or torch.device("cuda", torch.cuda.current_device())
        z = lambda *s, dt: torch.zeros(s, dtype=dt, device=device)  # noqa: E731
        one = lambda: torch.ones((n_blocks, kv_heads), dtype=torch.float32, device=device)  # noqa: E731
        return cls(z(n_blocks, kv_heads, block, dim, dt=torch.int8), z(n_blocks, kv_heads, block, dim, dt=torch.int8),
                   one(), one(), z(n_slots, 2, kv_heads, block, dim, dt=dtype),
                   z(n_slots, 2, kv_heads, block, dim, dt=dtype))

    def _batch(self, who, table, lens, starts, slots, rows, max_new, max_len):
        import torch

        i32, dev = torch.int32, self._dev
        if torch.cuda.current_device() != dev:
            raise ValueError(f"{who}: the cache is on another device than the current one")
        ts, n_slots = table.shape, self.n_slots
        if table.dtype != i32 or len(ts) != 2 or ts[0] != n_slots or ts[1] > _MAX32 or not table.is_contiguous():
            raise ValueError(f"{who}: table must be contiguous int32 [{n_slots}, width]")
        if lens.dtype != i32 or lens.shape != (n_slots,) or not lens.is_contiguous():
            raise ValueError(f"{who}: lens must be contiguous int32 [{n_slots}]")
        n, ps, pt = rows, None, None
        if slots is not None:
            if slots.dtype != i32 or slots.dim() != 1 or not slots.is_contiguous():
                raise ValueError(f"{who}: slots must be contiguous int32 [n]")
            n, ps = slots.shape[0], slots.data_ptr()
        if starts is not None:
            if starts.dtype != i32 or starts.dim() != 1 or not starts.is_contiguous() or starts.shape[0] < 2:
                raise ValueError(f"{who}: starts must be contiguous int32 [n + 1]")
            if slots is not None and starts.shape[0] != n + 1:
                raise ValueError(f"{who}: starts must have {n + 1} entries")
            n, pt = starts.shape[0] - 1, starts.data_ptr()
        if n > 65535 or not 0 <= rows <= 1 << 22:
            raise ValueError(f"{who}: at most 65535 sequences and 2^22 rows")
        if (table.get_device() != dev or lens.get_device() != dev or (ps is not None and slots.get_device() != dev)
                or (pt is not None and starts.get_device() != dev)):
            raise ValueError(f"{who}: table, lens, slots and starts must be on the cache's device")
        return KV8BatchC(n, ps, lens.data_ptr(), table.data_ptr(), ts[1], pt, rows, min(max_new or 0, _MAX32),
                         min(max_len or 0, _MAX32))

    def _rows(self, who, name, t, heads=None):
        """(rows, heads, distance of rows, distance of heads) of [rows, heads, dim]."""
        s = t.shape
        if len(s) != 3 or t.dtype != self.dtype or s[2] != self.dim or (heads is not None and s[1] != heads):
            raise ValueError(f"{who}: {name} must be {self.dtype} [rows, {'heads' if heads is None else heads}, {self.dim}]")
        if t.get_device() != self._dev:
            raise ValueError(f"{who}: {name} must be on the cache's device")
        d = t.stride()
        if d[2] != 1:
            raise ValueError(f"{who}: {name}'s last dimension must be adjacent")
        return s[0], s[1], d[0], d[1]

    def append(self, k, v, table, lens, starts=None, slots=None, max_new: Optional[int] = None, stream=None):
        """Appends rows of keys and values [rows, kv_heads, dim] (``tsd_kv8_append``)."""
        who = "KV8Cache.append"
        rows, _, kr, kh = self._rows(who, "k", k, self.kv_heads)
        rows_v, _, vr, vh = self._rows(who, "v", v, self.kv_heads)
        if rows != rows_v:
            raise ValueError(f"{who}: k and v must have the same rows")
        b = self._batch(who, table, lens, starts, slots, rows, max_new, None)
        st = lib().tsd_kv8_append(self._pc, ctypes.byref(b), k.data_ptr(), kr, kh, v.data_ptr(), vr, vh,
                                  _raw_stream(stream, self._dev))
        if st:
            _check(st)

    def read(self, table, lens, rows: int, starts=None, slots=None, out=None, stream=None):
        """(k, v) float32 [rows, kv_heads, dim]: the values held for the rows'
        tokens (``tsd_kv8_read``)."""
        import torch

        who = "KV8Cache.read"
        b = self._batch(who, table, lens, starts, slots, rows, None, None)
        shape = (rows, self.kv_heads, self.dim)
        if out is None:
            out = _empty(shape, torch.float32, self._dev, stream), _empty(shape, torch.float32, self._dev, stream)
        for t in out:
            if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous() or t.get_device() != self._dev:
                raise ValueError(f"{who}: out must be two contiguous float32 {list(shape)} on the cache's device")
        st = lib().tsd_kv8_read(self._pc, ctypes.byref(b), out[0].data_ptr(), out[1].data_ptr(),
                                _raw_stream(stream, self._dev))
        if st:
            _check(st)
        return out

    def attend(self, q, table, lens, starts=None, slots=None, scale: Optional[float] = None, window: int = 0,
               sinks: int = 0, out=None, max_new: Optional[int] = None, max_len: Optional[int] = None, stream=None):
        """Causal attention of queries [rows, heads, dim] over the cached tokens
        (``tsd_kv8_attend``): window > 0 limits a token's sight to the last
        `window` tokens and the first `sinks`.  scale: 1 / sqrt(dim) if None."""
        import torch

        who = "KV8Cache.attend"
        rows, heads, qr, qh = self._rows(who, "q", q)
        window, sinks = min(window, _MAX32), min(sinks, _MAX32)  # no sequence is longer
        b = self._batch(who, table, lens, starts, slots, rows, max_new, max_len)
        pb = ctypes.byref(b)
        L = lib()
        dev = self._dev
        key = (dev, self.dim, self.kv_heads, self.block, b.n, rows, heads, b.table_width, max_new, max_len, window, sinks)
        need = _sizes.get(key)
        if need is None:
            x = _i64()
            _check(L.tsd_kv8_attend_workspace(self._pc, pb, heads, window, sinks, ctypes.byref(x)))
            need = _remember(key, x.value)
        ws = None
        if need:
            ws = _empty(need, torch.uint8, dev, stream)
        if out is None:
            out = _empty((rows, heads, self.dim), self.dtype, dev, stream)
            orow, oh = heads * self.dim, self.dim
        else:
            orows, _, orow, oh = self._rows(who, "out", out, heads)
            if orows != rows:
                raise ValueError(f"{who}: out must have {rows} rows")
        st = L.tsd_kv8_attend(self._pc, pb, heads, q.data_ptr(), qr, qh, self.dim ** -0.5 if scale is None else scale,
                              window, sinks, out.data_ptr(), orow, oh, ws.data_ptr() if ws is not None else None, need,
                              _raw_stream(stream, dev))
        if st:
            _check(st)
        return out
