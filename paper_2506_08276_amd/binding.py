"""Thin ctypes binding of libleann.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/leann.h).
Device buffers are torch CUDA tensors (PyTorch is used for device memory and
the stream, nothing else); the raw data_ptr() values are handed to the library.
There is no fallback: if the shared library is missing, loading raises.
"""
import ctypes as C
import os

import numpy as np
import torch  # imported before libleann.so so that both share the HIP runtime torch ships (same soname)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libleann.so")
_lib = None

LEANN_F32, LEANN_BF16, LEANN_F16 = 0, 1, 2
STATUS = {0: "LEANN_OK", -1: "LEANN_EINVAL", -2: "LEANN_ENOMEM", -3: "LEANN_EDEVICE", -4: "LEANN_ESHAPE",
          -5: "LEANN_ECAPACITY"}
EXPORTS = ["leann_last_error", "leann_create", "leann_destroy", "leann_embed", "leann_build_pq", "leann_pq_export",
           "leann_pq_import", "leann_pq_wrap", "leann_pq_info", "leann_pq_free", "leann_adc", "leann_adc_noalloc", "leann_search",
           "leann_search_updates", "leann_build_graph", "leann_top_degree",
           "leann_set_limits", "leann_set_call_memo", "leann_set_gemm_tiles", "leann_profile_begin", "leann_profile_end", "leann_bench_mfma", "leann_bench_gather", "leann_bench_l1pull",
           "leann_dropout", "leann_layernorm", "leann_layernorm_backward",
           "leann_projection_create", "leann_projection_free", "leann_adapter_rows_create", "leann_adapter_rows_free",
           "leann_adapter_project", "leann_adapter_project_backward",
           "leann_position_buckets", "leann_attention_create", "leann_attention_free", "leann_attention",
           "leann_attention_backward", "leann_checkpoint", "leann_checkpoint_restore", "leann_activation", "leann_activation_backward"]
PROF_KINDS = ["gemm_qkv", "gemm_o", "gemm_ffn1", "gemm_ffn2", "attention", "layernorm", "enc_other", "traverse",
              "collect", "score_insert", "lut", "adc"]


class LeannError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class EncoderDesc(C.Structure):
    _fields_ = [("layers", C.c_int32), ("hidden", C.c_int32), ("heads", C.c_int32), ("ffn", C.c_int32),
                ("vocab", C.c_int32), ("max_pos", C.c_int32), ("ln_eps", C.c_float)]


class Graph(C.Structure):
    _fields_ = [("row_ptr", C.c_void_p), ("col_idx", C.c_void_p), ("n", C.c_int64), ("entry", C.c_uint32)]


class Chunks(C.Structure):
    _fields_ = [("tokens", C.c_void_p), ("lengths", C.c_void_p), ("n", C.c_int64), ("seq", C.c_int32)]


class EmbCache(C.Structure):
    _fields_ = [("slot_of", C.c_void_p), ("emb", C.c_void_p), ("rows", C.c_int64)]


class SearchStats(C.Structure):
    _fields_ = [("hops", C.c_int64), ("adc_candidates", C.c_int64), ("recomputed_chunks", C.c_int64),
                ("encoded_chunks", C.c_int64), ("encoded_tokens", C.c_int64), ("flushes", C.c_int64),
                ("rounds", C.c_int64), ("cache_hits", C.c_int64), ("memo_hits", C.c_int64), ("encoder_ms", C.c_float),
                ("traverse_ms", C.c_float),
                ("total_ms", C.c_float)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class Profile(C.Structure):
    _fields_ = [("ms", C.c_double * len(PROF_KINDS)), ("launches", C.c_int64 * len(PROF_KINDS)),
                ("tokens", C.c_int64)]


def load_library(path=LIB_PATH):
    """Load libleann.so; raises when it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise FileNotFoundError(f"{path} not found: build it with `python -m paper_2506_08276_amd.build` "
                                    "(or __graft_entry__.build())")
        lib = C.CDLL(path)
        lib.leann_last_error.restype = C.c_char_p
        for name in EXPORTS:
            getattr(lib, name)
        lib.leann_destroy.restype = None
        for name in ("leann_pq_free", "leann_projection_free", "leann_adapter_rows_free", "leann_attention_free"):
            getattr(lib, name).restype = None
        V, I, N, F = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        for name, args in {  # argument types: plain numbers are converted by ctypes, which small calls are faster with
                "leann_dropout": [V, V, N, V, N, N, N, I, V, V, N],
                "leann_layernorm": [V, V, N, V, N, N, I, I, V, V, V, F, V, N, V, N, V, V],
                "leann_layernorm_backward": [V, V, N, V, N, N, I, I, V, V, V, V, N, V, V, N, V, N, V, V],
                "leann_projection_create": [V, V, V, I, I, I, I, V], "leann_projection_free": [V],
                "leann_adapter_rows_create": [V, V, V, I, V, V, I, I, V], "leann_adapter_rows_free": [V],
                "leann_adapter_project": [V, V, V, V, N, V, V, V, N, V],
                "leann_adapter_project_backward": [V, V, V, V, N, V, N, V, V, V, V, N, V, V],
                "leann_position_buckets": [I, I, I, V],
                "leann_attention_create": [V, V, V, V, I, V, V], "leann_attention_free": [V],
                "leann_attention": [V, V, V, N, V, N, V, N, I, F, V, V, N, V],
                "leann_attention_backward": [V, V, V, N, V, N, V, N, V, N, V, N, V, I, F, V, V, N, V, N, V, N, V],
                "leann_checkpoint": [V, V, N, N, N, I, V, N, V], "leann_checkpoint_restore": [V, V, N, V, N, N, I, V, N],
                "leann_activation": [V, V, N, N, N, I, I, V, N, V, N, V],
                "leann_activation_backward": [V, V, N, V, N, V, N, V, N, N, I, I, V, N, V, N]}.items():
            getattr(lib, name).argtypes = args
        _lib = lib
    return _lib


def _check(rc):
    if rc != 0:
        raise LeannError(rc, load_library().leann_last_error(None).decode())


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


def _dev(t, dtype, what):
    assert isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous() and t.dtype == dtype, \
        f"{what}: need a contiguous CUDA tensor of {dtype}"
    return t


def leann_create(desc, weights, device=0, stream=None):
    """desc: dict of encoder dimensions; weights: packed CUDA tensor (float32 or bfloat16).  Returns a ctx handle."""
    lib = load_library()
    assert weights.is_cuda and weights.is_contiguous() and weights.dtype in (torch.float32, torch.bfloat16)
    d = EncoderDesc(desc["layers"], desc["hidden"], desc["heads"], desc["ffn"], desc["vocab"], desc["max_pos"],
                    desc.get("ln_eps", 1e-12))
    ctx = C.c_void_p()
    if stream is None:
        stream = torch.cuda.current_stream(device).cuda_stream
    _check(lib.leann_create(C.byref(ctx), C.byref(d), _ptr(weights),
                            LEANN_F32 if weights.dtype == torch.float32 else LEANN_BF16, C.c_int(device),
                            C.c_void_p(stream)))
    return ctx


def leann_destroy(ctx):
    load_library().leann_destroy(ctx)


def leann_set_limits(ctx, max_tokens_per_pass=0, aq_capacity=0):
    _check(load_library().leann_set_limits(ctx, C.c_int64(max_tokens_per_pass), C.c_int32(aq_capacity)))


def leann_set_call_memo(ctx, max_rows):
    """Per-call embedding memo of leann_search: up to max_rows embeddings kept within a call (0 = off)."""
    _check(load_library().leann_set_call_memo(ctx, C.c_int64(max_rows)))


def leann_set_gemm_tiles(ctx, large_tile=0, small_rows=2048):
    _check(load_library().leann_set_gemm_tiles(ctx, C.c_int32(large_tile), C.c_int32(small_rows)))


def _chunks(tokens, lengths):
    _dev(tokens, torch.int32, "tokens")
    _dev(lengths, torch.int32, "lengths")
    assert tokens.dim() == 2 and lengths.numel() == tokens.shape[0]
    return Chunks(tokens.data_ptr(), lengths.data_ptr(), tokens.shape[0], tokens.shape[1])


def leann_embed(ctx, tokens, lengths, ids=None, n_ids=None, hidden=None, out=None):
    """Embeddings fp32 [n_ids][hidden] of chunks `ids` (int64 CUDA tensor) or of the first n_ids chunks."""
    lib = load_library()
    ch = _chunks(tokens, lengths)
    if ids is not None:
        _dev(ids, torch.int64, "ids")
        n_ids = ids.numel()
    elif n_ids is None:
        n_ids = tokens.shape[0]
    if out is None:
        out = torch.empty((n_ids, hidden), dtype=torch.float32, device=tokens.device)
    _dev(out, torch.float32, "out")
    _check(lib.leann_embed(ctx, C.byref(ch), _ptr(ids), C.c_int64(n_ids), _ptr(out)))
    return out


def leann_build_pq(ctx, emb, m_sub, iters, seed):
    _dev(emb, torch.float32, "emb")
    pq = C.c_void_p()
    _check(load_library().leann_build_pq(ctx, _ptr(emb), C.c_int64(emb.shape[0]), C.c_int32(emb.shape[1]),
                                         C.c_int32(m_sub), C.c_int32(iters), C.c_uint64(seed), C.byref(pq)))
    return pq


def leann_pq_info(pq):
    n, d, m = C.c_int64(), C.c_int32(), C.c_int32()
    _check(load_library().leann_pq_info(pq, C.byref(n), C.byref(d), C.byref(m)))
    return n.value, d.value, m.value


def leann_pq_export(ctx, pq):
    """Returns (codebook float32 [m_sub][256][dsub], codes uint8 [n][m_sub]) as numpy arrays."""
    n, d, m = leann_pq_info(pq)
    cb = np.empty((m, 256, d // m), dtype=np.float32)
    codes = np.empty((n, m), dtype=np.uint8)
    _check(load_library().leann_pq_export(ctx, pq, cb.ctypes.data_as(C.c_void_p), codes.ctypes.data_as(C.c_void_p)))
    return cb, codes


def leann_pq_import(ctx, codebook, codes):
    codebook = np.ascontiguousarray(codebook, dtype=np.float32)
    codes = np.ascontiguousarray(codes, dtype=np.uint8)
    m, ksub, dsub = codebook.shape
    assert ksub == 256 and codes.shape[1] == m
    pq = C.c_void_p()
    _check(load_library().leann_pq_import(ctx, codebook.ctypes.data_as(C.c_void_p), codes.ctypes.data_as(C.c_void_p),
                                          C.c_int64(codes.shape[0]), C.c_int32(m * dsub), C.c_int32(m), C.byref(pq)))
    return pq


def leann_pq_wrap(ctx, codebook, codes_dev):
    codebook = np.ascontiguousarray(codebook, dtype=np.float32)
    _dev(codes_dev, torch.uint8, "codes")
    m, ksub, dsub = codebook.shape
    assert ksub == 256 and codes_dev.shape[1] == m
    pq = C.c_void_p()
    _check(load_library().leann_pq_wrap(ctx, codebook.ctypes.data_as(C.c_void_p), _ptr(codes_dev),
                                        C.c_int64(codes_dev.shape[0]), C.c_int32(m * dsub), C.c_int32(m),
                                        C.byref(pq)))
    return pq


def leann_pq_free(pq):
    load_library().leann_pq_free(pq)


def leann_adc(ctx, queries, pq, cand_ids, out=None):
    """ADC similarities fp32 [nq][nc] of candidate node ids (uint32 stored in an int32 CUDA tensor)."""
    _dev(queries, torch.float32, "queries")
    _dev(cand_ids, torch.int32, "cand_ids")
    nq, nc = cand_ids.shape
    if out is None:
        out = torch.empty((nq, nc), dtype=torch.float32, device=queries.device)
    _check(load_library().leann_adc(ctx, _ptr(queries), C.c_int64(nq), pq, _ptr(cand_ids), C.c_int32(nc), _ptr(out)))
    return out


def leann_adc_noalloc(ctx, queries, pq, cand_ids, out):
    """leann_adc through the library's fixed workspace (no allocation, no synchronisation); `out` is required."""
    _dev(queries, torch.float32, "queries")
    _dev(cand_ids, torch.int32, "cand_ids")
    _dev(out, torch.float32, "out")
    nq, nc = cand_ids.shape
    assert out.shape == (nq, nc)
    _check(load_library().leann_adc_noalloc(ctx, _ptr(queries), C.c_int64(nq), pq, _ptr(cand_ids), C.c_int32(nc),
                                            _ptr(out)))
    return out


class Updates(C.Structure):
    _fields_ = [("deleted_bits", C.c_void_p), ("buffer_emb", C.c_void_p), ("buffer_ids", C.c_void_p),
                ("buffer_n", C.c_int64)]


def _search(entry_point, ctx, queries, graph, pq, tokens, lengths, ef, k, rerank_ratio, batch, cache, updates):
    _dev(queries, torch.float32, "queries")
    row_ptr, col_idx, entry = graph
    _dev(row_ptr, torch.int64, "row_ptr")
    _dev(col_idx, torch.int32, "col_idx")
    g = Graph(row_ptr.data_ptr(), col_idx.data_ptr(), row_ptr.numel() - 1, int(entry))
    ch = _chunks(tokens, lengths)
    nq = queries.shape[0]
    ids = torch.empty((nq, k), dtype=torch.int64, device=queries.device)
    scores = torch.empty((nq, k), dtype=torch.float32, device=queries.device)
    st = SearchStats()
    cref = None
    if cache is not None:
        slot_of, emb = cache
        _dev(slot_of, torch.int32, "slot_of")
        _dev(emb, torch.float32, "cache emb")
        cstruct = EmbCache(slot_of.data_ptr(), emb.data_ptr(), emb.shape[0])
        cref = C.byref(cstruct)
    head = (ctx, _ptr(queries), C.c_int64(nq), C.byref(g), pq, C.byref(ch), cref)
    tail = (C.c_int32(ef), C.c_int32(k), C.c_float(rerank_ratio), C.c_int32(batch), _ptr(ids), _ptr(scores), C.byref(st))
    if entry_point == "leann_search":
        _check(load_library().leann_search(*head, *tail))
    else:
        deleted_bits, buffer = updates
        u = Updates(None, None, None, 0)
        if deleted_bits is not None:
            _dev(deleted_bits, torch.int32, "deleted_bits")
            assert deleted_bits.numel() >= (g.n + 31) // 32
            u.deleted_bits = deleted_bits.data_ptr()
        if buffer is not None:
            buf_ids, buf_emb = buffer
            _dev(buf_ids, torch.int32, "buffer ids")
            _dev(buf_emb, torch.float32, "buffer emb")
            assert buf_emb.shape == (buf_ids.numel(), queries.shape[1])
            u.buffer_emb, u.buffer_ids, u.buffer_n = buf_emb.data_ptr(), buf_ids.data_ptr(), buf_ids.numel()
        _check(load_library().leann_search_updates(*head, C.byref(u), *tail))
    return ids, scores, st.as_dict()


def leann_search(ctx, queries, graph, pq, tokens, lengths, ef, k, rerank_ratio, batch, cache=None):
    """graph = (row_ptr int64 CUDA tensor holding uint64 values, col_idx int32 CUDA tensor holding uint32, entry).
    cache = (slot_of int32 [n], emb float32 [rows][d]) or None.
    Returns (ids int64 [nq][k], scores float32 [nq][k], stats dict)."""
    return _search("leann_search", ctx, queries, graph, pq, tokens, lengths, ef, k, rerank_ratio, batch, cache, None)


def leann_search_updates(ctx, queries, graph, pq, tokens, lengths, ef, k, rerank_ratio, batch, cache=None,
                         deleted_bits=None, buffer=None):
    """leann_search with pending updates: deleted_bits = int32 CUDA tensor of (n + 31) // 32 words (bit v set: node v
    is soft-deleted) or None; buffer = (ids int32 CUDA tensor holding uint32 [nb], emb float32 [nb][d]) or None."""
    return _search("leann_search_updates", ctx, queries, graph, pq, tokens, lengths, ef, k, rerank_ratio, batch, cache,
                   (deleted_bits, buffer))


def leann_build_graph(ctx, emb, efC, M, m=None, is_hub=None, batch=256, ramp=8):
    """Algorithm 3 on the device.  emb float32 CUDA [n][d]; is_hub uint8 CUDA [n] or None.
    Returns (row_ptr int64 CUDA tensor holding uint64 [n+1], col_idx int32 CUDA tensor holding uint32 [E])."""
    _dev(emb, torch.float32, "emb")
    n, d = emb.shape
    m = M if m is None else m
    if is_hub is not None:
        _dev(is_hub, torch.uint8, "is_hub")
        assert is_hub.numel() == n
    row_ptr = torch.empty(n + 1, dtype=torch.int64, device=emb.device)
    col_idx = torch.empty(n * M, dtype=torch.int32, device=emb.device)
    edges = C.c_int64(0)
    _check(load_library().leann_build_graph(ctx, _ptr(emb), C.c_int64(n), C.c_int32(d), _ptr(is_hub), C.c_int32(efC),
                                            C.c_int32(M), C.c_int32(m), C.c_int32(batch), C.c_int32(ramp),
                                            _ptr(row_ptr), _ptr(col_idx), C.byref(edges)))
    return row_ptr, col_idx[:edges.value].clone()


def leann_top_degree(ctx, row_ptr, beta):
    """uint8 CUDA flags [n] of the ceil(beta * n) nodes of largest out-degree (ties: lower id)."""
    _dev(row_ptr, torch.int64, "row_ptr")
    n = row_ptr.numel() - 1
    out = torch.empty(n, dtype=torch.uint8, device=row_ptr.device)
    _check(load_library().leann_top_degree(ctx, _ptr(row_ptr), C.c_int64(n), C.c_double(beta), _ptr(out)))
    return out


def leann_profile_begin(ctx):
    _check(load_library().leann_profile_begin(ctx))


def leann_profile_end(ctx):
    """Returns {"ms": {kind: summed ms}, "launches": {kind: count}, "tokens": valid tokens encoded}."""
    p = Profile()
    _check(load_library().leann_profile_end(ctx, C.byref(p)))
    return {"ms": {k: p.ms[i] for i, k in enumerate(PROF_KINDS)},
            "launches": {k: p.launches[i] for i, k in enumerate(PROF_KINDS)}, "tokens": p.tokens}


def leann_bench_mfma(ctx, operand_kind, blocks_per_cu=2, iters=4000, launches=40):
    """(TFLOP/s, ms per launch) of a loop of independent bf16 MFMAs; operand_kind 0 zeros, 1 near one, 2 random bits."""
    tf, ms = C.c_double(), C.c_double()
    _check(load_library().leann_bench_mfma(ctx, C.c_int32(operand_kind), C.c_int32(blocks_per_cu), C.c_int32(iters),
                                           C.c_int32(launches), C.byref(tf), C.byref(ms)))
    return tf.value, ms.value


def leann_bench_gather(ctx, table, launches=5):
    """(rows/s, ms per launch) of uniformly random 32-byte row gathers from `table` (uint8 CUDA tensor [rows][32])."""
    _dev(table, torch.uint8, "table")
    assert table.dim() == 2 and table.shape[1] == 32
    rps, ms = C.c_double(), C.c_double()
    _check(load_library().leann_bench_gather(ctx, _ptr(table), C.c_int64(table.shape[0]), C.c_int32(launches),
                                             C.byref(rps), C.byref(ms)))
    return rps.value, ms.value


def leann_bench_l1pull(ctx, panel_rows, launches=5):
    """(bytes/s, ms per launch) of eight waves per CU doing only the GEMM's operand loads over a panel of 1536-byte rows."""
    bps, ms = C.c_double(), C.c_double()
    _check(load_library().leann_bench_l1pull(ctx, C.c_int64(panel_rows), C.c_int32(launches), C.byref(bps), C.byref(ms)))
    return bps.value, ms.value


# ---- operators for adapting an encoder
class DropoutDesc(C.Structure):
    _fields_ = [("p", C.c_float), ("seed", C.c_uint64), ("offset", C.c_uint64)]


_DTYPES = {torch.float32: LEANN_F32, torch.bfloat16: LEANN_BF16, torch.float16: LEANN_F16}


def _rows(t, what, like=None):
    """(pointer, distance of rows) of a 2-D CUDA tensor with unit column stride, (None, 0) for None."""
    if t is None:
        return None, 0
    assert t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] <= 1), f"{what}: need a 2-D CUDA tensor with unit column stride"
    assert like is None or (t.shape == like.shape and t.dtype == like.dtype), f"{what}: shape or type differs"
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1]  # a single row's stride is none


def _rows_or_new(t, what, like):
    """(t, pointer, distance of rows) of an output like a tensor that _rows has looked at; None: a new one, whose rows lie side by side."""
    if t is None:
        t = torch.empty_like(like)
        return t, t.data_ptr(), like.shape[1]
    return t, *_rows(t, what, like)


def _drop(drop):
    return None if drop is None else C.byref(DropoutDesc(*drop))


def _vector(t, n, what):
    assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == n, f"{what}: need {n} contiguous float32 values"
    return t.data_ptr()


def _dtype(t):
    assert t.dtype in _DTYPES, "need float32, bfloat16 or float16"
    return _DTYPES[t.dtype]


def leann_dropout(ctx, x, drop, residual=None, out=None):
    """dropout(x) (+ residual) of a 2-D tensor; drop = (p, seed, offset).  The gradient is the same call on the gradient."""
    if out is None:
        out = torch.empty_like(x)
    (xp, ldx), (rp, ldr), (op, ldo) = _rows(x, "x"), _rows(residual, "residual", x), _rows(out, "out", x)
    _check(load_library().leann_dropout(ctx, xp, ldx, rp, ldr, x.shape[0], x.shape[1], _dtype(x), _drop(drop), op, ldo))
    return out


def leann_layernorm(ctx, x, gamma, beta, eps, residual=None, drop=None, keep=False, out=None):
    """LayerNorm of dropout(x) (+ residual) over the rows of a 2-D tensor; drop = (p, seed, offset) or None.
    keep: returns (out, total, mean, rstd), what the backward pass needs (total is x where it would hold the same); else out."""
    rows, cols = x.shape
    if out is None:
        out = torch.empty_like(x)
    total = mean = rstd = None
    if keep:
        if residual is not None or drop is not None:
            total = torch.empty_like(x)
        mean, rstd = gamma.new_empty(rows), gamma.new_empty(rows)
    (xp, ldx), (rp, ldr), (op, ldo), (tp, ldt) = (_rows(x, "x"), _rows(residual, "residual", x), _rows(out, "out", x),
                                                  _rows(total, "total", x))
    _check(load_library().leann_layernorm(ctx, xp, ldx, rp, ldr, rows, cols, _dtype(x), _drop(drop), _vector(gamma, cols, "gamma"),
                                          _vector(beta, cols, "beta"), eps, op, ldo, tp, ldt,
                                          mean.data_ptr() if keep else None, rstd.data_ptr() if keep else None))
    return (out, x if total is None else total, mean, rstd) if keep else out


def leann_layernorm_backward(ctx, dout, total, mean, rstd, gamma, drop=None, dtotal=None):
    """(dresidual, dx, dgamma, dbeta) from the gradient of leann_layernorm's output and what it kept; dtotal: the gradient that
    reaches the kept total besides.  Without dropout dx is dresidual."""
    rows, cols = dout.shape
    dres = torch.empty_like(dout)
    dx = dres if drop is None else torch.empty_like(dres)
    dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(gamma)
    (dp, ldd), (tp, ldt), (ep, lde), (rp, ldr), (xp, ldx) = (_rows(dout, "dout"), _rows(total, "total", dout), _rows(dtotal, "dtotal", dout),
                                                             _rows(dres, "dresidual"), _rows(dx, "dx"))
    _check(load_library().leann_layernorm_backward(ctx, dp, ldd, tp, ldt, rows, cols, _dtype(dout), _vector(gamma, cols, "gamma"),
                                                   _vector(mean, rows, "mean"), _vector(rstd, rows, "rstd"), ep, lde, _drop(drop), rp, ldr,
                                                   xp, ldx, dgamma.data_ptr(), dbeta.data_ptr()))
    if drop is not None and round(DropoutDesc(*drop).p * 65536) == 0:
        dx = dres
    return dres, dx, dgamma, dbeta


class _Handle(C.c_void_p):
    """A handle of the library with the sizes that its calls' tensors have to have."""


def leann_projection_create(ctx, w, bias=None, gradient=False):
    """A projection's shared weight [n_out][n_in] (bfloat16 or float16, contiguous) and bias; gradient: also for the backward pass."""
    assert w.is_cuda and w.dim() == 2 and w.is_contiguous() and w.dtype in (torch.bfloat16, torch.float16), "w: need a contiguous 16-bit matrix"
    h = _Handle()
    _check(load_library().leann_projection_create(ctx, w.data_ptr(), None if bias is None else _vector(bias, w.shape[0], "bias"), w.shape[0],
                                                  w.shape[1], _dtype(w), int(gradient), C.byref(h)))
    h.n_out, h.n_in, h.dtype = w.shape[0], w.shape[1], w.dtype
    return h


def leann_projection_free(proj):
    load_library().leann_projection_free(proj)


def _int32(values):
    a = np.asarray(values, dtype=None if len(values) else np.int32)
    assert a.dtype.kind in "iu" and (a.size == 0 or -2**31 <= int(a.min()) and int(a.max()) < 2**31), "need whole numbers of 32 bits"
    return np.ascontiguousarray(a, dtype=np.int32)


def leann_adapter_rows_create(ctx, rows_of_request, adapter_of_request, rank, scale, max_rank):
    """Which rows go through which adapter: row counts and adapters (-1: none) of the requests, ranks and scales of the adapters."""
    n, of, rank = _int32(rows_of_request), _int32(adapter_of_request), _int32(rank)
    scale = np.ascontiguousarray(scale, dtype=np.float32)
    assert n.ndim == of.ndim == rank.ndim == scale.ndim == 1 and len(n) == len(of) and len(rank) == len(scale)
    h = _Handle()
    _check(load_library().leann_adapter_rows_create(ctx, n.ctypes.data, of.ctypes.data, len(n), rank.ctypes.data, scale.ctypes.data, len(rank),
                                                    max_rank, C.byref(h)))
    h.T, h.n_adapters, h.max_rank = int(n.sum(dtype=np.int64)), len(rank), max_rank
    return h


def leann_adapter_rows_free(rows):
    load_library().leann_adapter_rows_free(rows)


def _pools(proj, rows, down, up):
    assert down.is_cuda and up.is_cuda and down.is_contiguous() and up.is_contiguous() and down.dtype == up.dtype == proj.dtype
    assert down.shape == (rows.n_adapters, rows.max_rank, proj.n_in) and up.shape == (rows.n_adapters, proj.n_out, rows.max_rank)
    return down.data_ptr(), up.data_ptr()


def leann_adapter_project(ctx, proj, rows, x, down, up, keep=False, out=None):
    """x W^T + bias + each request's adapter's part, x [T][n_in]; keep: returns (out, low), what the backward pass needs; else out."""
    if out is None:
        out = x.new_empty((rows.T, proj.n_out))
    assert x.shape == (rows.T, proj.n_in) and out.shape == (rows.T, proj.n_out) and x.dtype == out.dtype == proj.dtype
    low = torch.empty((rows.T, rows.max_rank), dtype=torch.float32, device=x.device) if keep else None
    (xp, ldx), (op, ldo), (dp, up) = _rows(x, "x"), _rows(out, "out"), _pools(proj, rows, down, up)
    _check(load_library().leann_adapter_project(ctx, proj, rows, xp, ldx, dp, up, op, ldo, low.data_ptr() if keep else None))
    return (out, low) if keep else out


def leann_adapter_project_backward(ctx, proj, rows, dout, x, low, down, up, need_dx=True, need_adapters=True):
    """(dx, ddown, dup) from the gradient of leann_adapter_project's output, its input and what it kept; None for what is not needed
    (x and low may be None without need_adapters)."""
    assert dout.shape == (rows.T, proj.n_out) and dout.dtype == proj.dtype
    dx = dout.new_empty((rows.T, proj.n_in)) if need_dx else None
    ddown = torch.empty_like(down, dtype=torch.float32) if need_adapters else None
    dup = torch.empty_like(up, dtype=torch.float32) if need_adapters else None
    if need_adapters:
        assert x.shape == (rows.T, proj.n_in) and x.dtype == proj.dtype
        assert low.is_cuda and low.is_contiguous() and low.shape == (rows.T, rows.max_rank) and low.dtype == torch.float32
    (gp, ldd), (xp, ldx), (op, lddx), (dp, up) = _rows(dout, "dout"), _rows(x, "x"), _rows(dx, "dx"), _pools(proj, rows, down, up)
    _check(load_library().leann_adapter_project_backward(ctx, proj, rows, gp, ldd, xp, ldx, None if low is None else low.data_ptr(), dp, up, op, lddx,
                                                         ddown.data_ptr() if need_adapters else None, dup.data_ptr() if need_adapters else None))
    return dx, ddown, dup


# ---- attention over ragged sequences
class AttentionDesc(C.Structure):
    _fields_ = [("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32), ("left", C.c_int32), ("right", C.c_int32),
                ("sinks", C.c_int32), ("buckets", C.c_int32), ("distance", C.c_int32), ("bucket_of", C.c_void_p)]


def leann_position_buckets(buckets, distance, both=True):
    """int32 [2 distance + 1]: the bucket of each relative position (key minus query), single distances first, then ranges that grow by equal factors."""
    found = np.empty(2 * max(0, int(distance)) + 1, np.int32)
    _check(load_library().leann_position_buckets(buckets, distance, int(both), found.ctypes.data))
    return found


def leann_attention_create(ctx, q_rows, k_rows=None, *, heads, head_dim, kv_heads=None, first=None, window=None, sinks=0, bucket_of=None):
    """The sequences of a batch: rows of queries, rows of keys (None: the same rows), position of each first query (None: 0); window = (left, right)
    keys that a query sees to either side (-1 or None: all), the first `sinks` keys beside it; bucket_of: int [2 distance + 1], the bias's
    bucket of each relative position (leann_position_buckets makes one)."""
    q = _int32(q_rows)
    k, at = None if k_rows is None else _int32(k_rows), None if first is None else _int32(first)
    assert q.ndim == 1 and (k is None or k.shape == q.shape) and (at is None or at.shape == q.shape), "q_rows, k_rows, first: need one number per sequence"
    table = None if bucket_of is None else _int32(bucket_of)
    assert table is None or table.ndim == 1 and len(table) >= 3 and len(table) % 2 == 1, "bucket_of: need 2 distance + 1 buckets"
    left, right = (-1, -1) if window is None else window
    h = _Handle()
    h.heads, h.kv_heads, h.dim = heads, heads if kv_heads is None else kv_heads, head_dim
    h.buckets = 0 if table is None else max(0, int(table.max())) + 1
    desc = AttentionDesc(heads, h.kv_heads, head_dim, left, right, sinks, h.buckets, 0 if table is None else len(table) // 2,
                         None if table is None else table.ctypes.data)
    _check(load_library().leann_attention_create(ctx, q.ctypes.data, None if k is None else k.ctypes.data, None if at is None else at.ctypes.data,
                                                 len(q), C.byref(desc), C.byref(h)))
    h.Tq = int(q.sum(dtype=np.int64))
    h.Tk = h.Tq if k is None else int(k.sum(dtype=np.int64))
    return h


def leann_attention_free(plan):
    load_library().leann_attention_free(plan)


def _attention_inputs(plan, q, k, v, bias):
    """Pointers and distances of the rows of q, k and v, and the bias's pointer."""
    assert q.shape == (plan.Tq, plan.heads * plan.dim), "q: need [Tq][heads * head_dim]"
    assert k.shape == v.shape == (plan.Tk, plan.kv_heads * plan.dim), "k, v: need [Tk][kv_heads * head_dim]"
    assert q.dtype == k.dtype == v.dtype and q.dtype in (torch.bfloat16, torch.float16), "q, k, v: need bfloat16 or float16"
    assert (bias is None) == (plan.buckets == 0), "bias: goes with a plan that has buckets"
    assert bias is None or bias.dim() == 2 and bias.shape[0] >= plan.buckets and bias.shape[1] == plan.heads, "bias: need [buckets][heads]"
    return (*_rows(q, "q"), *_rows(k, "k"), *_rows(v, "v")), None if bias is None else _vector(bias, bias.numel(), "bias")


def leann_attention(ctx, plan, q, k, v, scale=None, bias=None, keep=False, out=None):
    """softmax(scale q k^T + bias) v for every sequence and head of the plan; q [Tq][heads * head_dim], k and v [Tk][kv_heads * head_dim], bias float32
    [buckets][heads]; scale None: head_dim ** -0.5.  keep: returns (out, lse), what the backward pass needs; else out."""
    (qp, ldq, kp, ldk, vp, ldv), bp = _attention_inputs(plan, q, k, v, bias)
    out, op, ldo = _rows_or_new(out, "out", q)
    lse = q.new_empty((plan.heads, plan.Tq), dtype=torch.float32) if keep else None
    scale = plan.dim ** -0.5 if scale is None else scale
    _check(load_library().leann_attention(ctx, plan, qp, ldq, kp, ldk, vp, ldv, _dtype(q), scale, bp, op, ldo, lse.data_ptr() if keep else None))
    return (out, lse) if keep else out


def leann_attention_backward(ctx, plan, dout, q, k, v, out, lse, scale=None, bias=None, dq=None, dk=None, dv=None, need_bias=True):
    """(dq, dk, dv, dbias) from the gradient of leann_attention's output, its inputs and what it kept; dbias None without a bias or need_bias.  dq, dk, dv may be
    given, as slices of one projection's gradient, say."""
    (qp, ldq, kp, ldk, vp, ldv), bp = _attention_inputs(plan, q, k, v, bias)
    assert dout.shape == out.shape == q.shape and dout.dtype == out.dtype == q.dtype, "dout, out: shape or type differs"
    assert lse.is_cuda and lse.is_contiguous() and lse.shape == (plan.heads, plan.Tq) and lse.dtype == torch.float32, "lse: need float32 [heads][Tq]"
    (dq, dqp, lddq), (dk, dkp, lddk), (dv, dvp, lddv) = _rows_or_new(dq, "dq", q), _rows_or_new(dk, "dk", k), _rows_or_new(dv, "dv", v)
    dbias = None
    if bias is not None and need_bias:  # rows that no relative position has stay zero
        dbias = torch.empty_like(bias) if bias.shape[0] == plan.buckets else torch.zeros_like(bias)
    (gp, ldd), (op, ldo) = _rows(dout, "dout"), _rows(out, "out")
    scale = plan.dim ** -0.5 if scale is None else scale
    _check(load_library().leann_attention_backward(ctx, plan, gp, ldd, qp, ldq, kp, ldk, vp, ldv, op, ldo, lse.data_ptr(), _dtype(q), scale, bp, dqp, lddq,
                                                   dkp, lddk, dvp, lddv, None if dbias is None else dbias.data_ptr()))
    return dq, dk, dv, dbias


# ---- activations, and their checkpoints in 8 bits
ACTIVATIONS = {"gelu": 0, "gelu_tanh": 1}


def _kind(kind):
    assert kind in ACTIVATIONS, f"kind: need one of {', '.join(ACTIVATIONS)}"
    return ACTIVATIONS[kind]


def _checkpoint_like(x):
    """A new checkpoint for x, which _rows has looked at, and what _checkpoint gives of it."""
    rows, cols = x.shape
    codes, scales = torch.empty_like(x, dtype=torch.int8), x.new_empty((rows, (cols + 127) // 128), dtype=torch.float32)
    return (codes, scales), (codes.data_ptr(), cols, scales.data_ptr())


def _checkpoint(kept):
    """(codes' pointer and distance of rows, scales' pointer) of a checkpoint."""
    codes, scales = kept
    assert codes.dtype == torch.int8, "checkpoint: codes have to be int8"
    return *_rows(codes, "codes"), _vector(scales, codes.shape[0] * ((codes.shape[1] + 127) // 128), "scales")


def leann_checkpoint(ctx, x):
    """A 2-D tensor in 8 bits: (codes int8 [rows][cols], scales float32 [rows][ceil(cols / 128)]), the largest of 128 columns being 127 steps."""
    xp, ldx = _rows(x, "x")
    kept, to = _checkpoint_like(x)
    _check(load_library().leann_checkpoint(ctx, xp, ldx, *x.shape, _dtype(x), *to))
    return kept


def leann_checkpoint_restore(ctx, kept, dtype=None, out=None):
    """The tensor that a checkpoint stands for, in `dtype` (or into `out`)."""
    cp, ldc, sp = _checkpoint(kept)
    rows, cols = kept[0].shape
    if out is None:
        assert dtype in _DTYPES, "need float32, bfloat16 or float16"
        out = torch.empty_like(kept[0], dtype=dtype)
        op, ldo = out.data_ptr(), cols
    else:
        assert out.shape == kept[0].shape and dtype in (None, out.dtype), "out: shape or type differs"
        op, ldo = _rows(out, "out")
    _check(load_library().leann_checkpoint_restore(ctx, cp, ldc, sp, rows, cols, _dtype(out), op, ldo))
    return out


def leann_activation(ctx, x, kind="gelu", keep=False, out=None):
    """GELU of a 2-D tensor ("gelu", or "gelu_tanh" for its approximation); keep: returns (out, checkpoint of x), what the backward pass needs; else out."""
    xp, ldx = _rows(x, "x")
    out, op, ldo = _rows_or_new(out, "out", x)
    kept, to = _checkpoint_like(x) if keep else (None, (None, 0, None))
    _check(load_library().leann_activation(ctx, xp, ldx, *x.shape, _dtype(x), _kind(kind), op, ldo, *to))
    return (out, kept) if keep else out


def leann_activation_backward(ctx, dout, kept, kind="gelu", again=False, dx=None):
    """The gradient of leann_activation's input from that of its output and the input, a checkpoint or the tensor itself; again: (dx, output once more)."""
    plain = isinstance(kept, torch.Tensor)
    assert plain or kept[0].shape == dout.shape, "checkpoint: shape differs"
    gp, ldd = _rows(dout, "dout")
    dx, dp, lddx = _rows_or_new(dx, "dx", dout)
    y, yp, lda = _rows_or_new(None, "again", dout) if again else (None, None, 0)
    (xp, ldx), (cp, ldc, sp) = (_rows(kept, "x", dout), (None, 0, None)) if plain else ((None, 0), _checkpoint(kept))
    _check(load_library().leann_activation_backward(ctx, gp, ldd, xp, ldx, cp, ldc, sp, dout.shape[0], dout.shape[1], _dtype(dout), _kind(kind), dp, lddx, yp, lda))
    return (dx, y) if again else dx
