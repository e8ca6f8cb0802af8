"""The library's own rules for a launch's shape, by their C++ names (they are not part of the C ABI).  Not a test module."""
import ctypes

from paper_2503_05840_amd import binding


def _rule(name, restype, *argtypes):
    f = getattr(binding.load(), name)
    f.restype, f.argtypes = restype, argtypes
    return f


def batch_tiles(B, rows, e, units):
    """Batch tiles of 16 sequences that a workgroup of a product takes (units: heads, times matrices for a block's products)."""
    i = ctypes.c_int
    return _rule("_ZN4slim16proj_batch_tilesEiiii", i, i, i, i, i)(B, rows, e, units)


def batch_chunks(B, rows, e, units):
    per = 16 * batch_tiles(B, rows, e, units)
    return (B + per - 1) // per


def row_splits(units, rows, e, B):
    i = ctypes.c_int
    return _rule("_ZN4slim15proj_row_splitsEiiii", i, i, i, i, i)(units, rows, e, B)


def read_once(weight_bytes, cache_bytes):
    """Whether a call's loads of its weights are nontemporal, where one batch chunk reads a matrix."""
    return _rule("_ZN4slim9read_onceEmm", ctypes.c_bool, ctypes.c_size_t, ctypes.c_size_t)(weight_bytes, cache_bytes)


def xcache_read_once(B, T, d_model, e, ragged, one_pass):
    i, b = ctypes.c_int, ctypes.c_bool
    return _rule("_ZN4slim16xcache_read_onceEiiiibb", b, i, i, i, i, b, b)(B, T, d_model, e, ragged, one_pass)


def one_pass_splits(B, H, T, d_model):
    """Context splits of the one-pass X-cache kernel, and the most that any context up to T takes."""
    i = ctypes.c_int
    return tuple(_rule("_ZN4slim%sEiiii" % name, i, i, i, i, i)(B, H, T, d_model) for name in ("13xfused_splits", "18xfused_most_splits"))


def one_pass_through(nbytes):
    """Whether that many bytes of the one-pass X-cache kernel's partials leave through the L2s."""
    return _rule("_ZN4slim14xfused_throughEm", ctypes.c_bool, ctypes.c_size_t)(nbytes)


def one_pass_tiles(B, H, T, d_model):
    """Head tiles of a workgroup of the one-pass X-cache kernel."""
    i = ctypes.c_int
    return _rule("_ZN4slim12xfused_tilesEiiii", i, i, i, i, i)(B, H, d_model, one_pass_splits(B, H, T, d_model)[0])


class _PromptCut(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("parts", ctypes.c_int)]


def prompt_cut(dtype, B, rows_q, rows_k, H, H_kv, d_k):
    """Queries of a workgroup of prompt attention, and parts of the keys."""
    i = ctypes.c_int
    c = _rule("_ZN4slim10prompt_cutEiiiiiii", _PromptCut, *[i] * 7)(binding.DTYPES[dtype], B, rows_q, rows_k, H, H_kv, d_k)
    return c.rows, c.parts


def quant_cut(dtype, B, H, T, d):
    """Of the decode step over a cache in 4 or 8 bits: blocks of 64 rows a split, splits, row splits of W and their rows; then the sequences x splits and sequences x row
    splits that a workspace has place for."""
    i, p = ctypes.c_int, ctypes.POINTER(ctypes.c_int)
    out = [i() for _ in range(4)]
    _rule("_ZN4slim11qdecode_cutEiiiiiPiS0_S0_S0_", None, *[i] * 5, *[p] * 4)(binding.DTYPES[dtype], B, H, T, d, *[ctypes.byref(x) for x in out])
    return (*[x.value for x in out], _rule("_ZN4slim19qdecode_most_splitsEiiiii", ctypes.c_size_t, *[i] * 5)(binding.DTYPES[dtype], B, H, T, d),
            _rule("_ZN4slim23qdecode_most_row_splitsEiii", ctypes.c_size_t, *[i] * 3)(B, H, d))
