"""Host-only: the mixture-of-experts and AdamW entry points reject bad arguments before any launch."""
import ctypes as C

import pytest

import paper_2507_16099_amd as fp8
from paper_2507_16099_amd.fp8 import _CAdamwTensor

NULL, SHAPE, ENUM, ALIGN, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    return fp8.load_library()


@pytest.fixture(scope="module")
def p():
    buf = (C.c_char * 8192)()
    p.buf = buf      # kept alive
    return (C.addressof(buf) + 255) // 256 * 256


def test_enum_values():
    import os
    import re
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fp8mi355.h")).read()
    for name in ("FP8_ROUTE_RENORM", "FP8_ROUTE_FP32", "FP8_ADAMW_PARAM_FP32", "FP8_ADAMW_GRAD_FP32", "FP8_ADAMW_STATE_FP8"):
        assert int(re.search(name + r"\s*=\s*(\d+)", src).group(1)) == getattr(fp8, name)


def test_route(lib, p):
    def call(logits=p, T=4, E=8, ld=8, k=2, flags=0, gates=p, experts=p, offsets=p, rows=p, slots=p, ws=p, n=4096):
        return lib.fp8_moe_route(logits, T, E, ld, k, flags, gates, experts, offsets, rows, slots, ws, n, None)

    for what in ("logits", "gates", "experts", "offsets", "rows", "slots", "ws"):
        assert call(**{what: None}) == NULL, what
        assert call(**{what: p + 1}) == ALIGN, what
    assert call(logits=p + 2, flags=fp8.FP8_ROUTE_FP32) == ALIGN
    for bad in ({"T": -1}, {"T": 1 << 31}, {"T": 1 << 26}, {"E": 0}, {"E": 513, "ld": 513}, {"k": 0}, {"k": 9}, {"E": 64, "ld": 64, "k": 17}, {"ld": 7}, {"T": 1 << 30, "k": 4}):
        assert call(**bad) == SHAPE, bad
        assert fp8.fp8_last_error()
    assert call(flags=1) == ENUM
    assert call(n=16) == WORKSPACE
    assert lib.fp8_moe_route_workspace_bytes(100, 513, 2) == 0 and lib.fp8_moe_route_workspace_bytes(100, 512, 2) > 0

    def back(dgates=p, logits=p, T=4, E=8, ld=8, k=2, flags=0, gates=p, experts=p, out=p, ld_out=8):
        return lib.fp8_moe_route_bwd(dgates, logits, T, E, ld, k, flags, gates, experts, out, ld_out, None)

    for what in ("dgates", "logits", "gates", "experts", "out"):
        assert back(**{what: None}) == NULL, what
        assert back(**{what: p + 1}) == ALIGN, what
    assert back(ld_out=7) == SHAPE and back(flags=2) == ENUM
    assert back(T=0) == 0 and fp8.fp8_last_error() == ""


def test_combine(lib, p):
    def call(y=p, M=8, ld=16, gates=p, slots=p, T=4, D=16, k=2, out=p, ld_out=16):
        return lib.fp8_moe_combine(y, M, ld, gates, slots, T, D, k, out, ld_out, None)

    for what in ("y", "slots", "out"):
        assert call(**{what: None}) == NULL, what
        assert call(**{what: p + 1}) == ALIGN, what
    assert call(gates=p + 1) == ALIGN
    for bad in ({"M": -1}, {"T": -1}, {"D": 12}, {"k": 0}, {"ld": 8}, {"ld_out": 8}, {"T": 1 << 30, "k": 4}, {"T": 1 << 29, "D": 64, "ld": 64, "ld_out": 64}):
        assert call(**bad) == SHAPE, bad
    assert call(ld=20) == ALIGN and call(ld_out=20) == ALIGN
    assert call(T=0) == 0 and call(D=0) == 0

    def back(dout=p, ld_dout=16, y=p, M=8, ld=16, gates=p, slots=p, rows=p, T=4, D=16, k=2, dy=p, ld_dy=16, dgates=p):
        return lib.fp8_moe_combine_bwd(dout, ld_dout, y, M, ld, gates, slots, rows, T, D, k, dy, ld_dy, dgates, None)

    for what in ("dout", "y", "slots", "rows"):
        assert back(**{what: None}) == NULL, what
        assert back(**{what: p + 1}) == ALIGN, what
    for what in ("gates", "dy", "dgates"):
        assert back(**{what: p + 1}) == ALIGN, what
    for bad in ({"ld_dout": 8}, {"ld": 8}, {"ld_dy": 8}, {"T": 1 << 24}, {"M": 1 << 31}):
        assert back(**bad) == SHAPE, bad
    assert back(dy=None, dgates=None) == 0


def test_grouped_linear(lib, p):
    row = fp8.Recipe(gran=fp8.FP8_ROW).c()

    def bytes_(M=8, E=4, K=32, N=16, r=row, bwd=0):
        return lib.fp8_grouped_linear_workspace_bytes(M, E, K, N, None if r is None else C.byref(r), bwd)

    assert bytes_() >= 8 * 32 + 4 * 16 * 32 + 4 * (8 + 64)
    assert bytes_(bwd=1) >= 8 * 16 + 4 * 32 * 16 + (16 + 32) * (8 + 4 * 127)
    for bad in ({"K": 24}, {"N": 12}, {"E": 0}, {"M": -1}, {"M": 1 << 24}, {"r": None}, {"r": fp8.Recipe(gran=fp8.FP8_TENSOR).c()},
                {"r": fp8.Recipe(gran=fp8.FP8_ROW, flags=fp8.FP8_SAVE_FOR_BWD).c()}, {"N": 24, "bwd": 1}, {"K": 1 << 23}, {"E": 1 << 20, "N": 4096},
                {"M": 1 << 23, "bwd": 1}):
        assert bytes_(**bad) == 0, bad
        assert fp8.fp8_last_error()

    def fwd(x=p, T=8, rows=p, w=p, offs=p, E=4, M=8, K=32, N=16, r=row, y=p, ws=p, n=1 << 20):
        return lib.fp8_grouped_linear_fwd(x, T, rows, w, offs, E, M, K, N, None if r is None else C.byref(r), y, ws, n, None)

    for what in ("x", "w", "offs", "y", "ws"):
        assert fwd(**{what: None}) == NULL, what
        assert fwd(**{what: p + 2}) == ALIGN, what
    assert fwd(r=None) == NULL and fwd(rows=p + 1) == ALIGN
    assert fwd(rows=None, T=7) == SHAPE and "row_token" in fp8.fp8_last_error()
    assert fwd(r=fp8.Recipe(gran=fp8.FP8_TENSOR).c()) == ENUM and fwd(r=fp8.Recipe(gran=fp8.FP8_ROW, fmt_x=5).c()) == ENUM
    assert fwd(K=24) == SHAPE and fwd(T=-1) == SHAPE and fwd(n=64) == WORKSPACE
    assert fwd(M=0, T=0, rows=None) == 0 and fwd(N=0) == 0

    def bwd(dy=p, x=p, T=8, rows=p, w=p, offs=p, E=4, M=8, K=32, N=16, r=row, dx=p, dw=p, ws=p, n=1 << 20):
        return lib.fp8_grouped_linear_bwd(dy, x, T, rows, w, offs, E, M, K, N, C.byref(r), dx, dw, ws, n, None)

    for what in ("dy", "x", "w", "offs", "ws"):
        assert bwd(**{what: None}) == NULL, what
        assert bwd(**{what: p + 2}) == ALIGN, what
    for what in ("dx", "dw"):
        assert bwd(**{what: p + 8}) == ALIGN, what
    assert bwd(N=24) == SHAPE and bwd(n=64) == WORKSPACE and bwd(dx=None, dw=None) == 0

    def infer(x=p, T=8, rows=p, fx=0, flags=0, wq=p, ldw=32, fw=0, sw=p, offs=p, E=4, M=8, K=32, N=16, y=p, ws=p, n=1 << 20):
        return lib.fp8_grouped_linear_fwd_prequantized(x, T, rows, fx, flags, wq, ldw, fw, sw, offs, E, M, K, N, y, ws, n, None)

    for what in ("x", "wq", "sw", "offs", "y", "ws"):
        assert infer(**{what: None}) == NULL, what
        assert infer(**{what: p + 2}) == ALIGN, what
    assert infer(fx=2) == ENUM and infer(fw=-1) == ENUM and infer(flags=2) == ENUM
    assert infer(ldw=16) == SHAPE and infer(ldw=40) == ALIGN and infer(ldw=1 << 23) == SHAPE and infer(n=64) == WORKSPACE
    assert lib.fp8_grouped_linear_prequantized_workspace_bytes(8, 32) >= 8 * 36
    assert lib.fp8_grouped_linear_prequantized_workspace_bytes(8, 24) == 0


def test_adamw_table(lib, p):
    q = fp8.FP8_ADAMW_STATE_FP8

    def call(fields=(p, p, p, p, p, p, 8), count=1, flags=q, none=False, table=p, n=4096):
        t = (_CAdamwTensor * 1)(_CAdamwTensor(*fields))
        blocks = C.c_int64(-7)
        at = None if none else C.addressof(t)
        rc = lib.fp8_adamw_table(at, count, flags, table, n, C.byref(blocks))
        assert (lib.fp8_adamw_table_bytes(at, count, flags) > 0) == (rc in (0, WORKSPACE) or table is None)
        return rc if rc else ("ok", blocks.value)

    for i in range(6):
        f = [p, p, p, p, p, p, 8]
        f[i] = None
        assert call(f) == NULL, i
        f[i] = p + (8 if i < 4 else 2)
        assert call(f) == ALIGN, i
    assert call((p, p, p, p, p, p, -1)) == SHAPE and call((p, p, p, p, p, p, 1 << 38)) == SHAPE
    assert call((None,) * 6 + (0,)) == ("ok", 0) and call(count=0) == ("ok", 0) and call(none=True) == NULL and call(count=-1) == SHAPE
    assert call((p, p, p, p, None, None, 8), flags=0) == ("ok", 1)
    assert call(flags=1) == ENUM and call(table=None) == NULL and call(n=8) == WORKSPACE
    assert lib.fp8_adamw_table(p, 0, 0, p, 4096, None) == NULL


@pytest.mark.parametrize("sizes", [[1], [2048, 2049, 0, 5], [16384 * 2048, 1], [16384 * 2048 + 1, 8193, 0, 3]])
def test_adamw_table_covers_every_element_once(sizes):
    """A header (blocks, flags), then 64 bytes for each workgroup: the pointers of its piece and how long it is."""
    import numpy as np
    base = [1 << 44, 2 << 44, 3 << 44, 4 << 44, 5 << 44, 6 << 44]
    for flags, bytes_of in ((0, (2, 2, 4, 4)), (fp8.FP8_ADAMW_PARAM_FP32 | fp8.FP8_ADAMW_STATE_FP8, (4, 2, 1, 1)), (fp8.FP8_ADAMW_GRAD_FP32, (2, 4, 4, 4))):
        array = (_CAdamwTensor * len(sizes))(*[_CAdamwTensor(*[b + (i << 40) for b in base], n) for i, n in enumerate(sizes)])
        table, blocks = fp8.fp8_adamw_table(array, len(sizes), flags)
        raw = table.numpy()
        assert raw[:8].view(np.int64)[0] == blocks and raw[8:12].view(np.int32)[0] == flags
        pieces = raw[64:].view(np.int64).reshape(-1, 8)
        assert len(pieces) == blocks
        want, q = [], flags & fp8.FP8_ADAMW_STATE_FP8
        for i, n in enumerate(sizes):
            for d in range(0, n, 2048):
                ptrs = [b + (i << 40) + d * s for b, s in zip(base, bytes_of)] + [b + (i << 40) + d // 256 * 4 if q else 0 for b in base[4:]]
                want.append(ptrs + [min(n - d, 2048), 0])
        assert np.array_equal(pieces, np.array(want, dtype=np.int64).reshape(-1, 8))


def test_adamw_step(lib, p):
    def call(table=p, blocks=1, flags=0, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.1, step=1, scale=None):
        return lib.fp8_adamw_step(table, blocks, flags, lr, b1, b2, eps, wd, step, scale, None)

    nan = float("nan")
    for bad in ({"lr": -1.0}, {"lr": nan}, {"b1": 1.0}, {"b1": nan}, {"b2": -0.1}, {"eps": -1.0}, {"wd": -1.0}, {"step": 0}, {"blocks": -1}, {"blocks": 1 << 24}):
        assert call(**bad) == SHAPE, bad
    assert call(flags=1) == ENUM and call(scale=p + 1) == ALIGN and call(table=None) == NULL and call(table=p + 8) == ALIGN
    assert call(blocks=0) == 0
