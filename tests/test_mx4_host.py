"""CPU-only checks of the MXFP4 operators: sizes, refusals of the C ABI and of the Python calls (no kernel is launched), and the plain
64-bit form that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import synthetic_inputs as si
from tests import mx4_plain as plain


@pytest.fixture(scope="module")
def P():
    import paper_2410_06916_amd as P
    P.lib()
    return P


def test_packed_sizes(P):
    from paper_2410_06916_amd import mx4
    # whole tiles: 17 bytes for every 32 weights
    assert mx4.packed_bytes(4096, 4096) == 4096 * 4096 // 32 * 17
    assert mx4.packed_bytes(11008, 4096, True) == 2 * 11008 * 4096 // 32 * 17
    # 16 rows x 128 of depth are the least (8 + 8 rows of a gated pair)
    assert mx4.packed_bytes(1, 1) == mx4.packed_bytes(16, 128) == 1088
    assert mx4.packed_bytes(1, 1, True) == mx4.packed_bytes(8, 128, True) == 1088
    assert mx4.packed_bytes(17, 129) == 4 * 1088
    # sizes past 32 bits
    assert mx4.packed_bytes(1 << 22, 1 << 22) == (1 << 44) // 32 * 17
    for bad in ((0, 1), (1, 0), (-1, 5), ((1 << 22) + 1, 1), (1, (1 << 22) + 1)):
        with pytest.raises(P.SwiftError):
            mx4.packed_bytes(*bad)
    assert P.lib().swift_mx4_bytes(1, 1, 0, None) == -1


def test_refusals_of_the_c_abi(P):
    """Nothing is launched: every call has one argument wrong (the pointers are never followed)."""
    L = P.lib()
    a = 1 << 20  # some aligned address
    n = C.c_uint64()
    assert L.swift_mx4_workspace(64, 256, 0, 4, 1, C.byref(n)) == 0
    ws = n.value
    quant = dict(packed=a, w=a, ld_w=256, up=None, ld_up=0, dtype=1, rows=64, depth=256, stream=None)
    for change, code in ((dict(packed=None), -1), (dict(w=None), -1), (dict(packed=a + 128), -1), (dict(w=a + 1), -1), (dict(ld_w=255), -1),
                         (dict(up=a, ld_up=255), -1), (dict(up=a + 1, ld_up=256), -1), (dict(dtype=2), -1), (dict(dtype=0, w=a + 2), -1), (dict(rows=0), -1),
                         (dict(depth=0), -1), (dict(rows=(1 << 22) + 1), -1), (dict(depth=1 << 23), -1)):
        assert L.swift_mx4_quantize(*{**quant, **change}.values()) == code, change
    deq = dict(w=a, ld_w=256, dtype=1, packed=a, rows=64, depth=256, gated=0, stream=None)
    for change in (dict(w=None), dict(packed=None), dict(ld_w=255), dict(dtype=3), dict(packed=a + 16), dict(w=a + 1), dict(rows=-1), dict(depth=0)):
        assert L.swift_mx4_dequantize(*{**deq, **change}.values()) == -1, change
    lin = dict(y=a, ld_y=64, y_dtype=1, x=a, ld_x=256, x_dtype=1, n=4, packed=a, rows=64, depth=256, residual=None, ld_r=0, ws=a, ws_bytes=ws, stream=None)
    wrong = ((dict(y=None), -1), (dict(x=None), -1), (dict(packed=None), -1), (dict(ld_y=63), -1), (dict(ld_x=255), -1), (dict(residual=a, ld_r=63), -1),
             (dict(residual=a + 1, ld_r=64), -1), (dict(y_dtype=2), -1), (dict(x_dtype=-1), -1), (dict(n=-1), -1), (dict(rows=0), -1), (dict(depth=0), -1),
             (dict(y=a + 1), -1), (dict(x=a + 1), -1), (dict(x=a + 2, x_dtype=0), -1), (dict(packed=a + 64), -1))
    for change, code in wrong:
        assert L.swift_mx4_linear(*{**lin, **change}.values()) == code, change
    glu = {k: v for k, v in lin.items() if k not in ("residual", "ld_r")}
    for change, code in wrong:
        if not change.keys() & {"residual", "ld_r"}:
            assert L.swift_mx4_swiglu(*{**glu, **change}.values()) == code, change
    # no rows: nothing to do, and nothing is looked at
    assert L.swift_mx4_linear(*{**lin, "n": 0, "x": None, "y": None, "ws": None, "ws_bytes": 0}.values()) == 0
    assert L.swift_mx4_swiglu(*{**glu, "n": 0, "x": None, "y": None, "ws": None, "ws_bytes": 0}.values()) == 0
    for bad in ((0, 256, 0, 4, 1), (64, 256, 0, -1, 1), (64, 256, 0, 4, 2)):
        assert L.swift_mx4_workspace(*bad, C.byref(n)) == -1
    assert L.swift_mx4_workspace(64, 256, 0, 4, 1, None) == -1


def test_a_workspace_too_small_is_refused(P):
    """Wherever a workspace is asked for, one byte less of it is refused before anything is enqueued."""
    L, a, n = P.lib(), 1 << 20, C.c_uint64()
    for rows, depth, m, dt in ((64, 256, 4, 0), (64, 257, 4, 1), (4096, 4096, 9, 0), (4096, 4096, 2000, 1), (4096, 4096, 2000, 0)):
        assert L.swift_mx4_workspace(rows, depth, 0, m, dt, C.byref(n)) == 0
        for ws, size in ((a, n.value - 1), (None, n.value), (a + 128, n.value)):
            if n.value:
                assert L.swift_mx4_linear(a, rows, 0, a, depth, dt, m, a, rows, depth, None, 0, ws, size, None) == -2
        if n.value:
            assert "workspace" in L.swift_last_error().decode()


def test_refusals_of_the_python_calls(P):
    w = torch.zeros(8, 64)
    with pytest.raises(ValueError, match="GPU"):
        P.mx4_quantize(w)
    with pytest.raises(TypeError):
        P.mx4_quantize(w.half())
    with pytest.raises(TypeError):
        P.mx4_quantize(w.double())
    with pytest.raises(ValueError):
        P.Mx4Weight(8, 64, False, torch.zeros(1087, dtype=torch.uint8))
    with pytest.raises(ValueError):
        P.Mx4Weight(8, 64, False, torch.zeros(1088, dtype=torch.int8))
    m = P.Mx4Weight(8, 64, False, torch.zeros(1088, dtype=torch.uint8))
    g = P.Mx4Weight(8, 64, True, torch.zeros(1088, dtype=torch.uint8))
    with pytest.raises(ValueError, match="gated"):
        P.mx4_linear(w, g)
    with pytest.raises(ValueError, match="gated"):
        P.mx4_swiglu(w, m)
    with pytest.raises(ValueError, match="GPU"):
        P.mx4_linear(w, m)
    with pytest.raises(TypeError):
        P.mx4_linear(w.to(torch.float64), m)
    with pytest.raises(TypeError):
        P.mx4_dequantize(m, torch.float16)


def test_a_model_of_mxfp4_matrices_is_sized_and_accounted_for(P):
    import dataclasses

    from paper_2410_06916_amd import binding as B
    bf = si.LLAMA2_7B
    mx = dataclasses.replace(bf, dtype="mxfp4")
    c16, c4 = B.make_config(bf, 1024), B.make_config(mx, 1024)
    assert P.check_config(c4) == 0
    layers = bf.n_layers * (bf.attn_sublayer_elems() + bf.mlp_sublayer_elems())
    assert P.device_bytes(c16) - P.device_bytes(c4) == 2 * layers - layers // 32 * 17
    assert P.pass_bytes(c16, None, 100, 1) - P.pass_bytes(c4, None, 100, 1) == 2 * layers - layers // 32 * 17
    m = np.zeros(64, np.uint8)
    m[2 * 5 + 1] = 1
    assert P.pass_bytes(c4, None, 100, 1) - P.pass_bytes(c4, m, 100, 1) == bf.mlp_sublayer_elems() // 32 * 17 + 4 * bf.hidden
    # a depth that fills no block: what is left of a row's last block has a scale too
    odd = dataclasses.replace(si.TINY, hidden=264, ffn=40, n_q_heads=4, dtype="mxfp4")
    got = P.pass_bytes(B.make_config(odd, 64), None, 0, 1)
    q, kv, h, f = odd.q_dim, odd.kv_dim, odd.hidden, odd.ffn
    blocks = lambda rows, k: rows * (-(-k // 32)) * 17  # noqa: E731
    want = odd.vocab * h * 2 + 4 * h + 2 * h
    want += odd.n_layers * (blocks(q + 2 * kv, h) + blocks(h, q) + 4 * h + 4 * kv + blocks(2 * f, h) + blocks(h, f) + 4 * h)
    assert got == want


def test_the_plain_form_of_the_format():
    """Values worked out by hand: a block's scale, ties to even codes, saturation, a short last block, what no scale reaches."""
    w = torch.zeros(4, 40)
    w[0, :8] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])   # scale 1: every tie
    w[1, :4] = torch.tensor([7.9, -7.9, 0.3, -0.2])                          # scale 1: past 6 stays 6
    w[2, 32:] = 3.0                                                          # a block of 8: scale 1/2, 6 x 1/2
    w[3, :2] = torch.tensor([2.0 ** -126, 2.0 ** -128])                      # least scale 2^-127: 2 and 1/2
    v = plain.values(w)
    assert v[0, :8].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    assert v[1, :4].tolist() == [6.0, -6.0, 0.5, 0.0]
    assert v[2, 32:].tolist() == [3.0] * 8
    assert v[3, :2].tolist() == [2.0 ** -126, 2.0 ** -128]
    assert torch.equal(plain.values(v.float()), v)                           # reading back and quantising again changes nothing
    w[0, 5] = float("inf")
    w[1, 6] = float("nan")
    v = plain.values(w)
    assert v[:2, :32].isnan().all() and not v[:2, 32:].isnan().any() and not v[2:].isnan().any()


def test_sizes_past_32_bits_are_refused_not_cut(P):
    """2^32 + 16 would arrive in the library as 16; a great number of rows (three columns each in fp32) still asks for the blocked product's
    workspace, which is that of 5376 rows whatever lies beyond."""
    from paper_2410_06916_amd import mx4
    for sides in (((1 << 32) + 16, 128), (128, (1 << 32) + 16), (1 << 31, 1)):
        with pytest.raises(ValueError):
            mx4.packed_bytes(*sides)
        with pytest.raises(ValueError):
            mx4.Mx4Weight(*sides, False, torch.zeros(1088, dtype=torch.uint8))
    n, least = C.c_uint64(), C.c_uint64()
    for dt in (0, 1):
        assert P.lib().swift_mx4_workspace(16, 128, 0, 128 * 42, dt, C.byref(least)) == 0
        for rows in (128 * 42 + 1, 715827883, 1431655766, (1 << 31) - 1):
            assert P.lib().swift_mx4_workspace(16, 128, 0, rows, dt, C.byref(n)) == 0
            assert n.value == least.value, (dt, rows)
