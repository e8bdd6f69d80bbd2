"""CPU-only checks of the operators around the attention: what their entry points refuse on the host, before anything is
launched, and what the binding refuses."""
import ctypes

import pytest

from paper_2506_04648_amd import fps

torch = pytest.importorskip("torch")
GOOD, ODD = 0x10000, 0x10004               # an aligned address and one that is not; never followed by a refused call


def shape(**kw):
    return fps.make_shape(kw.pop("heads", 2), kw.pop("grid", (2, 3, 5)), kw.pop("tile", (1, 2, 2)), **kw)


def view(data=GOOD, dt=fps.OUT_BF16, B=1, heads=2, rows=30, cols=128, stride_b=0, stride_h=30 * 128, stride_r=128):
    return fps.View(data, dt, B, heads, rows, cols, stride_b, stride_h, stride_r)


def rotation(pairs=(22, 21, 21), table=GOOD, stride_b=0, pairing=0):
    return fps.Rotation(table, stride_b, *pairs, pairing)


BAD_VIEWS = [None, view(data=None), view(data=ODD), view(dt=2), view(B=2), view(heads=3), view(rows=29), view(cols=64),
             view(rows=0), view(stride_r=-128), view(stride_r=129), view(stride_h=30 * 128 + 4), view(stride_r=1 << 41)]
BAD_OUTPUTS = [view(stride_r=0), view(stride_h=0), view(stride_h=128), view(stride_h=29 * 128), view(stride_r=120)]
BAD_NORMS = [fps.Norm(ODD, 0, 1e-6)] + [fps.Norm(GOOD, 0, eps) for eps in (0.0, -1e-6, 1e-40, float("nan"), float("inf"))]
BAD_ROTATIONS = [rotation(table=None), rotation(table=ODD), rotation(pairs=(22, 21, 22)), rotation(pairs=(-1, 3, 3)),
                 rotation(pairs=(0, 65, 0)), rotation(stride_b=3), rotation(stride_b=-2), rotation(pairing=2)]


def refused(status, code=fps.FPS_ERR_INVALID_ARG):
    assert status == code and fps.last_error()


@pytest.mark.parametrize("i", range(len(BAD_VIEWS)))
def test_bad_inputs(i):
    L, s, v, bad, norm = fps.lib(), shape(), view(), BAD_VIEWS[i], fps.Norm(GOOD, 0, 1e-6)
    refused(L.fps_norm_rotate(s, bad, None, None, v, None))
    refused(L.fps_norm_rotate_operand(s, bad, None, None, 0, 1, GOOD, GOOD, None))
    refused(L.fps_norm_rotate_bwd(s, bad, norm, None, v, v, None, None, 0, None))
    refused(L.fps_norm_rotate_bwd(s, v, norm, None, bad, v, None, None, 0, None))


@pytest.mark.parametrize("i", range(len(BAD_VIEWS) + len(BAD_OUTPUTS)))
def test_bad_outputs(i):
    L, s, v, bad = fps.lib(), shape(), view(), (BAD_VIEWS + BAD_OUTPUTS)[i]
    refused(L.fps_norm_rotate(s, v, None, None, bad, None))
    refused(L.fps_norm_rotate_bwd(s, v, None, None, v, bad, None, None, 0, None))


@pytest.mark.parametrize("i", range(len(BAD_NORMS)))
def test_bad_norms(i):
    L, s, v, bad = fps.lib(), shape(), view(), BAD_NORMS[i]
    refused(L.fps_norm_rotate(s, v, bad, None, v, None))
    refused(L.fps_norm_rotate_operand(s, v, bad, None, 0, 1, GOOD, GOOD, None))
    refused(L.fps_norm_rotate_bwd(s, v, bad, None, v, v, None, None, 0, None))
    assert L.fps_norm_rotate_bwd_bytes(s, bad) == 0


@pytest.mark.parametrize("i", range(len(BAD_ROTATIONS)))
def test_bad_rotations(i):
    L, s, v, bad = fps.lib(), shape(), view(), BAD_ROTATIONS[i]
    refused(L.fps_norm_rotate(s, v, None, bad, v, None))
    refused(L.fps_norm_rotate_operand(s, v, None, bad, 0, 1, GOOD, GOOD, None))
    refused(L.fps_norm_rotate_bwd(s, v, None, bad, v, v, None, None, 0, None))


def test_the_rest_of_the_arguments():
    L, s, v = fps.lib(), shape(), view()
    norm, plain = fps.Norm(GOOD, 0, 1e-6), fps.Norm(None, 0, 1e-6)
    refused(L.fps_norm_rotate(None, v, None, None, v, None))
    refused(L.fps_norm_rotate(shape(head_dim=64), v, None, None, v, None), fps.FPS_ERR_UNSUPPORTED)
    long = shape(heads=1, grid=(1 << 20, 64, 64), tile=(32, 32, 32))
    refused(L.fps_norm_rotate(long, v, None, None, v, None), fps.FPS_ERR_UNSUPPORTED)
    for role, prec, out, scales in ((2, 1, GOOD, GOOD), (-1, 1, GOOD, GOOD), (0, 2, GOOD, GOOD), (0, 1, None, GOOD), (0, 1, GOOD, None),
                                    (0, 1, ODD, GOOD), (1, 1, GOOD, ODD), (1, 0, None, None)):
        refused(L.fps_norm_rotate_operand(s, v, norm, None, role, prec, out, scales, None))
    need = L.fps_norm_rotate_bwd_bytes(s, norm)
    assert need >= 512 and L.fps_norm_rotate_bwd_bytes(s, fps.Norm(GOOD, 1, 1e-6)) >= 1024
    refused(L.fps_norm_rotate_bwd(s, v, norm, None, v, v, GOOD, GOOD, need - 1, None), fps.FPS_ERR_WORKSPACE)
    refused(L.fps_norm_rotate_bwd(s, v, norm, None, v, v, GOOD, None, need, None))
    refused(L.fps_norm_rotate_bwd(s, v, norm, None, v, v, ODD, GOOD, need, None))
    refused(L.fps_norm_rotate_bwd(s, v, plain, None, v, v, GOOD, GOOD, need, None))
    refused(L.fps_norm_rotate_bwd(s, v, None, None, v, v, GOOD, GOOD, need, None))
    refused(L.fps_norm_rotate_bwd(s, v, norm, None, view(dt=1), v, None, None, 0, None))
    refused(L.fps_norm_rotate_bwd(s, v, norm, None, v, view(dt=1), None, None, 0, None))
    for role, vscale, dt, a, b, c in ((3, 0, 0, GOOD, GOOD, GOOD), (0, 2, 0, GOOD, GOOD, GOOD), (0, 0, 2, GOOD, GOOD, GOOD), (0, 0, 0, None, GOOD, GOOD),
                                      (0, 0, 0, GOOD, None, GOOD), (0, 0, 0, GOOD, GOOD, None), (0, 0, 0, GOOD, GOOD, ODD)):
        refused(L.fps_dequantize(s, a, b, role, vscale, dt, c, None))


def test_rotation_tables():
    L, s = fps.lib(), shape()
    assert L.fps_rotation_floats(s, rotation(table=None)) == 2 * (2 * 22 + 3 * 21 + 5 * 21)
    assert L.fps_rotation_floats(s, None) == 0 and L.fps_rotation_floats(s, rotation(pairs=(60, 5, 0))) == 0
    out, start = (ctypes.c_float * 1024)(), (ctypes.c_int64 * 3)(0, 0, 0)
    for base in (0.0, -1.0, float("nan"), float("inf")):
        refused(L.fps_rotation_table_host(s, rotation(), start, base, out))
    refused(L.fps_rotation_table_host(s, rotation(), (ctypes.c_int64 * 3)(1 << 53, 0, 0), 10.0, out))
    refused(L.fps_rotation_table_host(s, rotation(), start, 10.0, None))
    with pytest.raises(fps.FpsError):
        fps.rotation_table(s, (60, 5, 0))
    table = fps.rotation_table(s, (4, 4, 4), base=100.0)
    assert table.shape == (40, 2) and bool((table[0] == torch.tensor([1.0, 0.0])).all())


def test_the_binding_refuses():
    s = shape()
    x = torch.zeros(1, 2, 30, 128, dtype=torch.bfloat16)
    for call in (lambda: fps.norm_rotate(s, x), lambda: fps.norm_rotate_operand(s, x, 0), lambda: fps.norm_rotate_bwd(s, x, x)):
        with pytest.raises(ValueError, match="current device"):
            call()
    for weight in (torch.ones(64), torch.ones(128, dtype=torch.bfloat16), torch.ones(1, 2, 128), torch.ones(128, 2)[:, 0], torch.ones(2, 256)[:, ::2]):
        with pytest.raises(ValueError):
            fps.make_norm(weight)
    with pytest.raises(ValueError, match="heads"):
        fps.norm_rotate(s, x, fps.make_norm(torch.ones(3, 128)))
    for table in (torch.ones(10), torch.ones(10, 3), torch.ones(10, 2, dtype=torch.float64), torch.ones(2, 10).t()):
        with pytest.raises(ValueError):
            fps.make_rotation(table, (1, 1, 1))
    with pytest.raises(ValueError, match="entries"):
        fps.norm_rotate(s, x, rotation=fps.make_rotation(torch.ones(9, 2), (1, 1, 1)))
    with pytest.raises(ValueError, match="batch"):
        fps.norm_rotate(s, x, rotation=fps.make_rotation(torch.ones(2, 10, 2), (1, 1, 1)))
    for bad in (x[0], x[..., ::2], torch.zeros(1, 2, 3, 10, 128)[:, :, ::2, ::2]):
        with pytest.raises(ValueError):
            fps._view(bad, "x")
    with pytest.raises(ValueError):
        fps._view(x.to(torch.float16), "x")
    six = torch.zeros(1, 2, 2, 3, 5, 128)
    assert [getattr(fps._view(six, "x"), n) for n in ("dt", "rows", "stride_h", "stride_r")] == [1, 30, 30 * 128, 128]
    wide = torch.zeros(1, 30, 3, 2, 128)[:, :, 1].transpose(1, 2)
    assert [getattr(fps._view(wide, "x"), n) for n in ("rows", "stride_h", "stride_r")] == [30, 128, 768]


# ---- microscaled 4-bit floating point -----------------------------------------------------------
def matrix(data=GOOD, dt=fps.OUT_BF16, B=1, heads=1, rows=5, cols=70, stride_b=0, stride_h=0, stride_r=71):
    return fps.View(data, dt, B, heads, rows, cols, stride_b, stride_h, stride_r)


def test_packed_sizes():
    """32 rows by 256 columns are 4352 bytes."""
    L = fps.lib()
    for rows, cols, units in ((1, 1, 1), (32, 256, 1), (33, 256, 2), (32, 257, 2), (75600, 5120, 2363 * 20)):
        assert L.fps_mx4_bytes(rows, cols) == L.fps_mx4_linear_bytes(rows, cols) == 4352 * units
    for rows, cols in ((0, 5), (5, 0), (-1, 5), (1 << 31, 5), (5, 1 << 31), (1 << 30, 1 << 20)):
        assert L.fps_mx4_bytes(rows, cols) == 0 and "packed" in fps.last_error()
        with pytest.raises(fps.FpsError):
            fps.mx4_bytes(rows, cols)


BAD_MATRICES = [None, matrix(data=None), matrix(data=ODD), matrix(dt=2), matrix(rows=0), matrix(cols=0), matrix(stride_r=-1),
                matrix(heads=2, stride_h=71, stride_r=142), matrix(B=0)]
BAD_RESULTS = [matrix(stride_r=69), matrix(stride_r=0), matrix(B=2, stride_b=71), matrix(heads=2, cols=32, stride_h=0, stride_r=64)]


@pytest.mark.parametrize("i", range(len(BAD_MATRICES) + len(BAD_RESULTS)))
def test_bad_matrices(i):
    L, good = fps.lib(), matrix()
    bad, need = (BAD_MATRICES + BAD_RESULTS)[i], fps.mx4_bytes(5, 70)
    if i < len(BAD_MATRICES):
        refused(L.fps_mx4_quantize(bad, GOOD, None))
        refused(L.fps_mx4_linear(bad, GOOD, None, good, GOOD, need, None))
    refused(L.fps_mx4_dequantize(GOOD, bad, None))
    refused(L.fps_mx4_matmul(70, GOOD, GOOD, None, bad, None))
    refused(L.fps_mx4_linear(good, GOOD, None, bad, GOOD, need, None))


def test_the_rest_of_a_products_arguments():
    L, v = fps.lib(), matrix()
    need = fps.mx4_bytes(5, 70)
    big = matrix(rows=1 << 30, cols=1 << 14, stride_r=1 << 14)
    refused(L.fps_mx4_quantize(big, GOOD, None), fps.FPS_ERR_UNSUPPORTED)
    for p in (None, ODD):
        refused(L.fps_mx4_quantize(v, p, None))
        refused(L.fps_mx4_dequantize(p, v, None))
        refused(L.fps_mx4_matmul(70, p, GOOD, None, v, None))
        refused(L.fps_mx4_matmul(70, GOOD, p, None, v, None))
        refused(L.fps_mx4_linear(v, p, None, v, GOOD, need, None))
        refused(L.fps_mx4_linear(v, GOOD, None, v, p, need, None))
    refused(L.fps_mx4_matmul(70, GOOD, GOOD, ODD, v, None))
    refused(L.fps_mx4_linear(v, GOOD, ODD, v, GOOD, need, None))
    for K in (0, -1, 1 << 31, 1 << 40):
        refused(L.fps_mx4_matmul(K, GOOD, GOOD, None, v, None))
    refused(L.fps_mx4_linear(v, GOOD, None, matrix(rows=6), GOOD, need, None))
    assert "rows" in fps.last_error()
    refused(L.fps_mx4_linear(v, GOOD, None, v, GOOD, need - 1, None), fps.FPS_ERR_WORKSPACE)


def test_the_binding_refuses_products():
    x, w = torch.zeros(5, 70), torch.zeros(fps.mx4_bytes(9, 70), dtype=torch.uint8)
    for call in (lambda: fps.mx4_quantize(x), lambda: fps.mx4_dequantize(w, 9, 70), lambda: fps.mx4_linear(x, w, 9),
                 lambda: fps.mx4_matmul(w, w, 9, 9, 70)):
        with pytest.raises(ValueError, match="current device"):
            call()
    for bad in (torch.zeros(70), torch.zeros(70, 5).t(), x.to(torch.float16)):
        with pytest.raises(ValueError):
            fps.mx4_quantize(bad)
    for out in (torch.zeros(5, 8), torch.zeros(6, 9), torch.zeros(1, 3, 5, 32)):
        with pytest.raises(ValueError, match="not a matrix"):
            fps.mx4_linear(x, w, 9, out=out)
    three = torch.zeros(2, 5, 70)[:, 1:]
    assert [getattr(fps._matrix(three, "x")[0], n) for n in ("B", "heads", "rows", "cols", "stride_b", "stride_r")] == [2, 1, 4, 70, 350, 70]


def test_the_build_links_objects_alone(tmp_path, monkeypatch):
    """hipcc takes an object that follows a source for a source: each source is compiled by itself, once, and the link has objects only."""
    from paper_2506_04648_amd import build
    log, stub = tmp_path / "log", tmp_path / "hipcc"
    stub.write_text(f'#!/bin/sh\necho "$@" >> {log}\n')
    stub.chmod(0o755)
    monkeypatch.setenv("HIPCC", str(stub))
    monkeypatch.setattr(build, "OUT", str(tmp_path / "lib.so"))
    build.build_lib()
    commands = [line.split() for line in log.read_text().splitlines()]
    sources = sorted(a.rsplit("/", 1)[-1] for c in commands[:-1] for a in c if a.endswith((".hip", ".cpp")))
    assert sources == sorted(build.SOURCES) and all(sum(a.endswith((".hip", ".cpp")) for a in c) == 1 for c in commands[:-1])
    assert "-shared" in commands[-1] and not any(a.endswith((".hip", ".cpp")) for a in commands[-1])
    assert sum(a.endswith(".o") for a in commands[-1]) == len(build.SOURCES)
