"""Host-side checks of the 4-bit operands that need no GPU: the reference's own tables, exported symbols, structures, planner, refusals."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import fp4_reference as ref
from paper_2512_02551_b200 import build as hbuild
from paper_2512_02551_b200 import fp4, hgemm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FORMS = ["forward", "input_grad", "weight_grad"]


@pytest.fixture(scope="module", autouse=True)
def lib():
    hbuild.build()
    return hgemm.lib()


def test_header_symbols_are_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hgemm_fp4.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(hgemm_[a-z0-9_]+)\s*\(", text))
    assert declared == set(fp4.EXPORTS)
    fp4.lib()
    checked = ctypes.CDLL(hbuild.build(checked=True))
    for name in declared:
        assert hasattr(lib, name) and hasattr(checked, name), name


def test_structures_match_the_header(tmp_path):
    """Sizes and field offsets of the mirrors, against a C program that includes the header."""
    mirrors = {"hgemm_fp4_quantize_t": fp4.Quantize, "hgemm_fp4_config_t": fp4.Config}
    lines = []
    for c_name, cls in mirrors.items():
        lines.append(f'printf("%zu\\n", sizeof({c_name}));')
        lines += [f'printf("%zu\\n", offsetof({c_name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "hgemm_fp4.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in mirrors.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def test_reference_tables():
    """The tests' own e4m3 and e2m1 against torch's types and against differences of neighbours."""
    e4m3 = torch.arange(128, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.E4M3, e4m3, equal_nan=True)
    v = np.linspace(0, 460, 40001).astype(np.float32)
    want = torch.from_numpy(np.minimum(v, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.nearest_e4m3(v), want)
    assert [int(c) for c in ref.nearest_code(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, 7.0, -0.0]))] == [0, 2, 2, 4, 4, 6, 6, 14, 7, 8]
    assert list(fp4.VALUES) == list(ref.decode(np.arange(16)))


def test_reference_layout_round_trips():
    rng = np.random.default_rng(1)
    for fmt in ("nvfp4", "mxfp4"):
        for R, C in ((1, 1), (128, 64), (130, 300), (300, 129)):
            b = rng.integers(0, 256, (R, ref.blocks(C, fmt)), dtype=np.uint8)
            t = torch.from_numpy(ref.tiles_from(b, fmt))
            assert t.numel() == fp4.lib().hgemm_fp4_scale_bytes(R, C, fp4.FORMATS[fmt])
            assert tuple(t.shape) == tuple(fp4.empty_rows(R, C, format=fmt, device="cpu")[1].shape)
            assert np.array_equal(ref.scale_bytes(t, R, C, fmt), b)
            assert np.array_equal(fp4.scale_matrix(t, R, C, fmt).view(torch.uint8).numpy(), b)
            c = rng.integers(0, 16, (R, C), dtype=np.uint8)
            assert np.array_equal(ref.codes(torch.from_numpy(ref.pack(c)), C), c)


def test_buffers():
    q, s = fp4.empty_rows(5, 77, device="cpu")
    assert q.shape == (5, 39) and q.stride(0) == 48 and s.shape == (1, 2, 512)
    q, s = fp4.empty_cols(5, 77, format="mxfp4", device="cpu")
    assert q.shape == (77, 3) and q.stride(0) == 16 and s.shape == (1, 1, 512)
    rows = fp4.padded_rows(300, 4)
    q, s = fp4.empty_cols(300, 77, groups=4, device="cpu")
    assert q.shape == (77, rows // 2) and s.shape == (1, rows // 64, 512)
    q, s = fp4.empty_rows(300, 77, groups=4, device="cpu")
    assert q.shape == (300, 39) and s.shape == (rows // 128, 2, 512)
    q, s = fp4.empty_rows(3, 200, 64, device="cpu")
    assert q.shape == (3, 200, 32) and s.shape == (3, 2, 1, 512)


@pytest.mark.parametrize("form", FORMS)
def test_planner_is_legal_everywhere(form):
    for M in (0, 1, 15, 16, 17, 33, 65, 129, 500, 1024, 8192, 1 << 22):
        for N in (1, 64, 100, 1024, 4096, 16384):
            for K in (1, 64, 127, 2048, 16384):
                for groups in (0, 1, 8, 64, 1024):
                    c = fp4.planned_config(form, M, N, K, groups)
                    assert (c.cta_group, c.block_q) in [(2, 256), (2, 128), (1, 64), (1, 128)]
                    assert c.split_k in (1, 2, 4, 8) and (c.cta_group == 1 or c.split_k == 1)


def test_refusals_before_any_gpu_work():
    L = fp4.lib()
    bad = hgemm.ERR_INVALID_ARG
    c = fp4.Config()
    for args in ((3, 1, 1, 1, 0), (-1, 1, 1, 1, 0), (0, -1, 1, 1, 0), (0, 1, 0, 1, 0), (0, 1, 1, 0, 0), (0, (1 << 22) + 1, 1, 1, 0), (0, 1, 1, 1, -1), (0, 1, 1, 1, 1025)):
        assert L.hgemm_fp4_planned_config(*args, 148, ctypes.byref(c)) == bad, args
    assert L.hgemm_fp4_planned_config(0, 1, 1, 1, 0, 0, ctypes.byref(c)) == bad
    assert L.hgemm_fp4_planned_config(0, 1, 1, 1, 0, 148, None) == bad
    h = ctypes.c_void_p()
    assert L.hgemm_fp4_plan(None, 0, 1, 1, 1, 0, 0, 0, ctypes.byref(h)) == bad
    assert L.hgemm_fp4_plan_destroy(None) == bad
    assert L.hgemm_fp4_plan_get_config(None, ctypes.byref(c)) == bad and L.hgemm_fp4_plan_set_config(None, ctypes.byref(c)) == bad
    assert L.hgemm_fp4_run(None, None, 0, None, None, None, 0, None, None, None, 0, None, 0, None) == bad
    assert L.hgemm_fp4_quantize(None, None, None) == bad
    assert L.hgemm_fp4_tensor_factor(None, 0, 1, 1, 1, None, 1, None, None) == bad
    assert L.hgemm_fp4_dequantize(None, 0, 0, 1, 1, 1, None, 16, None, None, None, 0, None, 1, None) == bad
    assert L.hgemm_fp4_scale_bytes(-1, 1, 0) == -1 and L.hgemm_fp4_scale_bytes(1, 1, 2) == -1


def test_binding_refuses_what_does_not_fit():
    """Shapes, types and factors are looked at before the library is called (CPU tensors: none of these calls reaches a GPU)."""
    x = torch.zeros(4, 64)
    q, s = fp4.empty_rows(4, 64, device="cpu")
    for call in (lambda: fp4.quantize_rows(None, x, q, s, factor=torch.ones(1)), lambda: fp4.quantize_rows(None, x, q, s), lambda: fp4.quantize_rows(None, x, q, s, format="int4"),
                 lambda: fp4.tensor_factor(None, x, torch.ones(1)), lambda: fp4.tensor_factor(None, x[0], torch.ones(1)), lambda: fp4.dequantize(None, q, s, x, factor=torch.ones(1)),
                 lambda: fp4.Plan(None, 1, 1, 1, form="backward"), lambda: fp4.Plan(None, 1, 1, 1, out_dtype=torch.int8), lambda: fp4.empty_rows(4, 64, format="fp4")):
        with pytest.raises(ValueError):
            call()
