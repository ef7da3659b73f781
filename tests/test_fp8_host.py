"""Host-side checks of the 8-bit products and the routing that need no GPU: exported symbols, planner, refusals."""
import ctypes
import os
import re

import numpy as np
import pytest

from paper_2512_02551_b200 import build as hbuild
from paper_2512_02551_b200 import fp8, hgemm, routing

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FORMS = ["forward", "input_grad", "weight_grad"]


@pytest.fixture(scope="module", autouse=True)
def lib():
    hbuild.build()
    return hgemm.lib()


@pytest.mark.parametrize("header,module", [("hgemm_fp8.h", fp8), ("hgemm_routing.h", routing)])
def test_header_symbols_are_exported(lib, header, module):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    declared = set(re.findall(r"\b(hgemm_[a-z0-9_]+)\s*\(", text))
    assert declared == set(module.EXPORTS)
    module.lib()
    checked = ctypes.CDLL(hbuild.build(checked=True))
    for name in declared:
        assert hasattr(lib, name) and hasattr(checked, name), name


def test_structures_match_the_headers(tmp_path):
    """Sizes and field offsets of the mirrors, against a C program that includes the headers."""
    import subprocess
    mirrors = {"hgemm_fp8_quantize_t": fp8.Quantize, "hgemm_fp8_config_t": fp8.Config, "hgemm_routing_t": routing.Routing}
    lines = []
    for c_name, cls in mirrors.items():
        lines.append(f'printf("%zu\\n", sizeof({c_name}));')
        lines += [f'printf("%zu\\n", offsetof({c_name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "hgemm_routing.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in mirrors.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def test_padded_rows():
    rng = np.random.default_rng(0)
    assert fp8.padded_rows(0, 0) == 0 and fp8.padded_rows(128, 0) == 128 and fp8.padded_rows(129, 0) == 256
    assert fp8.padded_rows(-1, 1) == -1 and fp8.padded_rows(5, 1025) == -1 and fp8.padded_rows((1 << 22) + 1, 1) == -1
    for _ in range(200):
        groups = int(rng.integers(1, 20))
        counts = rng.integers(0, 400, groups)
        need = int((-(-counts // 128) * 128).sum())
        assert need <= fp8.padded_rows(int(counts.sum()), groups) <= counts.sum() + 127 * groups + 128


@pytest.mark.parametrize("form", FORMS)
def test_planner_is_legal_everywhere(form):
    for M in (0, 1, 15, 16, 17, 33, 65, 129, 500, 1024, 8192, 1 << 22):
        for N in (1, 64, 100, 1024, 4096, 16384):
            for K in (1, 64, 127, 2048, 16384):
                for groups in (0, 1, 8, 64, 1024):
                    c = fp8.planned_config(form, M, N, K, groups)
                    assert (c.cta_group, c.block_q) in ([(2, 256), (1, 128)] if form == "weight_grad" else [(2, 256), (1, 16), (1, 32), (1, 64), (1, 128)])
                    assert c.split_k in (1, 2, 4, 8) and (c.cta_group == 1 or c.split_k == 1)


def test_refusals_before_any_gpu_work():
    L = fp8.lib()
    bad = hgemm.ERR_INVALID_ARG
    c = fp8.Config()
    for args in ((3, 1, 1, 1, 0), (-1, 1, 1, 1, 0), (0, -1, 1, 1, 0), (0, 1, 0, 1, 0), (0, 1, 1, 0, 0), (0, (1 << 22) + 1, 1, 1, 0), (0, 1, 1, 1, -1), (0, 1, 1, 1, 1025)):
        assert L.hgemm_fp8_planned_config(*args, 148, ctypes.byref(c)) == bad, args
    assert L.hgemm_fp8_planned_config(0, 1, 1, 1, 0, 0, ctypes.byref(c)) == bad
    assert L.hgemm_fp8_planned_config(0, 1, 1, 1, 0, 148, None) == bad
    h = ctypes.c_void_p()
    assert L.hgemm_fp8_plan(None, 0, 1, 1, 1, 0, 3, 3, 0, ctypes.byref(h)) == bad
    assert L.hgemm_fp8_plan_destroy(None) == bad
    assert L.hgemm_fp8_plan_get_config(None, ctypes.byref(c)) == bad and L.hgemm_fp8_plan_set_config(None, ctypes.byref(c)) == bad
    assert L.hgemm_fp8_run(None, None, 0, None, None, 0, None, None, 0, None, 0, None) == bad
    assert L.hgemm_fp8_quantize(None, None, None) == bad
    R = routing.lib()
    r = routing.Routing(8, 2, 0, 1, 1, 0, 1, 1.0)
    assert R.hgemm_route(None, ctypes.byref(r), 0, None, 0, 8, None, None, None, None) == bad
    assert R.hgemm_route_backward(None, ctypes.byref(r), 0, None, 0, 8, None, None, None, 8, None) == bad
    assert R.hgemm_route_sort(None, None, 0, 8, None, None, None, None) == bad
