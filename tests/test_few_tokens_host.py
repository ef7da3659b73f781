"""Host-side checks of the layer of experts for a few tokens that need no GPU."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2512_02551_b200 import build as hbuild
from paper_2512_02551_b200 import few_tokens, hgemm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    hbuild.build()
    return hgemm.lib()


def test_header_symbols_are_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hgemm_few_tokens.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(hgemm_[a-z0-9_]+)\s*\(", text))
    assert declared == set(few_tokens.EXPORTS)
    few_tokens.lib()
    checked = ctypes.CDLL(hbuild.build(checked=True))
    for name in declared:
        assert hasattr(lib, name) and hasattr(checked, name), name


def test_structures_match_the_header(tmp_path):
    mirrors = {"hgemm_few_tokens_t": few_tokens.Description, "hgemm_expert_weights_t": few_tokens.Weights}
    lines = []
    for c_name, cls in mirrors.items():
        lines.append(f'printf("%zu\\n", sizeof({c_name}));')
        lines += [f'printf("%zu\\n", offsetof({c_name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "hgemm_few_tokens.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in mirrors.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def test_scratch_and_descriptions():
    L, D = few_tokens.lib(), few_tokens.Description
    good = dict(hidden=100, inner=130, experts=4, top_k=2, weights=16, activation=1, type=2, reserved=0)
    size = lambda tokens, **kw: L.hgemm_few_tokens_scratch(ctypes.byref(D(**{**good, **kw})), tokens)  # noqa: E731
    assert size(0) == 0 and size(3, weights=2) == 3 * 2 * 160 * 4
    assert 3 * 2 * (8 * 80 + 4 * 260) < size(3) < 1 << 20 and size(64) > size(3) and size(3) % 256 == 0
    for kw in (dict(hidden=0), dict(inner=0), dict(hidden=(1 << 20) + 1), dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=33), dict(weights=0), dict(weights=1), dict(activation=2),
               dict(type=0)):
        assert size(1, **kw) == -1, kw
    assert size(-1) == -1 and size(65) == -1 and L.hgemm_few_tokens_scratch(None, 1) == -1
    assert L.hgemm_few_tokens(None, None, 1, None, 1, None, None, None, None, None, 1, None, 0, None) == hgemm.ERR_INVALID_ARG


def test_binding_refuses_what_does_not_fit():
    for kw in (dict(weights="int4"), dict(activation="relu"), dict(dtype=torch.float32), dict(weights="f16"), dict(weights="bf16", dtype=torch.float16)):
        with pytest.raises(ValueError):
            few_tokens.Layer(None, 64, 64, 2, 1, **kw)
    layer = few_tokens.Layer(None, 64, 64, 2, 1)
    assert layer.scratch_bytes(2) > 2 * 128 * 4 and layer.empty_scratch(0, device="cpu").numel() == 16
    with pytest.raises(ValueError):
        layer.scratch_bytes(65)
