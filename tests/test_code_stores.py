"""Stores of sixteen codes promise the compiler no alignment: a tensor of codes may begin at any byte, and a compiler that is told otherwise may use it."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCE = """#include "%s/paper_2505_20524_amd/csrc/common.h"
extern "C" __global__ void codes(uint8_t* p, const uint4* v) { %s(p, *v); }
extern "C" __global__ void halves(uint16_t* p, const uint4* v) { %s(p, *v); }
"""


@pytest.mark.parametrize("store", ["st_any16", "st_any_nt16"])
def test_alignment_of_the_stores(tmp_path, store):
    source = tmp_path / "stores.hip"
    source.write_text(SOURCE % (ROOT, store, store))
    out = subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-device-only", "-O1", "-std=c++17", "-S", "-emit-llvm", "-o", "-", str(source)], capture_output=True, text=True)
    assert out.returncode == 0, out.stderr
    for kernel, want in (("codes", "1"), ("halves", "2")):
        body = re.search(r"define [^\n]*@%s\(.*?\n}" % kernel, out.stdout, re.S).group(0)
        assert re.findall(r"store <4 x i32>.*?align (\d+)", body) == [want], body
