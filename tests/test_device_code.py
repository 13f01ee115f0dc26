"""The GPU code that the compiler is given (CPU only: LLVM IR of code built here): the alignment that each access of global
memory is taken to have, and what inline assembly says that it changes.

The header promises 16 bytes for logits, codes and scales and an element's size for rows; an access that claims more is
undefined for what the header allows."""
import concurrent.futures
import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def ir(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not installed")
    spec = importlib.util.spec_from_file_location("eqb_build_flags", os.path.join(ROOT, "paper_2609_28053_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    flags = [f for f in build.FLAGS if f not in ("-shared", "-O3")]
    out = tmp_path_factory.mktemp("ir")

    def compiled(name):
        to = str(out / (name + ".ll"))
        subprocess.run([HIPCC, *flags, "-O1", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S",
                        "-emit-llvm", os.path.join(build.CSRC, name + ".hip"), "-o", to], check=True, capture_output=True)
        with open(to) as f:
            return f.read()

    names = ("codes", "scored", "products")
    with concurrent.futures.ThreadPoolExecutor(3) as pool:
        return dict(zip(names, pool.map(compiled, names)))


def accesses(text):
    """(type, alignment) of every access of global memory."""
    found = re.findall(r"(?:load|store) (<\d+ x \w+>|\w+)(?: [^,\n]+)?, ptr addrspace\(1\) [^,]+, align (\d+)", text)
    return [(t, int(a)) for t, a in found]


@pytest.mark.parametrize("name", ["codes", "scored", "products"])
def test_no_access_claims_more_than_sixteen_bytes(ir, name):
    found = accesses(ir[name])
    assert len(found) > 100
    assert not [f for f in found if f[1] > 16]


@pytest.mark.parametrize("name", ["codes", "products"])
def test_rows_may_begin_at_any_element(ir, name):
    """Eight elements of a row (as the compiler has them: a vector, or what stores of results were cast to)."""
    size = {"i16": 2, "half": 2, "bfloat": 2, "float": 4}
    rows = [(t, a) for t, a in accesses(ir[name]) if re.fullmatch(r"<8 x (i16|half|bfloat|float)>", t)]
    assert len(rows) > 50
    assert not [(t, a) for t, a in rows if a > size[t[5:-1]]]


def test_assembly_that_writes_m0_says_so(ir):
    calls = re.findall(r'asm sideeffect "([^"]*)", "([^"]*)"', ir["products"])
    written = [c for c in calls if re.search(r"s_mov_b32 m0", c[0])]
    assert len(written) > 50 and all("~{m0}" in c[1] for c in written)
