"""Registers and private memory of the kernels in the built library, as its own
metadata has them: a kernel laid out for registers does not go through memory."""
import os
import re
import shutil
import struct
import subprocess

import pytest
import yaml

from paper_2607_24981_amd import build, ilw

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(data):
    """The device code objects of the bundles that lie in the library's bytes."""
    for m in re.finditer(MAGIC, data):
        at, (n,) = m.start(), struct.unpack_from("<Q", data, m.end())
        p = m.end() + 8
        for _ in range(n):
            offset, size, name = struct.unpack_from("<QQQ", data, p)
            target = data[p + 24:p + 24 + name].decode()
            p += 24 + name
            if "gfx950" in target:
                yield data[at + offset:at + offset + size]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """name -> metadata of every kernel."""
    root = os.path.dirname(os.path.dirname(os.path.realpath(build.hipcc())))
    tool = next((t for t in (os.path.join(root, "llvm", "bin", "llvm-readelf"),
                             "/opt/rocm/llvm/bin/llvm-readelf", shutil.which("llvm-readelf"))
                 if t and os.path.exists(t)), None)
    if tool is None or not os.path.exists(ilw.LIB_PATH):
        pytest.skip("needs the built library and llvm-readelf")
    out = {}
    with open(ilw.LIB_PATH, "rb") as f:
        objects = list(code_objects(f.read()))
    for i, obj in enumerate(objects):
        path = tmp_path_factory.mktemp("co") / f"{i}.co"
        path.write_bytes(obj)
        text = subprocess.run([tool, "--notes", str(path)], capture_output=True, text=True,
                              check=True).stdout
        for doc in re.findall(r"^\s*---$(.*?)^\.\.\.$", text, re.S | re.M):
            for k in yaml.safe_load(doc).get("amdhsa.kernels", []):
                out[k[".name"]] = k
    return out


def named(kernels, name):
    """Those of one kernel template or function (by its length-prefixed name)."""
    return {k: v for k, v in kernels.items() if f"{len(name)}{name}" in k}


@pytest.mark.parametrize("name,instances", [
    ("append_kernel", 2), ("cache_rows_kernel", 24), ("cache_few_kernel", 12),
    ("split_scores_kernel", 12), ("split_values_kernel", 12), ("split_join_kernel", 4), ("grouped_kernel", 8)])
def test_no_private_memory(kernels, name, instances):
    """No spills, and no array that is indexed in memory."""
    found = named(kernels, name)
    assert len(found) == instances
    bad = {k: (v[".private_segment_fixed_size"], v[".vgpr_spill_count"]) for k, v in found.items()
           if v[".private_segment_fixed_size"] or v[".vgpr_spill_count"]}
    assert not bad


@pytest.mark.parametrize("name", ["cache_rows_kernel", "cache_few_kernel", "split_scores_kernel",
                                  "split_values_kernel"])
def test_two_waves_a_simd(kernels, name):
    """256 registers a lane at most, accumulation registers among them."""
    assert max(v[".vgpr_count"] for v in named(kernels, name).values()) <= 256
