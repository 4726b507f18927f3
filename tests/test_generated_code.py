"""The library's machine code has no trace of a fault of its compiler (clang 22.0.0git of ROCm 7.2.0),
which loses the value of a short-circuited condition that writes part of a vector:

    for (int e = 0; e < 4; ++e)
      if (k + e >= K || (mask && !mask[k + e])) v[e] = -INFINITY;

leaves v[e] as it was where the mask closes it. What is left of the lost branch is an
empty one: the lanes are chosen (s_and_saveexec) and given back (s_or exec) with nothing between."""
import os
import re
import struct
import subprocess

import pytest

import paper_2506_09282_amd as hd
from paper_2506_09282_amd import build

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
LLVM = "/opt/rocm/llvm/bin"
LOSES = r"""
#include <hip/hip_runtime.h>
#include <stdint.h>
typedef float f32x4 __attribute__((ext_vector_type(4)));
__global__ void closed(const f32x4* s, const uint8_t* mask, int64_t K, f32x4* out) {
  const int64_t k = 4 * (int64_t)threadIdx.x;
  f32x4 v = {0, 0, 0, 0};
  if (k < K) v = s[threadIdx.x];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (k + e >= K || (mask && !mask[k + e])) v[e] = -INFINITY;
  out[threadIdx.x] = v;
}
"""


pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC) or not os.path.exists(LLVM),
                                reason="no hipcc")


def code_objects(blob: bytes):
    """The GPU code of a host library: every entry of its offload bundles."""
    at = blob.find(MAGIC)
    while at >= 0:
        (count,) = struct.unpack_from("<Q", blob, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(count):
            start, size, n = struct.unpack_from("<QQQ", blob, p)
            name = blob[p + 24:p + 24 + n]
            p += 24 + n
            if name.startswith(b"hip") and size:
                yield blob[at + start:at + start + size]
        at = blob.find(MAGIC, at + len(MAGIC))


def empty_branches(lines):
    """Functions that choose lanes and give them back at once: {name: how often}."""
    found, name, chosen = {}, "?", None
    for line in lines:
        m = re.match(r"^(?:[0-9a-f]+ )?<?(\w+)>?:", line)
        if m and not line.startswith("\t"):
            name, chosen = m.group(1), None
            continue
        s = line.split("//")[0].split(";")[0].strip()
        if not s or s.startswith("."):
            continue
        if chosen and re.match(r"s_or_b64 exec, exec, " + re.escape(chosen), s):
            found[name] = found.get(name, 0) + 1
        m = re.match(r"s_and_saveexec_b64 (s\[\d+:\d+\])", s)
        chosen = m.group(1) if m else None
    return found


def disassembled(path):
    r = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn",
                        "--no-leading-addr", path], capture_output=True, text=True, check=True)
    return r.stdout.splitlines()


def test_the_library(tmp_path):
    hd.lib()
    with open(hd.LIB_PATH, "rb") as f:
        objects = list(code_objects(f.read()))
    assert objects
    found, waits = {}, 0
    for i, code in enumerate(objects):
        path = tmp_path / f"{i}.co"
        path.write_bytes(code)
        lines = disassembled(str(path))
        waits += sum("s_and_saveexec_b64" in s for s in lines)
        found.update(empty_branches(lines))
    assert waits > 100  # (the code was read)
    assert not found, found


def test_the_form_that_is_lost_shows(tmp_path):
    """The search finds the fault where it is; a compiler without it makes this test void."""
    src, out = tmp_path / "closed.hip", tmp_path / "closed.co"
    src.write_text(LOSES)
    subprocess.run([build.HIPCC, *build.CFLAGS, "--cuda-device-only", "-c", str(src), "-o",
                    str(out)], capture_output=True, check=True)
    code = out.read_bytes()
    for i, c in enumerate(code_objects(code) if MAGIC in code else [code]):
        (tmp_path / f"{i}.co").write_bytes(c)
        if empty_branches(disassembled(str(tmp_path / f"{i}.co"))):
            return
    pytest.skip("this compiler keeps the value")
