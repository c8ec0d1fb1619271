"""The host side of the multi-token step under the undefined-behaviour sanitizer: its translation unit is built again with
-fsanitize=undefined and float-cast-overflow beside libpad.so, and plans of every kind (host only, nothing is launched) and
rotary specs go through it in a process of their own, whose reports are read from its standard error."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2607_02963_gb300 import build
from paper_2607_02963_gb300 import binding as B

HEAD = f"""
import ctypes, sys
sys.path.insert(0, {build.ROOT!r})
import numpy as np, torch
from paper_2607_02963_gb300 import binding as B
L = ctypes.CDLL(sys.argv[1])
for name, (res, args) in B._SIGNATURES.items():
    f = getattr(L, name)
    f.restype, f.argtypes = res, args
B._lib = L
"""

PLANS = HEAD + """
def plan(fmt, lens, news, prefix=None, video=None, h_q=28, h_kv=4, d=128, page=16, flags=0, sms=152):
    prob = B.make_problem(h_q, h_kv, d, page, flags=flags, num_sms=sms)
    B.pad_chunk_workspace_size(prob, prefix, video, lens, news, kv_format=fmt)
    table = torch.full((len(lens), 4096), -1, dtype=torch.int32)
    p = B.pad_chunk_plan(prob, None, prefix, video, lens, news, page_table=table, n_pages=9000, kv_format=fmt)
    return p.info()

count = 0
for fmt in (B.KV_BF16, B.KV_FP8, B.KV_FP4):
    for flags in (0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC):
        for shape in (dict(), dict(h_q=14, h_kv=2, d=64, page=64), dict(h_q=16, h_kv=1, page=4), dict(h_q=2, h_kv=2, sms=1)):
            for lens, news in (([5], [1]), ([0, 40], [0, 0]), ([0], [300]), ([9000, 3, 0], [1, 7, 0]), ([100] * 40, [5] * 40)):
                for prefix in (None, [0], [3001]):
                    plan(fmt, lens, news, prefix, None if prefix is None else [0] * len(lens), flags=flags, **shape)
                    count += 1
    plan(fmt, [], [])
print(count + 1, "plans")
"""

ROPES = HEAD + """
count = 0
for scaling in B.Rope.SCALINGS:
    for rotary in (4, 54, 128):
        for theta in (1e-3, 1.5, 1e4, 1e300):
            for factor in (1e-3, 4.0, 1e300):
                try:
                    B.Rope(128, rotary, theta, scaling=scaling, factor=factor, original_len=4096.0, low=1.0, high=32.0)
                except B.PadError:
                    pass
                count += 1
print(count, "specs")
"""


@pytest.fixture(scope="module")
def sanitized(padlib, tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    out = tmp_path_factory.mktemp("sanitized")
    obj, so, at = out / "api.o", out / "libpad_chunk_sanitized.so", os.path.dirname(B.lib_path())
    flags = [f for f in build.CFLAGS if f not in ("-O3", "-lineinfo")] + ["-O1"]
    subprocess.run([build._nvcc(), "-c", os.path.join(build.CSRC, "pad_chunk_api.cu"), "-o", obj, *flags, "-Xcompiler",
                    "-fsanitize=undefined,-fsanitize=float-cast-overflow"], check=True)
    subprocess.run([build._nvcc(), obj, "-o", so, *(f for f in build.LDFLAGS if f != "-lcuda"), "-Xcompiler", "-fsanitize=undefined", "-L" + at, "-l:libpad.so",
                    "-Xlinker", "-rpath," + at], check=True)
    return str(so)


@pytest.mark.parametrize("script", [PLANS, ROPES], ids=["plans", "ropes"])
def test_no_undefined_behaviour(sanitized, script):
    r = subprocess.run([sys.executable, "-c", script, sanitized], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout, r.stderr
    assert "runtime error" not in r.stderr, r.stderr
