"""The library's host code without a GPU: a script of calls over a CUDA runtime that does nothing (fake_runtime.c), in a process of its own."""
import json
import os
import shutil
import subprocess
import sys
from pathlib import Path

import pytest

from paper_2608_08020_gb300 import binding as B

HERE = Path(__file__).resolve().parent
CUDA = "/usr/local/cuda/include"

# What a script begins with: pools of every type, and calls of each entry.
CALLS = """
import ctypes, json, sys
from paper_2608_08020_gb300 import binding as B
fake, lib = ctypes.CDLL(sys.argv[1]), B.load()
AT, ROT = 1 << 20, B.GbRotation(1 << 20, 64, 32, 0)       # (addresses that nothing reads)


def pool(dtype):
    cfg = B.GbPoolConfig(2, 8, 2, 64 if dtype == B.GB_F32 else 128, 16, dtype, 64, 4, 8, 0)
    return B.gb_pool_init(cfg, AT, AT, 0)


def calls(p):
    yield "seed", lambda: B.gb_pool_seed(p, 2, 20, AT, AT, 0)
    for layer in range(2):
        yield f"append {layer}", lambda: B.gb_append_kv(p, layer, 3, AT, AT, 0)
    for layer in range(2):
        yield f"append rotated {layer}", lambda: B.gb_append_kv_rotated(p, layer, 3, ROT, AT, AT, 0)
    for flags in range(3):
        for layer in range(2):
            yield f"decode {flags} {layer}", lambda: B.gb_decode_attention(p, layer, AT, AT, AT, 0.1, AT, flags, 0)
        for layer in range(2):
            yield f"decode rotated {flags} {layer}", lambda: B.gb_decode_attention_rotated(p, layer, ROT, AT, AT, AT, 0.1, 2 * AT, flags, 0)
    yield "read_kv", lambda: B.gb_read_kv(p, 0, AT, 3, AT, AT, 0)
    yield "truncate", lambda: B.gb_truncate(p, AT, 0)
    yield "fork", lambda: B.gb_fork_slots(p, AT, 0)
    yield "release", lambda: B.gb_release(p, AT, 1, 0)
    yield "selftest", lambda: B.gb_pool_wait_selftest(p, 0)
    yield "mlp", lambda: B.gb_score_mlp(p, AT, 128, AT, AT, AT, 0.0, 64, None, None, 0)


def code(f):
    try:
        f()
        return 0, ""
    except B.GambitError as e:
        return e.code, str(e)


"""


@pytest.fixture(scope="module")
def host_only(tmp_path_factory):
    if not B.LIB_PATH.exists() or shutil.which("gcc") is None or not Path(CUDA).exists():
        pytest.skip("libgambit.so, gcc or the CUDA headers missing")
    so = tmp_path_factory.mktemp("fake") / "fake.so"
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-I", CUDA, "-o", str(so), str(HERE / "fake_runtime.c")], check=True)

    def go(script):
        r = subprocess.run([sys.executable, "-c", script, str(so)], cwd=HERE.parent, capture_output=True, text=True, timeout=120,
                           env={**os.environ, "LD_PRELOAD": str(so)})
        assert r.returncode == 0, r.stdout + r.stderr
        return json.loads(r.stdout)

    return go
