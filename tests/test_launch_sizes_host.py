"""A launch has less than 2^32 threads in each direction, and up to 65536 workgroups across it, at the largest shapes that the towers' calls take.  (The stand-in is that of
test_failed_launch_host, which keeps the sizes of what would be launched: nothing reaches a GPU.)"""
import json
import os
import shutil
import subprocess
import sys

import pytest

from .test_failed_launch_host import ROOT, STAND_IN

PUSH = "int __hipPushCallConfiguration() { return 0; }"
SIZES = """
typedef struct { unsigned x, y, z; } dim3;
static unsigned long long threads; static unsigned across;
void stand_in_sizes(unsigned long long* t, unsigned* a) { *t = threads; *a = across; threads = across = 0; }
static void most(unsigned n, unsigned of) { unsigned long long t = (unsigned long long)n * of; if (t > threads) threads = t; }
int __hipPushCallConfiguration(dim3 grid, dim3 block, unsigned long lds, void* stream) {
  most(grid.x, block.x); most(grid.y, block.y); most(grid.z, block.z);
  if (grid.y > across) across = grid.y;
  if (grid.z > across) across = grid.z;
  return 0;
}
"""

CALLS = """
import ctypes, json, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # before the runtime, so that the library's launches come here
import paper_2304_08480_amd as dl
A = 0x1000
calls = {}

for d in (8, 128, 256, 512, 16384):
    for rows in (1 << 26, 1 << 27):
        for bits in (32, 64):
            s = dl.DiscoEmbedding(rows=rows, vocabulary=1 << 20, places=1 << 20, d=d, id_bits=bits, table_dtype=dl.DISCO_F32, y_dtype=dl.DISCO_BF16,
                                  grad_dtype=dl.DISCO_F32, scale=1.0)
            calls[f"embedding forward {d} {rows} {bits}"] = lambda s=s: dl.disco_embedding_fwd(s, *[A] * 5, check=False)
            calls[f"embedding backward {d} {rows} {bits}"] = lambda s=s: dl.disco_embedding_bwd(s, A, A, A, 0, A, A, A, 1 << 50, check=False)

for dim in (8, 256):
    s = dl.DiscoHeadNorm(tokens=(1 << 31) - 1, places=0, heads=1 << 16, kv_heads=1 << 16, head_dim=dim, rotated=0, norm=dl.DISCO_NORM_RMS, pairs=0, x_dtype=1,
                         y_dtype=1, eps=1e-5, **{m + w: (1 << 24 if w == "_row" else 256) for m in ("q", "k", "qn", "kn") for w in ("_row", "_head")})
    calls[f"heads forward {dim}"] = lambda s=s: dl.disco_head_norm_fwd(s, *[A] * 10, check=False)
    calls[f"heads backward {dim}"] = lambda s=s: dl.disco_head_norm_bwd(s, *[A] * 10, A, A, A, A, A, 1 << 50, check=False)

def cross(name, q, k, sequences, q_longest, k_longest, dim, heads, kv_heads):
    s = dl.DiscoCrossAttention(q_tokens=q, k_tokens=k, sequences=sequences, q_longest=q_longest, k_longest=k_longest, heads=heads, kv_heads=kv_heads, head_dim=dim,
                               dtype=dl.DISCO_BF16, scale=0.125, **{m + w: (1024 if w == "_row" else dim) for m in "qkvo" for w in ("_row", "_head")})
    assert dl.disco_cross_attention_workspace_bytes(s), name
    calls["cross forward " + name] = lambda: dl.disco_cross_attention_fwd(s, *[A] * 8, 1 << 60, check=False)
    calls["cross backward " + name] = lambda: dl.disco_cross_attention_bwd(s, *[A] * 12, 1 << 60, check=False)

most = (1 << 31) - 513
for dim in (8, 128):
    cross(f"many queries {dim}", most, 1, 1, 0, 0, dim, 1, 1)
    cross(f"many keys {dim}", 1, most, 1, 1, 0, dim, 1, 1)
    cross(f"many of both {dim}", most, most, 1, 0, 0, dim, 1, 1)
    cross(f"many short ones {dim}", 1 << 23, 1 << 23, 1 << 20, 8, 8, dim, 4, 1)
    cross(f"many sequences of one query {dim}", 1 << 20, 1 << 27, 1 << 20, 1, 300, dim, 4, 4)
    cross(f"heads on shared keys {dim}", 1 << 20, 1 << 10, 1, 0, 0, dim, 1024, 1)
got = {}
for name, call in calls.items():
    stand_in.stand_in_reset(0)
    threads, across = ctypes.c_ulonglong(), ctypes.c_uint()
    status = call()
    stand_in.stand_in_sizes(ctypes.byref(threads), ctypes.byref(across))
    got[name] = [status, stand_in.stand_in_launches(), threads.value, across.value]
print(json.dumps(got))
"""


@pytest.fixture(scope="module")
def got(tmp_path_factory):
    cc = shutil.which("cc") or shutil.which("gcc") or shutil.which("g++")
    if cc is None:
        pytest.skip("no C compiler for the stand-in")
    at = tmp_path_factory.mktemp("stand_in")
    assert PUSH in STAND_IN
    (at / "s.c").write_text(STAND_IN.replace(PUSH, SIZES))
    subprocess.run([cc, "-x", "c", "-std=gnu11", "-w", "-shared", "-fPIC", "-o", str(at / "s.so"), str(at / "s.c")], check=True)
    r = subprocess.run([sys.executable, "-c", CALLS, str(at / "s.so")], cwd=ROOT, check=True, capture_output=True, text=True, timeout=300,
                       env=os.environ | {"PYTHONPATH": ROOT})
    return json.loads(r.stdout.splitlines()[-1])


@pytest.mark.parametrize("kind,calls", [("embedding forward", 20), ("embedding backward", 20), ("heads", 4), ("cross", 24)])
def test_threads_of_the_largest_calls(got, kind, calls):
    import paper_2304_08480_amd as dl
    of_kind = {name: v for name, v in got.items() if name.startswith(kind)}
    # the exact number says that no call of a kind was left out
    assert len(of_kind) == calls
    for name, (status, launches, threads, across) in of_kind.items():
        assert status == dl.DISCO_OK and launches > 0, name
        assert 0 < threads < 1 << 32 and across <= 65536, (name, threads, across)
