"""A launch that fails is a status code, whichever of a call's launches it is, and the ones behind it are left out.

The calls run in a process of their own, where launches go to a stand-in that counts them, does nothing and reports an error for one of them, the way
the runtime does: kept until it is asked for, once.  Nothing reaches a GPU, so the addresses need not exist."""
import json
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_IN = """
static int failing, launches, kept;
void stand_in_reset(int n) { failing = n; launches = kept = 0; }
int stand_in_launches(void) { return launches; }
int __hipPushCallConfiguration() { return 0; }
int __hipPopCallConfiguration() { return 0; }
int hipLaunchKernel() { return ++launches == failing ? (kept = 1) : 0; }
int hipGetLastError(void) { int e = kept; kept = 0; return e; }
int hipPeekAtLastError(void) { return kept; }
"""

CALLS = """
import ctypes, json, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)      # before the runtime, so that the library's launches come here
import paper_2304_08480_amd as dl
from paper_2304_08480_amd import binding
A = 0x1000

def attention(lengths, tokens, dim, backward, kv_heads=8):
    s = dl.DiscoAttention(tokens=tokens, sequences=lengths, heads=8, kv_heads=kv_heads, head_dim=dim, causal=0, dtype=dl.DISCO_BF16, scale=0.125,
                          **{m + w: (1024 if w == "_row" else dim) for m in "qkvo" for w in ("_row", "_head")})
    if backward:
        return lambda: dl.disco_attention_bwd(s, *[A] * 11, 1 << 40, check=False)
    return lambda: dl.disco_attention_fwd(s, *[A] * 6, check=False)

def norm(backward):
    s = dl.DiscoBlockNorm(rows=5000, d=512, post=dl.DISCO_NORM_LAYER, pre=dl.DISCO_NORM_LAYER, gate=dl.DISCO_GATE_CHANNEL, x_dtype=dl.DISCO_BF16,
                          h_dtype=dl.DISCO_BF16, eps_post=1e-5, eps_pre=1e-5, x_scale=1.0, h_scale=1.0)
    if backward:
        return lambda: dl.disco_block_norm_bwd(s, *[A] * 16, A, 1 << 40, check=False)
    return lambda: dl.disco_block_norm_fwd(s, *[A] * 10, check=False)

def gradients(count, elements, given):
    at, n, types = (ctypes.c_void_p * count)(*[A] * count), (ctypes.c_int64 * count)(*[elements] * count), (ctypes.c_int32 * count)(*[dl.DISCO_F32] * count)
    if given is None:
        return lambda: binding._lib.disco_grad_norm(at, n, types, count, 0, A, A, 1 << 40, None)
    return lambda: binding._lib.disco_grad_clip(at, at, n, types, count, 1.0, given or None, A, A, 1 << 40, None)

calls = {
    "attention forward, short": attention(1000, 40000, 64, False),
    "attention forward, short, wide": attention(1000, 40000, 128, False),
    "attention forward, short, no longer ones": attention(2, 60, 64, False),
    "attention forward, long": attention(3, 40000, 64, False),
    "attention forward, few rows": attention(1, 2000, 64, False),
    "attention backward, short": attention(1000, 40000, 64, True),
    "attention backward, short, wide": attention(1000, 40000, 128, True),
    "attention backward, short, no longer ones": attention(2, 60, 64, True),
    "attention backward, shared heads": attention(1000, 40000, 64, True, 2),
    "attention backward, long": attention(3, 40000, 64, True),
    "attention backward, few rows": attention(1, 2000, 64, True),
    "norm forward": norm(False),
    "norm backward": norm(True),
    "gradient norm": gradients(300, 9000, None),
    "clipping, few pieces": gradients(3, 9000, 0),
    "clipping, many pieces": gradients(300, 1 << 20, 0),
    "clipping, a given norm": gradients(300, 9000, 2 * A),
}
got = {}
for name, call in calls.items():
    stand_in.stand_in_reset(0)
    got[name] = [[0, call(), stand_in.stand_in_launches()]]
    for n in range(1, got[name][0][2] + 1):
        stand_in.stand_in_reset(n)
        got[name].append([n, call(), stand_in.stand_in_launches()])
print(json.dumps(got))
"""

LAUNCHES = {
    "attention forward, short": 2, "attention forward, short, wide": 2, "attention forward, short, no longer ones": 1, "attention forward, long": 1,
    "attention forward, few rows": 1, "attention backward, short": 3, "attention backward, short, wide": 3,
    "attention backward, short, no longer ones": 1, "attention backward, shared heads": 2, "attention backward, long": 2,
    "attention backward, few rows": 2, "norm forward": 1, "norm backward": 2, "gradient norm": 4, "clipping, few pieces": 2, "clipping, many pieces": 7,
    "clipping, a given norm": 4,
}


@pytest.fixture(scope="module")
def got(tmp_path_factory):
    cc = shutil.which("cc") or shutil.which("gcc") or shutil.which("g++")
    if cc is None:
        pytest.skip("no C compiler for the stand-in")
    at = tmp_path_factory.mktemp("stand_in")
    (at / "s.c").write_text(STAND_IN)
    subprocess.run([cc, "-x", "c", "-std=gnu11", "-w", "-shared", "-fPIC", "-o", str(at / "s.so"), str(at / "s.c")], check=True)
    r = subprocess.run([sys.executable, "-c", CALLS, str(at / "s.so")], cwd=ROOT, check=True, capture_output=True, text=True, timeout=300)
    return json.loads(r.stdout.splitlines()[-1])


@pytest.mark.parametrize("name", LAUNCHES)
def test_every_launch_of_a_call(got, name):
    import paper_2304_08480_amd as dl
    (_, ok, launches), *failed = got[name]
    assert ok == dl.DISCO_OK and launches == LAUNCHES[name]
    for n, status, done in failed:
        assert (status, done) == (dl.DISCO_ERR_HIP, n), f"launch {n} of {launches} failed"
