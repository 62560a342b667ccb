"""Results that lie on what a call reads are refused before any device work (the pointers
here are never followed), and those that only lie beside it are not.  A call that
is taken fails for want of a device, which is made sure of first."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import ctypes as C, sys
sys.path.insert(0, sys.argv[1])
sys.path.insert(0, sys.argv[1] + "/tests")
import network_refusals as N
from paper_1609_06119_amd._lib import lib
L = lib()
count = C.c_int(0)
assert C.CDLL("libamdhip64.so").hipGetDeviceCount(C.byref(count)) != 0 and count.value == 0
A, M = N.A, 1 << 20


def call(name, **change):
    args = {**N.BASE[name], **change}
    return getattr(L, name)(*args.values())


def refused(name, what, **change):
    assert call(name, **change) == -1, (name, change)
    text = L.fbdt_last_error()
    assert b"overlaps " + what in text, (name, change, text)


def taken(name, **change):
    assert call(name, **change) == -6, (name, change, L.fbdt_last_error())


E = "fbdt_embed"                 # a table of 48 x 64 of 2 bytes, 10 tokens of 4, 10 rows out
apart = dict(tokens=2 * M, out=3 * M)
taken(E, **apart)
refused(E, b"table", tokens=2 * M)                                    # out = table
refused(E, b"table", **{**apart, "out": A + 47 * 128 + 126})          # its last element
refused(E, b"table", **{**apart, "table": 3 * M + 9 * 128 + 126})     # the result's last element
taken(E, **{**apart, "out": A + 48 * 128})                            # just behind the table
taken(E, **{**apart, "out": A - 10 * 128})                            # just before it
refused(E, b"tokens", **{**apart, "out": 2 * M + 38})
taken(E, **{**apart, "out": 2 * M + 40})
side = dict(ldt=200, ldo=200, tokens=2 * M)                           # columns of one matrix
taken(E, out=A + 64 * 2, **side)
taken(E, out=A + 136 * 2, **side)
taken(E, out=A + (5 * 200 + 64) * 2, **side)
refused(E, b"table", out=A + 63 * 2, **side)
refused(E, b"table", out=A + 137 * 2, **side)
refused(E, b"table", out=A - 63 * 2, **side)
refused(E, b"table", out=A + 64 * 2, ldt=200, ldo=300, tokens=2 * M)  # other strides among each other
taken(E, out=A + 64 * 2, ldt=200, ldo=2 ** 40, n=1, tokens=2 * M)     # one row between rows
refused(E, b"table", out=A + 140 * 2, ldt=200, ldo=2 ** 40, n=1, tokens=2 * M)
taken(E, out=A + 64 * 2, ldt=2 ** 40, rows=1, ldo=128, tokens=2 * M)
refused(E, b"table", out=A + 62 * 2, ldt=2 ** 40, rows=1, ldo=128, tokens=2 * M)
refused(E, b"table", out=A + 2, ldt=2 ** 62, ldo=2 ** 62, n=2 ** 31 - 1, rows=2 ** 31 - 1, tokens=2 * M)

G = "fbdt_embed_grad"            # 10 rows of 64 bfloat16 into 48 x 64 float32
apart = dict(tokens=2 * M, dout=3 * M, work=8 * M)
taken(G, **apart)
refused(G, b"dout", **{**apart, "dout": A})
refused(G, b"dout", **{**apart, "dout": A + 47 * 256 + 254})
refused(G, b"dout", **{**apart, "dout": A, "grad_dtype": N.BF16, "rows": 10})   # out = dout
refused(G, b"tokens", **{**apart, "tokens": A + 47 * 256 + 252})
taken(G, **{**apart, "dout": A + 48 * 256})
assert call(G, n=0, tokens=None, dout=None) == -6                     # nothing is read

T = "fbdt_event_tokens"          # 3 rows of 10 codes, 120 bytes of tokens
taken(T, tokens=2 * M)
refused(T, b"xb")
refused(T, b"xb", tokens=A + 2 * 16 + 8)
taken(T, tokens=A + 48)

P = "fbdt_packed_product"        # a: 4 rows, b: 9 rows of 200; 4 x 9 of 2 bytes
apart = dict(a_scales=2 * M, b=3 * M, b_scales=4 * M, out=5 * M)
taken(P, **apart)
taken(P, **{**apart, "a": 3 * M, "a_scales": 4 * M, "m": 4})          # a and b may be one
for at, what in ((A, b"a"), (A + 3 * 256 + 198, b"a"), (2 * M + 12, b"a"), (3 * M, b"b"),
                 (3 * M + 8 * 256 + 198, b"b"), (4 * M + 8 * 4, b"b")):
    refused(P, what, **{**apart, "out": at})
taken(P, **{**apart, "out": A + 3 * 256 + 200})
taken(P, **{**apart, "out": A + 200, "ldo": 128, "m": 4})             # in the rows' last 56 bytes
refused(P, b"a", **{**apart, "out": A + 240, "ldo": 128})             # 18 bytes from 240 on

W = "fbdt_packed_weight_grad"    # dy: 4 x 9 of 2 bytes, x: 4 rows of 200; 9 x 200 float32
apart = dict(x=2 * M, x_scales=3 * M, out=4 * M)
taken(W, **apart)
refused(W, b"dy", **{**apart, "out": A + 3 * 32 + 16})
refused(W, b"x", **{**apart, "out": 2 * M})
refused(W, b"x", **{**apart, "out": 3 * M - 9 * 800 + 4})
taken(W, **{**apart, "out": A - 9 * 800})
print("overlaps ok")
"""


def test_results_on_what_a_call_reads_are_refused():
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")
    run = subprocess.run([sys.executable, "-c", SCRIPT, ROOT], capture_output=True, text=True, env=env,
                         timeout=120)
    assert run.returncode == 0, (run.stdout[-1000:], run.stderr[-3000:])
    assert "overlaps ok" in run.stdout
