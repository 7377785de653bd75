"""What the calls that make rollouts launch, at the ends of the sizes they take: grids, workgroups and LDS that a launch can have.  A library in
front of the runtime writes each launch down and makes none, so nothing needs a GPU or the memory that the sizes stand for."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

IN_FRONT = r"""
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
typedef struct { uint32_t x, y, z; } sizes;
unsigned __hipPushCallConfiguration(sizes grid, sizes block, size_t shared, void* stream) {
    printf("launch %u %u %u %u %u %u %zu\n", grid.x, grid.y, grid.z, block.x, block.y, block.z, shared);
    fflush(stdout);
    return 1;                  /* (anything but 0: the launch is not made) */
}
int hipGetLastError(void) { return 0; }
"""

CALLS = r"""
import ctypes as C, sys
sys.path.insert(0, sys.argv[1])
C.CDLL(sys.argv[2], mode=C.RTLD_GLOBAL)
import paper_2203_16340_amd as L
from paper_2203_16340_amd import losses as S, rollouts as R
lib, at, room = L.lib(), 1 << 40, 1 << 62
def say(rc, *what):
    print("call", rc, *what, flush=True)
for dtype in (1, 2):
    for rows, vocab in ((1, 1), (1, 1 << 21), (128, 1 << 21), (129, 1 << 21), (257, 1 << 21), ((1 << 23) + 5, 50000), ((1 << 31) - 1, 100)):
        say(lib.lbfgsb_draw_tokens(C.byref(S.Logits(dtype, rows, vocab, vocab, at, 1.0, None, 0)), at, at, at, at, room, None), "draw", dtype, rows, vocab)
    for n, k, vocab in ((1, 0, 1), (1, 128, 1 << 21), (159, 128, 1 << 21), (160, 128, 1 << 21), (1 << 22, 0, 1 << 21), (1 << 22, 1, 1 << 17), ((1 << 23) + 1, 1, 40000),
                        ((1 << 30) - 1, 1, 10)):
        for draft, logp in ((None, None), (at, None), (at, at)):
            d = R.Drafts(dtype, n, k, vocab, at, vocab, vocab * (k + 1), 1.0, draft, vocab, vocab * max(k, 1), 1.0, logp, at, None, at, at)
            say(lib.lbfgsb_verify_draft(C.byref(d), at, at, at, at, room, None), "verify", dtype, n, k, vocab, bool(draft), bool(logp))
for rows, cols in ((1, 1), (1 << 28, 128), (1 << 11, 1 << 24), (16400, 1 << 20), (32800, 1 << 19), (49200, 130), (100, 1 << 24)):
    for group, scale in ((32, 1), (64, 2), (128, 3), (1 << 24, 1)):
        w = R.Weights4Struct(rows, cols, group, scale, at, at, at)
        n = lib.lbfgsb_packed4_bytes(C.byref(w))
        say(lib.lbfgsb_quantize4(1, cols, at, C.byref(w), None), "quantize", rows, cols, group)
        say(lib.lbfgsb_pack4(C.byref(w), at, n, None), "pack", rows, cols, group)
        for x in (1, 2, 3):
            for tokens in (1, 2, 16, 17, 33, 49, 64, 1 << 21):
                if tokens * cols < 1 << 34:
                    say(lib.lbfgsb_matvec4(C.byref(w), 1 << 50, tokens, x, cols, at, x, rows, 1 << 60, 256, room, None), "product", rows, cols, group, tokens, x)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    at = tmp_path_factory.mktemp("launches")
    (at / "front.c").write_text(IN_FRONT)
    (at / "calls.py").write_text(CALLS)
    subprocess.run(["gcc", "-shared", "-fPIC", str(at / "front.c"), "-o", str(at / "front.so")], check=True)
    out = subprocess.run([sys.executable, str(at / "calls.py"), ROOT, str(at / "front.so")], check=True, capture_output=True, text=True).stdout
    calls, made = [], []
    for line in out.splitlines():
        what, *rest = line.split()
        if what == "launch":
            made.append([int(v) for v in rest])
        else:
            calls.append((" ".join(rest[1:]), int(rest[0]), made))
            made = []
    return calls


def test_every_call_launches(launches):
    assert len(launches) > 300
    for what, rc, made in launches:
        assert rc == 0 and made, what


def test_launches_are_what_a_launch_can_be(launches):
    for what, _, made in launches:
        for gx, gy, gz, bx, by, bz, shared in made:
            assert gx > 0 and 0 < gy <= 65535 and gz == by == bz == 1, what
            assert 64 <= bx <= 1024 and bx % 64 == 0 and shared <= 160 << 10, what
            assert gx * bx < 1 << 32 and gy * by < 1 << 32, (what, gx, bx)
