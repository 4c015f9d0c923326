"""How the distillation kernel shares out shared memory, on the CPU: csrc/apc_distill_plan.h
compiled as it is."""
import ctypes
import subprocess

import pytest

from paper_2609_18178_gb300 import _build

SOURCE = """
#include "apc_distill_plan.h"
extern "C" void plan(unsigned k, int loss, int grad, unsigned *out) {
  const apc::Layout l = apc::distill_layout(k, loss, grad);
  out[0] = l.teachers, out[1] = l.chunks * l.chunk * 16, out[2] = l.chunks, out[3] = l.bytes();
  out[4] = l.room, out[5] = 1u << l.slots_log2, out[6] = l.tables;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    so = str(d / "libplan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", _build.CSRC, str(d / "plan.cpp"), "-o", so], check=True)
    f = ctypes.CDLL(so).plan

    def call(k, form):
        out = (ctypes.c_uint * 7)()
        f(k, form in ("loss", "both"), form in ("grad", "both"), out)
        return dict(zip(("teachers", "ring", "chunks", "bytes", "room", "slots", "tables"), out))

    return call


@pytest.mark.parametrize("form", ["loss", "grad", "both"])
def test_as_many_teachers_as_there_is_room_for(plan, form):
    """Whatever k is (at 279 and 280, at 511 to 513 and everywhere else): a ring of 32 KB
    at least, and no teacher fewer than that leaves room for."""
    room = 228 * 1024 // 2 - 1024  # two blocks on an SM
    for k in range(1025):
        p = plan(k, form)
        assert p["ring"] >= 32 * 1024 and 1 <= p["chunks"] <= 16, (k, p)
        assert p["bytes"] <= room
        assert p["room"] >= k + 1 and p["slots"] >= 2 * (k + 1)
        assert p["tables"] == (0 if form == "loss" else p["teachers"] * p["slots"])
        one_more = p["room"] * 12 + (3 * 256 * 4 if form == "loss" else p["slots"] * 4)
        fixed = p["bytes"] - p["ring"]
        assert p["teachers"] == 4 or 1 <= p["teachers"] < 4 and fixed + one_more + 32 * 1024 > room, (k, p)


def test_no_step_at_512(plan):
    for form in ("loss", "grad", "both"):
        assert plan(512, form)["teachers"] == plan(513, form)["teachers"] == 4
