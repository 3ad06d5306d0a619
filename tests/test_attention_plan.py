"""The calls of attention_kernel_cases.py reach every kernel of attention, by the rules that
the library itself goes by. Without a GPU."""
import ctypes as C
import itertools
import os
import subprocess

import pytest

import attention_kernel_cases as K

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34244_amd", "csrc")
SOURCE = """
#include "attention_plan.h"
using namespace heddle::attn;
extern "C" void plan(const int64_t *z, int *out)
{
    const Sizes s = {z[0], z[1], z[2], (int)z[3], (int)z[4]};
    const ForwardPlan f = plan_forward(s);
    out[0] = f.split, out[1] = f.rows, out[2] = f.parts, out[3] = plan_keys(s);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(at / "plan.so"), str(at / "plan.cpp")], check=True)
    L = C.CDLL(str(at / "plan.so"))

    def ask(*z):
        out = (C.c_int * 4)()
        L.plan((C.c_int64 * 5)(*z), out)
        split, rows, parts, keys = out
        return ("parts" if parts > 1 else "one part") if split else f"{rows} rows", parts, keys

    return ask


def reached(plan):
    """{(kernel, padded width, mode): names}, and the same of packed calls by the way their sequences are found"""
    forms, found = {}, {}
    for name, c in K.cases().items():
        rows, _, keys = plan(*K.sizes(c))
        for kernel in [rows] + [f"{keys} keys"] * c.get("train", True):
            forms.setdefault((kernel, 64 if c["dim"] <= 64 else 128, K.mode(c)), []).append(name)
            if c.get("packed"):
                found.setdefault((kernel, len(c["queries"]) <= 64), []).append(name)
    return forms, found


def test_every_kernel_is_reached(plan):
    forms, found = reached(plan)
    for form in itertools.product(["parts", "one part", "128 rows", "256 rows", "32 keys", "128 keys", "256 keys"], (64, 128), ("", "cap", "slopes", "capslopes")):
        assert form in forms, form
    for form in itertools.product(["parts", "128 rows", "256 rows", "128 keys", "256 keys"], (True, False)):
        assert form in found, form


def test_rules(plan):
    """what their comments say"""
    assert plan(1, 1, 2048, 32, 32)[0] == "parts" and plan(32, 32, 32 * 8192, 64, 8)[:2] == ("parts", 2)
    assert plan(4, 8192, 8192, 64, 8) == ("256 rows", 1, 256) and plan(11, 4092, 4092, 32, 32) == ("128 rows", 1, 128)
    assert plan(3, 999, 999, 12, 4) == ("128 rows", 1, 32) and plan(1, 8192, 8192, 32, 8)[0] == "256 rows"
    assert plan(8, 16, 32000, 32, 8)[0] == "parts" and plan(8, 512, 32000, 32, 8)[0] != "parts" and plan(1, 64, 16000, 32, 8)[0] == "parts"
    assert plan(1, 1, 1 << 20, 1, 1)[1] == 64 and plan(1, 0, 0, 1, 1)[1] == 1
