"""A preparation goes through the kernels of both epilogues and reports what either of them does (compiled with gcc; no device)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2407_19644_amd", "csrc")

DRIVER = r"""
#include <cstdio>
#include "ubp_internal.h"

static int plain_calls, wide_calls;
template <ubp_status RC> ubp_status plain(int x, bool) { plain_calls += x; return RC; }
template <ubp_status RC> ubp_status wide(int x, bool) { wide_calls += x; return RC; }

#define CHECK(c) do { if (!(c)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main() {
    using ubp::launch_either;
    for (int on = 0; on <= 2; ++on) {
        ubp::Epilogue ep = {};
        ep.on = on;
        // a preparation: both, and the first error of the two
        plain_calls = wide_calls = 0;
        CHECK(launch_either(plain<UBP_OK>, wide<UBP_OK>, ep, true, 1) == UBP_OK && plain_calls == 1 && wide_calls == 1);
        CHECK(launch_either(plain<UBP_OK>, wide<UBP_ERR_DEVICE>, ep, true, 1) == UBP_ERR_DEVICE);
        CHECK(launch_either(plain<UBP_ERR_UNSUPPORTED>, wide<UBP_OK>, ep, true, 1) == UBP_ERR_UNSUPPORTED);
        CHECK(launch_either(plain<UBP_ERR_UNSUPPORTED>, wide<UBP_ERR_DEVICE>, ep, true, 1) == UBP_ERR_UNSUPPORTED);
        // a launch: one of them
        plain_calls = wide_calls = 0;
        CHECK(launch_either(plain<UBP_OK>, wide<UBP_ERR_DEVICE>, ep, false, 1) == (on == 2 ? UBP_ERR_DEVICE : UBP_OK));
        CHECK(plain_calls == (on == 2 ? 0 : 1) && wide_calls == (on == 2 ? 1 : 0));
    }
    return 0;
}
"""


def test_a_preparation_reports_both_epilogues(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "driver.cpp", tmp_path / "driver"
    src.write_text(DRIVER)
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", CSRC, str(src), "-o", str(exe)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
