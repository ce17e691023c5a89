"""Which form of the selection kernel an eviction takes (csrc/launch_rules.h), on the CPU."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_15619_b200", "csrc")
SOURCE = r"""
#include "launch_rules.h"
extern "C" void form(int T, long long rows, int sms, int* out) {
    const moda::EvictForm f = moda::evict_form(T, rows, sms);
    out[0] = f.ranks; out[1] = f.most; out[2] = f.threads; out[3] = f.ctas; out[4] = moda::evict_run(T, f.ranks, f.threads);
}
"""


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    (d / "forms.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(d / "forms.so"), str(d / "forms.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "forms.so"))

    def call(T, rows, sms=148):
        out = (ctypes.c_int * 5)()
        lib.form(T, ctypes.c_longlong(rows), sms, out)
        return tuple(out)
    return call


def test_the_share_of_a_thread_fits_its_form(form):
    rng = random.Random(3)
    for _ in range(20000):
        T, rows, sms = int(2 ** rng.uniform(0, 24)), int(2 ** rng.uniform(0, 14)), rng.choice((148, 132, 16))
        ranks, most, threads, ctas, run = form(T, rows, sms)
        case = (T, rows, sms, ranks, most, threads, ctas, run)
        assert ranks in (1, 2, 4, 8, 16) and run % 2 == 1 and run * threads * ranks >= T, case
        assert (most, threads, ctas) in ((5, 512, 2), (9, 512, 2), (17, 512, 2), (33, 512, 2), (33, 512, 1), (33, 1024, 1), (0, 512, 1)), case
        assert run <= most or (most == 0 and T > 16 * 33 * 1024 and ranks == 16), case


def test_the_sms_of_the_device_count(form):
    # clusters while the SMs have room for all CTAs; the keys in registers where a CTA has its SM to itself
    assert form(131001, 8)[:4] == (8, 33, 512, 1) and form(131001, 8, 132)[:4] == (8, 33, 512, 1) and form(131001, 8, 40)[:4] == (4, 33, 1024, 1)
    assert form(16001, 148)[:4] == (1, 33, 512, 1) and form(16001, 148, 132)[:4] == (1, 33, 512, 2) and form(16001, 149)[:4] == (1, 33, 512, 2)
