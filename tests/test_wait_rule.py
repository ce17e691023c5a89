"""Every kernel that can wait on a barrier, in whatever way it spells the wait, is on one list and reports a wait that ran out."""
import os
import re

from paper_2603_15619_b200 import build

from test_wait_reporting import kernels, source

# all of them, by how the report leaves the kernel: in its tear-down (abort_teardown), or from the wait itself
TEAR_DOWN = {"moda_fwd_kernel", "moda_fwd2_kernel", "bwd_rows_kernel", "moda_bwd_fused_kernel", "moda_bwd_dq_kernel", "moda_bwd_dkdv_kernel",
             "moda_kv_project_kernel", "wait_timeout_selftest_kernel", "key_mass_kernel", "shared_prefix_kernel"}
FROM_THE_WAIT = {"decode_split_tma_kernel"}


def block(text, at):
    """From `at` to the end of the braces that open behind it."""
    end = text.index("{", at)
    depth = 0
    while True:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
        if depth == 0:
            return text[at:end]


def device_code():
    files = [source(f) for f in sorted(os.listdir(build.CSRC)) if f.endswith((".cu", ".cuh", ".h"))]
    named, found = {}, {}
    for text in files:
        for name, body in kernels(text):
            found[name] = found.get(name, "") + body
        for m in re.finditer(r"\bstruct\s+(?:__align__\(\d+\)\s*)?(\w+)[^;{()]*\{", text):
            named[m.group(1)] = named.get(m.group(1), "") + block(text, m.start())
        for m in re.finditer(r"\b__device__[^;{}()]*?(?:__launch_bounds__\([^)]*\)\s*)?\b(\w+)\(", text):
            if text[:m.start()].rstrip().endswith("__global__") or "{" not in text[m.end():]:
                continue
            rest = text[m.end():]
            if ";" in rest[:rest.index("{")]:                                # a declaration
                continue
            named[m.group(1)] = named.get(m.group(1), "") + block(text, m.end())
    for name in found:
        named.pop(name, None)
    return named, found


def waiting(named):
    """Functions and types that wait, themselves or through others."""
    names = {n for n, body in named.items() if re.search(r"mbarrier\.(try|test)_wait", body)}
    while True:
        more = {n for n, body in named.items() if n not in names and any(re.search(rf"\b{w}\b", body) for w in names)}
        if not more:
            return names
        names |= more


def test_every_kernel_that_waits_is_on_the_list():
    named, found = device_code()
    waits = waiting(named)
    assert {"mbar_try_wait", "mbar_wait", "mbar_wait2", "decode_wait", "PipeWait"} <= waits
    there = {n for n, body in found.items() if any(re.search(rf"\b{w}\b", body) for w in waits) or re.search(r"mbarrier\.(try|test)_wait", body)}
    assert there == TEAR_DOWN | FROM_THE_WAIT, there ^ (TEAR_DOWN | FROM_THE_WAIT)
    for name in TEAR_DOWN:
        assert "abort_teardown(" in found[name], name
    for name in FROM_THE_WAIT:
        assert "decode_wait(" in found[name] and "report_abort(" in named["decode_wait"], name


def test_a_probe_outside_of_a_wait_is_bounded():
    # mbar_try_wait alone neither gives up nor reports: only loops with a limit of their own probe with it
    for f in sorted(os.listdir(build.CSRC)):
        if not f.endswith((".cu", ".cuh")):
            continue
        for name, body in kernels(source(f)):
            for m in re.finditer(r"\bmbar_try_wait\(", body):
                line = body[body.rindex("\n", 0, m.start()):body.index("\n", m.end())]
                before = body[:m.start()].rstrip().splitlines()
                assert re.search(r"globaltimer_ns\(\) - \w+ < \d+ull", line) or re.search(r"for \(int spin = 0; spin < ", "\n".join(before[-2:])), (name, line)


def test_a_wait_of_a_new_kind_would_be_seen():
    # the rule itself: a function that wraps a wait, and one that wraps that one
    named, _ = device_code()
    named["outer"], named["inner"] = "{ inner(bar); }", "{ mbar_wait(bar, 0, f, 1); }"
    assert {"outer", "inner"} <= waiting(named)
