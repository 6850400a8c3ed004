"""The host code of the calls on pages (sa_pages_api.hip) built for the CPU with
AddressSanitizer and UndefinedBehaviorSanitizer over launchers that only count: the refusals
of test_host_pages.py, accepted calls, and arguments at the ends of their types."""
import itertools
import os
import subprocess

import pytest

import paper_2608_15522_amd as sa
from test_host_pages import (INVALID, _attend, _compact, _copy, _fork, _free, _reserve,
                             _write)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "host_asan")
CSRC = os.path.join(ROOT, "paper_2608_15522_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
INT_MAX, INT_MIN = 2 ** 31 - 1, -2 ** 31
REFUSALS = [c & 0xffffffffffffffff for c in (sa.SA_ERR_INVALID_ARG, sa.SA_ERR_UNSUPPORTED,
                                              sa.SA_ERR_WORKSPACE)]
CALLS = (_reserve, _write, _fork, _free, _compact, _copy, _attend)

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    out = tmp_path_factory.mktemp("pages_asan")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all"]
    common = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang",
              "-target-feature", "-Xclang", "-packed-fp32-ops", "-I",
              os.path.join(ROOT, "include"), "-DSA_SRC_ID=\"host-asan\"", *san]
    sources = [os.path.join(CSRC, "sa_pages_api.hip"), os.path.join(CSRC, "sa_api.hip"),
               os.path.join(HERE, "stub_launchers.hip"),
               os.path.join(HERE, "stub_page_launchers.hip"),
               os.path.join(HERE, "pages_checks.cpp")]
    objs = [os.path.join(out, os.path.basename(s) + ".o") for s in sources]
    procs = []
    for src, obj in zip(sources, objs):
        lang = ["-x", "hip"] if src.endswith(".cpp") else []
        procs.append(subprocess.Popen([*common, *lang, "-c", src, "-o", obj],
                                      stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for p in procs:
        text = p.communicate()[0]
        assert p.returncode == 0, text[-3000:]
    exe = os.path.join(out, "pages_checks")
    subprocess.run([HIPCC, "--offload-arch=gfx950", *san, *objs, "-o", exe], check=True,
                   capture_output=True, text=True)
    return exe


def run(exe, lines):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True,
                         env=env, timeout=120)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-3000:]
    got = [line.split(" ", 2) for line in res.stdout.splitlines()]
    assert len(got) == len(lines)
    return [(int(code), int(n), text) for code, n, text in got]


def line(call, **kw):
    args = {**call.defaults, **kw}
    return " ".join([call.name] + ["0" if v is None else repr(v) if isinstance(v, float)
                                   else str(int(v)) for v in args.values()])


def test_refusals_launch_nothing(built):
    got = run(built, [line(call, **kw) for call, kw, _, _ in INVALID])
    for (call, kw, code, needle), (rc, launches, text) in zip(INVALID, got):
        assert rc == code & 0xffffffffffffffff, (call.name, kw, rc)  # printed as 64 bits
        assert launches == 0 and needle in text, (call.name, kw, text)


def accepted(rc, launches, text):
    """Reached its launcher; without a GPU HIP reports that behind the launch."""
    return launches == 1 and (text == "-" if rc == 0 else rc == sa.SA_ERR_HIP
                              and "kernel launch failed" in text)


def test_accepted_calls_launch_once(built):
    for got, call in zip(run(built, [line(c) for c in CALLS]), CALLS):
        assert accepted(*got), (call.name, got)


def test_ends_of_the_types(built):
    """Every number alone and every two together at the ends of 32 bits: refused or accepted,
    without overflow."""
    lines = []
    for call in CALLS:
        ints = [k for k, v in call.defaults.items() if isinstance(v, int) and v < 1 << 30]
        for one, two in itertools.combinations_with_replacement(ints, 2):
            for x, y in itertools.product((INT_MAX, INT_MIN, 1, 1 << 20), repeat=2):
                kw = {one: x, two: y}
                if call is _copy and "page_bytes" in kw:
                    kw["page_bytes"] = kw["page_bytes"] & (2 ** 64 - 1)
                lines.append(line(call, **kw))
    for args, got in zip(lines, run(built, lines)):
        rc, launches, text = got
        nothing = args.startswith("sa_pages_copy") and (rc, launches, text) == (0, 0, "-")  # n = 0
        refused = rc in REFUSALS and launches == 0 and text != "-"
        assert accepted(*got) or refused or nothing, (args, got)


def test_workspace_sizes_agree_with_the_library(built):
    cases = [(B, Hq, Hkv, S, d, t, g) for B in (1, 4, 1023, INT_MAX) for Hq, Hkv in
             ((1, 1), (8, 2), (INT_MAX, 1), (INT_MAX, INT_MAX), (3, 2)) for S in (1, 33, 262144)
             for d in (64, 128, 96) for t in (0, 1, 7) for g in (0, 1, B, INT_MIN)]
    got = run(built, ["sa_prefix_attention_workspace " + " ".join(map(str, c)) for c in cases])
    for c, (size, _, _) in zip(cases, got):
        assert size == sa.lib().sa_prefix_attention_workspace(*c), c
