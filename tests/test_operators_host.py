"""The sequence operators' host side (launch shapes, workspace, streams, event
pairs) on the CPU: tests/host_calls.cpp stands in for the HIP runtime and writes
down what libpolyglot.so asks of it."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_1404_1521_amd")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("host") / "host_calls")
    r = subprocess.run(
        ["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
         "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host_calls.cpp"), "-o", out,
         "-rdynamic", "-L", PKG, "-lpolyglot", f"-Wl,-rpath,{PKG}", f"-Wl,-rpath,{ROCM}/lib",
         "-Wl,--unresolved-symbols=ignore-in-shared-libs"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return out


def run(program, what):
    r = subprocess.run([program, what], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)


def test_scores_of_more_rows_than_a_launch_has(program):
    """A launch has fewer than 2^32 threads; more rows take several launches."""
    run(program, "many_rows")


def test_a_change_of_the_stream_keeps_the_order(program):
    run(program, "streams")


def test_event_pairs_do_not_pile_up(program):
    run(program, "times")


def test_reserving_takes_no_host_memory_of_its_size(program):
    run(program, "reserve")
