"""How much device memory the library's workspaces take as calls grow, on the
host alone (a double of the HIP runtime that counts allocations)."""

import os
import subprocess

import pytest

import paper_2609_02846_amd as ue
from host_launches import HERE, fp8_call, gemm_call
from paper_2609_02846_amd import build as ue_build


@pytest.fixture(scope="module")
def counter(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("host_workspaces") / "host_workspaces")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-rdynamic", "-pthread", os.path.join(HERE, "host_workspaces.cpp"),
                           "-o", exe, "-ldl"])
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)

    def run(calls):
        """(status, allocations, bytes, largest) after each call of a list."""
        r = subprocess.run([exe, ue.LIB_PATH], input="\n".join(calls) + "\n", capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr
        return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    return run


def tokens(T, K):
    """Bytes of a serving call's quantized tokens, E8M0."""
    return T * K + K // 128 * ((T + 15) // 16 * 16)


GROWING = {
    "serving, one token more each call": [fp8_call(T, 256, 8192, "linear", scale="e8m0") for T in range(65, 2000)],
    "serving, K grows": [fp8_call(200, 256, K, "linear") for K in range(128, 30000, 128)],
    "products in blocks of 32": [gemm_call("nt", M, 256, 2048, block=32) for M in range(64, 4096, 32)],
}


@pytest.mark.parametrize("what", GROWING)
def test_calls_that_grow_keep_memory_within_a_few_times_the_largest(what, counter):
    """A replaced workspace is never freed: were each as large as its call
    asked, n growing calls would hold n of them."""
    got = counter(GROWING[what])
    one = counter(GROWING[what][-1:])[0]              # what the last call needs by itself
    assert all(status == 0 for status, *_ in got)
    status, allocations, total, largest = got[-1]
    assert allocations <= 30 and largest <= 2 * one[3] and total <= 4 * one[2], (got[-1], one)


def test_the_same_calls_allocate_once(counter):
    calls = [fp8_call(T, 256, 8192, "linear", scale="e8m0") for T in (900, 70, 900, 300)]
    got = counter(calls)
    assert {n for _, n, _, _ in got} == {1} and got[-1][2] < 1.01 * tokens(900, 8192) + (64 << 20)


def test_room_for_the_call_but_not_for_twice_the_last(counter):
    """The call gets what it needs."""
    a, b = (fp8_call(T, 25600, 8192, "linear", scale="e8m0") for T in (1000, 1100))
    need = [counter([c])[0][2] for c in (a, b)]
    got = counter([f"memory {sum(need) + 4096}", a, b])
    assert [s for s, *_ in got] == [0, 0] and got[1][2] == sum(need)
    short = counter([f"memory {sum(need) - 4096}", a, b])
    assert short[0][0] == 0 and short[1][0] != 0


def test_a_call_without_room_does_not_spoil_the_next(counter):
    """Its error is its own status and not what the next call's launches find."""
    a, b = fp8_call(100, 25600, 8192, "linear"), fp8_call(1100, 25600, 8192, "linear")
    room = counter([a])[0][2]
    assert [s == 0 for s, *_ in counter([f"memory {room + 4096}", a, b, a])] == [True, False, True]
