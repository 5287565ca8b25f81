"""What calls allocate, free and launch, without a GPU: tests/host_calls_main.cpp stands in for the HIP runtime."""
import os
import subprocess

import pytest

from paper_2410_10989_amd import _build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if _build.is_stale():
        _build.build()
    exe = str(tmp_path_factory.mktemp("host_calls") / "host_calls")
    # (-rdynamic: the program's functions stand before the runtime's when the library's calls are resolved)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-rdynamic",
                    os.path.join(HERE, "host_calls_main.cpp"), "-o", exe, "-ldl"], check=True)
    return exe


@pytest.mark.parametrize("scenario", ["short_lists", "backward_with_little_memory", "workspace_of_a_captured_call"])
def test_host_calls(program, scenario):
    res = subprocess.run([program, _build.LIB_PATH, scenario], stdout=subprocess.PIPE, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout
