"""What the embedding's, the layer norm's and the orthogonalisation's calls launch, from the smallest to the largest sizes, without a
GPU: tests/step_calls_main.cpp stands in for the HIP runtime."""
import os
import subprocess

import pytest

from paper_2410_10989_amd import _build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if _build.is_stale():
        _build.build()
    exe = str(tmp_path_factory.mktemp("step_calls") / "step_calls")
    # (-rdynamic: the program's functions stand before the runtime's when the library's calls are resolved)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-rdynamic",
                    os.path.join(HERE, "step_calls_main.cpp"), "-o", exe, "-ldl"], check=True)
    return exe


@pytest.mark.parametrize("scenario", ["embeddings", "layer_norms", "orthogonalisations", "orthogonalisation_with_little_memory"])
def test_step_calls(program, scenario):
    res = subprocess.run([program, _build.LIB_PATH, scenario], stdout=subprocess.PIPE, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.endswith("ok\n"), res.stdout[:4000]
