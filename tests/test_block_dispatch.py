"""Which kernels the transformer-block calls launch, on both sides of each rule (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import re
import subprocess

import pytest

from block_rounds import ROUNDS, kernels
from paper_1902_04610_amd import build


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    return kernels([r[:3] for r in ROUNDS], tmp_path_factory.mktemp("recorder"))


def test_kernels_of_each_round(launched):
    wrong = [(r[:2], got, r[3]) for r, got in zip(ROUNDS, launched) if got != r[3]]
    assert not wrong, wrong[:3]


def test_every_kernel_has_a_round(launched):
    names = subprocess.run(["nm", "-C", build.LIB], stdout=subprocess.PIPE, text=True, check=True).stdout
    names = re.sub(r"\((salus::)?Epilogue\)", "E", names).replace("salus::", "")
    built = set(re.findall(r"__device_stub__((?:block|gradients|weight_grad|clip)_\w+(?:<.*>)?)\(", names))
    assert len(built) > 50
    assert built <= {k for ks in launched for k in ks}, built - {k for ks in launched for k in ks}
