"""The rules that choose the forms of the operators around a model's matrices, and that the GPU tests reach each form (no GPU needed)."""
import subprocess
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    exe = tmp_path_factory.mktemp("shape") / "lm_shape"
    build = subprocess.run(["g++", "-O2", "-std=c++17", f"-I{ROOT / 'include'}", f"-I{ROOT / 'paper_2410_01799_amd' / 'csrc'}",
                            str(ROOT / "tests" / "lm_shape_driver.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr

    def run(calls):
        got = subprocess.run([str(exe)], input="\n".join("%s %d %d %d" % c for c in calls), capture_output=True, text=True, timeout=120)
        assert got.returncode == 0
        answers = [a.split("\n") for a in got.stdout.split("--\n")[:len(calls)]]
        assert len(answers) == len(calls)
        return set(line for a in answers for line in a if line)

    return run


def needed(found):
    """Forms to be tested: a form whose ring of buffers is never filled again counts only where no size fills it."""
    return {f for f in found if not (f.endswith(" short") and f[:-len(" short")] in found)}


NAMES = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}


def test_the_gpu_tests_reach_every_form_of_the_cross_entropy(forms):
    from test_gpu_lm_forms import XENT

    sizes = [(n, d, v) for n in (1, 2, 17, 33, 64, 65, 100, 129, 200, 300, 513, 1000, 2048, 2900, 4096, 9000)
             for d in (1, 8, 40, 63, 64, 72, 129, 256, 520, 1000, 1001, 1024, 2048, 2056, 4096, 4099, 8192)
             for v in (1, 8, 65, 200, 333, 700, 1024, 2003, 2049, 4097, 5003, 8199, 16000, 20001, 32000, 70000, 128256)]
    for dtype, name in NAMES.items():
        all_of = needed(forms([(name, *s) for s in sizes]))
        tested = forms([(name, n, d, v) for t, n, d, v in XENT if t == dtype])
        assert len(all_of) > 40 and all_of <= tested, sorted(all_of - tested)


def test_the_gpu_tests_reach_every_form_of_the_8_bit_products(forms):
    from test_gpu_lm_forms import Q8

    sizes = [(m, k, n) for m in (1, 2, 3, 4, 5, 9, 16, 17, 33, 64, 65, 100, 129, 200, 333, 600, 1000, 2048, 4096, 20000)
             for k in (1, 8, 200, 1000, 1024, 4096, 14336, 40000, 131072) for n in (1, 17, 64, 193, 1000, 1501, 4096, 8192, 14336, 128256)]
    all_of = needed(forms([("q8", *s) for s in sizes]))
    tested = forms([("q8", *s) for s in Q8])
    assert len(all_of) >= 9 and all_of <= tested, sorted(all_of - tested)


@pytest.mark.parametrize("dtype", [0, 2, 3])
@pytest.mark.parametrize("N,D,V", [(4096, 4096, 32000), (16384, 4096, 128256), (32768, 1024, 128256), (1, 4096, 32000), (2048, 2048, 200)])
def test_work_space_of_the_loss_is_two_sums_for_each_row_and_strip(dtype, N, D, V):
    """8 bytes for each token and 128 rows of the vocabulary (tiles of 128, as f32 takes them: 64; of few tokens: 32), besides what is rounded up.
    Logits in shares: up to 16 of them."""
    from paper_2410_01799_amd import scd

    strip = 32 if N <= 64 else 64 if dtype == 0 else 128
    most = -(-V // strip) * N * 8 if V > 2048 else 16 * N * 4 * (V + 64)
    assert scd.lib().scd_xent_workspace_bytes(dtype, N, D, V) <= most + 4 * N + 4096
