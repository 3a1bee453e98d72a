"""The product tile's loads into LDS as the compiler lays them out (no GPU needed): the wait states that the instruction asks for."""
import re
import subprocess

import pytest

from paper_2410_01799_amd import build

SOURCE = """
#include "scd_lm_tile.h"
using namespace scd::lm;
template <class Q>
__device__ void product(TileRows a, TileRows b, int steps, float* out)
{
    __shared__ __align__(128) char lds[Q::kLds];
    typename Q::Acc acc[Q::FA][Q::FB];
    Q::run(a, b, blockIdx.x * Q::TA, blockIdx.y * Q::TB, steps, lds, acc);
    for (int i = 0; i < Q::FA; ++i)
        for (int j = 0; j < Q::FB; ++j) *(typename Q::Acc*)(out + ((threadIdx.x * Q::FA + i) * Q::FB + j) * 4) = acc[i][j];
}
extern "C" __global__ __launch_bounds__(256) void both_along(TileRows a, TileRows b, int s, float* o) { product<Tile<OpBf16, 2, 2, 2, 2, true, true, 3>>(a, b, s, o); }
extern "C" __global__ __launch_bounds__(256) void one_along(TileRows a, TileRows b, int s, float* o) { product<Tile<OpF16, 4, 4, 2, 2, false, true, 2>>(a, b, s, o); }
extern "C" __global__ __launch_bounds__(256) void two_planes(TileRows a, TileRows b, int s, float* o) { product<Tile<OpBf16, 2, 2, 2, 2, false, false, 3, 2>>(a, b, s, o); }
extern "C" __global__ __launch_bounds__(256) void split(TileRows a, TileRows b, int s, float* o) { product<Tile<OpSplit, 2, 2, 2, 2, false, true, 3>>(a, b, s, o); }
extern "C" __global__ __launch_bounds__(512) void bytes(TileRows a, TileRows b, int s, float* o) { product<Tile<OpI8, 8, 4, 2, 4, true, true, 2>>(a, b, s, o); }
"""


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    where = tmp_path_factory.mktemp("tile")
    (where / "tile.hip").write_text(SOURCE)
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-Wall")]
    got = subprocess.run([build.hipcc(), *flags, f"-I{build.ROOT / 'include'}", f"-I{build.PKG / 'csrc'}", "--cuda-device-only", "-S", str(where / "tile.hip"),
                          "-o", str(where / "tile.s")], capture_output=True, text=True)
    assert got.returncode == 0, got.stderr
    lines = [line.split(";")[0].strip() for line in (where / "tile.s").read_text().splitlines()]
    return [line for line in lines if line and not line.startswith(".") and not line.endswith(":")]


def scalars(text):
    """Numbers of the scalar registers that an operand names."""
    found = set()
    for low, high, one in re.findall(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        found |= set(range(int(low), int(high) + 1)) if low else {int(one)}
    return found


def test_loads_into_lds_keep_their_distance_from_what_they_read(code):
    """One state between a write of M0 and a load with the LDS bit, five between a vector instruction that writes a scalar register and a
    load that takes its resource from it.  An instruction is a state, s_nop n is n + 1."""
    loads = 0
    for i, line in enumerate(code):
        if not (line.startswith("buffer_load") and line.endswith(" lds")):
            continue
        loads += 1
        resource, states = scalars(line.split(",")[1]), 0
        for before in reversed(code[max(0, i - 8):i]):
            name, _, operands = before.partition(" ")
            if name == "s_nop":
                states += int(operands, 0) + 1
                continue
            to = operands.split(",")[0].strip()
            assert to != "m0" or states >= 1, f"{before} / {line}"
            assert not (name.startswith("v_") and scalars(to) & resource) or states >= 5, f"{before} / {line}"
            states += 1
    assert loads >= 5 * 8
