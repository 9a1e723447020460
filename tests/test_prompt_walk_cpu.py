"""How a launch over packed prompts goes about its rows, compiled for the host: the choice of
walk as the GPU tests state it, and the order of the workgroups."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2512_11221_amd import build
from tests import _walks

HERE = os.path.dirname(os.path.abspath(__file__))
CUS = 256


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("walk") / "prompt_check.so")
    subprocess.run([build.hipcc(), "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-shared",
                    os.path.join(HERE, "split", "prompt_check.cpp"), "-o", out], check=True,
                   stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    return ctypes.CDLL(out)


def _choice(lib, Hq, Hkv, D, dtype, lens):
    lens = [n for n in lens if n]
    walk, rows = ctypes.c_int(), ctypes.c_int()
    waves = lib.prompt_choice(dtype == "bf16", D, Hq // Hkv, Hkv, (ctypes.c_int32 * len(lens))(*lens), len(lens),
                              ctypes.byref(walk), ctypes.byref(rows))
    name = {(0, 4): _walks.TEAM4, (0, 8): _walks.TEAM8, (1, 4): _walks.SPLIT, (2, 8): _walks.HALVES}[walk.value, waves]
    return name, walk.value, waves, rows.value


def _order(lib, D, dtype, walk, waves, blocks, Hkv):
    units = (ctypes.c_int32 * blocks)()
    fold = lib.prompt_order(dtype == "bf16", D, walk, waves, blocks, Hkv, units)
    return fold, list(units)


def _layout(rng):
    dtype = rng.choice(["bf16", "f32"])
    D = rng.choice([64, 128, 256] if dtype == "bf16" else [64, 128])
    group, Hkv = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
    return group * Hkv, Hkv, D, dtype


def test_walks_as_the_gpu_tests_state_them(lib):
    rng = random.Random(2)
    seen = set()
    for _ in range(4000):
        Hq, Hkv, D, dtype = _layout(rng)
        n = rng.choice([1, 1, 2, 3, 8, 30, 128])
        lens = [rng.choice([0, 1]) if rng.random() < 0.1 else int(2 ** rng.uniform(0, 14 if n < 8 else 11)) for _ in range(n)] + [1]
        lens = lens[-128:]
        want = _choice(lib, Hq, Hkv, D, dtype, lens)[0]
        assert _walks.walk(Hq, Hkv, D, dtype, lens) == want
        seen.add((want, dtype, D))
    assert {w for w, _, _ in seen} == {_walks.TEAM4, _walks.TEAM8, _walks.SPLIT, _walks.HALVES}


def test_every_block_is_taken_once(lib):
    rng = random.Random(3)
    for _ in range(500):
        Hq, Hkv, D, dtype = _layout(rng)
        blocks = rng.randint(1, 700)
        for walk, waves in ((0, 4), (0, 8), (1, 4), (2, 8)):
            fold, units = _order(lib, D, dtype, walk, waves, blocks, Hkv)
            assert sorted(units) == list(range(blocks)) and units[:fold] == list(range(fold))


def _greedy(work, slots):
    """The time at which the last of `slots` ends, each taking the next piece of work when it is free."""
    free = [0] * slots
    for w in work:
        i = min(range(slots), key=free.__getitem__)
        free[i] += w
    return max(free)


@pytest.mark.parametrize("lens", [[2048, 2048], [4000], [1500, 2500], [700] * 5], ids=str)
def test_rows_of_256_keep_the_longest_blocks_in_front(lib, lens):
    """A CU has room for one workgroup of four waves with rows of 256.  In the order of the launch the
    last CU ends no later than with every prompt's blocks from its longest on."""
    Hq, Hkv, D = 16, 8, 256
    name, walk, waves, rows = _choice(lib, Hq, Hkv, D, "bf16", lens)
    assert name == _walks.TEAM4
    tiles = []                                   # of every unit of a KV head: the last block of a prompt first
    for n in sorted(lens, reverse=True):
        blocks = -(-n * (Hq // Hkv) // rows)
        tiles += [min(n - 1, ((b + 1) * rows - 1) // (Hq // Hkv)) // 32 + 1 for b in reversed(range(blocks))]
    _, units = _order(lib, D, "bf16", walk, waves, len(tiles), Hkv)
    assert CUS < len(tiles) * Hkv <= 2 * CUS
    ends = _greedy([tiles[u] for u in units for _ in range(Hkv)], CUS)
    straight = _greedy([t for t in tiles for _ in range(Hkv)], CUS)
    assert ends <= straight, (ends, straight)


@pytest.mark.parametrize("Hq,Hkv,D,dtype", [(64, 32, 64, "bf16"), (64, 8, 128, "bf16"), (64, 8, 256, "bf16"), (64, 16, 64, "f32")])
def test_the_longest_launch_fits_a_grid(lib, Hq, Hkv, D, dtype):
    """The threads of a launch with as many tokens as are taken into one, whatever memory would hold:
    a workgroup for every block of rows and for every 16 tokens' store."""
    lib.prompt_max_tokens.restype = ctypes.c_int64
    top = lib.prompt_max_tokens()
    for lens in ([top], [top // 128] * 128, [top - 127] + [1] * 127):
        _, _, waves, rows = _choice(lib, Hq, Hkv, D, dtype, lens)
        blocks = sum(-(-n * (Hq // Hkv) // rows) for n in lens) * Hkv + sum(-(-n // 16) for n in lens)
        assert blocks * waves * 64 < 1 << 32


def test_offsets_within_a_tile(lib):
    """... of the longest token stride are 32-bit, the last row's end included."""
    lib.prompt_max_stride.restype = ctypes.c_int64
    assert (lib.prompt_max_tile() - 1) * lib.prompt_max_stride() + 1024 < 1 << 31
