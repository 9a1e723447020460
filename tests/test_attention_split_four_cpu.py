"""The split of the attention kernel's work over rows held in 4 bits (tiles of 64 tokens, of 32 with
rows of 256, and their room for relevance values), compiled for the host, as
tests/test_attention_split_cpu.py has it for rows of 16 and 32 bits."""
import ctypes
import random

import pytest

from tests.test_attention_split_cpu import GRID, _check, _ints, lib  # noqa: F401


def _heads(lib, plen, hkv, dim, t=1):
    launch = ctypes.c_int()
    hw = lib.split_layout_four(_ints(plen), len(plen), t, hkv, dim, GRID, ctypes.byref(launch))
    assert 1 <= launch.value <= GRID
    return hw, launch.value


def test_tiles_and_room(lib):  # noqa: F811
    """A wave's room holds whole tiles of every head that the workgroup's waves take (each of eight
    query heads under the softmax reading)."""
    for dim, tile in ((64, 64), (128, 64), (256, 32)):
        assert lib.split_tile_four(dim) == tile
        per_wave = lib.split_room_four(dim) // 8
        assert per_wave * tile * 4 <= (4096 if dim == 256 else 6144)
        assert per_wave // 8 >= 1


def test_launch_covers_the_workgroups_with_work(lib):  # noqa: F811
    """Lists up to plen + t long, and shorter ones after freezing: every tile falls to one workgroup,
    and the launched ones are at least those with work."""
    rng = random.Random(19)
    heads = set()
    for _ in range(600):
        batch = rng.choice([1, 2, 8, 33, 64, 65, 100])
        hkv, dim = rng.choice([(1, 64), (2, 128), (8, 128), (8, 256), (32, 128), (32, 64), (16, 256)])
        t = rng.randint(1, 40)
        plen = [rng.randint(0, int(2 ** rng.uniform(0, 15 if batch < 9 else 12))) for _ in range(batch)]
        hw, launch = _heads(lib, plen, hkv, dim, t)
        heads.add(hw)
        full = [p + t for p in plen]
        for n in (full, [max(1, int(x * rng.uniform(0.2, 1))) for x in full]):
            _, live, _ = _check(lib, n, hkv, hw, lib.split_tile_four(dim))
            assert live <= launch
    assert {1, 8} <= heads


# the lists of the GPU tests: (lengths at the first step, KV heads, head dim) -> heads together, and
# whether a workgroup has more tiles than room (under the softmax reading a plane per query head)
SHORT = lambda batch: [2 + (37 * b * b + 11 * b) % 90 for b in range(batch)]   # noqa: E731
GPU_CASES = {
    "long-shared": ([20001, 9001], 2, 128, 1, 1, False),
    "long-heads": ([33001] * 8 + [2, 701], 8, 64, 1, 1, False),
    "long-softmax": ([33001] * 4, 8, 64, 4, 1, True),
    "long-rows256": ([17001] * 5, 8, 256, 1, 1, False),
    "longer-rows64": ([50001] * 8 + [2, 701], 8, 64, 1, 8, True),
    "longer-rows128": ([50001] * 8 + [2, 701], 8, 128, 1, 8, True),
    "longer-rows256": ([33001] * 8 + [301], 8, 256, 1, 8, True),
    "longer-softmax": ([50001] * 8, 8, 64, 8, 8, True),
    "together-40": (SHORT(40), 8, 128, 1, 2, False),
    "together-70": (SHORT(70), 8, 64, 1, 4, False),
    "together-70-rows256": (SHORT(70), 8, 256, 1, 4, False),
    "together-300": (SHORT(300), 8, 128, 1, 8, False),
}


@pytest.mark.parametrize("name", sorted(GPU_CASES))
def test_forms_of_the_gpu_cases(lib, name):  # noqa: F811
    n, hkv, dim, planes, want_hw, want_full = GPU_CASES[name]
    hw, _ = _heads(lib, [x - 1 for x in n], hkv, dim)
    _, _, p = _check(lib, n, hkv, hw, lib.split_tile_four(dim))
    longest = (p[:, 5] - p[:, 4]).max() * hw           # of one piece, a tile of every head
    assert (hw, bool(longest > lib.split_room_four(dim) // planes)) == (want_hw, want_full)
