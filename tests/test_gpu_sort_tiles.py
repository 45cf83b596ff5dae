"""The plain ID sort around the sizes at which its tiles change: 512 keys up to
131,072 (65,536 where a digit has 11 bits), 1024 up to 262,144, 2048 above;
against a stable sort, which the outputs equal element for element."""
import pytest
import torch

import paper_2205_11048_amd as gba
import test_gpu_small_sort as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [1, 8, 9, 10, 11, 16, 18, 20, 22, 24, 27, 32])
@pytest.mark.parametrize("n", [32_769, 65_535, 65_536, 65_537, 131_071, 131_072, 131_073, 262_143, 262_144, 262_145])
def test_sort_tile_lines(n, bits):
    R = 1 << bits
    ids = base._ids(n, R, n % 1013 + bits, 3.0)
    keys, index, err = base._sort(ids, R)
    ref, ref_index = torch.sort(ids, stable=True)
    assert err == 0
    assert torch.equal(keys, ref) and torch.equal(index, ref_index)


@pytest.mark.parametrize("n", [65_537, 131_073, 262_145])
def test_one_id_and_bad_ids(n):
    base.test_sort_one_id_and_bad_ids(n)


@pytest.mark.parametrize("bits", [9, 11, 18, 22, 27])
@pytest.mark.parametrize("n", [65_537, 131_073, 262_145])
def test_the_largest_sizes_workspace_serves_smaller_ones(n, bits):
    """Scratch asked for at one size is taken by every smaller one."""
    R = 1 << bits
    room = gba.gba_sort_ids_workspace_size(n, R, gba.SORT_PLAIN)
    for m in (n, n - 1, n // 2 + 1, n // 4 + 1):
        assert gba.gba_sort_ids_workspace_size(m, R, gba.SORT_PLAIN) <= room
