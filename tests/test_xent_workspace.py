"""What the head's loss asks for as a workspace (no GPU needed): nothing for copies that are not made, pieces of bounded size."""
import pytest

pytest.importorskip("torch")

from paper_2510_20271_amd import _lib, api

MB = 1 << 20
F32, F16, BF16 = 2, 3, 6
HALVES = (F16, BF16)


def _bytes(rows, dim, classes, dtype, backward, aligned=True):
    return api.ecc_xent_workspace_bytes(rows, dim, classes, dtype, backward, aligned)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,dim,classes", [(1, 4096, 131072), (8, 16384, 131072), (64, 65536, 131072), (1, 8, 8)])
def test_few_rows_of_whole_chunks(rows, dim, classes, dtype):
    """No copy of the weight: a maximum and a sum for each row and 32 classes or more, dz, and split sums of hidden's gradient."""
    assert _bytes(rows, dim, classes, dtype, False) <= rows * (classes + 128) // 32 * 8 + 64 * rows + MB
    assert _bytes(rows, dim, classes, dtype, True) <= 4 * rows * (classes + 8) + 256 * MB + MB


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_voxels(dtype):
    """A 256^3 volume's voxels, 64 features, 21 classes: no copy of the features (2.1 GB in 16 bits), 4 bytes a logit's gradient."""
    rows = 256 ** 3
    assert _bytes(rows, 64, 21, dtype, False) <= rows * 24 + MB
    assert _bytes(rows, 64, 21, dtype, True) <= rows * (24 * 4 + 8) + 2 * 256 * MB


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,dim,classes", [(1, 4095, 131072), (8, 16383, 131072), (64, 65535, 131072)])
def test_copies_of_odd_rows_are_made_in_pieces(rows, dim, classes, dtype, backward):
    size = 4 if dtype == F32 else 2
    room = 1024 * MB + rows * (dim + 8) * size + 4 * rows * (classes + 8) + 2 * 256 * MB + MB
    assert _bytes(rows, dim, classes, dtype, backward) <= room
    # operands off their alignment need the same copies where their rows are whole chunks
    assert _bytes(rows, dim + 1, classes, dtype, backward, aligned=False) <= room


def test_flags():
    query = _lib.load().ecc_xent_workspace_bytes
    for dtype in (F32, F16, BF16):
        for rows, dim, classes in ((1, 64, 1000), (300, 96, 5000), (4096, 512, 10007), (100000, 64, 21), (7, 63, 100)):
            for back in (0, api.ECC_XENT_BACKWARD):
                any_alignment, aligned = query(rows, dim, classes, dtype, back), query(rows, dim, classes, dtype, back | api.ECC_XENT_ALIGNED)
                assert 0 < aligned <= any_alignment
                assert (aligned == any_alignment) == (dim % (4 if dtype == F32 else 8) != 0)
    assert query(4, 8, 16, F32, 4) == 0 and query(4, 8, 16, F32, -1) == 0


def test_largest_sizes():
    """Rows and classes up to 2^31 - 256: one tile of the smallest kind more would be a grid of 2^32 threads."""
    for back in (0, 1):
        assert _lib.load().ecc_xent_workspace_bytes(2 ** 31 - 256, 1, 2, F32, back) > 0
        for rows, classes in ((2 ** 31 - 255, 2), (2, 2 ** 31 - 255)):
            assert _lib.load().ecc_xent_workspace_bytes(rows, 1, classes, F32, back) == 0
            assert "2^31 - 256" in _lib.load().ecc_last_error().decode()
