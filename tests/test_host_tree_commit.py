"""tree_commit on the host side (a fake CUDA runtime, no GPU): a call that fails changes nothing."""
import pytest

from fake_library import FakeLayer, load


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return load(tmp_path_factory.mktemp("fake"))


UNEQUAL = [[0, 2, 5], [1], []]


def test_lengths_and_launches(lib):
    lay = FakeLayer(lib, 3, 2, 64, 256, 32, lens=[100, 40, 7])
    lay.launched()
    assert lay.tree_commit(UNEQUAL, 8) == 0
    assert lay.lens() == [103, 41, 7] and lay.launched() == ["tree_commit_kernel"]
    assert lay.tree_commit([[0, 1]] * 3, 8) == 0                 # a chain: nothing to move
    assert lay.lens() == [105, 43, 9] and lay.launched() == []
    assert lay.tree_commit([[1, 3]] * 3, 8) == 0
    assert lay.lens() == [107, 45, 11] and lay.launched() == ["tree_commit_kernel"]


def test_a_failed_upload_of_the_lengths_moves_no_row(lib):
    lay = FakeLayer(lib, 3, 2, 64, 256, 32, lens=[100, 40, 7])
    lay.launched()
    lib.fake_fail(b"cudaMemcpyAsync", 1)
    assert lay.tree_commit(UNEQUAL, 8) == lay.B.EA_ERR_CUDA
    assert lay.lens() == [100, 40, 7] and lay.launched() == []
    assert lay.tree_commit(UNEQUAL, 8) == 0                      # the same call again does all of it
    assert lay.lens() == [103, 41, 7] and lay.launched() == ["tree_commit_kernel"]


@pytest.mark.parametrize("paths", [UNEQUAL, [[1, 3]] * 3])
def test_a_failed_launch_leaves_the_lengths(lib, paths):
    lay = FakeLayer(lib, 3, 2, 64, 256, 32, lens=[100, 40, 7])
    lay.launched()
    lib.fake_fail(b"cudaLaunchKernel", 1)
    assert lay.tree_commit(paths, 8) == lay.B.EA_ERR_CUDA
    assert lay.lens() == [100, 40, 7] and lay.launched() == []


def test_refusals_change_nothing(lib):
    lay = FakeLayer(lib, 3, 2, 64, 256, 32, lens=[100, 40, 7])
    lay.launched()
    for paths, T, status in (([[0, 0], [], []], 8, -1), ([[2, 1], [], []], 8, -1), ([[8], [], []], 8, -1), ([[-1], [], []], 8, -1),
                             ([[], [], []], 65, -2), ([[], [], []], 0, -2)):
        assert lay.tree_commit(paths, T) == status
    lib.fake_capture(1)
    assert lay.tree_commit(UNEQUAL, 8) == lay.B.EA_ERR_UNSUPPORTED
    lib.fake_capture(0)
    assert lay.lens() == [100, 40, 7] and lay.launched() == []
