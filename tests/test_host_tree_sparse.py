"""Tree attention and decode over selected blocks on the host side (a fake CUDA runtime, no GPU): refusals come before any
launch, a failure leaves the handle as it was, and what is launched follows the lengths."""
import ctypes

import pytest

from fake_library import FakeLayer, aligned, load


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return load(tmp_path_factory.mktemp("fake"))


class Layer(FakeLayer):
    """With buffers large enough for every call here."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.data, self.at = aligned(1 << 20)

    def tree(self, T, group=1, flags=0, **bad):
        a = dict(q=self.at, k=self.at, v=self.at, mask=self.at, out=self.at)
        a.update(bad)
        return self.lib.eigen_attn_decode_tree(self.h, a["q"], 0, 0, group, a["k"], a["v"], 0, 0, T, a["mask"], a["out"], 0, 0, flags, None)

    def sparse_attach(self, block):
        n = ctypes.c_size_t(0)
        self.check(self.lib.eigen_attn_sparse_bytes(self.h, block, ctypes.byref(n)))
        self.sparse_buf, self.sparse_at = aligned(n.value)
        self.sparse_bytes = n.value
        return self.lib.eigen_attn_sparse_attach(self.h, block, self.sparse_at, n.value, None)

    def sync(self):
        return self.lib.eigen_attn_sparse_sync(self.h, None)

    def sparse_lens(self):
        out = self.ints([0] * self.batch)
        self.check(self.lib.eigen_attn_sparse_lens(self.h, out))
        return list(out)

    def blocks(self, n_blocks, group=1, sink=1, recent=1, flags=0, q=True, out=True):
        return self.lib.eigen_attn_decode_sparse(self.h, self.at if q else None, 0, group, n_blocks, sink, recent, self.at if out else None, 0,
                                                 None, flags, None)


def test_tree_refusals_launch_nothing(lib):
    lay = Layer(lib, 2, 2, 64, 256, 32, lens=[10, 40])
    lay.launched()
    B = lay.B
    assert lay.tree(4) == B.EA_ERR_INVALID_ARG                                   # no scratch
    lay.tree_attach(8)
    for status, call in (
        (B.EA_ERR_INVALID_ARG, lambda: lay.tree(4, q=None)), (B.EA_ERR_INVALID_ARG, lambda: lay.tree(4, k=None)),
        (B.EA_ERR_INVALID_ARG, lambda: lay.tree(4, v=None)), (B.EA_ERR_INVALID_ARG, lambda: lay.tree(4, mask=None)),
        (B.EA_ERR_INVALID_ARG, lambda: lay.tree(4, out=None)), (B.EA_ERR_INVALID_ARG, lambda: lay.tree(4, mask=lay.at + 4)),
        (B.EA_ERR_INVALID_ARG, lambda: lay.tree(4, flags=8)), (B.EA_ERR_SHAPE, lambda: lay.tree(0)), (B.EA_ERR_SHAPE, lambda: lay.tree(65)),
        (B.EA_ERR_SHAPE, lambda: lay.tree(4, group=0)), (B.EA_ERR_SHAPE, lambda: lay.tree(4, group=17)),
        (B.EA_ERR_CAPACITY, lambda: lay.tree(9)), (B.EA_ERR_CAPACITY, lambda: lay.tree(4, group=3)),
    ):
        assert call() == status
    lay.set_lens([10, 253])
    assert lay.tree(4) == B.EA_ERR_CAPACITY
    assert lay.launched() == []
    assert lay.tree(3) == 0 and lay.launched() == ["mq_project_few_kernel", "mq_mma_kernel", "mq_combine_few_kernel"]
    assert lay.lens() == [10, 253]


@pytest.mark.parametrize("fail", range(1, 4))
@pytest.mark.parametrize("dtype", [0, 1])
def test_a_launch_that_fails_is_returned(lib, dtype, fail):
    """Whichever of a tree's launches fails: the status says so and the lengths stay."""
    lay = Layer(lib, 2, 2, 64, 256, 32, dtype=dtype, lens=[10, 40])
    lay.tree_attach(8)
    lay.launched()
    if fail == 1:
        lib.fake_fail(b"cudaLaunchKernel", 1)
    else:
        lib.fake_fail(b"cudaLaunchKernelExC", fail - 1)
    assert lay.tree(4) == lay.B.EA_ERR_CUDA
    assert len(lay.launched()) == fail - 1 and lay.lens() == [10, 40]


def test_lengths_of_a_captured_call(lib):
    """Unequal lengths travel with a captured call; equal ones, and calls that are not captured, need no launch for them."""
    lay = Layer(lib, 2, 2, 64, 256, 32, lens=[100, 40])
    lay.tree_attach(8)
    assert lay.sparse_attach(16) == 0 and lay.sync() == 0
    lay.launched()
    tree = ["mq_project_few_kernel", "mq_mma_kernel", "mq_combine_few_kernel"]
    sparse = ["mq_query64_kernel", "block_scores_kernel", "block_select_kernel", "mq_mma_kernel", "mq_combine_few_kernel"]
    for lens, captured, first in (([100, 40], 0, []), ([100, 40], 1, ["write_lens_kernel"]), ([100, 100], 1, []), ([100, 100], 0, [])):
        lay.set_lens(lens)
        assert lay.sync() == 0
        lay.launched()
        lib.fake_capture(captured)
        assert lay.tree(4) == 0
        lib.fake_capture(0)
        assert lay.launched() == first + tree
        lib.fake_capture(captured)
        assert lay.blocks(4) == 0
        lib.fake_capture(0)
        assert lay.launched() == first + sparse


def test_block_refusals_and_bounds(lib):
    lay = Layer(lib, 2, 2, 64, 250, 32, lens=[200, 90])
    lay.launched()
    B = lay.B
    assert lay.blocks(4) == B.EA_ERR_INVALID_ARG and lay.sync() == B.EA_ERR_INVALID_ARG      # no buffer
    n = ctypes.c_size_t(0)
    for block in (0, -16, 8, 48, 256):
        assert lib.eigen_attn_sparse_bytes(lay.h, block, ctypes.byref(n)) == B.EA_ERR_SHAPE
    lib.fake_capture(1)
    assert lay.sparse_attach(16) == B.EA_ERR_UNSUPPORTED
    lib.fake_capture(0)
    assert lay.blocks(4) == B.EA_ERR_INVALID_ARG
    assert lay.sparse_attach(16) == 0 and lay.sparse_lens() == [0, 0]
    assert lib.eigen_attn_sparse_attach(lay.h, 16, lay.sparse_at + 16, lay.sparse_bytes, None) == B.EA_ERR_INVALID_ARG
    assert lib.eigen_attn_sparse_attach(lay.h, 16, lay.sparse_at, lay.sparse_bytes - 1, None) == B.EA_ERR_CAPACITY
    assert lay.blocks(4) == B.EA_ERR_INVALID_ARG                                 # no bounds yet
    lib.fake_capture(1)
    assert lay.sync() == B.EA_ERR_UNSUPPORTED and lay.sparse_lens() == [0, 0]
    lib.fake_capture(0)
    lib.fake_fail(b"cudaLaunchKernel", 1)
    assert lay.sync() == B.EA_ERR_CUDA and lay.sparse_lens() == [0, 0]
    assert lay.launched() == []
    assert lay.sync() == 0 and lay.sparse_lens() == [192, 80] and lay.launched() == ["block_bounds_kernel"]
    lib.fake_capture(1)
    assert lay.sync() == 0 and lay.launched() == []                              # nothing to do
    lib.fake_capture(0)
    for args, status in (((0,), -2), ((4, 0), -2), ((4, 17), -2), ((4, 1, -1), -2), ((4, 1, 1, 0), -2), ((4, 1, 3, 2), -2), ((4, 1, 2 ** 31 - 1, 1), -2),
                         ((4, 1, 1, 1, 4), -1), ((4, 1, 1, 1, 0, False), -1), ((4, 1, 1, 1, 0, True, False), -1)):
        assert lay.blocks(*args) == status, args
    assert lay.launched() == []
    lay.set_lens([200, 0])
    assert lay.blocks(4) == -2                                                   # a sequence without rows
    lay.set_lens([150, 90])                                                      # shorter: the blocks it no longer fills are forgotten
    assert lay.sparse_lens() == [144, 0]
    lay.set_lens([200, 90])
    assert lay.blocks(4) == B.EA_ERR_INVALID_ARG and lay.sync() == 0 and lay.blocks(4) == 0


def test_page_tables(lib):
    """Pages of a tree's and a block list's sequences: changes forget the bounds, refused tables change nothing."""
    lay = Layer(lib, 2, 1, 64, 256, 32, lens=[200, 90])
    lay.tree_attach(8)
    assert lay.sparse_attach(16) == 0 and lay.sync() == 0
    lay.launched()

    def table(entries, width, rows=128):
        return lib.eigen_attn_set_page_table(lay.h, lay.ints(entries), width, rows, None)
    for entries, width, rows in (([0, 1, 2, 4], 2, 128), ([0, 1, 1, 2], 2, 128), ([0, -1, 1, 2], 2, 128), ([-1, 0, 1, 2], 2, 128),
                                 ([0, 1, 2, 3], 2, 100), ([0, 1, 2, 3], 2, 64), ([0, 1, 2, 3], 0, 128)):
        assert table(entries, width, rows) != 0, entries
        assert lay.sparse_lens() == [192, 80]
    assert table([3, 1, 2, -1], 2) == 0 and lay.sparse_lens() == [0, 0]
    assert lay.blocks(4) == lay.B.EA_ERR_INVALID_ARG
    assert lay.sync() == 0 and lay.blocks(4) == 0 and lay.tree(8) == 0
    lay.set_lens([200, 122])
    assert lay.tree(7) == lay.B.EA_ERR_CAPACITY and lay.tree(6) == 0             # one page: 128 rows
    assert lay.tree_commit([[0], [0, 1, 2, 3, 4, 5, 6]], 7) == lay.B.EA_ERR_CAPACITY
    assert lay.tree_commit([[0], [0, 2, 5]], 6) == 0 and lay.lens() == [201, 125]
