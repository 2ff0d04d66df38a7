"""Host side of the training calls and of the learned bias (a fake CUDA runtime, no GPU): arguments, what is launched in which
order, what a failing call of the runtime leaves."""
import ctypes

import numpy as np
import pytest

from fake_library import FakeLayer, aligned, load
from oracle import training as oracle

BF16, FP32 = 0, 1
INVALID, SHAPE, UNSUPPORTED, CAPACITY, CUDA = "EA_ERR_INVALID_ARG", "EA_ERR_SHAPE", "EA_ERR_UNSUPPORTED", "EA_ERR_CAPACITY", "EA_ERR_CUDA"
NAMES = ["bias_expand_kernel", "bias_reduce_kernel", "train_pack_kernel", "train_forward_kernel", "train_backward_kernel",
         "train_simt_forward_kernel", "train_simt_dq_kernel", "train_simt_dkv_kernel"]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return load(tmp_path_factory.mktemp("fake"))


class Layer(FakeLayer):
    def __init__(self, lib, dtype=BF16, batch=2, n_max=256):
        super().__init__(lib, batch, 2, 64, n_max, 32, dtype=dtype, lens=[8] * batch)
        self.some, self.at = aligned(1 << 20)
        self.launched()

    def launched(self):
        text = self.lib.fake_log().decode()
        self.lib.fake_reset()
        return [next((k for k in NAMES if k in line), line) for line in text.split("\n") if line]

    def is_(self, status, want):
        assert status == (0 if want is None else getattr(self.B, want)), self.lib.eigen_attn_last_error(self.h)

    def bias_attach(self, n_buckets=8, far=20, want=None, less=0, shift=0):
        n = ctypes.c_size_t(0)
        self.check(self.lib.eigen_attn_bias_bytes(self.h, n_buckets, far, ctypes.byref(n)))
        self.bias_buf, at = aligned(n.value + 256)
        self.is_(self.lib.eigen_attn_bias_attach(self.h, n_buckets, far, at + shift, n.value - less, None), want)

    def train_attach(self, tokens=200, group=1, want=None, less=0, shift=0):
        n = ctypes.c_size_t(0)
        self.check(self.lib.eigen_attn_train_bytes(self.h, tokens, group, ctypes.byref(n)))
        self.train_buf, at = aligned(n.value + 256)
        self.is_(self.lib.eigen_attn_train_attach(self.h, tokens, group, at + shift, n.value - less), want)

    def forward(self, T=200, group=1, want=None, lens=None, null=None):
        at = [None if i == null else self.at for i in range(4)]
        self.is_(self.lib.eigen_attn_train_forward(self.h, at[0], at[1], at[2], T, group, lens, at[3], None), want)

    def backward(self, want=None, table=False, null=None):
        at = [None if i == null else self.at for i in range(4)]
        self.is_(self.lib.eigen_attn_train_backward(self.h, *at, self.at if table else None, None), want)

    def alibi(self, slopes):
        return self.lib.eigen_attn_set_alibi(self.h, (ctypes.c_float * 2)(*slopes) if slopes else None, None)


FORWARD = {BF16: ["train_pack_kernel", "train_forward_kernel"], FP32: ["train_simt_forward_kernel"]}
BACKWARD = {BF16: ["train_pack_kernel", "train_backward_kernel"], FP32: ["train_simt_dq_kernel", "train_simt_dkv_kernel"]}


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_launches(lib, dtype):
    lay = Layer(lib, dtype)
    lay.train_attach(group=4)
    lay.forward(group=4)
    assert lay.launched() == FORWARD[dtype]
    lay.backward()
    lay.backward()
    assert lay.launched() == 2 * BACKWARD[dtype]
    lay.bias_attach()
    assert lay.launched() == []
    lay.is_(lib.eigen_attn_bias_set(lay.h, lay.at, None), None)
    assert lay.launched() == ["bias_expand_kernel"]
    lay.forward()
    lay.backward()
    lay.backward(table=True)
    assert lay.launched() == FORWARD[dtype] + 2 * BACKWARD[dtype] + ["bias_reduce_kernel"]
    assert lay.lens() == [8, 8]


def test_refusals_of_the_training_calls(lib):
    lay = Layer(lib)
    lay.forward(want=INVALID)                                # no scratch
    lay.backward(want=INVALID)
    n = ctypes.c_size_t(0)
    for tokens, group in ((0, 1), ((1 << 20) + 1, 1), (5, 0), (5, 17)):
        lay.is_(lib.eigen_attn_train_bytes(lay.h, tokens, group, ctypes.byref(n)), SHAPE)
        lay.is_(lib.eigen_attn_train_attach(lay.h, tokens, group, lay.at, 1 << 20), SHAPE)
    lay.is_(lib.eigen_attn_train_bytes(lay.h, 5, 1, None), INVALID)
    lay.train_attach(want=CAPACITY, less=1)
    lay.train_attach(want=INVALID, shift=128)
    lay.forward(want=INVALID)
    lay.train_attach(200, 2)
    lay.backward(want=INVALID)                               # no forward pass yet
    for i in range(4):
        lay.forward(want=INVALID, null=i)
    lay.forward(T=0, want=SHAPE)
    lay.forward(group=0, want=SHAPE)
    lay.forward(T=201, want=CAPACITY)
    lay.forward(group=3, want=CAPACITY)
    assert lay.launched() == []
    lay.forward(T=7, group=2)
    lay.launched()
    for i in range(4):
        lay.backward(want=INVALID, null=i)
    lay.backward(table=True, want=INVALID)                   # no bias attached
    lay.forward(T=201, want=CAPACITY)                        # a refused call leaves the pass before it
    lay.backward()
    assert lay.launched() == BACKWARD[BF16]
    lay.train_attach()                                       # another scratch holds no pass
    lay.backward(want=INVALID)
    lay.is_(lib.eigen_attn_train_attach(lay.h, 0, 0, None, 0), None)
    lay.forward(want=INVALID)


def test_position_biases_of_the_training_calls(lib):
    lay = Layer(lib)
    lay.train_attach(group=2)
    lay.is_(lay.alibi([0.5, 0.25]), None)
    lay.forward(group=2, want=UNSUPPORTED)
    lay.forward()
    lay.is_(lay.alibi([0.5, 0.125]), None)
    lay.backward(want=INVALID)                               # not the bias that the forward pass had
    lay.forward()
    lay.backward()
    lay.is_(lay.alibi(None), None)
    lay.bias_attach()
    lay.forward(group=2, want=UNSUPPORTED)
    lay.forward()
    lay.is_(lib.eigen_attn_bias_set(lay.h, lay.at, None), None)
    lay.backward(want=INVALID)
    lay.forward()
    lay.is_(lib.eigen_attn_bias_attach(lay.h, 0, 0, None, 0, None), None)
    lay.backward(want=INVALID)


def test_refusals_of_the_learned_bias(lib):
    lay = Layer(lib)
    n = ctypes.c_size_t(0)
    for n_buckets, far in ((1, 5), (257, 1000), (8, 4), (8, 32769), (2, 1)):
        lay.is_(lib.eigen_attn_bias_bytes(lay.h, n_buckets, far, ctypes.byref(n)), SHAPE)
        lay.is_(lib.eigen_attn_bias_attach(lay.h, n_buckets, far, lay.at, 1 << 20, None), SHAPE)
    starts = (ctypes.c_int32 * 8)()
    lay.is_(lib.eigen_attn_bias_starts(lay.h, starts), INVALID)
    lay.is_(lib.eigen_attn_bias_set(lay.h, lay.at, None), INVALID)
    lay.bias_attach(want=CAPACITY, less=1)
    lay.bias_attach(want=INVALID, shift=16)
    lib.fake_capture(1)
    lay.bias_attach(want=UNSUPPORTED)
    lib.fake_capture(0)
    lay.is_(lib.eigen_attn_bias_starts(lay.h, starts), INVALID)          # none of them attached anything
    lay.is_(lay.alibi([0.5, 0.25]), None)
    lay.bias_attach(want=INVALID)
    lay.is_(lay.alibi(None), None)
    lay.bias_attach()
    lay.is_(lib.eigen_attn_bias_set(lay.h, None, None), INVALID)
    lay.is_(lay.alibi([0.5, 0.25]), INVALID)
    lay.is_(lay.alibi(None), None)                           # none to none
    lay.is_(lib.eigen_attn_bias_starts(lay.h, None), INVALID)
    lay.is_(lib.eigen_attn_bias_starts(lay.h, starts), None)
    lib.fake_capture(1)                                      # a table can be set inside a capture
    lay.is_(lib.eigen_attn_bias_set(lay.h, lay.at, None), None)
    lib.fake_capture(0)


def test_calls_that_do_not_know_the_learned_bias(lib):
    lay = Layer(lib)
    lay.tree_attach(4)
    n = ctypes.c_size_t(0)
    lay.is_(lib.eigen_attn_quant_bytes(lay.h, 4, 32, ctypes.byref(n)), None)
    lay.codes, at = aligned(n.value)
    lay.is_(lib.eigen_attn_quant_attach(lay.h, 4, 32, at, n.value, None), None)
    lay.is_(lib.eigen_attn_sparse_bytes(lay.h, 64, ctypes.byref(n)), None)
    lay.bounds, at = aligned(n.value)
    lay.is_(lib.eigen_attn_sparse_attach(lay.h, 64, at, n.value, None), None)
    lay.bias_attach()
    lay.launched()
    lay.is_(lib.eigen_attn_decode_gqa(lay.h, lay.at, 256, 2, lay.at, 256, 0, None), UNSUPPORTED)
    lay.is_(lib.eigen_attn_decode_quant(lay.h, lay.at, 128, lay.at, 128, 0, None), UNSUPPORTED)
    lay.is_(lib.eigen_attn_decode_tree(lay.h, lay.at, 256, 128, 1, lay.at, lay.at, 256, 128, 2, lay.at, lay.at, 256, 128, 0, None), UNSUPPORTED)
    lay.is_(lib.eigen_attn_decode_sparse(lay.h, lay.at, 128, 1, 2, 1, 1, lay.at, 128, None, 0, None), UNSUPPORTED)
    assert lay.launched() == [] and lay.lens() == [8, 8]


@pytest.mark.parametrize("n_buckets,far", [(2, 2), (3, 7), (5, 3), (32, 128), (64, 1024), (255, 130), (256, 32768)])
def test_starts_are_the_first_distances(lib, n_buckets, far):
    """A bucket starts at the first distance whose bucket is that one or a later one."""
    lay = Layer(lib)
    lay.bias_attach(n_buckets, far)
    starts = (ctypes.c_int32 * n_buckets)()
    lay.is_(lib.eigen_attn_bias_starts(lay.h, starts), None)
    assert list(starts) == sorted(starts) and starts[0] == 0 and starts[n_buckets - 1] <= far
    for u, d in enumerate(starts):
        if u % 16 in (0, 1) or n_buckets <= 64:              # (exact powers of large numbers take long)
            assert oracle.bucket_of(d, n_buckets, far) >= u
            assert d == 0 or oracle.bucket_of(d - 1, n_buckets, far) < u


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_failed_launch_leaves_no_pass(lib, dtype):
    lay = Layer(lib, dtype)
    lay.train_attach()
    lay.forward()
    for which in range(len(FORWARD[dtype])):
        fn = b"cudaLaunchKernelExC" if which == 1 else b"cudaLaunchKernel"
        lib.fake_fail(fn, 1)
        lay.forward(want=CUDA)
        lay.backward(want=INVALID)
        lay.forward()
    lay.launched()
    lib.fake_fail(b"cudaLaunchKernel", 1)
    lay.backward(want=CUDA)
    assert lay.launched() == []
    lay.backward()                                           # the same call again does all of it
    assert lay.launched() == BACKWARD[dtype]


@pytest.mark.parametrize("fn", [b"cudaMemcpyAsync", b"cudaMemsetAsync", b"cudaStreamSynchronize"])
def test_a_failed_attach_leaves_no_bias(lib, fn):
    lay = Layer(lib)
    lib.fake_fail(fn, 1)
    lay.bias_attach(want=CUDA)
    lay.is_(lib.eigen_attn_bias_set(lay.h, lay.at, None), INVALID)
    lay.is_(lay.alibi([0.5, 0.25]), None)                    # no bias in its way


def test_null_handles(lib):
    n = ctypes.c_size_t(0)
    for status in (lib.eigen_attn_bias_bytes(None, 8, 20, ctypes.byref(n)), lib.eigen_attn_bias_attach(None, 8, 20, None, 0, None),
                   lib.eigen_attn_bias_set(None, None, None), lib.eigen_attn_bias_starts(None, None),
                   lib.eigen_attn_train_bytes(None, 8, 1, ctypes.byref(n)), lib.eigen_attn_train_attach(None, 8, 1, None, 0),
                   lib.eigen_attn_train_forward(None, None, None, None, 1, 1, None, None, None),
                   lib.eigen_attn_train_backward(None, None, None, None, None, None, None)):
        assert status == -1
