"""Where the training calls' launches point to in the caller's scratch (a fake CUDA runtime that keeps what a launch gets, no
GPU)."""
import ctypes
import os
import subprocess

import pytest

from fake_library import FakeLayer, HERE, aligned

BF16, FP32 = 0, 1
WORDS = 40


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2408_05646_b200 import binding, build
    build.build_library()
    objects = [os.path.join(build.BUILD, src.replace(".cu", ".o")) for src in build.SOURCES]
    path = os.path.join(str(tmp_path_factory.mktemp("args")), "libargs.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", path,
                    os.path.join(HERE, "fake_launch_args.cpp")] + objects, check=True)
    lib = ctypes.CDLL(path)
    for name, (res, args) in binding.SYMBOLS.items():
        getattr(lib, name).restype, getattr(lib, name).argtypes = res, args
    return lib


def launches(lib):
    """Words of the first argument of every training kernel's launch since the last question."""
    out = []
    for i in range(lib.fake_launches()):
        words = (ctypes.c_size_t * WORDS)()
        lib.fake_args(i, words)
        out.append(list(words))
    lib.fake_forget_args()
    return out


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("attached", [1, 2, 16])
@pytest.mark.parametrize("T", [1, 33, 200])
def test_the_bias_sums_lie_inside_the_scratch(lib, dtype, attached, T):
    """Scratch for more query heads per K/V head, or more tokens, than the pass has: the area that its table gradient needs,
    (sequences x heads) x parts x buckets sums, ends where the scratch does or before."""
    batch, H, buckets, tokens = 2, 2, 8, 200
    lay = FakeLayer(lib, batch, H, 64, 256, 32, dtype=dtype, lens=[8] * batch)
    n = ctypes.c_size_t(0)
    lay.check(lib.eigen_attn_bias_bytes(lay.h, buckets, 20, ctypes.byref(n)))
    lay.bias_buf, at = aligned(n.value)
    lay.check(lib.eigen_attn_bias_attach(lay.h, buckets, 20, at, n.value, None))
    lay.check(lib.eigen_attn_train_bytes(lay.h, tokens, attached, ctypes.byref(n)))
    lay.train_buf, scratch = aligned(n.value)
    lay.check(lib.eigen_attn_train_attach(lay.h, tokens, attached, scratch, n.value))
    some_buf, some = aligned(1 << 16)
    launches(lib)
    lay.check(lib.eigen_attn_train_forward(lay.h, some, some, some, T, 1, None, some, None))
    lay.check(lib.eigen_attn_train_backward(lay.h, some, some, some, some, some, None))
    parts = -(-T // 32) if dtype == FP32 else -(-T // 128) * 8
    seen = launches(lib)
    assert len(seen) == (4 if dtype == FP32 else 5)
    for words in seen:
        top = max(w for w in words if scratch <= w <= scratch + n.value)
        assert scratch + n.value - top >= batch * H * parts * buckets * 4
