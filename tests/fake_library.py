"""The library's own objects linked against tests/fake_cudart.cpp: its host side (arguments, lengths, what it launches in
which order, what it does when a call of the CUDA runtime fails) runs without a GPU."""
import ctypes
import os
import subprocess

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))


def load(directory):
    from paper_2408_05646_b200 import binding, build
    build.build_library()
    objects = [os.path.join(build.BUILD, src.replace(".cu", ".o")) for src in build.SOURCES]
    path = os.path.join(str(directory), "libfake.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", path,
                    os.path.join(HERE, "fake_cudart.cpp")] + objects, check=True)
    lib = ctypes.CDLL(path)
    for name, (res, args) in binding.SYMBOLS.items():
        getattr(lib, name).restype, getattr(lib, name).argtypes = res, args
    lib.fake_log.restype = ctypes.c_char_p
    lib.fake_fail.argtypes = [ctypes.c_char_p, ctypes.c_int]
    return lib


def aligned(nbytes, fill=0):
    """(array that owns the memory, address on a 256-byte boundary)"""
    raw = np.full(nbytes + 256, fill, dtype=np.uint8)
    return raw, -(-raw.ctypes.data // 256) * 256


class FakeLayer:
    """A handle on the fake runtime.  `check` turns a status into an exception, as the binding does."""

    def __init__(self, lib, batch, H, d, n_max, r, dtype=0, lens=None):
        from paper_2408_05646_b200 import binding as B
        self.B, self.lib, self.batch = B, lib, batch
        U = [np.eye(d, dtype=np.float32)[:, :r] for _ in range(H)]
        desc, self.keep = B._make_desc(batch, H, d, n_max, dtype, [r] * H, [r] * H, U, U, 0, 0)
        cb, wb = ctypes.c_size_t(0), ctypes.c_size_t(0)
        self.check(lib.eigen_attn_cache_bytes(ctypes.byref(desc), ctypes.byref(cb), ctypes.byref(wb)))
        self.cache, cache = aligned(cb.value)
        self.ws, ws = aligned(wb.value)
        self.h = ctypes.c_void_p(0)
        lib.fake_reset()
        self.check(lib.eigen_attn_create(ctypes.byref(desc), cache, cb.value, ws, wb.value, None, ctypes.byref(self.h)))
        self.cache_at = cache - self.cache.ctypes.data
        if lens is not None:
            self.set_lens(lens)

    def check(self, status):
        if status != 0:
            raise self.B.EigenAttnError(status, "fake", "")

    def ints(self, values):
        return (ctypes.c_int32 * len(values))(*values)

    def set_lens(self, lens):
        self.check(self.lib.eigen_attn_set_lens(self.h, self.ints(lens), None))

    def lens(self):
        out = self.ints([0] * self.batch)
        self.check(self.lib.eigen_attn_get_lens(self.h, out))
        return list(out)

    def tree_attach(self, tokens, group=1):
        n = ctypes.c_size_t(0)
        self.check(self.lib.eigen_attn_tree_bytes(self.h, tokens, group, ctypes.byref(n)))
        self.tree_buf, at = aligned(n.value)
        self.check(self.lib.eigen_attn_tree_attach(self.h, tokens, group, at, n.value))
        self.tree_at, self.tree_bytes = at, n.value

    def tree_commit(self, paths, T):
        flat = [0] * (self.batch * T)
        for b, p in enumerate(paths):
            flat[b * T:b * T + len(p)] = p
        return self.lib.eigen_attn_tree_commit(self.h, self.ints(flat), self.ints([len(p) for p in paths]), T, None)

    def launched(self):
        """Short names of the kernels launched since the last question."""
        text = self.lib.fake_log().decode()
        self.lib.fake_reset()
        return [next((k for k in KERNELS if k in line), line) for line in text.split("\n") if line]


KERNELS = ["tree_commit_kernel", "write_lens_kernel", "mq_project_few_kernel", "mq_project_many_kernel", "mq_simt_kernel", "mq_mma_kernel",
           "mq_combine_few_kernel", "mq_combine_many_kernel", "mq_combine_mma_kernel", "block_bounds_kernel", "block_scores_kernel",
           "block_select_kernel", "mq_query64_kernel"]
