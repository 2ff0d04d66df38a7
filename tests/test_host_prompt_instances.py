"""Which instance of the prompt kernels a layer launches (a fake CUDA runtime, no GPU)."""
import ctypes

import pytest

from fake_library import FakeLayer, aligned, load

BF16, FP32 = 0, 1


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return load(tmp_path_factory.mktemp("fake"))


@pytest.mark.parametrize("dtype,impl,kernel,no,yes", [(BF16, 0, "prefill_tc_kernel", "ILb0E", "ILb1E"),
                                                      (BF16, 1, "prefill_simt_kernel", "Lb0EE", "Lb1EE"),
                                                      (FP32, 0, "prefill_simt_kernel", "Lb0EE", "Lb1EE")])
def test_a_learned_bias_has_an_instance_of_its_own(lib, monkeypatch, dtype, impl, kernel, no, yes):
    """Layers without one run the code that they ran before there was one."""
    from paper_2408_05646_b200 import binding
    make = binding._make_desc
    monkeypatch.setattr(binding, "_make_desc", lambda *a: make(*a[:9], 16, a[10]))           # prompts of up to 16 tokens
    lay = FakeLayer(lib, 1, 2, 64, 256, 32, dtype=dtype)
    lay.check(lib.eigen_attn_set_option(lay.h, lay.B.EA_OPT_PREFILL_IMPL, impl))
    some_buf, some = aligned(1 << 16)

    def instance():
        lay.check(lib.eigen_attn_set_len(lay.h, 0))
        lib.fake_reset()
        packed = lay.B.EA_Q_PREPROJECTED | lay.B.EA_KV_PREPROJECTED | lay.B.EA_OUT_LOWRANK
        lay.check(lib.eigen_attn_prefill(lay.h, some, some, some, 4, 512, 128, some, 512, 128, packed, None))
        lines = [line for line in lib.fake_log().decode().split("\n") if kernel in line]
        assert len(lines) == 1
        return lines[0]
    assert no in instance()
    n = ctypes.c_size_t(0)
    lay.check(lib.eigen_attn_bias_bytes(lay.h, 8, 20, ctypes.byref(n)))
    lay.bias_buf, at = aligned(n.value)
    lay.check(lib.eigen_attn_bias_attach(lay.h, 8, 20, at, n.value, None))
    assert yes in instance()
    lay.check(lib.eigen_attn_bias_attach(lay.h, 0, 0, None, 0, None))
    assert no in instance()
