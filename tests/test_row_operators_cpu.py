"""Host side of the operators on rows, and pins of their 64-bit reference, without a GPU."""
import os
import re

import numpy as np
import pytest

import row_reference as ref
from paper_1912_11040_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


@pytest.mark.parametrize("D,groups", [(1, 1), (127, 1), (128, 1), (129, 2), (257, 3), (16384, 128)])
def test_row_sizes(D, groups):
    assert binding.feat_mx_code_bytes(binding.ELEM_MX8, D) == 128 * groups
    assert binding.feat_mx_code_bytes(binding.ELEM_MX4, D) == 64 * groups
    assert binding.feat_mx_scale_bytes(D) == 4 * groups
    assert binding.feat_rms_norm_partial_floats(D) >= D


@pytest.mark.parametrize("call", [lambda: binding.feat_mx_code_bytes(binding.ELEM_F32, 8),
                                  lambda: binding.feat_mx_code_bytes(binding.ELEM_MX4, 0),
                                  lambda: binding.feat_mx_scale_bytes(-1),
                                  lambda: binding.feat_rms_norm_partial_floats(0),
                                  lambda: binding.feat_rms_norm_partial_floats(16385)])
def test_sizes_of_nothing_are_refused(call):
    with pytest.raises(binding.AugError) as e:
        call()
    assert e.value.code == binding.AUG_EINVAL


def test_calls_without_a_context_are_refused():
    L = binding.lib()
    assert L.feat_rms_norm(None, None, None, 0, None, None, 1, 1, 8, 1e-5, None, None, 0, None) == binding.AUG_EINVAL
    assert L.feat_rms_norm_grad(None, None, None, None, 0, None, None, 1, 1, 8, 1e-5, None, None, None) == binding.AUG_EINVAL
    assert L.feat_mx_quantize(None, None, 0, None, 1, 1, 8, None, 2, None) == binding.AUG_EINVAL
    assert L.feat_mx_dequantize(None, None, 2, None, None, 1, 1, 8, None, 0) == binding.AUG_EINVAL
    assert L.feat_mx_product(None, None, 2, None, None, None, None, None, 1, 1, 8, 8, None, 0) == binding.AUG_EINVAL


def test_reference_formats_have_their_largest_and_smallest_numbers():
    g = ref.e4m3_values()
    assert g[126] == 448.0 and g[1] == 2.0 ** -9 and g[8] == 2.0 ** -6 and np.all(np.diff(g) > 0)
    # ties go to the even code, as the published format asks; beyond the largest number that number
    v = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 7.9, -0.25, -5.0])
    assert ref.E2M1[ref.nearest_code(v, ref.E2M1) & 7].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 6, 0, 4]
    codes, scales = ref.quantize(np.array([[6.0] + [0.0] * 31 + [np.inf] + [1.0] * 31]), "mx4")
    assert scales[0].tolist() == [127, 255, 0, 0] and codes[0, 0] == 7 and not codes[0, 1:].any()


def test_reference_gradient_is_that_of_differences():
    rng = np.random.default_rng(0)
    x, dy, w = rng.normal(size=(3, 7)), rng.normal(size=(3, 7)), rng.normal(size=7)
    loss = lambda x, w: float((ref.rms_norm(x, None, w, 0.1)[1] * dy).sum())
    dx, dw, _, _ = ref.rms_norm_grad(x, dy, None, w, 0.1)
    for got, v, of in ((dx, x, lambda z: loss(z, w)), (dw, w, lambda z: loss(x, z))):
        for i in np.ndindex(*v.shape):
            up, down = v.copy(), v.copy()
            up[i] += 1e-5
            down[i] -= 1e-5
            assert (of(up) - of(down)) / 2e-5 == pytest.approx(got[i], abs=1e-8)


@pytest.mark.parametrize("name", ["rows.cu", "product.cu"])
def test_chained_kernels_wait_and_read_coherently(name):
    """Every kernel is launched behind one that may still be writing, so each waits for it, reads nothing through the
    non-coherent path, and lets nothing start early but the gradient's own second kernel."""
    at = os.path.join(os.path.dirname(binding.__file__), "csrc", name)
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(at).read(), flags=re.S)
    for word in ("__ldg", "__restrict__", "ld.global.nc", "<<<"):
        assert word not in text, word
    kernels = text.split("__global__")[1:]
    for k in kernels:
        body = k.split("\n}\n")[0]
        name = re.search(r"(\w+)\((?:const )?(?:__grid|Norm|Grad|float|T |uint8_t|Product)", body).group(1)
        assert body.count("chain_wait();") == 1, name
        assert body.count("chain_next();") == (name == "rms_norm_grad_kernel"), name
