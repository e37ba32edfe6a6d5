"""What can be told of the row operators' kernels from their source alone."""
import os
import re

from paper_1912_11040_b200 import binding


def kernels(name):
    """(name, body without comments) of the file's kernels."""
    text = open(os.path.join(os.path.dirname(binding.__file__), "csrc", name)).read()
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    for k in text.split("__global__")[1:]:
        body = k.split("\n}\n")[0]
        yield re.search(r"(\w+_kernel)\(", body).group(1), body


def test_tensor_memory_is_taken_behind_the_kernels_ahead():
    """Tensor memory is waited for without a limit.  A CTA that held it while it waits for the kernel ahead on the stream
    could keep that kernel, and so itself, from ever ending."""
    taken = [(name, body) for name, body in kernels("product.cu") if "tcgen05.alloc" in body]
    assert [name for name, _ in taken] == ["tile_product_kernel"]
    for _, body in taken:
        assert 0 <= body.index("chain_wait();") < body.index("tcgen05.alloc")
