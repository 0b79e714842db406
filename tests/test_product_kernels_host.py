"""Which kernel runs a product of 8-bit operands: the products that the GPU tests run reach every kernel there is."""
import pytest

from paper_2507_05829_amd import lop
from product_cases import CASES, FLAT
from test_operators_host import ARG, BAND, UNS, product_op


@pytest.mark.parametrize("kernel,dtype,m,k,n", FLAT)
def test_products_are_run_by_the_kernels_they_are_for(kernel, dtype, m, k, n):
    op = lop.lop_rowwise_f8_t(m + 7, n, k, lop.LOP_F32 if dtype == "f32" else lop.LOP_BF16)
    assert lop.lop_rowwise_f8_kernel(op, (3, m + 3)) == kernel.format("float" if dtype == "f32" else "__bf16")


def test_every_kernel_is_reached():
    """Over the whole range of sizes nothing is chosen that the cases do not have."""
    have = {kernel.format("float" if dtype == "f32" else "__bf16") for kernel, dtype, *_ in FLAT}
    sizes = [1, 7, 16, 40, 100, 300, 513, 1000, 2500, 6000, 16384]
    found = set()
    for dtype in (lop.LOP_F32, lop.LOP_BF16):
        for k in (16, 128, 272, 400, 656, 1040, 4096, 16384):
            for m in sizes:
                for n in sizes + [65536, 2097120]:
                    found.add(lop.lop_rowwise_f8_kernel(lop.lop_rowwise_f8_t(m, n, k, dtype), (0, m)))
    assert found == have and len(found) == 2 * len(CASES) - 1


def test_names_are_refused_as_products_are():
    assert lop.lop_rowwise_f8_kernel(product_op(), (5, 5)) == ""
    for code, rows, change in ((BAND, (0, 101), {}), (UNS, (0, 5), dict(k=100)), (UNS, (0, 5), dict(act=9)), (UNS, (0, 5), dict(dtype=7)), (ARG, (0, 5), dict(n=0))):
        op = product_op()
        for name, v in change.items():
            setattr(op, name, v)
        with pytest.raises(lop.LopError) as e:
            lop.lop_rowwise_f8_kernel(op, rows)
        assert e.value.code == code
    assert lop._lib.lop_rowwise_f8_kernel(None, 0, None, 5) == ARG
