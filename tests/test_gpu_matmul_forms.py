"""Products that take the forms of the kernel which the other products' sizes miss: whole blocks
of k alone, rows of more than 64 blocks, and loads that copies delay.  That the sizes of all
these tests between them take every form is checked in test_matmul_forms_cpu.py."""

import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")

from tests import test_gpu_dense as dense  # noqa: E402

MORE = [(1, 16, 1616), (1, 8328, 128), (1, 16631, 128), (17, 2143, 8544), (18, 4129, 9600), (18, 8267, 10880), (18, 16458, 16), (21, 4184, 256),
        (29, 18001, 400), (36, 32413, 9216), (70, 8377, 128), (70, 10936, 10240), (153, 32880, 16), (201, 32017, 272), (431, 1221, 15488),
        (441, 4819, 256), (4252, 68, 8576)]
DELAYED = [(1, 11287, 1664), (17, 8623, 1664), (18, 16, 1808), (19, 8227, 1024), (20, 4220, 1840), (33, 32731, 3456), (80, 9000, 1024),
           (110, 8660, 1024), (257, 1830, 4784), (274, 6790, 1024), (520, 7578, 1040), (4178, 17, 1952), (4533, 194, 1024), (4607, 17, 1024),
           (4721, 37, 1152)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", MORE)
def test_products(m, n, k, out):
    dense.test_large_products(m, n, k, out)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", DELAYED)
def test_products_while_copies_delay_their_loads(m, n, k, out):
    dense.test_products_while_copies_delay_their_loads(m, n, k, out)
