"""The sizes at which products are tested take every form of the kernel: each kernel that any
of many sizes takes is taken by one of a test's too, so that a change of the rule between
forms that leaves one untested fails here."""

import random

import pytest

pytest.importorskip("torch")

from paper_2608_15018_amd import _lib  # noqa: E402
from tests import test_dense_devices_cpu as devices  # noqa: E402
from tests import test_gpu_dense as dense  # noqa: E402
from tests import test_gpu_matmul_forms as more  # noqa: E402
from tests.matmul_forms import Forms  # noqa: E402
from tests.test_attention_devices_cpu import lib  # noqa: E402,F401

DTYPES = ("bf16", "f32")
# Sizes of which each kernel with more than 64 KB of LDS takes one.
DEVICES = devices.SIZES + [(1, 8558, 16), (17, 4135, 896), (17, 8623, 1664), (18, 16, 1808), (18, 16979, 16), (20, 4220, 1840), (21, 17, 16),
                           (65, 8309, 16), (110, 29437, 112), (125, 9651, 16), (135, 5826, 16), (257, 1830, 4784), (4100, 43, 256), (4178, 17, 1952)]


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    return Forms(tmp_path_factory.mktemp("forms"))


def sizes_of(test):
    """The sizes that a test is parametrized with."""
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == "m,n,k")


@pytest.fixture(scope="module")
def many():
    r = random.Random(5)
    some = lambda a, b: round(a * (b / a) ** r.random())  # noqa: E731
    out = []
    for i in range(40000):
        k = 128 * some(1, 140) if i % 2 else 16 * some(1, 1100)
        m, n = some(1, 5000), some(16, 33000)
        if m * n * k <= 1e10:
            out.append((m, n, k))
    return out


def kinds(m, n, k):
    """Whole blocks of k alone or a part of one; more blocks than a wave has weight scales of at a
    time."""
    return {"whole" if k % 128 == 0 else "part"} | ({"long"} if k > 64 * 128 else set())


def tokens_of_a_tile(kernel):
    kind, a = kernel[0], kernel[1:]
    return 16 * {"stream": lambda: a[1], "few_tokens": lambda: 1, "small_tiles": lambda: a[1] * a[3], "tiles": lambda: a[1] * a[3]}[kind]()


def covered(forms, sizes, of):
    """(type of result, kernel, kind) of sizes; products of one launch also by whether its tokens
    are one tile or several."""
    out = set()
    for s in sizes:
        for d in DTYPES:
            kernels = forms.kernels(*s, d)
            some = of(*s)
            if of is kinds and len(kernels) == 1:
                some.add("tiles" if s[0] > tokens_of_a_tile(kernels[0]) else "tile")
            out |= {(d, kernel, kind) for kernel in kernels for kind in some}
    return out


def test_products_take_every_form(forms, many):
    want = covered(forms, many, kinds)
    assert len({(d, kernel) for d, kernel, _ in want}) == 37
    got = covered(forms, dense.SIZES + dense.LARGE + dense.LONG + more.MORE, kinds)
    assert not want - got, sorted(want - got)


def test_delayed_products_take_every_form(forms, many):
    of = lambda m, n, k: {"steps"} if k >= 1000 else set()  # more than lie in LDS at a time  # noqa: E731
    want = covered(forms, many, of)
    assert len(want) == 37
    got = covered(forms, sizes_of(dense.test_products_while_copies_delay_their_loads) + more.DELAYED, of)
    assert not want - got, sorted(want - got)


def test_every_form_gets_its_attributes_on_each_device(forms, many, lib):  # noqa: F811
    of = lambda *s: {"any"}  # noqa: E731
    want, got = covered(forms, many, of), covered(forms, DEVICES, of)
    assert not want - got, sorted(want - got)
    for device in (0, 3, 0):
        lib.shim_device(device)
        for out in (_lib.F32, _lib.BF16):
            assert [devices.product(lib, *s, out) for s in DEVICES] == [_lib.OK] * len(DEVICES)
    assert lib.shim_missing() == 0 and lib.shim_sets() > 0
