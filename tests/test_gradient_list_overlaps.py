"""CPU: the list of gradients refuses results that would be written over something that the same launch still reads."""
import pytest

import test_ends_abi as base
from paper_2509_25149_amd import binding as nv

P, grad = base.P, base.grad
INVALID = -1


@pytest.fixture(scope="module")
def lib():
    return nv.load_library()


def build(lib, *grads):
    return base.build(lib, list(grads))[0]


def test_results_over_another_tensors_data(lib):
    a, b = P, 2 * P
    assert build(lib, grad(data=a, out=b), grad(data=b, out=a)) == INVALID                           # exchanged
    assert build(lib, grad(data=a, out=3 * P), grad(data=b, out=a)) == INVALID
    assert build(lib, grad(data=b, out=a), grad(data=a, out=3 * P)) == INVALID
    assert build(lib, grad(data=a), grad(data=a, out=3 * P)) == INVALID                              # one in its place, the other reads it
    assert build(lib, grad(data=a, out=3 * P), grad(data=a)) == INVALID
    for shift in (4, 396, -396):                                                                     # a part of it
        assert build(lib, grad(data=a), grad(data=a + shift, out=3 * P)) == INVALID
        assert build(lib, grad(data=a, out=b + shift), grad(data=b, out=3 * P)) == INVALID
    for shift in (400, -400):
        assert build(lib, grad(data=a), grad(data=a + shift, out=3 * P)) == 0
    long = grad(data=a, cols=100_000, ld=100_000, out=64 * P, ld_out=100_000)                        # another range begins and ends between its beginning and the result
    assert build(lib, long, grad(data=a + 40, out=32 * P), grad(data=32 * P + 4000, out=a + 4000)) == INVALID
    assert build(lib, long, grad(data=a + 40, out=32 * P), grad(data=32 * P + 4000, out=a + 400_000)) == 0


def test_results_over_a_part_of_their_own_data(lib):
    assert build(lib, grad()) == build(lib, grad(out=P)) == 0                                        # in its place
    assert build(lib, grad(out=P + 4)) == build(lib, grad(out=P - 4)) == INVALID
    assert build(lib, grad(out=P + 400)) == build(lib, grad(out=P - 400)) == 0
    assert build(lib, grad(dt=1, ot=1, out=P + 2)) == INVALID and build(lib, grad(dt=1, ot=0, out=P + 196)) == INVALID and build(lib, grad(dt=1, ot=0, out=P + 200)) == 0


def test_what_may_be_shared(lib):
    assert build(lib, grad(out=2 * P), grad(out=3 * P), grad(out=4 * P)) == 0                        # the same data for several results
    assert build(lib, grad(), grad(data=P + 400), grad(rows=0, data=P), grad(cols=0, data=P)) == 0
    apart = dict(rows=4, cols=10, ld=40, ld_out=40)                                                  # columns of one tensor between each other's rows
    assert build(lib, grad(**apart), grad(data=P + 40, **apart), grad(data=P + 80, out=P + 120, **apart)) == 0
    assert build(lib, grad(**apart), grad(data=P, out=2 * P, **apart)) == INVALID
    assert build(lib, grad(out=2 * P, **apart), grad(data=2 * P, out=3 * P, **apart)) == INVALID
    assert build(lib, grad(data=P, out=2 * P, **apart), grad(data=2 * P - 40, cols=100, out=3 * P)) == INVALID      # it begins in the middle of another's data
