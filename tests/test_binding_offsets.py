"""Host arrays of offsets as the binding hands them to the library: one 64-bit entry for every element of what the
caller gives, whatever holds the elements."""
import array

import numpy as np
import pytest
import torch

from paper_2608_03276_amd import binding as B

WANT = [0, 3, 3, 40, 41, 42, 43, 44]
HOLDERS = {
    "list": list, "tuple": tuple, "bytes": bytes, "bytearray": bytearray, "memoryview": lambda x: memoryview(bytes(x)),
    "array": lambda x: array.array("i", x), "int32": lambda x: np.array(x, dtype=np.int32),
    "float64": lambda x: np.array(x, dtype=np.float64), "tensor": torch.tensor,
    "float tensor": lambda x: torch.tensor(x, dtype=torch.float32), "floats": lambda x: [float(i) for i in x],
    "last a float": lambda x: x[:-1] + [float(x[-1])], "iterator": iter, "iterator of floats": lambda x: (float(i) for i in x),
}


@pytest.mark.parametrize("holder", HOLDERS)
def test_an_entry_for_every_element(holder):
    got = B._i64_array(HOLDERS[holder](WANT))
    assert list(got) == WANT
    assert B.ctypes.sizeof(got) == 8 * len(WANT)


def test_no_elements():
    assert len(B._i64_array([])) == 0


def test_the_array_is_a_copy():
    given = array.array("q", WANT)
    got = B._i64_array(given)
    given[1] = -1
    assert list(got) == WANT
