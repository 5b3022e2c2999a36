"""Arguments that are none, beside tensors that are fine: the error names the one that is wrong, and nothing is called after it."""
import pytest
import torch


class Broken:
    def data_ptr(self):
        raise RuntimeError("no storage")


class Counting:
    asked = 0

    def data_ptr(self):
        Counting.asked += 1
        return 256


@pytest.fixture
def calls():
    import paper_2609_16009_b200 as nm
    if nm._calls is None:
        pytest.skip("no Python headers here")
    return nm._calls


POINTERS = {"nm_moe_route": (16, (0, 2, 3, 4, 15)), "nm_matmul_act": (18, (0, 2, 3, 4, 6, 15, 17)), "nm_moe_ffn": (23, (0, 2, 3, 4, 5, 6, 8, 20, 22))}


@pytest.mark.parametrize("name", list(POINTERS))
@pytest.mark.parametrize("bad,error,words", [("x", AttributeError, "'str'"), (1.5, AttributeError, "'float'"), (Broken(), RuntimeError, "no storage")])
def test_a_pointer_that_is_none(calls, name, bad, error, words):
    count, pointers = POINTERS[name]
    t = torch.zeros(64)
    for at in pointers:
        args = [0] * count                                         # sizes of zero: refused, were it to come to that
        for i in pointers:
            args[i] = t if i < at else Counting() if i > at else bad
        Counting.asked = 0
        with pytest.raises(error, match=words) as err:
            getattr(calls, name)(*args)
        assert err.value.__cause__ is None and Counting.asked == 0, at


@pytest.mark.parametrize("name", list(POINTERS))
def test_a_number_that_is_none_beside_tensors(calls, name):
    count, pointers = POINTERS[name]
    for at in (i for i in range(count) if i not in pointers):
        args = [0] * count
        for i in pointers:
            args[i] = torch.zeros(64)
        args[at] = "x"
        with pytest.raises(TypeError, match="str"):
            getattr(calls, name)(*args)
