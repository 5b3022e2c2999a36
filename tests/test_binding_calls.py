"""The two ways from Python into the feed-forward entry points, the extension module's calls and ctypes: the same arguments arrive, the same errors come back."""
import pytest
import torch


@pytest.fixture(params=["extension", "ctypes"])
def nm(request, monkeypatch):
    import paper_2609_16009_b200 as nm
    monkeypatch.setattr(nm, "_stream", lambda s: 0)                # no device is asked for
    if request.param == "ctypes":
        monkeypatch.setattr(nm, "_calls", None)
    elif nm._calls is None:
        pytest.skip("no Python headers here")
    return nm


def tensors():
    return torch.zeros(64), torch.zeros(6, dtype=torch.int32), torch.zeros(6)


@pytest.mark.parametrize("change,status", [({}, -1), ({"T": 4, "E": 1025}, -2), ({"T": 4, "dtype": 2}, -2), ({"T": 4, "groups": 5}, -1), ({"T": 4, "top_k": 33, "ld_logits": 64}, -2)])
def test_statuses_of_route(nm, change, status):
    x, e, w = tensors()
    args = dict(T=0, E=64, top_k=6, dtype=0)
    args.update(change)
    if args["E"] > 64:
        args["ld_logits"] = args["E"]
    with pytest.raises(nm.NmError) as err:
        nm.nm_moe_route(x, None, e, w, **args)
    assert err.value.status == status


def test_every_argument_has_its_place(nm):
    """One argument at a time made wrong: each is refused for itself."""
    x = torch.zeros(4096, dtype=torch.bfloat16)
    ws = torch.zeros(nm.nm_matmul_act_workspace_bytes(4, 64, 128), dtype=torch.uint8)
    good = dict(A=256, B=512, C_out=1024, M=4, N=64, K=128, act=2, dtype=1, layout_B=1, workspace=ws[:8], gated=False, bias=None, residual=None)
    odd = x.data_ptr() + 1
    for name, value, status in [("A", None, -1), ("B", None, -1), ("C_out", None, -1), ("M", 0, -1), ("N", 0, -1), ("K", 0, -1), ("lda", 127, -1), ("ldc", 63, -1), ("act", 5, -2), ("dtype", 0, -2),
                                ("layout_B", 2, -2), ("A", odd, -3), ("B", odd, -3), ("C_out", odd, -3), ("bias", odd, -3), ("residual", odd, -3), ("workspace", None, -4), ("workspace", ws[:8], -4)]:
        with pytest.raises(nm.NmError) as err:
            nm.nm_matmul_act(**{**good, name: value})
        assert err.value.status == status, name
    with pytest.raises(nm.NmError) as err:
        nm.nm_matmul_act(**{**good, "residual": 256, "ld_residual": 63})
    assert err.value.status == -1
    moe = dict(x=256, experts=512, weights=1024, W_up=2048, W_down=4096, out=8192, T=4, d=64, inter=32, E=8, top_k=2, act=2, dtype=1, layout=1, workspace=ws[:8])
    for name, value, status in [("x", None, -1), ("experts", None, -1), ("W_up", None, -1), ("W_down", None, -1), ("out", None, -1), ("T", 0, -1), ("d", 0, -1), ("inter", 0, -1), ("E", 0, -1),
                                ("top_k", 0, -1), ("first_expert", -1, -1), ("ldx", 63, -1), ("ldo", 63, -1), ("act", 5, -2), ("dtype", 2, -2), ("layout", 2, -2), ("experts", 514, -3), ("weights", 1026, -3),
                                ("x", odd, -3), ("W_up", odd, -3), ("W_down", odd, -3), ("residual", odd, -3), ("out", odd, -3), ("workspace", ws[:8], -4)]:
        with pytest.raises(nm.NmError) as err:
            nm.nm_moe_ffn(**{**moe, name: value})
        assert err.value.status == status, name


def test_what_is_no_argument_is_an_error_of_python():
    import paper_2609_16009_b200 as nm
    if nm._calls is None:
        pytest.skip("no Python headers here")
    good = [1, 64, None, 2, 3, 0, 64, 6, 0, 0, 1, 1, 1, 1, 1.0, 0]
    assert nm._calls.nm_moe_route(*good) == -1
    for i, bad in [(0, "x"), (1, "x"), (5, 2 ** 40), (6, 1.5), (14, "x"), (15, [])]:
        with pytest.raises((TypeError, AttributeError, OverflowError)):
            nm._calls.nm_moe_route(*good[:i], bad, *good[i + 1:])
    with pytest.raises(TypeError):
        nm._calls.nm_moe_route(*good[:-1])
