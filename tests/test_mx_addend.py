"""What the products refuse of an addend, by the rule's tile and by a named one (stand-ins for tensors, no GPU)."""
import pytest
import torch

from paper_2501_17116_amd import binding as b
from tests.test_other_device import On, mx, reached  # noqa: F401

P, Q, Kc = 8, 32, 64


class Apart(On):
    def stride(self):
        return (self.shape[1] + 8, 1)


def host(rows, cols):
    t = On(0, rows, cols, torch.float32)
    t.is_cuda, t.device = False, torch.device("cpu")
    return t


BAD = [On(0, P - 1, Q, torch.float32), On(0, P, Q - 8, torch.float32), On(0, P, Q, torch.bfloat16), On(1, P, Q, torch.float32), host(P, Q),
       Apart(0, P, Q, torch.float32)]


@pytest.fixture
def calls(monkeypatch, reached):  # noqa: F811
    monkeypatch.setattr(b, "_out", lambda t, shape, dtype, device, name: On(0, *shape, dtype) if t is None else t)
    return {"mx_gemm": lambda add: b.mx_gemm(mx(0, P, Kc), mx(0, Q, Kc), addend=add),
            "mx_gemm_by_tile": lambda add: b.mx_gemm_by_tile(mx(0, P, Kc), mx(0, Q, Kc), 32, addend=add)}


@pytest.mark.parametrize("name", ["mx_gemm", "mx_gemm_by_tile"])
def test_addends(reached, calls, name):  # noqa: F811
    for add in BAD:
        with pytest.raises(ValueError):
            calls[name](add)
    assert not reached
    calls[name](None)
    calls[name](On(0, P, Q, torch.float32))
    assert reached == [name, name]


def test_operands_that_do_not_fit(reached, calls):  # noqa: F811
    for l, r in ((mx(0, P, Kc), mx(0, Q, Kc + 32)), (mx(0, P, Kc), mx(1, Q, Kc))):
        for call in (lambda: b.mx_gemm(l, r), lambda: b.mx_gemm_by_tile(l, r, 32)):
            with pytest.raises(ValueError):
                call()
    assert not reached
