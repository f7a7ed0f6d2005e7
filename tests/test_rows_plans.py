"""What a KeyOrder given by the caller has to hold before its addresses reach a
kernel (no GPU: the checks look at shapes only)."""

import pytest
import torch

from paper_2211_17111_amd import rows

CPU, META = torch.device("cpu"), torch.device("meta")


def _i32(n, dev=CPU):
    return torch.empty(n, dtype=torch.int32, device=dev)


def test_count_of_kept_slots_lies_inside_the_offsets():
    """offsets[n_keys] is read on the device: n_keys must name an element of them."""
    offsets = _i32(4)
    assert rows.KeyOrder(_i32(6), _i32(6), offsets, 3)._check(CPU, 6, 2) == offsets.data_ptr() + 12
    assert rows.KeyOrder(_i32(0), _i32(0), _i32(1), 0)._check(CPU, 0, 1) != 0
    for n in (0, 6):
        for n_keys in (-1, -2):
            with pytest.raises(ValueError):
                rows.KeyOrder(_i32(n), _i32(n), _i32(max(0, n_keys + 1)), n_keys)._check(CPU, n, 1)


def test_orders_past_32_bits_are_refused():
    """Slots and slots to a token reach the library as 32-bit integers."""
    n = 1 << 32
    for k in (1, n):
        with pytest.raises(ValueError):
            rows.KeyOrder(_i32(n, META), _i32(n, META), _i32(4, META), 3)._check(META, n, k)


def test_gradient_of_a_dispatch_holds_no_false_order(monkeypatch):
    """Its order keeps positions and offsets only: no other tensor stands in for the slots."""
    order = torch.tensor([1, 2, 3, 0], dtype=torch.int32)
    position = torch.tensor([3, 0, 1, 2], dtype=torch.int32)
    offsets = torch.tensor([0, 3, 4], dtype=torch.int32)
    seen = []
    monkeypatch.setattr(rows, "dispatch_forward",
                        lambda x, ids, n: (x[order.long()], rows.KeyOrder(order, position, offsets, n, 1)))
    monkeypatch.setattr(rows, "dispatch_backward", lambda g, plan, k: (seen.append(plan), g[plan.position.long()])[1])
    x = torch.randn(4, 3, requires_grad=True)
    r, plan = rows.dispatch(x, torch.tensor([[1], [0], [0], [0]]), 2)
    assert torch.equal(plan.order, order)
    r.backward(r.detach())
    assert torch.equal(x.grad, x.detach())
    assert seen[0].order is None and torch.equal(seen[0].position, position) and seen[0].n_keys == 2
