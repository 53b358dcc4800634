"""A ring has no gradients: rows that require them are refused by fill and step, and not answered without, unless torch makes none."""
import pytest
import torch

from tests.test_devices_cpu import on_gpu
from tests.test_forward_mode_cpu import machine, ring  # noqa: F401


def test_rows_that_require_gradients_are_refused(machine):  # noqa: F811
    cache = ring()
    for call, shapes in ((cache.fill, [(2, 2, 5, 64)] * 2), (cache.step, [(2, 4, 64), (2, 2, 64), (2, 2, 64)])):
        for i in range(len(shapes)):
            rows = [on_gpu(s) for s in shapes]
            call(*rows)
            n = len(machine.calls)
            rows[i].requires_grad_()
            with pytest.raises(ValueError, match="no_grad"):
                call(*rows)
            assert len(machine.calls) == n
            with torch.no_grad():
                call(*rows)
            assert len(machine.calls) == n + 1
