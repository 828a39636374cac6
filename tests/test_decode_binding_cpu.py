"""CPU-only tests of the binding of the decode operators: what it refuses before the library is called."""
import numpy as np
import pytest

import paper_2101_07948_amd as sd

torch = pytest.importorskip("torch")


def test_rope_refuses_frequencies_in_host_memory():
    for make in (lambda: sd.Rope(8, device="cpu"),
                 lambda: sd.Rope(frequencies=np.ones(4), device="cpu"),
                 lambda: sd.Rope(frequencies=torch.ones(4, dtype=torch.float64), device="cpu")):
        with pytest.raises(TypeError):
            make()
    for make in (lambda: sd.Rope(), lambda: sd.Rope(8, frequencies=np.ones(3), device="cpu"),
                 lambda: sd.Rope(frequencies=np.ones((2, 2)), device="cpu")):
        with pytest.raises(ValueError):
            make()
