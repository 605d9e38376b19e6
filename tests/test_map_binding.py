"""What the binding of the trained map's operators does with its arguments before the library is called: no GPU."""
import numpy as np
import pytest
import torch

from paper_2212_11506_amd import _binding as b


def values(coefficients, steps):
    c = b._coefficients(coefficients, steps)
    return [c[i] for i in range(3 * steps)]


def test_coefficients_are_read_at_each_call():
    """Numbers that a caller keeps in tensors or arrays and changes in place are taken as they are now."""
    for make in (torch.tensor, lambda v: torch.tensor(v, dtype=torch.float64), np.array):
        rows = [[make(1.5), make(-0.5), make(0.0)]]
        assert values(rows, 2) == [1.5, -0.5, 0.0] * 2
        rows[0][0] += 0.25
        assert values(rows, 2) == [1.75, -0.5, 0.0] * 2
        flat = [make(1.5), make(-0.5), make(0.0)]
        assert values(flat, 1) == [1.5, -0.5, 0.0]
        flat[1] -= 0.25
        assert values(flat, 1) == [1.5, -0.75, 0.0]
    table = np.array([[2.0, -1.5, 0.5], [1.5, -0.5, 0.0]])
    assert values(table, 2) == [2.0, -1.5, 0.5, 1.5, -0.5, 0.0]
    table[1, 0] = 1.25
    assert values(table, 2) == [2.0, -1.5, 0.5, 1.25, -0.5, 0.0]
    assert values(torch.tensor([2.0, -1.5, 0.5]), 2) == [2.0, -1.5, 0.5] * 2
    assert b._coefficients(None, 5) is None


@pytest.mark.parametrize("coefficients,steps", [((1.0, 2.0), 1), ([(1.0, 2.0, 3.0)] * 2, 3), (("a", 1.0, 2.0), 1)])
def test_coefficients_are_refused(coefficients, steps):
    with pytest.raises(ValueError):
        b._coefficients(coefficients, steps)


class Elsewhere:
    """What the binding asks of a tensor, on a GPU of any number."""

    def __init__(self, shape, gpu, dtype=torch.float32):
        self._t = torch.zeros(shape, dtype=dtype)
        self.gpu, self.is_cuda, self.requires_grad = gpu, True, False
        self.shape, self.dtype = self._t.shape, dtype

    def get_device(self):
        return self.gpu

    def __getattr__(self, name):
        return getattr(self._t, name)

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        return func(*[a._t if isinstance(a, cls) else a for a in args], **(kwargs or {}))


X, V, Y = (4, 8), (8,), (4,)


@pytest.mark.parametrize("which", range(5))
def test_tensors_of_another_gpu_are_refused(which, monkeypatch):
    """All of a call's tensors are on the current GPU: pointers of another one would be handed to its kernels."""
    monkeypatch.setattr(b, "_current_gpu", lambda: 0, raising=False)
    monkeypatch.setattr(b, "layer_norm_workspace_size", lambda n, d: 4096)
    at = lambda k, shape: Elsewhere(shape, 1 if k == which else 0)  # noqa: E731

    class Library:
        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} was called")

    monkeypatch.setattr(b, "load_library", Library)
    calls = [lambda: b.layer_norm(at(0, X), at(1, V), at(2, V), out=at(3, X) if which == 3 else None),
             lambda: b.layer_norm_backward(at(0, X), at(1, X), at(2, V), at(3, Y), at(4, Y)),
             lambda: b.orthogonalise(at(0, X), out=at(1, X), workspace=at(2, (4096,))),
             lambda: b.muon_step(at(0, X), at(1, X), at(2, X), 0.1, workspace=at(3, (4096,)))]
    count = [4, 5, 3, 4]
    for call, n in zip(calls, count):
        if which < n:
            with pytest.raises(ValueError, match="GPU 1"):
                call()


def test_a_call_runs_on_the_current_gpu(monkeypatch):
    monkeypatch.setattr(b, "_current_gpu", lambda: 1, raising=False)
    for call in (lambda: b.layer_norm(Elsewhere(X, 0)), lambda: b.orthogonalise(Elsewhere(X, 0)),
                 lambda: b.layer_norm_backward(*[Elsewhere(X, 0)] * 2, None, Elsewhere(Y, 0), Elsewhere(Y, 0)),
                 lambda: b.muon_step(*[Elsewhere(X, 0)] * 3, 0.1)):
        with pytest.raises(ValueError, match="current"):
            call()
