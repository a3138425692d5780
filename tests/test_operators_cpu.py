"""Host side of LocalTrain's operators without a GPU: workspace sizes, a context that is not there, and what the binding refuses
before it calls the library."""
import ctypes as C

import pytest

from paper_1709_09393_amd import binding

torch = pytest.importorskip("torch")


def rows(*r):
    return (C.c_uint64 * len(r))(*r)


def test_workspaces_are_pure_host_functions():
    L = binding.load()
    norm, lin = L.slimdp_layer_norm_workspace_bytes, L.slimdp_linear_workspace_bytes
    for dt in (0, 1, 2):
        assert norm(1, rows(1), 4096, dt) == 0 and norm(2, rows(0, 0), 100, dt) == 0
        big = norm(8, rows(*[2048] * 8), 4096, dt)
        assert 0 < big < 8 * 2048 * 4096                      # a fraction of the data
        assert big % (2 * 4 * 4096 * 8) == 0                  # whole rows of both sums for every worker
        assert lin(8, rows(*[2048] * 8), 4096, 4096, dt, binding.LINEAR_FORWARD) == 0      # tiles enough without splitting
        assert lin(3, rows(0, 0, 0), 64, 64, dt, binding.LINEAR_FORWARD) == 0
        for p in (0, 1, 2):
            assert lin(1, rows(4096), 64, 64, dt, p) <= 64 * 4096 * 64 * 4
    for bad in ((0, rows(1), 16, 0), (33, rows(*[1] * 33), 16, 0), (1, None, 16, 0), (1, rows(1), 0, 0), (1, rows(1), 65537, 0), (1, rows(1), 16, 3),
                (1, rows((1 << 24) + 1), 16, 0)):
        assert norm(*bad) == 0
    for bad in ((1, rows(99), 0, 5, 0, 0), (1, rows(99), 5, 0, 0, 1), (1, rows(99), 5, 5, 4, 2), (1, rows(99), 5, 5, 0, 3), (1, rows(99), 1 << 21, 5, 0, 0)):
        assert lin(*bad) == 0


def test_null_context_is_refused():
    L = binding.load()
    n, t = rows(1), (C.c_void_p * 1)()
    assert L.slimdp_layer_norm(None, 1, n, 8, 0, t, 8, None, None, 1e-5, t, 8, None, None) == binding.ERR_INVALID_ARG
    assert L.slimdp_layer_norm_backward(None, 1, n, 8, 0, t, 8, t, 8, None, t, t, t, 8, None, None, 0, None, 0) == binding.ERR_INVALID_ARG
    assert L.slimdp_linear(None, 1, n, 8, 8, 0, t, 8, t, 8, None, 0, None, 0, t, 8, None, 0, None, 0) == binding.ERR_INVALID_ARG
    assert L.slimdp_linear_epilogue_backward(None, 1, n, 8, 0, t, 8, t, 8, 1, t, 8, None, 0, None, 0) == binding.ERR_INVALID_ARG
    assert L.slimdp_linear_backward(None, 1, n, 8, 8, 0, t, 8, t, 8, t, 8, t, 8, None, 0, None, 0) == binding.ERR_INVALID_ARG
    assert L.slimdp_distill_loss(None, 1, n, 8, 0, t, 8, 0, None, None, 0, 1.0, None, None, None, t, 8) == binding.ERR_INVALID_ARG


class Host(binding.SlimDP):
    """The binding's checks with tensors of the host; a call that passes them reaches a library that only says so."""

    class Reached(Exception):
        pass

    class Library:
        def __getattr__(self, name):
            if name.endswith("workspace_bytes"):
                return lambda *a: 0

            def call(*a):
                raise Host.Reached(name)
            return call

    def __init__(self):
        self._torch, self._L, self._h, self.device = torch, self.Library(), None, torch.device("cpu")

    def _new(self, make):
        return make()


@pytest.mark.parametrize("compiled", [True, False])
def test_binding_refuses_what_does_not_fit(monkeypatch, compiled):
    """By the compiled checks, and as the binding spells them out."""
    if compiled:
        assert binding._tables() is not None, "the binding's helper is not built"
    else:
        monkeypatch.setattr(binding, "_helper", None)
    sd, Z = Host(), torch.zeros
    x, v = Z(4, 8), Z(8)

    def reached(f):
        with pytest.raises(Host.Reached):
            f()

    def refused(f):
        with pytest.raises(ValueError):
            f()
    reached(lambda: sd.layer_norm([x], [v], [v]))
    reached(lambda: sd.layer_norm([x, Z(0, 8)], [v, None], None))
    reached(lambda: sd.layer_norm([Z(4, 16)[:, :8]], [v], [v]))
    reached(lambda: sd.layer_norm([Z(4, 16)[:, :8], Z(1, 8)], None, None))                   # one row: any distance
    reached(lambda: sd.layer_norm([Z(5, 1).t().contiguous().t()], None, None))
    refused(lambda: sd.layer_norm([x.double()], [v], [v]))
    refused(lambda: sd.layer_norm([Z(8)], [v], [v]))
    refused(lambda: sd.layer_norm([x], [Z(7)], [v]))
    refused(lambda: sd.layer_norm([x], [v.half()], [v]))
    refused(lambda: sd.layer_norm([x], [Z(16)[::2]], [v]))
    refused(lambda: sd.layer_norm([x], [v, v], [v]))
    refused(lambda: sd.layer_norm([Z(8, 4).t()], [v], [v]))                                  # columns not consecutive
    refused(lambda: sd.layer_norm([x, Z(4, 16)[:, :8]], None, None))                         # two distances
    refused(lambda: sd.layer_norm([Z(1, 8).expand(4, 8)], None, None))                       # rows on top of each other
    refused(lambda: sd.layer_norm([x], None, None, y=[Z(4, 9)]))
    refused(lambda: sd.layer_norm([x], None, None, y=[x.half()]))
    refused(lambda: sd.layer_norm([x], None, None, mean=[Z(5)]))
    reached(lambda: sd.linear([x], [Z(5, 8)], [Z(5)], "gelu", [Z(4, 5)], keep=True))
    refused(lambda: sd.linear([x], [Z(5, 9)]))
    refused(lambda: sd.linear([x], [Z(5, 8).bfloat16()]))
    refused(lambda: sd.linear([x], [Z(5, 8)], [Z(8)]))
    refused(lambda: sd.linear([x], [Z(5, 8)], residual=[x]))
    refused(lambda: sd.linear([x], [Z(5, 8)], z=[x]))
    with pytest.raises(KeyError):
        sd.linear([x], [Z(5, 8)], activation="tanh")
    reached(lambda: sd.linear_epilogue_backward([x], [x], "relu"))
    refused(lambda: sd.linear_epilogue_backward([x], [Z(4, 9)], "relu"))
    reached(lambda: sd.linear_backward([Z(4, 5)], [x], [Z(5, 8)]))
    refused(lambda: sd.linear_backward([Z(4, 5)], [Z(3, 8)], [Z(5, 8)]))
    refused(lambda: sd.linear_backward([Z(4, 5)], [x], [Z(5, 8)], dweight=[Z(5, 16)[:, ::2]]))
    i, t = Z(4, 3, dtype=torch.int32), Z(4, 3)
    reached(lambda: sd.distill_loss([x], [i], [t]))
    reached(lambda: sd.distill_loss([x], [i[:, :0]], [t[:, :0]]))
    refused(lambda: sd.distill_loss([x], [i.long()], [t]))
    refused(lambda: sd.distill_loss([x], [i], [Z(4, 2)]))
    refused(lambda: sd.distill_loss([x], [i], [Z(4, 6)[:, :3]]))                             # index and value at different distances
    refused(lambda: sd.distill_loss([x], [i], [t], row_weight=[Z(3)]))


def test_compiled_tables_are_those_of_the_binding(monkeypatch):
    sd, Z = Host(), torch.zeros
    lists = [([Z(4, 16)[:, 3:11], Z(0, 8), Z(1, 8), Z(2, 16)[:, :8]], [4, 0, 1, 2], 8), ([Z(3, 1)], [3], 1), ((Z(5, 7), Z(5, 7)), [5, 5], 7)]
    for ts, rows, cols in lists:
        fast = sd._matrix("t", "x", ts, rows, cols, torch.float32)
        with monkeypatch.context() as m:
            m.setattr(binding, "_helper", None)
            slow = sd._matrix("t", "x", ts, rows, cols, torch.float32)
        assert list(fast[0]) == list(slow[0]) and fast[1] == slow[1]
    vs = [Z(6)[1:5], None, Z(2, 2), Z(0)]
    fast = sd._vectors("t", "v", vs, [4, 9, 4, 0], torch.float32)
    with monkeypatch.context() as m:
        m.setattr(binding, "_helper", None)
        slow = sd._vectors("t", "v", vs, [4, 9, 4, 0], torch.float32)
    assert list(fast) == list(slow)
