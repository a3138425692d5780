"""The binding's compiled helper on tensors that have no memory of their own: whatever they throw is an answer, never the end of the process."""
import subprocess
import sys
import textwrap

import pytest

torch = pytest.importorskip("torch")

COMMON = """
    import ctypes as C, sys, torch
    from paper_1709_09393_amd import _tables
    table = (C.c_void_p * 2)()
    def matrix(t, rows=4, cols=8):
        return _tables.matrix([t], [rows], cols, 0, -1, C.addressof(table))
    def vectors(t, n=8):
        return _tables.vectors([t], [n], 0, -1, C.addressof(table))
"""
CASES = {
    "vmap": """
        got = []
        def f(t):
            got.append((matrix(t), vectors(t, 32)))
            return t
        torch.vmap(f)(torch.zeros(3, 4, 8))
        assert got == [(-1, -1)], got
    """,
    "grad": """
        got = []
        def f(t):
            got.append((matrix(t), vectors(t, 32)))
            return t.sum()
        torch.func.grad(f)(torch.zeros(4, 8))
        assert got == [(-1, -1)], got
    """,
    "fake": """
        from torch._subclasses.fake_tensor import FakeTensorMode
        with FakeTensorMode():
            t = torch.zeros(4, 8)
        assert (matrix(t), vectors(t, 32)) == (-1, -1)
    """,
    "nested": """
        t = torch.nested.nested_tensor([torch.zeros(3), torch.zeros(8)])
        assert (matrix(t, 2), vectors(t, 11)) == (-1, -1)
    """,
    "sparse": """
        assert (matrix(torch.zeros(4, 8).to_sparse()), vectors(torch.zeros(8).to_sparse())) == (-1, -1)
    """,
    "freed": """
        t = torch.zeros(4, 8)
        t.untyped_storage().resize_(0)
        assert (matrix(t), vectors(t, 32)) == (-1, -1)
    """,
    "sound": """
        t = torch.zeros(4, 8)
        assert matrix(t) == 8 and table[0] == t.data_ptr() and vectors(t, 32) == 0 and table[0] == t.data_ptr()
        assert matrix(torch.zeros(4, 0), 4, 0) >= 0 and vectors(torch.zeros(0), 0) == 0
    """,
}


@pytest.mark.parametrize("case", sorted(CASES))
def test_helper_answers(case):
    """In a process of its own: an exception that leaves the helper would end it."""
    code = textwrap.dedent(COMMON) + textwrap.dedent(CASES[case])
    p = subprocess.run([sys.executable, "-W", "ignore", "-c", code], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, (p.returncode, p.stderr[-2000:])


def test_binding_says_what_is_wrong_with_such_a_tensor():
    """Inside a transformation a call of the binding is refused with an exception."""
    code = textwrap.dedent("""
        import torch
        from paper_1709_09393_amd import binding
        assert binding._tables() is not None
        class Host(binding.SlimDP):
            def __init__(self):
                self._torch, self._L, self._h, self.device = torch, None, None, torch.device("cpu")
        sd = Host()
        for wrong in (lambda t: sd._matrix("call", "x", [t], [4], 8, torch.float32), lambda t: sd._vectors("call", "w", [t], [32], torch.float32)):
            try:
                torch.vmap(lambda t: (wrong(t), t)[1])(torch.zeros(3, 4, 8))
            except (RuntimeError, ValueError) as e:
                continue
            raise SystemExit("accepted")
        t = torch.zeros(4, 8)
        t.untyped_storage().resize_(0)
        for wrong in (lambda: sd._matrix("call", "x", [t], [4], 8, torch.float32), lambda: sd._vectors("call", "w", [t], [32], torch.float32)):
            for helper in (binding._helper, None):
                binding._helper = helper
                try:
                    wrong()
                except (RuntimeError, ValueError):
                    continue
                raise SystemExit("accepted")
    """)
    p = subprocess.run([sys.executable, "-W", "ignore", "-c", code], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, (p.returncode, p.stderr[-2000:])
