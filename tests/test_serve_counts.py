"""The counts of a serving step's new tokens may be any integers that numpy takes: lists, arrays, tensors on the host (no GPU)."""
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("counts", [[3, 0, 5], (3, 0, 5), np.array([3, 0, 5]), np.array([3, 0, 5], np.int32),
                                    torch.tensor([3, 0, 5]), torch.tensor([3, 0, 5], dtype=torch.int32)])
def test_step_and_verify_take_counts_of_any_kind(monkeypatch, counts):
    from paper_2606_30391_amd import festina
    from paper_2606_30391_amd.serve import Server
    srv, said = object.__new__(Server), []
    srv.blocks, srv.drafts = types.SimpleNamespace(advance=lambda: None), None
    monkeypatch.setattr(Server, "_begin", lambda self, add: int(np.ascontiguousarray(add, np.int32).sum()))
    monkeypatch.setattr(Server, "_layers", lambda self, tokens, longest, *a: said.append((tokens, longest)) or [])
    assert srv.step(counts, None) == [] and said == [(8, 5)]

    def checked(t, name, dtypes, shape):
        said.append((name, shape))
        if name == "token":
            raise KeyboardInterrupt                          # (what comes next is the device's)
    monkeypatch.setattr(festina, "_check", checked)
    with pytest.raises(KeyboardInterrupt):
        srv.verify(counts, None, None, None, None)
    assert said[1:] == [("parent", (8,)), ("token", (8,))]
