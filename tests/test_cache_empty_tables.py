"""Tables of the rotation without rows or without columns are refused, not taken for none: the call's native form and its
Python form, on host tensors with the entry points replaced."""
import importlib.util

import pytest
import torch

import paper_2412_01447_gb300 as pk
from tests.test_cache_native import Recorder, _arguments
from tests.test_native_calls import _f, any_device  # noqa: F401  (a fixture)


@pytest.mark.parametrize("form", ["native", "python"])
@pytest.mark.parametrize("rows,columns", [(0, 16), (9, 0), (0, 0)])
def test_empty_tables_are_refused(any_device, monkeypatch, form, rows, columns):  # noqa: F811
    rec = Recorder(pk._load())
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    calls = None
    if form == "native":
        spec = importlib.util.spec_from_file_location("_pldp_calls", any_device)
        calls = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(calls)
        calls.bind_cache(rec.addresses)
    monkeypatch.setattr(pk, "_load", lambda: rec)
    monkeypatch.setattr(pk, "_calls", calls)
    args = _arguments()[0]["pldp_cache_append"]
    pk.pldp_cache_append(**args)
    assert len(rec.made) == 1
    with pytest.raises(pk.PldpError, match="rot"):
        pk.pldp_cache_append(**{**args, "cos": _f(rows, columns), "sin": _f(rows, columns)})
    assert len(rec.made) == 1                                     # nothing was launched without a rotation
