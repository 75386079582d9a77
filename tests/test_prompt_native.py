"""The binding's native form of the prompt and page calls against the Python form: the same calls are made,
with the same argument blocks, and what a check refuses is refused the same way."""
import ctypes
import importlib.util
import inspect

import pytest
import torch

import paper_2412_01447_gb300 as pk
from tests.test_cache_native import Recorder as CacheRecorder
from tests.test_native_calls import _f, _i, _variants, any_device  # noqa: F401  (a fixture)

B, R, Hq, H, D, page, n_pages = 3, 7, 6, 2, 32, 4, 9


class Recorder(CacheRecorder):
    def __init__(self, lib):
        self.made, self.rc, self.fns = [], 0, {}
        for f in pk._PROMPT_CALLS:
            self.fns[f] = ctypes.CFUNCTYPE(ctypes.c_int, *getattr(lib, f).argtypes)(self._entry(f))
        self.addresses = tuple(ctypes.cast(self.fns[f], ctypes.c_void_p).value for f in pk._PROMPT_CALLS)


def _arguments():
    pool = _f(n_pages, page, H, D, dtype=torch.bfloat16)
    cache = pk.pldp_cache(pool, pool.clone(), _i(B, 3))
    table = pk.pldp_page_table(_i(B, 3), _i(n_pages), page)
    q, kv, w, cos = _f(R, Hq + 1, D, dtype=torch.bfloat16)[:, :Hq], _f(R, H, D, dtype=torch.bfloat16), _f(D, dtype=torch.bfloat16), _f(9, D // 2)
    opt = dict(status=_i(B), stream=7)
    full = {
        "pldp_cache_append_prompt": dict(cache=cache, q=q, k=kv, v=kv.clone(), rows=_i(B + 1), q_out=q.clone(), start=_i(B), q_norm=w,
                                         k_norm=w, eps=1e-5, cos=cos, sin=cos.clone(), interleaved=True, **opt),
        "pldp_attend_prompt": dict(cache=cache, q=q, rows=_i(B + 1), out=q.clone(), workspace=_f(64), start=_i(B), lse=_f(R, Hq),
                                   scale=0.3, **opt),
        "pldp_pages_reserve": dict(table=table, start=_i(B), copies=_i(B, 2), workspace=_f(64), n=11, count=_i(B), **opt),
        "pldp_pages_fork": dict(table=table, parent=_i(B), len=_i(B), **opt),
        "pldp_pages_free": dict(table=table, keep_len=_i(B), stream=7),
        "pldp_pages_compact": dict(table=table, copies=_i(5, 2), n_copies=_i(1), workspace=_f(64), used=_i(1), stream=7),
        "pldp_cache_copy_pages": dict(cache=cache, copies=_i(5, 2), n_copies=_i(1), stream=7),
    }
    assert set(full) == set(pk._PROMPT_CALLS)
    needed = {f: [p.name for p in inspect.signature(getattr(pk, f)).parameters.values() if p.default is p.empty] for f in full}
    return full, {f: {**{k: a[k] for k in needed[f]}, "stream": 0} for f, a in full.items()}


def test_native_and_python_checks_agree(any_device, monkeypatch):  # noqa: F811
    """Every argument of every call in turn replaced by other things, on host tensors with the entry
    points replaced."""
    spec = importlib.util.spec_from_file_location("_pldp_calls", any_device)
    native = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(native)
    rec = Recorder(pk._load())
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    with pytest.raises(ValueError):
        native.bind_prompt((1, 2))
    both = _arguments()
    assert native.pages_free(both[0]["pldp_pages_free"]["table"].address, _i(B), None) is None    # not bound yet
    native.bind_prompt(rec.addresses)
    monkeypatch.setattr(pk, "_load", lambda: rec)

    def outcome(f, args, calls):
        monkeypatch.setattr(pk, "_calls", calls)
        rec.made.clear()
        try:
            getattr(pk, f)(**args)
            return list(rec.made)
        except Exception as e:
            return [*rec.made, type(e), str(e)]

    def agree(f, args, what):
        a, b = outcome(f, args, native), outcome(f, args, None)
        assert a == b, (f, what, a, b)
        return a

    for arguments in both:
        for f, args in arguments.items():
            taken = getattr(native, f[5:])
            made = agree(f, args, "as it is")
            assert len(made) == 1 and made[0][0] == f, made
            seen = []

            class Spy:
                def __getattr__(self, name):
                    return lambda *a: seen.append(taken(*a)) or seen[-1]

            outcome(f, args, Spy())
            assert seen == [0], (f, "not taken natively")
            rec.rc = 3
            assert agree(f, args, "refused by the library")[1] is pk.PldpError
            rec.rc = 0
            for name, x in args.items():
                if name in ("cache", "table"):
                    for y in (None, 3, both[0]["pldp_pages_free"]["table"] if name == "cache" else both[0]["pldp_attend_prompt"]["cache"]):
                        agree(f, {**args, name: y}, name)
                    continue
                for i, y in enumerate(_variants(x)):
                    agree(f, {**args, name: y}, (name, i, y))
