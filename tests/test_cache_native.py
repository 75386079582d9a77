"""The binding's native form of the cache and scoring calls against the Python form: the same calls are
made, with the same argument blocks, and what a check refuses is refused the same way."""
import ctypes
import importlib.util
import inspect

import pytest
import torch

import paper_2412_01447_gb300 as pk
from tests.test_native_calls import _f, _i, _variants, any_device  # noqa: F401  (a fixture)

B, n, Hq, H, D, page, C, V = 3, 2, 6, 2, 32, 4, 5, 16
NAMES = {"pldp_cache_append": "append", "pldp_cache_read": "read", "pldp_attend_cache": "attend", "pldp_rank_cache": "rank",
         "pldp_token_logprobs": "logprobs"}


class Recorder:
    def __init__(self, lib):
        self.made, self.rc, self.fns = [], 0, {}
        for f in pk._CACHE_CALLS:
            self.fns[f] = ctypes.CFUNCTYPE(ctypes.c_int, *getattr(lib, f).argtypes)(self._entry(f))
        self.addresses = tuple(ctypes.cast(self.fns[f], ctypes.c_void_p).value for f in pk._CACHE_CALLS)

    def _entry(self, name):
        def entry(*args):
            def flat(x):
                if isinstance(x, ctypes.Structure):            # field by field: padding holds anything
                    return tuple(flat(getattr(x, f)) for f, _ in x._fields_)
                return tuple(x) if isinstance(x, ctypes.Array) else repr(x)
            self.made.append((name, *(flat(a.contents) if hasattr(a, "contents") else repr(a) for a in args)))
            return self.rc
        return entry

    def pldp_last_error(self):
        return b"refused"

    def __getattr__(self, name):
        return self.fns[name]


def _arguments():
    pool = _f(7, page, H, D, dtype=torch.bfloat16)
    cache = pk.pldp_cache(pool, pool.clone(), _i(B, 3))
    q, kv = _f(B, n, Hq + 1, D, dtype=torch.bfloat16)[:, :, :Hq], _f(B, n, H, D, dtype=torch.bfloat16)
    opt = dict(status=_i(B), stream=7)
    w = _f(D, dtype=torch.bfloat16)
    cos = _f(9, D // 2)
    full = {
        "pldp_cache_append": dict(cache=cache, q=q, k=kv, v=kv.clone(), seq_len=_i(B), q_out=q.clone(), draft_len=_i(B), q_norm=w,
                                  k_norm=w, eps=1e-5, cos=cos, sin=cos.clone(), interleaved=True, **opt),
        "pldp_cache_read": dict(cache=cache, start=_i(B), count=_i(B), k_out=_f(B, 4, H, D), v_out=_f(B, 4, H, D), **opt),
        "pldp_attend_cache": dict(cache=cache, q=q, seq_len=_i(B), out=q.clone(), workspace=_f(64), draft_len=_i(B),
                                  lse=_f(B, n, Hq), scale=0.3, **opt),
        "pldp_rank_cache": dict(cache=cache, q=q, row=_i(B), kv_len=_i(B), lse=_f(B, n, Hq), cand_pos=_i(B, C), cand_count=_i(B),
                                best_pos=_i(B), heads=_i(3), agg="sum", scale=0.3, scores=_f(B, C), best_score=_f(B), accumulate=True,
                                **opt),
        "pldp_token_logprobs": dict(logits=_f(B, n, V), tokens=_i(B, n), logprob=_f(B, n), workspace=_f(64), entropy=_f(B, n),
                                    top_id=_i(B, n, 3), top_logprob=_f(B, n, 3), temperature=0.7, stream=7),
    }
    assert set(full) == set(pk._CACHE_CALLS)
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
        native.bind_cache((1, 2))
    both = _arguments()
    assert native.cache_read(both[0]["pldp_cache_read"]["cache"].address, B, *[None] * 6) is None    # not bound yet
    native.bind_cache(rec.addresses)
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
                if name == "cache":
                    agree(f, {**args, name: None}, name)
                    continue
                for i, y in enumerate(_variants(x)):
                    agree(f, {**args, name: y}, (name, i, y))
