"""The cache and scoring calls without a GPU: argument blocks as the header lays them out, and
the host's checks before anything is launched."""
import ctypes
import os
import subprocess

import pytest

import paper_2412_01447_gb300 as pk

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "pldp.h")
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def so():
    pk.build()
    return pk._load()


@pytest.mark.parametrize("struct,cls", [("pldp_cache", pk.pldp_cache_args), ("pldp_cache_append_args", pk.pldp_cache_append_args),
                                        ("pldp_cache_read_args", pk.pldp_cache_read_args), ("pldp_attend_args", pk.pldp_attend_args),
                                        ("pldp_rank_cache_args", pk.pldp_rank_cache_args)])
def test_blocks_match_the_header(tmp_path, struct, cls):
    names = [f for f, _ in cls._fields_]
    src = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{HEADER}"', "int main(void) {",
           f'printf("%zu\\n", sizeof({struct}));']
    src += [f'printf("%zu\\n", offsetof({struct}, {n}));' for n in names] + ["return 0; }"]
    (tmp_path / "layout.c").write_text("\n".join(src))
    subprocess.check_call(["gcc", str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")])
    out = [int(x) for x in subprocess.check_output([str(tmp_path / "layout")]).split()]
    assert out == [ctypes.sizeof(cls)] + [getattr(cls, n).offset for n in names]


def _cache(**kw):
    c = pk.pldp_cache_args(k=P(256), v=P(256), dtype=1, n_pages=4, page_size=16, heads=2, head_dim=64, page_stride=2048,
                           pos_stride=128, head_stride=64, pages=P(256), pages_stride=2, max_pages=2)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _three(*x):
    return (ctypes.c_int64 * 3)(*x)


def _append(**kw):
    a = pk.pldp_cache_append_args(cache=_cache(**kw.pop("cache", {})), q=P(256), k=P(256), v=P(256), dtype=1, B=2, n=3, q_heads=4,
                                  q_strides=_three(768, 256, 64), k_strides=_three(768, 256, 64), v_strides=_three(768, 256, 64),
                                  eps=1e-6, seq_len=P(256), q_out=P(256), q_out_strides=_three(768, 256, 64))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_CACHES = [(dict(dtype=0), 2, "dtype"), (dict(head_dim=24), 2, "multiple of 16"), (dict(head_dim=272), 2, "heads of"),
              (dict(heads=0), 2, "heads"), (dict(n_pages=0), 1, "n_pages"), (dict(max_pages=3), 1, "pages_stride"),
              (dict(page_size=1 << 30, max_pages=2, pages_stride=2), 1, "2\\^31"), (dict(k=None), 1, "null"),
              (dict(dtype=2), 1, "k_scale"), (dict(pos_stride=132), 1, "16 bytes"), (dict(v=P(264)), 1, "aligned")]


@pytest.mark.parametrize("bad,rc,match", BAD_CACHES)
def test_cache_descriptions(so, bad, rc, match):
    a = _append(cache=bad)
    assert so.pldp_cache_append(ctypes.byref(a), None) == rc
    assert __import__("re").search(match, pk.pldp_last_error()), pk.pldp_last_error()


def test_append_checks(so):
    call = lambda **kw: so.pldp_cache_append(ctypes.byref(_append(**kw)), None)
    assert so.pldp_cache_append(None, None) == 1
    assert call(B=-1) == 1 and call(n=0) == 1 and call(q_heads=0) == 1 and call(dtype=2) == 2
    assert call(q=None) == 1 and "null" in pk.pldp_last_error()
    assert call(q=P(264)) == 1 and "aligned" in pk.pldp_last_error()
    assert call(k_strides=_three(768, 260, 64)) == 1 and "k strides" in pk.pldp_last_error()
    assert call(q_out_strides=_three(768, -256, 64)) == 1
    assert call(cos=P(256)) == 1 and "together" in pk.pldp_last_error()
    assert call(cos=P(256), sin=P(256), rot=3, rot_rows=4) == 1 and call(cos=P(256), sin=P(256), rot=66, rot_rows=4) == 1
    assert call(cos=P(256), sin=P(256), rot=64, rot_rows=0) == 1
    assert call(eps=float("nan")) == 1 and call(eps=-1.0) == 1
    assert call(B=0, q=None) == 0


def test_read_checks(so):
    def call(**kw):
        a = pk.pldp_cache_read_args(cache=_cache(), count=P(256), B=2, n=4, dtype=1, k_out=P(256), v_out=P(256),
                                    out_strides=_three(512, 128, 64))
        for k, v in kw.items():
            setattr(a, k, v)
        return so.pldp_cache_read(ctypes.byref(a), None)
    assert so.pldp_cache_read(None, None) == 1
    assert call(B=-1) == 1 and call(n=-1) == 1 and call(dtype=2) == 2 and call(count=None) == 1 and call(B=70000) == 2
    assert call(out_strides=_three(512, 129, 64)) == 1 and call(n=0, count=None) == 0


def test_attend_checks(so):
    def call(**kw):
        a = pk.pldp_attend_args(cache=_cache(), q=P(256), B=2, n=3, q_heads=4, q_strides=_three(768, 256, 64), seq_len=P(256), scale=0.1,
                                out=P(256), out_strides=_three(768, 256, 64), workspace=P(256),
                                workspace_bytes=pk.pldp_attend_workspace_size(2, 3, 4, 2, 64))
        for k, v in kw.items():
            setattr(a, k, v)
        return so.pldp_attend_cache(ctypes.byref(a), None)
    assert so.pldp_attend_cache(None, None) == 1
    assert call(n=0) == 1 and call(q_heads=3) == 1 and call(scale=float("inf")) == 1 and call(workspace_bytes=8) == 1
    assert call(workspace=P(272)) == 1 and call(seq_len=None) == 1 and call(out=P(264)) == 1 and call(B=0, q=None) == 0
    size = pk.pldp_attend_workspace_size
    assert size(-1, 1, 1, 1, 64) == 0 and size(1, 0, 1, 1, 64) == 0 and size(1, 1, 3, 2, 64) == 0 and size(8, 13, 32, 8, 128) % 256 == 0


def test_rank_checks(so):
    def call(**kw):
        a = pk.pldp_rank_cache_args(cache=_cache(), q=P(256), B=2, n=3, q_heads=4, q_strides=_three(768, 256, 64), kv_len=P(256),
                                    lse=P(256), scale=0.1, cand_pos=P(256), cand_count=P(256), C_cap=8, best_pos=P(256))
        for k, v in kw.items():
            setattr(a, k, v)
        return so.pldp_rank_cache(ctypes.byref(a), None)
    assert so.pldp_rank_cache(None, None) == 1
    assert call(C_cap=-1) == 1 and call(agg=2) == 1 and call(heads=P(256), n_sel=0) == 1 and call(heads=P(256), n_sel=800) == 2
    assert call(accumulate=1) == 1 and call(scale=float("nan")) == 1 and call(lse=None) == 1 and call(q_heads=5) == 1
    assert call(B=0, q=None) == 0


def test_logprobs_checks(so):
    def call(**kw):
        a = dict(logits=P(256), dtype=1, rows=2, V=100, T=1.0, tokens=P(256), logprob=P(256), entropy=None, top=0, top_id=None,
                 top_logprob=None, ws=P(256), bytes=pk.pldp_token_logprobs_workspace_size(2, 100), stream=None) | kw
        return so.pldp_token_logprobs(*a.values())
    assert call(rows=-1) == 1 and call(V=0) == 1 and call(dtype=2) == 2 and call(tokens=None) == 1 and call(ws=P(264)) == 1
    for t in (0.0, -1.0, float("inf"), float("nan")):
        assert call(T=t) == 1 and "temperature" in pk.pldp_last_error()
    assert call(top=-1) == 1 and call(top=33) == 1 and call(top=11, V=10) == 1 and call(logits=None) == 1 and call(bytes=4) == 1
    assert call(rows=0, logits=None) == 0
    assert pk.pldp_token_logprobs_workspace_size(-1, 5) == 0 and pk.pldp_token_logprobs_workspace_size(5, 0) == 0


def test_host_tensors_are_refused():
    import torch
    x = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        pk.pldp_cache(x, x, torch.zeros((1, 2), dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        pk.pldp_token_logprobs(x, None, None, x)
