"""The native argument marshalling of the rotation's calls against the general path, without a GPU."""
import pytest
import torch

import paper_2608_27370_gb300 as P
import _native_harness as H
from test_binding_layer_ops import harness  # noqa: F401

T, HQ, HK, D, ROT = 6, 3, 2, 64, 32
bf16, f32, i32, i64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


class Recorder(H.Recorder):
    def _note(self, name, where, args):
        heads = (0, 1, 9, 10) if name in ("puro_rope", "puro_rope_backward") else ()
        args = [[getattr(P.puro_heads_t.from_address(a), f) for f, _ in P.puro_heads_t._fields_] if i in heads else a
                for i, a in enumerate(args)]
        return super()._note(name, where, args)


def _arguments():
    e = lambda dt, *s: torch.zeros(s, dtype=dt)  # noqa: E731
    qkv = e(bf16, T, (HQ + 2 * HK) * D)
    q, k = qkv[:, :HQ * D].view(T, HQ, D), qkv[:, HQ * D:(HQ + HK) * D].view(T, HK, D)
    qo, ko = e(bf16, HQ, T, D).transpose(0, 1), e(bf16, T, HK, D)
    return {"puro_rope": (q, k, e(i64, ROT // 2), e(i32, T), True, qo, ko, 0.75, None),
            "puro_rope_backward": (qo, ko, e(i64, ROT // 2), e(i32, T), False, q, k, 1.0, None),
            "puro_rope_tables": (e(i64, ROT // 2), 11, e(f32, 9, ROT // 2), e(f32, 9, ROT // 2), 1.5, None)}


@pytest.fixture
def both(harness, monkeypatch):  # noqa: F811
    lib = Recorder()
    m = H.load(harness, lib.addresses)
    monkeypatch.setattr(P, "_lib", lib)
    monkeypatch.setattr(P, "_native", P._CtypesOnly())
    monkeypatch.setattr(P, "_stream", lambda stream: H.STREAM if stream is None else int(stream))
    monkeypatch.setattr(P, "_current_device", lambda: 0)

    def calls(name, args, shown=True):
        args = [H.shown_as_cuda(m, a) for a in args] if shown else args
        lib.calls.clear()
        native = getattr(m, name)(*args)
        assert native in (None, lib.STATUS)
        got = lib.calls[0] if native is not None else None
        lib.calls.clear()
        kw = {}
        positional = list(args)
        if name == "puro_rope_tables":  # (the native order)
            kw = {"scale": positional[4], "stream": positional[5]}
            positional = positional[:4]
        try:
            getattr(P, name)(*positional, **kw)
        except P.PuroError:
            return got, lib.calls[0]
        except (ValueError, TypeError, AttributeError) as e:
            return got, type(e)
        raise AssertionError("the recorder's status was not reported")

    calls.module = m
    return calls


@pytest.mark.parametrize("name", sorted(_arguments()))
def test_both_paths_call_the_library_alike(name, both):
    ordinary = _arguments()[name]
    native, general = both(name, ordinary)
    assert native is not None and native == general
    if name != "puro_rope_tables":
        native, general = both(name, [*ordinary[:3], None, *ordinary[4:]])
        assert native is not None and native == general


@pytest.mark.parametrize("name", sorted(_arguments()))
def test_odd_arguments_are_left_to_the_general_path(name, both):
    ordinary = [H.shown_as_cuda(both.module, a) for a in _arguments()[name]]
    for i, a in enumerate(ordinary):
        if not torch.is_tensor(a):
            continue
        odd = [both.module.as_cuda(torch.zeros(a.shape, dtype=torch.float64)), both.module.as_cuda(torch.zeros((*a.shape, 2), dtype=a.dtype)[..., 0]),
               both.module.as_cuda(torch.zeros(tuple(s + 1 for s in a.shape), dtype=a.dtype)), torch.zeros(a.shape, dtype=a.dtype),
               both.module.as_cuda(torch.zeros(0, dtype=a.dtype)), object()]
        for o in odd:
            native, general = both(name, [*ordinary[:i], o, *ordinary[i + 1:]], shown=False)
            assert native is None or native == general, (i, o)
