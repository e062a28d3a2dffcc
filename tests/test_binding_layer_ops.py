"""The native argument marshalling of the calls beside the linears (gates,
epilogues, query and key norms) against the general path, without a GPU."""
import pytest
import torch

import paper_2608_27370_gb300 as P
import _native_harness as H

u8, i32, bf16, f32 = torch.uint8, torch.int32, torch.bfloat16, torch.float32
M, F, K, T, HQ, HK, D = 256, 384, 128, 6, 3, 2, 64


class Recorder(H.Recorder):
    """Also notes the fields of the heads' structures and of the gated operands."""

    def _note(self, name, where, args):
        if name == "puro_fp8_gated_fprop":
            where = (0, 1)
        heads = {"puro_qk_norm_rope": (0, 1, 13, 14), "puro_qk_norm_rope_backward": (0, 1, 2, 3, 15, 16)}.get(name, ())
        args = [[getattr(P.puro_heads_t.from_address(a), f) for f, _ in P.puro_heads_t._fields_] if i in heads else a
                for i, a in enumerate(args)]
        return super()._note(name, where, args)


def _arguments():
    e = lambda dt, *s: torch.zeros(s, dtype=dt)  # noqa: E731
    op = lambda r, c, role=P.ROLE_ACT: P.FP8Operand(e(u8, r, c), e(u8, *P.scale_vec_shape(r, c)), role=role)  # noqa: E731
    st = (e(i32, 1), None)
    copies = lambda r, c: (e(u8, r, c), e(u8, *P.scale_vec_shape(r, c)), e(u8, c, r), e(u8, *P.scale_vec_shape(c, r)))  # noqa: E731
    gu, qkv = e(bf16, M, 2 * F), e(bf16, T, (HQ + 2 * HK) * D)
    q, k = qkv[:, :HQ * D].view(T, HQ, D), qkv[:, HQ * D:(HQ + HK) * D].view(T, HK, D)
    qo, ko = e(bf16, HQ, T, D).transpose(0, 1), e(bf16, T, HK, D)
    tab, pos, ws = (e(f32, 9, D // 2), e(f32, 9, D // 2)), e(i32, T), e(u8, 64)
    wide = e(bf16, M, F + 24)
    return {
        "puro_fp8_linear_fprop_epilogue": (op(M, K), op(F, K, 1), e(bf16, M, F), e(bf16, F), 3, wide[:, 8:F + 8], e(bf16, M, F), ws, *st),
        "puro_bf16_linear_fprop_epilogue": (e(bf16, 5, K), e(bf16, F, K), e(bf16, 5, F), e(bf16, F), 2, e(bf16, 5, F), e(bf16, 5, F), *st),
        "puro_fp8_gated_fprop": (op(M, K), op(2 * F, K, 1), 2, 1, gu, e(bf16, M, F), *copies(M, F), *st),
        "puro_bf16_gated_fprop": (e(bf16, 5, K), e(bf16, 2 * F, K), 2, e(bf16, 5, 2 * F), e(bf16, 5, F), *st),
        "puro_fp8_quantize_act_backward": (e(bf16, M, F), e(bf16, M, F), 4, 0, e(bf16, M, F), e(f32, F), ws, *copies(M, F), *st),
        "puro_act_backward_bf16": (e(bf16, M, F), e(bf16, M, F), 1, e(bf16, M, F), e(f32, F), ws, None),
        "puro_fp8_quantize_gated_backward": (e(bf16, M, F), gu[:, :F], gu[:, F:], 2, 0, e(bf16, M, 2 * F), *copies(M, 2 * F), *st),
        "puro_gated_backward_bf16": (e(bf16, M, F), gu[:, :F], gu[:, F:], 3, e(bf16, M, 2 * F), None),
        "puro_qk_norm_rope": (q, k, e(bf16, D), e(bf16, D), 1e-6, *tab, pos, True, qo, ko, e(f32, T, HQ + HK), *st),
        "puro_qk_norm_rope_backward": (qo, ko, q, k, e(f32, T, HQ + HK), e(bf16, D), e(bf16, D), *tab, pos, False, q, k, e(f32, D),
                                       e(f32, D), ws, *st),
    }


OPTIONAL = {"puro_fp8_linear_fprop_epilogue": (3, 5, 6, 7, 8), "puro_bf16_linear_fprop_epilogue": (3, 5, 6, 7), "puro_fp8_gated_fprop": (4, 5, 10),
            "puro_bf16_gated_fprop": (3, 5), "puro_fp8_quantize_act_backward": (1, 4, 5, 6, 11), "puro_act_backward_bf16": (1, 3, 4, 5),
            "puro_fp8_quantize_gated_backward": (5, 10), "puro_gated_backward_bf16": (), "puro_qk_norm_rope": (2, 3, 7, 11, 12),
            "puro_qk_norm_rope_backward": (5, 6, 9, 13, 14, 15, 16)}


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    return H.build(tmp_path_factory.mktemp("harness"))


@pytest.fixture
def both(harness, monkeypatch):
    """calls(name, args): how the native and the general path call the library (None: declined, or an error's type)."""
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
        try:
            getattr(P, name)(*args)
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
    for i in OPTIONAL[name]:
        args = list(ordinary)
        args[i] = None
        native, general = both(name, args)
        assert native is not None and native == general, i


@pytest.mark.parametrize("name", sorted(_arguments()))
def test_odd_arguments_are_left_to_the_general_path(name, both):
    """Another type, shape, layout or place of each tensor in turn: what the native function takes reaches the library as
    in the general path, and what that refuses is not taken."""
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


def test_a_tensor_on_another_device_is_refused(monkeypatch):
    class Elsewhere:
        is_cuda = True

        def get_device(self):
            return 1

    monkeypatch.setattr(P, "_current_device", lambda: 0)
    with pytest.raises(ValueError):
        P._on_current_device(None, Elsewhere())
