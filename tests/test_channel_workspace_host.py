"""Checks of the wrappers of the operators over channels, and the scratch memory that
they keep (no GPU needed: the memory is the CPU's, and streams are numbers)."""
import itertools
import types
import weakref

import pytest

torch = pytest.importorskip("torch")
L = pytest.importorskip("paper_2307_15034_amd.layer")


def test_a_workspace_that_was_handed_out_stays(monkeypatch):
    """A captured graph holds the address of the workspace that its calls got.  A
    later call that needs more gets another one; the first is not given back."""
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: types.SimpleNamespace(cuda_stream=0))
    ws, cpu = L._Workspace(), torch.device("cpu")
    seen = []
    for nbytes in (256, 1024, 512, 4096):
        at, n = ws.get(nbytes, cpu, 0)
        assert n >= nbytes and at == ws._t.data_ptr()
        seen.append((at, weakref.ref(ws._t)))
    assert all(t() is not None and t().data_ptr() == at for at, t in seen)
    assert seen[1][0] == seen[2][0] and len({at for at, _ in seen}) == 3


def test_a_gate_in_the_place_of_another_parameter_is_refused():
    """The same tensor as gate and as a parameter of one row: its shape is not the
    parameter's."""
    op = L.ResidualNorm(8, 16)
    one = torch.ones(1, 16)
    for k in ("post_w", "post_b", "scale", "pre_w", "pre_b"):
        p = {**dict.fromkeys(op.PARAMS), "gate": one, k: one}
        with pytest.raises(ValueError, match=k):
            op._params(tuple(p.values()), False)  # (layout checks alone: no GPU)


def test_a_buffer_for_two_results_is_refused():
    """Refused before any device call, whichever two they are."""
    B = L.B
    at = 1 << 20  # aligned addresses that are never reached
    d = B.make_residual_norm_desc(96, 64, 4)
    names = ("g_x", "g_u") + L.ResidualNorm.PARAMS
    params = B.FnoResidualNormParams(gate=at)
    for a, b in itertools.combinations(names, 2):
        to = {k: (i + 2) * at for i, k in enumerate(names)}
        to[b] = to[a]
        grads = B.FnoResidualNormParams(**{k: v for k, v in to.items() if k not in ("g_x", "g_u")})
        assert B.fno_residual_norm_bwd(d, params, at, at, at, at, at, to["g_x"], to["g_u"], grads, at, 1 << 40,
                                       0, check=False) == B.FNO_ERR_INVALID_ARGUMENT, (a, b)
    d = B.make_fp8_quantize_desc(96, 64)
    names = ("codes", "scale", "codes_t", "scale_t", "col_sums")
    for a, b in itertools.combinations(names, 2):
        to = {k: (i + 2) * at for i, k in enumerate(names)}
        to[b] = to[a]
        assert B.fno_fp8_quantize(d, at, ws=at, ws_bytes=1 << 40, stream=0, check=False,
                                  **to) == B.FNO_ERR_INVALID_ARGUMENT, (a, b)
