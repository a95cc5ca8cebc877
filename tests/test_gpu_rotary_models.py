"""Models whose rotary positions are not the plain ones over the whole head (pahq_set_rotary): a part of the head, neighbouring
elements paired, stretched frequencies, a magnitude, against the oracle with those positions in 64 bits on the weights as
they are given."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(__file__), "golden"))
sys.path.insert(0, os.path.dirname(__file__))
import workloads                                    # noqa: E402
from fp32_spread import SpreadModel, kl_with_spread  # noqa: E402
from tolerance import bound, check_kl_cases         # noqa: E402

from oracle.acdc import MODE_PAHQ, MODE_ALL_FP32   # noqa: E402

pytestmark = pytest.mark.gpu

FORMS = {
    "part": dict(rot_dim=16),
    "neighbours": dict(rot_dim=64, layout="interleaved"),
    "part of neighbours, stretched": dict(rot_dim=20, layout="interleaved", theta=500.0, scaling="linear", factor=4.0),
    "whole, bands": dict(rot_dim=64, theta=100.0, scaling="bands", factor=8.0, original=64.0, turns=(1.0, 4.0), magnitude=1.25),
}


def rotated(a, B, S, dh, rot_dim, layout="half", theta=10000.0, scaling="none", factor=1.0, original=0.0, turns=(1.0, 32.0), magnitude=1.0):
    """Rows [B * S][dh] turned by their positions, by the definition."""
    f = theta ** (-2.0 * np.arange(rot_dim // 2) / rot_dim)
    if scaling == "linear":
        f = f / factor
    if scaling == "bands":
        g = np.clip((original * f / (2 * np.pi) - turns[0]) / (turns[1] - turns[0]), 0, 1)
        f = f * (g + (1 - g) / factor)
    phi = np.tile(np.arange(S)[:, None] * f, (B, 1))
    i = np.arange(rot_dim // 2)
    ia, ib = (i, i + rot_dim // 2) if layout == "half" else (2 * i, 2 * i + 1)
    out = a.copy()
    out[:, ia] = magnitude * (a[:, ia] * np.cos(phi) - a[:, ib] * np.sin(phi))
    out[:, ib] = magnitude * (a[:, ia] * np.sin(phi) + a[:, ib] * np.cos(phi))
    return out


def oracle_with(form):
    class Model(SpreadModel):
        def _rope(self, a, B, S):
            return rotated(a, B, S, self.dh, **form)
    return Model


@pytest.mark.parametrize("name", list(FORMS))
@pytest.mark.parametrize("precision", [2, 0])
def test_edges_of_models_with_other_positions(name, precision):
    import paper_2510_23264_amd as P
    form = FORMS[name]
    shape, w, clean, corrupt = workloads.make("midllama_hi2")
    assert shape.d_head == 64
    mode = MODE_PAHQ if precision == 2 else MODE_ALL_FP32
    om = oracle_with(form)(shape, w)
    gm = P.Model(shape, w, clean.shape[0], clean.shape[1], precision=precision, max_batch_edges=8, rotary=form)
    try:
        gm.clean_cache(clean, corrupt)
        g = om.g
        cases, got = [], []
        for r in (g.headin(0, 0, 0), g.headin(shape.n_layers - 1, 1, 1), g.headin(0, shape.n_heads - 1, 2), g.OUT):
            senders = np.arange(g.n_upstream(r), dtype=np.int32)
            got.append(np.concatenate([[gm.eval_current(r)], gm.eval_edges(r, senders)]))
            cases.append((r, g.empty_removed(), senders))
        res = kl_with_spread(om, clean, corrupt, mode, cases, seeds=4)
        want = np.concatenate([[c["kl_current"]] + list(c["kl_new"]) for c in res])
        sigma = np.concatenate([[c["sigma_current"]] + list(c["sigma_new"]) for c in res])
        check_kl_cases(np.concatenate(got), want, sigma, what=name)
        # the positions matter here: with the plain ones many edges are outside the bound
        plain = P.Model(shape, w, clean.shape[0], clean.shape[1], precision=precision, max_batch_edges=8)
        plain.clean_cache(clean, corrupt)
        other = np.concatenate([np.concatenate([[plain.eval_current(r)], plain.eval_edges(r, q)]) for r, _, q in cases])
        plain.close()
        assert (np.abs(other - want) > 3 * bound(want, sigma)).sum() >= 4
        if precision == 2:              # the codes come back in the order the weights were given in
            from oracle.e4m3 import quantize_rows
            for which, key in ((P.W_Q, "W_Q"), (P.W_K, "W_K"), (P.W_V, "W_V")):
                slice_ = w[key][0, 1]
                codes, scale = gm.get_weight_q(which, 0, 1, slice_.shape)
                want_codes, want_scale = quantize_rows(slice_.reshape(1, -1))
                assert (codes.reshape(1, -1) == want_codes).all() and np.float32(np.ravel(want_scale)[0]) == scale
    finally:
        gm.close()


def test_refusals_and_the_dropped_caches():
    import ctypes as C
    import paper_2510_23264_amd as P
    shape, w, clean, corrupt = workloads.make("midllama_hi")
    gm = P.Model(shape, w, clean.shape[0], clean.shape[1], precision=2, max_batch_edges=8)
    try:
        gm.clean_cache(clean, corrupt)
        before = gm.eval_edges(0, np.arange(1, dtype=np.int32))
        t = P.rotary_entries(64, theta=shape.rope_theta)
        tp = t.ctypes.data_as(C.POINTER(C.c_uint64))
        call = P.lib().pahq_set_rotary
        assert [call(None, tp, 64, 1.0), call(gm.h, None, 64, 1.0), call(gm.h, tp, 0, 1.0), call(gm.h, tp, 31, 1.0), call(gm.h, tp, 66, 1.0),
                call(gm.h, tp, 64, float("inf")), call(gm.h, tp, 64, float("nan"))] == [-1] * 7
        assert np.array_equal(gm.eval_edges(0, np.arange(1, dtype=np.int32)), before)      # a refused call changes nothing
        assert call(gm.h, tp, 64, 1.0) == 0
        with pytest.raises(P.PahqError) as e:
            gm.eval_edges(0, np.arange(1, dtype=np.int32))
        assert e.value.code == -2
        gm.clean_cache(clean, corrupt)
        # the same positions by another road: cosines may differ in the last place
        assert np.allclose(gm.eval_edges(0, np.arange(1, dtype=np.int32)), before, rtol=1e-2)
    finally:
        gm.close()
    shape, w, clean, corrupt = workloads.make("mid_hi")
    with pytest.raises(P.PahqError) as e:               # learned positions
        P.Model(shape, w, clean.shape[0], clean.shape[1], precision=2, max_batch_edges=8, rotary=dict(rot_dim=16))
    assert e.value.code == -2
    for bad in (dict(rot_dim=33), dict(rot_dim=66), dict(rot_dim=16, layout="other"), dict(rot_dim=16, scaling="other")):
        with pytest.raises((ValueError, P.PahqError)):
            P.Model(*workloads.make("midllama_hi")[:2], 4, 4, rotary=bad)
