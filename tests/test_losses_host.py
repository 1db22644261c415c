"""Refusals of the losses on rows of logits and of gradient clipping: arguments that no kernel is launched for.
Checked before anything touches a device."""
import ctypes

import numpy as np
import pytest

import paper_1906_08879_amd as pl
from paper_1906_08879_amd import binding as b

NULL, SHAPE = -1, -2
SOME = 4096                                               # stands for device memory; nothing is launched


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(pl.library_path()):
        from paper_1906_08879_amd.build import build
        build()
    return pl.load_library()


def _x(**kw):
    v = dict(data=SOME, n_rows=8, row_stride=5, n_actions=5, dtype=0)
    v.update(kw)
    return b.LogitsView(*[v[k] for k, _ in b.LogitsView._fields_])


def _rows(**kw):
    v = dict(n_seqs=2, order=0, bounds=None, mask=None)
    v.update(kw)
    return b.RowsView(*[v[k] for k, _ in b.RowsView._fields_])


def _policy(lib, x=None, rows=None, ws=SOME, ws_bytes=1 << 20, grad=SOME, stride=5, actions=SOME, adv=SOME, stats=SOME, **cfg):
    c = dict(clip_low=0.2, clip_high=0.2, kl_coeff=0.0, entropy_coeff=0.0, grad_scale=1.0, reduction=0, advantage_per_seq=0)
    c.update(cfg)
    c = b.PolicyLossCfg(*[c[k] for k, _ in b.PolicyLossCfg._fields_])
    return lib.pl_clipped_policy_loss(ctypes.byref(_x() if x is None else x), None if rows is None else ctypes.byref(rows),
                                      ctypes.byref(c), actions, adv, None, None, stats, grad, stride, None, None, None, None, ws,
                                      ws_bytes, None)


def _preference(lib, rows=None, n_pairs=1, pairs=None, stats=SOME, **cfg):
    c = dict(beta=0.1, label_smoothing=0.0, grad_scale=1.0, average=0)
    c.update(cfg)
    c = b.PreferenceCfg(*[c[k] for k, _ in b.PreferenceCfg._fields_])
    return lib.pl_preference_loss(ctypes.byref(_x()), ctypes.byref(_rows() if rows is None else rows), ctypes.byref(c), SOME, None,
                                  n_pairs, pairs, stats, None, 0, None, None, None, None, SOME, 1 << 20, None)


BAD_LOGITS = [dict(dtype=3), dict(dtype=-1), dict(n_actions=0), dict(n_actions=(1 << 24) + 1, row_stride=1 << 25), dict(n_rows=-1),
              dict(n_rows=1 << 31), dict(row_stride=4), dict(row_stride=(1 << 31) + 1), dict(data=SOME + 2)]


@pytest.mark.parametrize("bad", BAD_LOGITS)
def test_logits_are_refused(lib, bad):
    assert _policy(lib, x=_x(**bad)) == SHAPE
    if "data" not in bad:
        assert lib.pl_loss_workspace(ctypes.byref(_x(**bad)), None, 0) == 0
        assert lib.pl_action_logp(ctypes.byref(_x(**bad)), SOME, SOME, None, SOME, 1 << 20, None) == SHAPE


@pytest.mark.parametrize("bad,code", [(dict(n_seqs=0), SHAPE), (dict(n_seqs=3), SHAPE), (dict(order=3), SHAPE), (dict(order=2), NULL),
                                      (dict(n_seqs=(1 << 24) + 1), SHAPE)])
def test_rows_are_refused(lib, bad, code):
    assert _policy(lib, rows=_rows(**bad)) == code
    assert _preference(lib, rows=_rows(**bad)) == code


@pytest.mark.parametrize("bad", [dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-1.0), dict(clip_low=float("nan")),
                                 dict(kl_coeff=float("inf")), dict(entropy_coeff=float("nan")), dict(grad_scale=float("inf")),
                                 dict(reduction=3), dict(advantage_per_seq=2), dict(stride=4), dict(grad=SOME + 1), dict(ws=SOME + 8),
                                 dict(ws_bytes=16)])
def test_policy_loss_refuses(lib, bad):
    assert _policy(lib, **bad) == SHAPE


def test_policy_loss_needs_its_arrays(lib):
    assert _policy(lib, x=_x(data=None)) == NULL
    for missing in ("actions", "adv", "stats", "ws"):
        assert _policy(lib, **{missing: None}) == NULL
    assert lib.pl_clipped_policy_loss(None, *[None] * 8, 0, *[None] * 5, 0, None) == NULL
    assert _policy(lib, x=_x(row_stride=7), grad=SOME, stride=5) == SHAPE        # in place with another stride
    assert b"row_stride" in lib.pl_last_error()


@pytest.mark.parametrize("bad", [dict(beta=-1.0), dict(beta=float("inf")), dict(label_smoothing=1.5), dict(average=2), dict(n_pairs=-1),
                                 dict(n_pairs=2), dict(grad_scale=float("nan")), dict(rows=_rows(n_seqs=1))])
def test_preference_loss_refuses(lib, bad):
    assert _preference(lib, **bad) == SHAPE


def test_preference_loss_needs_its_arrays(lib):
    assert _preference(lib, stats=None) == NULL


def test_log_probabilities_need_their_arrays(lib):
    x = ctypes.byref(_x())
    assert lib.pl_action_logp(None, SOME, SOME, None, SOME, 1 << 20, None) == NULL
    assert lib.pl_action_logp(x, None, SOME, None, SOME, 1 << 20, None) == NULL
    assert lib.pl_action_logp(x, SOME, None, None, SOME, 1 << 20, None) == NULL
    assert lib.pl_action_logp(x, SOME, SOME, None, None, 1 << 20, None) == NULL
    assert lib.pl_action_logp(x, SOME, SOME, None, SOME, 4, None) == SHAPE
    assert lib.pl_action_logp(ctypes.byref(_x(n_rows=0)), None, None, None, None, 0, None) == 0


def _clip(lib, n=1, src=SOME, dst=None, numel=4, dtype=0, max_norm=1.0, norm=SOME, ws=SOME, ws_bytes=1 << 20):
    one = lambda t, v: (t * 1)(v)  # noqa: E731
    return lib.pl_clip_gradients(n, one(ctypes.c_void_p, src), None if dst is None else one(ctypes.c_void_p, dst),
                                 one(ctypes.c_int64, numel), one(ctypes.c_int32, dtype), max_norm, norm, ws, ws_bytes, None)


def test_clipping_refuses(lib):
    for bad in (dict(n=-1), dict(numel=-1), dict(numel=(1 << 44) + 1), dict(dtype=3), dict(max_norm=-1.0), dict(max_norm=float("nan")),
                dict(src=SOME + 1), dict(dst=SOME + 2), dict(ws=SOME + 4), dict(ws_bytes=8)):
        assert _clip(lib, **bad) == SHAPE, bad
    for bad in (dict(src=None), dict(norm=None), dict(ws=None)):
        assert _clip(lib, **bad) == NULL, bad
    assert lib.pl_clip_gradients(1, None, None, None, None, 1.0, SOME, SOME, 1 << 20, None) == NULL
    assert lib.pl_clip_gradients_workspace(-1) == 0
    assert lib.pl_clip_gradients_workspace(0) > 0
    sizes = [lib.pl_clip_gradients_workspace(n) for n in (1, 100, 1000, 100000)]
    assert sizes == sorted(sizes)


def test_workspace_grows_with_rows_and_sequences(lib):
    size = lambda n, V, S: lib.pl_loss_workspace(ctypes.byref(_x(n_rows=n, n_actions=V, row_stride=V)),  # noqa: E731
                                                 ctypes.byref(_rows(n_seqs=S, order=2)), 0)
    assert 0 < size(1, 1, 1) <= size(100, 1, 1) <= size(100, 1, 100) <= size(1 << 20, 1, 100)
    assert size(1, 1 << 24, 1) > 0
    assert size(8, 5, 0) == 0 and lib.pl_loss_workspace(None, None, 0) == 0


def test_binding_refuses_tensors_off_the_device():
    import torch
    x, a, f = torch.zeros(4, 3), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(pl.PlacetoError):
        pl.action_logp(x, a, f)
    with pytest.raises(pl.PlacetoError):
        pl.clipped_policy_loss(x, a, f, torch.zeros(5))
    with pytest.raises(pl.PlacetoError):
        pl.clip_gradients([f], 1.0, f)
    with pytest.raises(pl.PlacetoError):
        pl.DecisionRows(4, 2, "sideways")
    with pytest.raises(pl.PlacetoError):
        pl.DecisionRows(4, 2, bounds=torch.zeros(2, dtype=torch.int32))
    assert np.isfinite(pl.load_library().pl_clip_gradients_workspace(3))


@pytest.mark.parametrize("grads,norm,out", [([], None, None), ([np.zeros(3, np.float32)], "norm", None), ([None], "norm", None), ([], "norm", [None])])
def test_binding_refuses_what_is_no_tensor(grads, norm, out):
    import torch
    with pytest.raises(pl.PlacetoError):
        pl.clip_gradients(grads, 1.0, torch.zeros(1) if norm else None, out=out)
