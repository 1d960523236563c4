"""What the entry points of the feed-forward block refuse, before anything reaches a device: status, and a text that names the reason."""

import ctypes

import pytest

from paper_2001_00138_amd import binding as B

L = B.lib
P = 1 << 20                   # stands for device addresses that no call gets as far as reading
Q, R, S, T, U, V, W = (P << i for i in range(8, 15))


def _refused(status, word, call, *args):
    assert call(*args) == status
    assert word in L().patdnn_last_error().decode()


def _each(call, good, bad):
    for at, value, word in bad:
        _refused(B.PATDNN_EINVAL, word, call, *[value if i == at else v for i, v in enumerate(good)])


def test_quantise():
    q, d = L().patdnn_fp8_quantize, L().patdnn_fp8_dequantize
    for transposed in (0, 1):
        for blocks in (0, 1):
            _each(q, [P, 0, 3, 40, 40, blocks, transposed, Q, R, None],
                  [(1, 3, "type"), (1, 4, "type"), (2, -1, "rows"), (3, 0, "positive"), (4, -1, "strides"), (5, 2, "blocks"), (5, -1, "blocks"), (0, None, "NULL"),
                   (7, None, "NULL"), (8, None, "NULL"), (7, Q + 8, "aligned"), (0, P + 2, "aligned"), (7, P + 16, "overlap"), (8, P + 4, "overlap"), (8, Q, "overlap")])
    # 40 x 128 bytes of codes of the transpose, 3 x 128 of the matrix
    _refused(B.PATDNN_EINVAL, "overlap", q, P, 0, 3, 40, 40, 0, 1, Q, Q + 39 * 128, None)
    _each(d, [Q, R, 3, 40, 0, P, 0, 40, None],
          [(4, 2, "blocks"), (6, 3, "type"), (7, 39, "overlap"), (5, None, "NULL"), (0, P + 16, "overlap"), (1, P + 4, "overlap")])
    for change in (dict(rows=3, cols=2 ** 31 - 1), dict(rows=2 ** 31 - 1, cols=300), dict(rows=2 ** 31 - 1, cols=2 ** 20)):
        for transposed in (0, 1):
            _refused(B.PATDNN_EUNSUPPORTED, "large", q, P, 0, change["rows"], change["cols"], 1, 1, transposed, Q, R, None)
    assert q(None, 0, 0, 40, 40, 0, 1, None, None, None) == B.PATDNN_OK and d(None, None, 0, 40, 0, None, 0, 40, None) == B.PATDNN_OK


def _rms(**change):
    d = dict(rows=4, cols=40, type=0, y_type=0, eps=1e-6, x_row=40, residual_row=40, sum_row=40, y_row=40)
    d.update(change)
    return ctypes.byref(B.RmsDesc(*(d[k] for k, _ in B.RmsDesc._fields_)))


def test_rms_norm():
    f, b, room = L().patdnn_rms_norm, L().patdnn_rms_norm_backward, L().patdnn_rms_norm_workspace_floats
    good_f, big = [_rms(), P, Q, R, S, T, None, U, None], 1 << 20
    good_b = [_rms(), P, Q, R, S, T, U, V, W, big, None]
    for change, word in [(dict(rows=-1), "rows"), (dict(cols=0), "positive"), (dict(type=3), "type"), (dict(type=4), "type"), (dict(y_type=3), "type"), (dict(x_row=-1), "strides"),
                         (dict(residual_row=-1), "strides"), (dict(sum_row=-1), "strides"), (dict(y_row=-1), "strides"), (dict(sum_row=39), "overlap")]:
        _each(f, good_f, [(0, _rms(**change), word)])
        _each(b, good_b, [(0, _rms(**change), word)])
    assert room(_rms(rows=-1)) == 0 and room(_rms(y_type=4)) == 0 and room(None) == 0 and room(_rms(rows=0)) == 0
    needs = room(_rms())
    assert needs > 0
    _each(b, good_b, [(0, _rms(y_type=4), "type"), (8, None, "workspace"), (9, needs - 1, "workspace"), (8, V, "overlaps"), (8, U, "overlaps"), (8, P, "overlaps"),
                      (1, None, "NULL"), (3, None, "NULL"), (4, None, "NULL"), (6, None, "NULL"), (7, V + 2, "aligned"), (1, P + 1, "aligned"), (2, Q + 2, "aligned"),
                      (6, P, "overlaps"), (6, R + 4, "overlaps"), (6, Q + 160, "overlaps"), (7, T, "overlaps"), (7, S, "overlaps")])
    for eps in (-1.0, float("nan"), float("inf")):
        _each(f, good_f, [(0, _rms(eps=eps), "eps")])
    _each(f, good_f, [(0, None, "desc"), (0, _rms(y_row=39), "overlap"), (0, _rms(y_type=4), "NULL"), (1, None, "NULL"), (5, None, "NULL"), (1, P + 2, "aligned"),
                      (3, R + 2, "aligned"), (4, S + 1, "aligned"), (7, U + 1, "aligned"), (4, P, "overlaps"), (5, Q, "overlaps"), (4, Q + 160, "overlaps"),
                      (5, S, "overlaps"), (7, T, "overlaps"), (7, R, "overlaps")])
    codes = [_rms(y_type=4), P, Q, R, S, T, V, U, None]
    _each(f, codes, [(5, T + 8, "aligned"), (6, T + 511, "overlaps"), (6, P, "overlaps"), (4, T + 508, "overlaps")])
    # sum in place of residual only with its stride
    _each(f, good_f[:4] + [Q] + good_f[5:], [(0, _rms(sum_row=48), "overlaps")])
    _each(b, good_b[:6] + [Q] + good_b[7:], [(0, _rms(residual_row=48), "overlaps")])
    _refused(B.PATDNN_EUNSUPPORTED, "large", f, _rms(cols=2 ** 31 - 1, x_row=0, sum_row=2 ** 31, y_row=2 ** 31), *good_f[1:])
    _refused(B.PATDNN_EUNSUPPORTED, "large", f, _rms(rows=2 ** 31 - 1, cols=1000, sum_row=1000, y_row=1000), *good_f[1:])
    _refused(B.PATDNN_EUNSUPPORTED, "large", f, _rms(x_row=1 << 60), *good_f[1:])
    # backward: 64 threads for a column of a long row, in one grid
    wide = dict(rows=1, x_row=0, residual_row=0, sum_row=1 << 30, y_row=0)
    assert room(_rms(cols=2 ** 26 - 1024, **wide)) == 2 ** 26 - 1024 and room(_rms(cols=2 ** 26 - 1023, **wide)) == 0
    _refused(B.PATDNN_EUNSUPPORTED, "large", b, _rms(cols=2 ** 26 - 1023, **wide), *good_b[1:])
    _refused(B.PATDNN_EINVAL, "NULL", b, _rms(cols=2 ** 26 - 1024, **wide), None, *good_b[2:])
    _refused(B.PATDNN_EINVAL, "NULL", f, _rms(cols=2 ** 31 - 8321, **{**wide, "sum_row": 1 << 31}), None, *good_f[2:])
    _refused(B.PATDNN_EUNSUPPORTED, "large", f, _rms(cols=2 ** 31 - 8320, **{**wide, "sum_row": 1 << 31}), *good_f[1:])
    assert f(_rms(rows=0), None, None, None, None, None, None, None, None) == B.PATDNN_OK
    assert b(_rms(rows=0), None, None, None, None, None, None, None, None, 0, None) == B.PATDNN_OK


def _product(**change):
    d = dict(rows=3, in_features=200, out_features=20, w_blocks=0, out_type=0, act=0, dh_type=0, out_row=20, dh_row=20)
    d.update(change)
    return ctypes.byref(B.Fp8Desc(*(d[k] for k, _ in B.Fp8Desc._fields_)))


CALLS = {      # name: (good arguments, where x, x_scales, weights ..., the outputs, the workspace and its size are)
    "linear": ([P, P << 1, P << 2, P << 3, P << 4, P << 5], [0, 1, 2, 3], [5]),
    "gated": ([P, P << 1, P << 2, P << 3, P << 4, P << 5, P << 6, None], [0, 1, 2, 3, 4, 5], [6]),
    "gated_backward": ([P << i for i in range(9)], [0, 1, 2, 3, 4, 5, 6], [7, 8]),
}


@pytest.mark.parametrize("name", CALLS)
def test_products(name):
    f, room = getattr(L(), f"patdnn_fp8_{name}"), getattr(L(), f"patdnn_fp8_{name}_workspace_bytes")
    args, inputs, outputs = CALLS[name]
    big = P << 20
    tail = [big, 1 << 30, None]
    for change, word in [(dict(rows=-1), "rows"), (dict(in_features=0), "positive"), (dict(out_features=-3), "positive"), (dict(w_blocks=2), "blocks"), (dict(out_type=3), "type"),
                         (dict(act=3), "activation"), (dict(act=-1), "activation"), (dict(out_row=19), "overlap"), (dict(out_row=-1), "strides")]:
        _refused(B.PATDNN_EINVAL, word, f, _product(**change), *args, *tail)
        assert room(_product(**change)) == 0
    _refused(B.PATDNN_EINVAL, "desc", f, None, *args, *tail)
    for i in inputs + outputs:
        _refused(B.PATDNN_EINVAL, "NULL", f, _product(), *[None if j == i else v for j, v in enumerate(args)], *tail)
    for o in outputs:
        _refused(B.PATDNN_EINVAL, "aligned", f, _product(), *[v + 2 if j == o else v for j, v in enumerate(args)], *tail)
        for i in inputs:
            _refused(B.PATDNN_EINVAL, "overlaps", f, _product(), *[args[i] if j == o else v for j, v in enumerate(args)], *tail)
    _refused(B.PATDNN_EUNSUPPORTED, "large", f, _product(in_features=2 ** 31 - 1), *args, *tail)
    _refused(B.PATDNN_EUNSUPPORTED, "large", f, _product(out_features=2 ** 27, out_row=2 ** 27), *args, *tail)
    _refused(B.PATDNN_EUNSUPPORTED, "large", f, _product(rows=2 ** 31 - 1), *args, *tail)
    assert f(_product(rows=0), *[None] * len(args), None, 0, None) == B.PATDNN_OK and room(_product(rows=0)) == 0


def test_products_of_their_own_kind():
    args = CALLS["gated"][0]
    codes = [*args[:7], P << 9]
    needs = L().patdnn_fp8_gated_workspace_bytes(_product(out_type=4))
    f = L().patdnn_fp8_gated
    _refused(B.PATDNN_EINVAL, "NULL", f, _product(out_type=4), *args, P << 20, 1 << 30, None)
    _refused(B.PATDNN_EINVAL, "aligned", f, _product(out_type=4), *[v + 8 if i == 6 else v for i, v in enumerate(codes)], P << 20, 1 << 30, None)
    _refused(B.PATDNN_EINVAL, "overlaps", f, _product(out_type=4), *codes[:7], codes[6] + 3 * 128 - 1, P << 20, 1 << 30, None)
    if needs:
        _refused(B.PATDNN_EINVAL, "workspace", f, _product(out_type=4), *codes, P << 20, needs - 1, None)
        _refused(B.PATDNN_EINVAL, "workspace", f, _product(out_type=4), *codes, (P << 20) + 4, needs, None)
        _refused(B.PATDNN_EINVAL, "overlaps", f, _product(out_type=4), *codes, codes[0], needs, None)
    for name, word in (("linear", "type"), ("gated_backward", "type")):
        _refused(B.PATDNN_EINVAL, word, getattr(L(), f"patdnn_fp8_{name}"), _product(out_type=4), *CALLS[name][0], P << 20, 1 << 30, None)
    b = CALLS["gated_backward"][0]
    _refused(B.PATDNN_EINVAL, "type", L().patdnn_fp8_gated_backward, _product(dh_type=4), *b, P << 20, 1 << 30, None)
    _refused(B.PATDNN_EINVAL, "strides", L().patdnn_fp8_gated_backward, _product(dh_row=-1), *b, P << 20, 1 << 30, None)
    # slices of one wider tensor beside each other, and over each other
    wide = _product(out_row=40)
    _refused(B.PATDNN_EINVAL, "overlaps", L().patdnn_fp8_gated_backward, wide, *b[:7], b[7], b[7] + 19 * 4, P << 20, 1 << 30, None)


def test_the_binding_refuses():
    import torch
    x = torch.zeros(4, 128)
    b = torch.zeros(4, 128, dtype=torch.uint8)
    s = torch.zeros(4, 1, dtype=torch.uint8)
    for call in (lambda: B.patdnn_fp8_quantize(x), lambda: B.patdnn_fp8_dequantize(b, s, 128), lambda: B.patdnn_rms_norm(x), lambda: B.patdnn_rms_norm_backward(x, x, x[:, 0]),
                 lambda: B.patdnn_fp8_linear(b, s, b, s), lambda: B.patdnn_fp8_gated(b, s, b, s, b, s), lambda: B.patdnn_fp8_gated_backward(x, b, s, b, s, b, s)):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError, match="blocks"):
        B.patdnn_fp8_quantize(x, blocks="columns")
