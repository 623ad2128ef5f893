"""What the operators of a layer of experts refuse, on the host, before anything is launched; and their sizes."""
import pytest

from paper_2102_10485_amd import binding as B

P = 1 << 20                                                         # an address that no refused call touches


def refused(call, status, word):
    with pytest.raises(B.GanError) as e:
        call()
    assert e.value.status == status and word in str(e.value), str(e.value)


def each(call, ok, changes):
    for change, status, word in changes:
        refused(lambda: call(**{**ok, **change}), status, word)


ARG, SHAPE = B.GAN_E_ARG, B.GAN_E_SHAPE


def test_linear_act():
    ok = dict(precision=B.BF16, x=P, x_stride=64, w=P, offs=P, groups=4, rows=10, n_in=64, n_out=32, bias=P, act=B.ACT_GELU, residual=P, residual_stride=32, z=P, z_stride=32,
              y=P, y_stride=32)
    each(B.group_linear_act, ok, [(dict(precision=2), ARG, "precision"), (dict(x=0), ARG, "NULL"), (dict(y=0), ARG, "NULL"), (dict(w=0), ARG, "NULL"), (dict(offs=0), ARG, "NULL"),
                                  (dict(x_stride=63), ARG, "x_stride"), (dict(y_stride=31), ARG, "y_stride"), (dict(residual_stride=31), ARG, "residual_stride"),
                                  (dict(z_stride=31), ARG, "z_stride"), (dict(act=4), ARG, "activation"), (dict(act=-1), ARG, "activation"), (dict(rows=-1), ARG, "negative"),
                                  (dict(n_in=0), ARG, "inputs"), (dict(groups=65536), SHAPE, "65535"), (dict(rows=(1 << 30) + 1), SHAPE, "2^30")])
    B.group_linear_act(**{**ok, "rows": 0, "x": 0, "y": 0})
    ok = dict(precision=B.FP32, dy=P, dy_stride=32, w=P, offs=P, groups=4, rows=10, n_in=64, n_out=32, other=P, other_stride=64, act=B.ACT_SILU, z=P, z_stride=64, dx=P,
              dx_stride=64)
    each(B.group_linear_dgrad_act, ok, [(dict(dy=0), ARG, "NULL"), (dict(dx=0), ARG, "NULL"), (dict(z=0), ARG, "z is NULL"), (dict(z_stride=63), ARG, "z_stride"),
                                        (dict(other_stride=63), ARG, "other_stride"), (dict(dy_stride=31), ARG, "dy_stride"), (dict(dx_stride=63), ARG, "dx_stride"),
                                        (dict(act=9), ARG, "activation"), (dict(groups=-1), ARG, "negative")])
    B.group_linear_dgrad_act(**{**ok, "rows": 0, "z": 0})
    ok = dict(x8=P, x_scale=P, w8=P, w_scale=P, offs=P, groups=4, rows=10, n_in=100, n_out=64, bias=0, act=B.ACT_RELU, residual=P, residual_stride=64, y_precision=B.BF16, y=P,
              y_stride=64)
    each(B.group_linear8_act, ok, [(dict(x_scale=0), ARG, "NULL"), (dict(w_scale=0), ARG, "NULL"), (dict(x8=P + 8), ARG, "aligned"), (dict(w8=P + 8), ARG, "aligned"),
                                   (dict(y_stride=63), ARG, "y_stride"), (dict(residual_stride=0), ARG, "residual_stride"), (dict(y_precision=7), ARG, "precision"),
                                   (dict(act=5), ARG, "activation"), (dict(n_in=(1 << 22) + 1), SHAPE, "2^22")])


def test_act_backward():
    ok = dict(precision=B.BF16, dy=P, dy_stride=32, act=B.ACT_GELU, z=P, z_stride=32, offs=P, groups=4, rows=1000, cols=32, dz=P, dz_stride=32, dbias=P, work=P,
              work_bytes=B.group_act_backward_bytes(4, 1000, 32))
    each(B.group_act_backward, ok, [(dict(precision=3), ARG, "precision"), (dict(act=4), ARG, "activation"), (dict(dy=0), ARG, "NULL"), (dict(z=0), ARG, "NULL"),
                                    (dict(offs=0), ARG, "NULL"), (dict(dy_stride=31), ARG, "dy_stride"), (dict(z_stride=31), ARG, "z_stride"), (dict(dz_stride=31), ARG, "dz_stride"),
                                    (dict(work=0), ARG, "work"), (dict(work_bytes=4), ARG, "work"), (dict(work=P + 4), ARG, "work"), (dict(groups=-1), ARG, "negative"),
                                    (dict(groups=65536), SHAPE, "65535"), (dict(cols=0), ARG, "columns"), (dict(rows=1 << 31), SHAPE, "2^30")])
    assert B.group_act_backward_bytes(4, 0, 32) == 0 and B.group_act_backward_bytes(0, 4, 32) == 0 and B.group_act_backward_bytes(1, 512, 32) == 0 and B.group_act_backward_bytes(1, 513, 32) > 0
    B.group_act_backward(**{**ok, "dz": 0, "dbias": 0, "rows": 0})


def test_route():
    ok = dict(precision=B.BF16, logits=P, logits_stride=64, rows=10, experts=64, k=2, normalize=1, expert=P, weight=P, counts=P, mean=P, balance=P, work=P,
              work_bytes=B.route_bytes(10, 64))
    each(B.route, ok, [(dict(precision=2), ARG, "precision"), (dict(logits=0), ARG, "NULL"), (dict(expert=0), ARG, "NULL"), (dict(k=0), ARG, "k is"), (dict(k=65), ARG, "k is"),
                       (dict(logits_stride=63), ARG, "stride"), (dict(rows=-1), ARG, "negative"), (dict(experts=0), ARG, "columns"), (dict(counts=0), ARG, "counts"),
                       (dict(work=0, rows=500), ARG, "work"), (dict(work_bytes=0, rows=500), ARG, "work"), (dict(work=P + 8), ARG, "work"), (dict(k=17), SHAPE, "16 choices"),
                       (dict(experts=4097, logits_stride=4097), SHAPE, "4096"), (dict(rows=1 << 30), SHAPE, "2^30")])
    B.route(**{**ok, "rows": 0, "counts": 0, "mean": 0, "balance": 0})
    ok = dict(precision=B.BF16, logits=P, logits_stride=64, rows=10, experts=64, k=2, normalize=1, expert=P, dweight=P, counts=P, balance_grad=0.1, dlogits=P, dlogits_stride=64)
    each(B.route_backward, ok, [(dict(logits=0), ARG, "NULL"), (dict(dlogits=0), ARG, "NULL"), (dict(expert=0), ARG, "NULL"), (dict(dlogits_stride=63), ARG, "stride"),
                                (dict(logits_stride=1), ARG, "stride"), (dict(k=65), ARG, "k is")])
    B.route_backward(**{**ok, "rows": 0})
    assert B.route_bytes(0, 5) == 0 and B.route_bytes(1, 5) == 0 and B.route_bytes(5000, 5) > 0 and B.route_bytes(5, 5000) == 0


def test_rows():
    ok = dict(labels=P, n=5000, groups=10, offs=P, order=P, place=P, work=P, work_bytes=B.sort_by_label_bytes(5000, 10))
    each(B.sort_by_label, ok, [(dict(n=-1), ARG, "negative"), (dict(groups=-1), ARG, "negative"), (dict(labels=0), ARG, "NULL"), (dict(offs=0), ARG, "NULL"),
                               (dict(work=0), ARG, "work"), (dict(work_bytes=8), ARG, "work"), (dict(work=P + 4), ARG, "work"), (dict(groups=4097), SHAPE, "4096"),
                               (dict(n=(1 << 30) + 1), SHAPE, "2^30")])
    assert B.sort_by_label_bytes(100, 10) == 0 and B.sort_by_label_bytes(-1, 10) == 0 and B.sort_by_label_bytes(5000, 5000) == 0
    ok = dict(precision=B.BF16, x=P, x_stride=64, place=P, offs=P, groups=4, k=2, rows=10, cols=64, out=P, out_stride=64)
    both = [(dict(precision=2), ARG, "precision"), (dict(place=0), ARG, "NULL"), (dict(offs=0), ARG, "NULL"), (dict(out=0), ARG, "NULL"), (dict(out_stride=63), ARG, "out_stride"),
            (dict(k=0), ARG, "choices"), (dict(groups=-1), ARG, "negative"), (dict(groups=65536), SHAPE, "65535"), (dict(rows=1 << 30), SHAPE, "2^30"), (dict(rows=-1), ARG, "negative"),
            (dict(cols=0), ARG, "columns")]
    each(B.gather_rows, ok, both + [(dict(x=0), ARG, "NULL"), (dict(x_stride=63), ARG, "x_stride")])
    B.gather_rows(**{**ok, "rows": 0, "x": 0, "out": 0})
    ok = dict(precision=B.BF16, out=P, out_stride=64, place=P, weight=P, offs=P, groups=4, k=2, residual=P, residual_stride=64, rows=10, cols=64, y=P, y_stride=64)
    each(B.combine_rows, ok, both + [(dict(y=0), ARG, "NULL"), (dict(y_stride=63), ARG, "y_stride"), (dict(residual_stride=63), ARG, "residual_stride")])
    B.combine_rows(**{**ok, "rows": 0})
    ok = dict(precision=B.BF16, dy=P, dy_stride=64, out=P, out_stride=64, place=P, weight=P, offs=P, groups=4, k=2, rows=10, cols=64, dout=P, dout_stride=64, dweight=P)
    each(B.combine_rows_backward, ok, both + [(dict(dy=0), ARG, "NULL"), (dict(dy_stride=63), ARG, "dy_stride"), (dict(dout_stride=63), ARG, "dout_stride")])
    B.combine_rows_backward(**{**ok, "rows": 0})


def test_dropout():
    ok = dict(precision=B.BF16, x=P, x_stride=64, residual=P, residual_stride=64, rows=10, cols=64, p=0.1, seed=1, site=0, step=0, step_device=0, y=P, y_stride=64)
    each(B.dropout, ok, [(dict(precision=2), ARG, "precision"), (dict(x=0), ARG, "NULL"), (dict(y=0), ARG, "NULL"), (dict(p=1.0), ARG, "p is"), (dict(p=-0.1), ARG, "p is"),
                         (dict(p=float("nan")), ARG, "p is"), (dict(p=1 - 2.0 ** -18), ARG, "2^-16"), (dict(x_stride=63), ARG, "x_stride"),
                         (dict(residual_stride=63), ARG, "residual_stride"), (dict(y_stride=63), ARG, "y_stride"), (dict(rows=(1 << 30) + 1), SHAPE, "2^30"), (dict(cols=0), ARG, "columns")])
    B.dropout(**{**ok, "rows": 0, "x": 0, "y": 0})
