"""gan_combine_rows_backward on the host: `out` is what dweight is made of, and asked for with it alone; without either result nothing is launched."""
import pytest

from paper_2102_10485_amd import binding as B

P = 1 << 20                                                         # an address that no refused call touches
OK = dict(precision=B.BF16, dy=P, dy_stride=64, out=P, out_stride=64, place=P, weight=P, offs=P, groups=4, k=2, rows=10, cols=64, dout=P, dout_stride=64, dweight=P)


def call(**change):
    B.combine_rows_backward(**{**OK, **change})


def test_out_goes_with_dweight():
    for change in (dict(out=0), dict(out=0, dout=0)):
        with pytest.raises(B.GanError) as e:
            call(**change)
        assert e.value.status == B.GAN_E_ARG and "out" in str(e.value) and "NULL" in str(e.value)


def test_neither_result():
    call(dout=0, dweight=0)
    call(out=0, dout=0, dweight=0)
    call(out=0, dout=0, dweight=0, rows=0, dy=0, place=0)
    for change, word in ((dict(dy=0), "NULL"), (dict(place=0), "NULL"), (dict(offs=0), "NULL"), (dict(dy_stride=63), "dy_stride"), (dict(out_stride=63), "out_stride")):
        with pytest.raises(B.GanError) as e:
            call(**{**dict(dout=0, dweight=0), **change})
        assert e.value.status == B.GAN_E_ARG and word in str(e.value)
