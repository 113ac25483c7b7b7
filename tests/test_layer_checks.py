"""What the MoE layer's constructor refuses before it makes a context or a buffer."""
import pytest

from paper_2508_12801_b200 import binding as ms
from paper_2508_12801_b200.layer import MoELayer


class Made(Exception):
    pass


@pytest.fixture(autouse=True)
def no_context(monkeypatch):
    def create(params, device):
        raise Made
    monkeypatch.setattr(ms, "create", create)


def make(d, f, io=ms.BF16, **form):
    return MoELayer(ms.make_params(16, d, 4, 2, io_dtype=io), f, **form)


SERVE = dict(int8=True, training=False)


@pytest.mark.parametrize("d, f, io, form, bad", [
    (72, 64, ms.BF16, SERVE, "d_model"), (64, 1000, ms.BF16, SERVE, "d_ff"), (64, 8, ms.BF16, SERVE, "d_ff"), (64, 0, ms.BF16, SERVE, "d_ff"),
    (64, -16, ms.BF16, SERVE, "d_ff"), (64, 1 << 17, ms.BF16, SERVE, "d_ff"), (1 << 17, 64, ms.BF16, SERVE, "d_model"),
    (64, 36, ms.BF16, dict(keep8=True), "d_ff"), (60, 64, ms.BF16, {}, "d_model"), (64, (1 << 17) + 8, ms.BF16, {}, "d_ff"),
    (64, (1 << 18) + 8, ms.BF16, dict(training=False), "d_ff"), (64, 100, ms.BF16, dict(training=False), "d_ff"),
    (64, 30, ms.F32, {}, "d_ff"), (30, 32, ms.F32, {}, "d_model")])
def test_widths(d, f, io, form, bad):
    with pytest.raises(ValueError, match=bad):
        make(d, f, io, **form)


@pytest.mark.parametrize("d, f, io, form", [
    (64, 48, ms.BF16, SERVE), (16, 16, ms.BF16, SERVE), (64, (1 << 17) - 16, ms.BF16, SERVE), (72, 1000, ms.BF16, {}), (72, 1000, ms.BF16, dict(keep8=True)),
    (72, 1000, ms.BF16, dict(training=False)), (36, 20, ms.F32, {}), (64, 1 << 17, ms.BF16, {}), (64, 1 << 18, ms.BF16, dict(training=False))])
def test_widths_that_are_served(d, f, io, form):
    with pytest.raises(Made):
        make(d, f, io, **form)


@pytest.mark.parametrize("io, form, why", [(ms.F32, SERVE, "bf16"), (ms.F32, dict(keep8=True), "bf16"), (ms.BF16, dict(int8=True), "training"),
                                           (ms.BF16, dict(keep8=True, training=False), "training")])
def test_forms(io, form, why):
    with pytest.raises(ValueError, match=why):
        make(64, 64, io, **form)
