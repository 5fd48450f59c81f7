"""A norm's output in place of an input keeps the input's rows: another row stride would
overwrite rows that are not read yet, and is refused (no GPU needed)."""
import pytest

from test_linear8_host import GRAD, NORM, P, ctx  # noqa: F401

Q = P + (1 << 16)  # another fake device address: never dereferenced


@pytest.mark.parametrize("bad", [dict(h=P, ldh=512), dict(x=Q, r=P, ldr=256, h=P, ldh=512), dict(ldx=512, h=P, ldh=256)])
def test_rmsnorm8(ctx, bad):
    L, h = ctx
    assert L.jagg_rmsnorm8(h, *{**NORM, **bad}.values()) == 1 and b"in place" in L.jagg_last_error()


@pytest.mark.parametrize("bad", [dict(lddx=512), dict(lddy=512), dict(dy=Q, dh=P, lddh=512), dict(dy=Q, dh=P, lddh=256, lddx=257)])
def test_rmsnorm8_grad(ctx, bad):
    L, h = ctx
    assert L.jagg_rmsnorm8_grad(h, *{**GRAD, **bad}.values()) == 1 and b"in place" in L.jagg_last_error()
