"""What the entry points say about how exact the gated block's backward pass is.  Host only."""
import pytest

from test_int8_gated_host import Matrix, gvq, made  # noqa: F401  (fixtures)

ROUNDED, PRECISE = 0x100, 0x200


def test_workspaces(gvq):      # noqa: F811
    need = gvq.lib().gvq_gated_workspace_bytes
    for M, F, K in ((1, 1, 1), (300, 333, 165), (1024, 256, 256), (1024, 256, 257), (1300, 1029, 520), (8192, 8192, 4096)):
        by_size, rounded, precise = (need(M, F, K, 1 | mode, 1) for mode in (0, ROUNDED, PRECISE))
        assert by_size == (precise if M * F * K <= 2 ** 26 else rounded)
        assert precise - rounded == 2 * (-(-(M * -(-F // 8) * 16) // 256) * 256)
        assert need(M, F, K, 1 | ROUNDED | PRECISE, 1) == -1
        for mode in (ROUNDED, PRECISE):      # one that is enough for every smaller call
            assert need(M, F, K, 1 | mode, 1) <= need(M + 1, F, K, 1 | mode, 1) and need(M, F, K, 1 | mode, 1) <= need(M, F, K + 1, 1 | mode, 1)
            assert need(M, F, K, 1 | mode, 0) == need(M, F, K, 1 | mode, 1) + need(M, F, K, 0, 0)


def test_arguments(made):      # noqa: F811
    ctx, fake = made
    M, F, K = 10, 24, 16
    x, w, h = Matrix(M, K), Matrix(F, K), Matrix(M, F)
    asked = []
    fake.gvq_gated_workspace_bytes = lambda *a: asked.append(a) or 4096
    for precise, mode in ((None, 0), (False, ROUNDED), (True, PRECISE)):
        ctx.gated_backward(h, h, h, x, w, w, act="gelu", dx=x, precise=precise)
        assert fake.calls[-1][0] == "gvq_gated_backward" and fake.calls[-1][1][17] == 1 | mode and asked[-1][3] == 1 | mode
    n = len(fake.names())
    for precise in ("yes", 2, 0.5):
        with pytest.raises(ValueError):
            ctx.gated_backward(h, h, h, x, w, w, dx=x, precise=precise)
    with pytest.raises(ValueError):
        ctx.gated_backward(h, h, h, x, w, w, act="none", dx=x, precise=True)
    assert len(fake.names()) == n
