"""4-bit and 8-bit matrices have the same attributes and are of different sizes: either is refused where the other is wanted, before
anything reaches the library.  Host only: the library is a stand-in, and no pointer is followed."""
import pytest

from test_int8_gated_host import F32, Matrix, gvq, made  # noqa: F401  (fixtures)


def _made(kind, rows, cols):
    q = object.__new__(kind)
    q.rows, q.cols, q.device, q.codes_ptr, q.scales_ptr = rows, cols, 0, 256, 512
    return q


def test_a_matrix_of_the_other_format_is_refused(made):      # noqa: F811
    from paper_1811_03617_b200.gvq import I8, Mx4
    ctx, fake = made
    x, out, back = Matrix(100, 128), Matrix(100, 70, F32), Matrix(100, 128, F32)
    for mine, other, what in ((I8, Mx4, "i8"), (Mx4, I8, "mx4")):
        def call(name):
            return getattr(ctx, f"{what}_{name}")
        a, b, a4, b4 = _made(mine, 100, 128), _made(mine, 70, 128), _made(other, 100, 128), _made(other, 70, 128)
        call("quantize")(x, out=a)
        call("quantize_both")(x, out=a, out_t=_made(mine, 128, 100))
        call("dequantize")(a, back)
        call("matmul")(a, b, out)
        calls = [lambda: call("quantize")(x, out=a4), lambda: call("quantize_transposed")(x, out=_made(other, 128, 100)),
                 lambda: call("quantize_both")(x, out=a, out_t=_made(other, 128, 100)), lambda: call("quantize_both")(x, out=a4, out_t=_made(mine, 128, 100)),
                 lambda: call("dequantize")(a4, back), lambda: call("dequantize")(a4), lambda: call("matmul")(a4, b, out), lambda: call("matmul")(a, b4, out)]
        if what == "i8":
            call("gated")(a, b, b, out)
            calls += [lambda: call("gated")(a4, b, b, out), lambda: call("gated")(a, b4, b, out), lambda: call("gated")(a, b, b4, out)]
        n = len(fake.names())
        for refused in calls:
            with pytest.raises(TypeError):
                refused()
        assert len(fake.names()) == n


def test_slices_of_the_exchange_are_4_bit_matrices(made):      # noqa: F811
    from paper_1811_03617_b200.gvq import I8, Mx4
    ctx, _ = made
    ctx.S, ctx.d = 100, 16
    assert ctx._slices([_made(Mx4, 100, 16)], 1, "exchange")
    with pytest.raises(TypeError):
        ctx._slices([_made(I8, 100, 16)], 1, "exchange")
