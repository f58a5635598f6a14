"""How attention's weights are held between its two products, by the kernel that a call's prefix goes through.

Two numbers of the values' type leave 2 (eps / 2)^2 of a weight; where a prefix of many rows goes through tensor memory they are rounded once, eps / 2.
Which of the two it is is asked of the library (a limit of no polls makes the tensor-memory kernel, and no other, give up), and the
tolerance follows it, so that losing the second numbers where they are promised is seen."""
import pytest

from test_gpu_attention import Case, serving, torch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def by_tensor_memory(torch, plan, c):  # noqa: F811
    from paper_2609_09800_b200 import hbf
    waits = hbf.lib().hbf_debug_operator_waits
    waits(0)
    try:
        out = plan(c.q)
        torch.cuda.synchronize()
    finally:
        waits(-1)
    gone = torch.isnan(out)
    assert gone.all() or not gone.any()
    return bool(gone.all())


def check(torch, c, out, lse, once):  # noqa: F811
    want, want_lse, A, S = c.expect()
    half = torch.finfo(c.dt).eps / 2
    rel = (half if once else 2 * half * half) + 2 * (c.d + 8) * 2.0 ** -23 * S + 2.0 ** -18          # (as tests/test_gpu_attention.py has it)
    tol = half * want.abs() + (1 + half) * A * rel[..., None] + torch.finfo(c.dt).tiny
    err = (out.double() - want).abs()
    assert torch.isfinite(out).all() and (err <= tol).all(), "off by %g of the tolerance" % float((err / tol).max())
    assert ((lse.double() - want_lse).abs() <= (c.d + 8) * 2.0 ** -23 * S + 2.0 ** -18 + 2.0 ** -22 * want_lse.abs()).all()


# B, Hq, Hk, d, page, prefix, own, and whether the prefix is through tensor memory.  There: heads a group of which a tile of 128 rows ends inside a
# request (5, 3, 7, 24), pages of 100 and 40 with them, a last tile of few rows, and one tile in the last pair
SHAPES = [
    (130, 40, 8, 64, 100, 1000, 11, True), (103, 40, 8, 128, 16, 515, 9, True), (90, 15, 5, 128, 40, 4000, 20, True), (201, 21, 3, 64, 24, 3001, 0, True),
    (29, 96, 4, 128, 100, 2100, 33, True), (129, 5, 1, 128, 16, 9000, 5, True), (257, 32, 32, 64, 16, 400, 3, True),
    (16, 32, 4, 128, 16, 200, 40, False), (33, 8, 1, 64, 16, 1111, 20, False), (64, 32, 4, 128, 16, 500, 90, False), (17, 10, 2, 64, 12, 777, 33, False),
    (40, 7, 7, 128, 16, 130, 9, False), (120, 40, 8, 64, 100, 300, 11, False), (5, 40, 2, 128, 100, 900, 40, False),
]


@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s[:7])) for s in SHAPES])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_against_64_bits_by_path(torch, serving, shape, dtype):  # noqa: F811
    *sizes, tensor_memory = shape
    c = Case(torch, *sizes, dtype=dtype, seed=sum(sizes))
    plan = c.plan(serving)
    once = by_tensor_memory(torch, plan, c)
    assert once == tensor_memory
    lse = torch.empty(c.B, c.Hq, device="cuda")
    check(torch, c, plan(c.q, lse=lse), lse, once)


@pytest.mark.parametrize("sharp", [1.0, 4.0, 12.0])
@pytest.mark.parametrize("shape", [(128, 32, 4, 128, 16, 640, 0), (101, 32, 4, 128, 12, 2000, 9), (1216, 64, 8, 64, 16, 300, 0), (3, 32, 4, 128, 16, 900, 40), (40, 8, 2, 64, 16, 300, 30)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_equal_values(torch, serving, shape, dtype, sharp):  # noqa: F811
    """sum w v / sum w with one v for all keys.  With two numbers a weight that is v to the bit: 2^-16 of it (bf16; 2^-22 fp16) and the 32-bit sums of at most
    2,012 weights move it by far less than the half step, 2^-9 (2^-12) at least, that would round to another value.  With weights rounded once, eps / 2
    of v, and the output's rounding of what then comes."""
    c = Case(torch, *shape, dtype=dtype, seed=sum(shape), poison=False, k_scale=sharp)
    c.v[:] = c.v[0, 0]
    plan = c.plan(serving)
    want = c.v[0, 0].repeat_interleave(c.Hq // c.Hk, 0).expand(c.q.shape)
    out = plan(c.q)
    if by_tensor_memory(torch, plan, c):
        half = torch.finfo(c.dt).eps / 2
        assert ((out.double() - want.double()).abs() <= want.double().abs() * (half + (1 + half) * (half + 2.0 ** -18)) + torch.finfo(c.dt).tiny).all()
    else:
        assert torch.equal(out, want)
