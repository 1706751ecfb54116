"""The shapes by which the products with a scale per 128 are tested reach every kernel, and the choice gives only kernels that
there are. Nothing here needs a GPU."""
import random

import pytest

from .gemm128_shapes import CODES, GATED, PLAIN, choice, flat

FEW = {("few", nt, split) for nt in (16, 32, 64, 128) for split in (1, 2, 4, 8)}
KINDS = {"plain": (PLAIN, FEW | {("many", 128, 1), ("many", 192, 1), ("many", 256, 1)}, {}),
         "gated": (GATED, FEW | {("many", 128, 1), ("many", 256, 1)}, dict(gated=True)),
         "codes": (CODES, FEW | {("many", 256, 1)}, dict(gated=True, codes=True))}


@pytest.mark.parametrize("kind", KINDS)
def test_every_kernel_has_its_shapes(kind):
    table, kernels, how = KINDS[kind]
    assert set(table) == kernels
    wrong = {s: choice(*s[3:], **how) for s in flat(table) if choice(*s[3:], **how) != s[:3]}
    assert not wrong, wrong


@pytest.mark.parametrize("kind", KINDS)
def test_the_shapes_end_inside_tiles_and_blocks(kind):
    for kernel, nt, split, rows, k, n in flat(KINDS[kind][0]):
        assert rows % (nt if kernel == "few" else 256) and k % 128 and n % 128, (nt, split, rows, k, n)


@pytest.mark.parametrize("kind", KINDS)
def test_the_choice_gives_what_is_there(kind):
    """Over all sizes, the largest among them: a kernel that is built, clusters that have a block each, grids that fit."""
    _, kernels, how = KINDS[kind]
    rng = random.Random(5)
    size = lambda lo, hi: min(hi, int(lo * 2 ** rng.uniform(0, (hi // lo).bit_length())))  # noqa: E731
    for _ in range(20000):
        rows, k, n = size(1, 1 << 30), 16 * size(1, 1 << 26), 16 * size(1, 1 << 26)
        if rows * n >= 1 << 44:
            continue
        kernel, nt, split = choice(rows, k, n, num_sms=rng.choice((152, 148, 132, 2)), **how)
        assert (kernel, nt, split) in kernels
        assert split <= -(-k // 128)
        if kernel == "few":
            assert -(-rows // nt) <= 65535 and -(-n // 128) * split < 1 << 31
        else:
            assert -(-rows // 256) * -(-n // (nt // (2 if how else 1))) <= 0x7fffffff // 2
