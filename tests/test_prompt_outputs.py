"""tkv_prompt_attn refuses outputs whose rows overlap and a reserved field that is not 0, before any GPU work (no GPU needed)."""
import pytest

from test_prompt_refusals import L, _call  # noqa: F401  (the library, a call on addresses that are never read)

TEN = ((0, 5), (5, 5), (0, 5), (5, 5))    # tokens 0 to 9
ONE = ((0, 3), (0, 1), (0, 5), (5, 5))    # token 3
TWO = ((0, 9), (1, 1), (0, 5), (5, 5))    # tokens 0 and 9


@pytest.mark.parametrize("lens,heads,stride", [
    (TEN, 32, (0, 128)), (TEN, 32, (4096, 0)), (TEN, 32, (0, 0)), (TEN, 32, (64, 4096)), (TEN, 32, (4096, 64)), (TEN, 32, (128, 128)),
    (TEN, 32, (2048, 128)), (TEN, 32, (4088, 128)), (TEN, 32, (384, 256)), (TEN, 32, (128, 1272)), (TEN, 1, (120, 0)), (TEN, 1, (0, 128)),
    (ONE, 32, (4096, 120)), (TWO, 1, (8, 0)), (TWO, 2, (128, 1216)), (TEN, 3, (640, 648)),
])
def test_rows_of_the_output_that_overlap(L, lens, heads, stride):  # noqa: F811
    assert _call(L, lens=lens, n_q_heads=heads, n_kv_heads=1, o_stride=stride, ws=16) == -1


@pytest.mark.parametrize("lens,heads,stride", [
    (TEN, 32, (4096, 128)), (TEN, 32, (4096 + 8, 128)), (TEN, 32, (128, 1280)), (TEN, 32, (256, 10 * 256 + 8)), (TEN, 8, (4096, 512)),
    (TEN, 3, (384, 256 + 384 * 10)), (TEN, 2, (256, 128)), (TEN, 2, (256, 384)), (TEN, 2, (256, 256 * 9 + 128)),
    (ONE, 32, (0, 128)), (TEN, 1, (128, 0)), (((0, 0), (0, 0), (0, 5), (5, 5)), 32, (0, 0)),
])
def test_rows_that_lie_apart_are_accepted(L, lens, heads, stride):  # noqa: F811
    """(Such a call then asks for its workspace, too small here.)"""
    assert _call(L, lens=lens, n_q_heads=heads, n_kv_heads=1, o_stride=stride, ws=16) == -4


def test_rows_apart_as_counted_one_by_one(L):  # noqa: F811
    """Against every pair of rows, for strides drawn at random."""
    import random
    rng, seen = random.Random(1), set()
    for _ in range(400):
        heads, n = rng.randint(1, 5), rng.randint(1, 6)
        st, sh = (8 * rng.randint(0, rng.choice((20, 60, 120))) for _ in range(2))
        at = sorted(t * st + h * sh for t in range(n) for h in range(heads))
        apart = all(b - a >= 128 for a, b in zip(at, at[1:]))
        lens = ((0, n - 1), (n - 1, 1), (0, 5), (5, 5))
        assert _call(L, lens=lens, n_q_heads=heads, n_kv_heads=1, o_stride=(st, sh), ws=16) == (-4 if apart else -1), (heads, n, st, sh)
        seen.add(apart)
    assert seen == {True, False}

def test_reserved(L):  # noqa: F811
    assert _call(L, reserved=1, ws=16) == -1
