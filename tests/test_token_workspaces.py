"""The workspace queries of the token operators over all sizes, on the CPU."""
import pytest

from paper_2108_02416_amd import aspis

NONE = 2 ** 64 - 1
LONGEST = 1 << 30      # rows of a call, and tokens


@pytest.mark.parametrize("rows,vocab", [(LONGEST + 1, 4), (LONGEST + 1, 0), (1 << 60, 1), (1 << 60, 0),
                                        ((1 << 63) - 1, 0), ((1 << 63) - 1, 1), (1 << 59, 2)])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_more_rows_than_a_call_takes(rows, vocab, kind):
    """(Their bytes, 24 a row and more, pass 64 bits.)"""
    assert aspis.lib().aspis_policy_workspace(rows, vocab, kind) == NONE


@pytest.mark.parametrize("rows", [0, 1, 127, 128, 8192, 8193, 300_000, LONGEST])
@pytest.mark.parametrize("vocab", [0, 1, 257, 131_072, 131_073, 1 << 24])
@pytest.mark.parametrize("kind", [0, 1])
def test_the_workspace_holds_a_rows_terms_and_units(rows, vocab, kind):
    """Three fp64 terms, a logit and 8 bytes a unit, at least one of 64 lanes of
    8 vectors; no more than one for every vector of 64 lanes."""
    got = aspis.lib().aspis_policy_workspace(rows, vocab, kind)
    vecs = (vocab * (2 if kind else 4) + 15) // 16
    low, high = (vecs + 511) // 512, max(vecs // 16, 64)
    assert rows * (24 + 4 + 8 * max(low, 1)) <= got <= rows * (28 + 8 * high) + 64 * 24 + 16
    assert got % 16 == 0


def test_bytes_of_the_embedding_gradient():
    for n in (0, 1, 768, 16_384, 16_385, LONGEST):
        for d in (0, 1, 4096):
            got = aspis.lib().aspis_embed_workspace(n, d)
            assert 16 * n <= got < 16 * (n + 16) + 64 + 4 * (d + 4) * (n / 8 + 2)
