"""CPU-only: the sets of the tile tests reach every tile width of every product."""
import pytest

from muon_sets import ONE_WORD_PAIRS, ONE_WORD_SINGLES, TWO_WORDS, shapes_of
from paper_2605_16341_amd import binding as b


def tiles(groups, dtype, precision, step):
    h = b.orthdion_muon_create(shapes_of(groups), dtype, dtype, precision=precision)
    got = b.orthdion_muon_get_tiles(h, step)
    b.orthdion_muon_destroy(h)
    return got


def reached(sets, dtype, precision):
    """{kind of product: {tile: smallest remainder a dimension of its sets leaves}}"""
    got = {}
    for groups in sets:
        for step in (False, True):
            for kind, widths in tiles(groups, dtype, precision, step).items():
                for w in widths:
                    rest = min(d % w for _, m, n in groups for d in (m, n))
                    got.setdefault(kind, {}).setdefault(w, []).append(rest)
    return got


@pytest.mark.parametrize("sets,dtype,precision,widths", [(ONE_WORD_SINGLES + [s for pair in ONE_WORD_PAIRS for s in pair], b.ORTHDION_BF16, b.ORTHDION_PREC_FAST, (64, 128, 192, 256)),
                                                         (TWO_WORDS, b.ORTHDION_F32, b.ORTHDION_PREC_EXACT, (64, 128, 256))])
def test_every_tile_of_every_product_is_reached_with_remainders(sets, dtype, precision, widths):
    got = reached(sets, dtype, precision)
    assert set(got) == set(b.MUON_PRODUCTS)
    for kind in b.MUON_PRODUCTS:
        assert set(got[kind]) == set(widths), (kind, got[kind])
        assert all(min(rests) > 0 for rests in got[kind].values())


@pytest.mark.parametrize("pair", ONE_WORD_PAIRS, ids=lambda p: str(p[0]))
def test_pairs_of_sets_differ_in_their_tiles(pair):
    first, second = (tiles(groups, b.ORTHDION_BF16, b.ORTHDION_PREC_FAST, False) for groups in pair)
    assert set(first) == set(second) and any(first[kind].isdisjoint(second[kind]) for kind in first)


def test_refusals():
    h = b.orthdion_muon_create([(64, 64)], b.ORTHDION_BF16, b.ORTHDION_BF16)
    assert b.load().orthdion_muon_get_tiles(None, 0, None) == b.ORTHDION_E_NULL_PTR
    assert b.load().orthdion_muon_get_tiles(h, 0, None) == b.ORTHDION_E_NULL_PTR
    for step in (-1, 2):
        with pytest.raises(b.OrthDionError) as e:
            b.orthdion_muon_get_tiles(h, step)
        assert e.value.status == b.ORTHDION_E_INVALID_ARG
    # small matrices have no p x p products but those of their own kernel
    assert set(b.orthdion_muon_get_tiles(h, 0)) == {"apply", "last_wide"}
    b.orthdion_muon_destroy(h)
