"""Layout.modulation_spans: the rows of a class, or a refusal."""
import pytest

import paper_2608_21229_amd as rc


@pytest.mark.parametrize("preset", ["perref", "paper", "isolated", "dense"])
def test_spans_cover_their_class(preset):
    L = rc.Layout([(0, 8), (1, 16), (2, 64), (3, 5), (3, 64)], preset)
    for which in (rc.ROWS_STATIC, rc.ROWS_LIVE, rc.ROWS_ALL):
        assert sum(n for n, _ in L.modulation_spans(which)) == L.rows(which)


@pytest.mark.parametrize("which", [rc.ROWS_CACHED, -1, 4, None])
def test_other_classes_are_refused(which):
    """The cached rows are keys, which no norm reads; under most masks they are not all static ones."""
    with pytest.raises(ValueError, match="ROWS_STATIC, ROWS_LIVE or ROWS_ALL"):
        rc.Layout([(0, 8), (1, 16), (2, 64), (3, 64)], "paper").modulation_spans(which)
