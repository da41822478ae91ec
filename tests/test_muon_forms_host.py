"""The lists of muon_cases.py reach the forms of the orthogonalised update that they are named for (no GPU)."""
import numpy as np
import pytest

from muon_cases import FORMS, chunks
from test_muon_host import plan  # noqa: F401  (the launch table's host build)


@pytest.mark.parametrize("name", sorted(FORMS))
def test_lists_reach_their_forms(plan, name):  # noqa: F811
    (tiles, alone, direct, in_a_row), shapes = FORMS[name]
    floats, unsupported, (_, _, per_block, got_tiles, got_alone, got_direct), _ = plan(shapes)
    assert floats > 0 and not unsupported
    assert (got_tiles, bool(got_alone), bool(got_direct)) == (tiles, alone, direct)
    waves = 8 if tiles < 4 else 4
    if not alone:
        assert per_block == waves * in_a_row
        if in_a_row > 1:   # a wide and a tall matrix with full wavefronts, and blocks that end in between
            assert max(chunks(s) for s in shapes if s[0] < s[1]) >= per_block
            assert any(chunks(s) % per_block for s in shapes)
    else:                  # wavefronts with several chunks, and with none
        assert max(chunks(s) for s in shapes) > waves and min(chunks(s) for s in shapes) < waves


def test_every_form_has_a_list():
    seen = {form[:3] for form, _ in FORMS.values()}
    assert seen == {(t, a, d) for t in (1, 2) for a, d in ((True, True), (False, True), (False, False))} | {(4, False, False)}
    several = {form[:3] for form, _ in FORMS.values() if form[3] and form[3] > 1}
    assert several == {form for form in seen if not form[1]}
    for several_tall in ("direct1_two", "direct2_two", "sums2_two", "sums4_two", "sums4_three"):
        form, shapes = FORMS[several_tall]
        assert any(r > c and chunks((r, c)) > (8 if form[0] < 4 else 4) * form[3] for r, c in shapes)


def test_what_two_halves_hold():
    """The documented precision of a product: two fp16 hold a scaled fp32 value to 2^-23 of it, or to 2^-25 where that is more, and
    three products of them miss at most 2^-21 of a product whose operands are above a quarter."""
    rng = np.random.default_rng(1)

    def halves(v):
        hi = v.astype(np.float16)
        return hi.astype(np.float64), (v - hi.astype(np.float32)).astype(np.float16).astype(np.float64)

    def draw(low):
        return (rng.choice([-1, 1], 10 ** 6) * rng.uniform(1, 2, 10 ** 6) * 2.0 ** rng.integers(low, 15, 10 ** 6)).astype(np.float32)

    v = np.concatenate([draw(-30), (1 + np.arange(2 ** 20, dtype=np.float32) * np.float32(2.0 ** -20 + 2.0 ** -23))])
    v = v[np.abs(v) < 2.0 ** 15]
    hi, lo = halves(v)
    off = np.abs(hi + lo - v)
    assert (off <= np.maximum(2.0 ** -23 * np.abs(v), 2.0 ** -25)).all() and (off > 2.0 ** -24 * np.abs(v))[np.abs(v) >= 0.25].any()
    a, b = draw(-2), draw(-2)
    (ah, al), (bh, bl) = halves(a), halves(b)
    exact = a.astype(np.float64) * b
    off = np.abs(ah * bh + ah * bl + al * bh - exact) / np.abs(exact)
    assert 2.0 ** -22 < off.max() <= 2.0 ** -21 and 2.0 ** -23.8 < np.sqrt((off * off).mean()) < 2.0 ** -23.6
