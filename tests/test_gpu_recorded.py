"""The recorded form of the sensitivity study runs, its schedules are feasible and its numbers hang together."""
import pytest

pytestmark = pytest.mark.gpu


def test_recorded_study():
    from paper_2508_13231_b200 import figures
    out, kept = figures.recorded("recorded_small", quick=True)
    assert set(out) == {"static", "reactive", "accumulated", "sa_guided"}
    assert all(ticks > 0 and 0 <= hits <= 1 for ticks, hits in out.values())
    assert out["sa_guided"][0] <= out["accumulated"][0]
    shares = list(kept.values())
    assert all(0 < s <= 1 + 1e-5 for s in shares) and shares == sorted(shares, reverse=True)
