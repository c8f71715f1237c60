"""The checks of sequence_sums themselves: rounded results pass, zeros and results that miss one row do not."""
import pytest

import sequence_sums as sums


def name(c):
    return f"{c[0]}-{'x'.join(map(str, c[1:6]))}"


CASES = [(sums.Conv, c) for c in sums.CONV] + [(sums.Scan, c) for c in sums.SCAN + sums.SETS] + [(sums.Norm, c) for c in sums.NORM]


@pytest.mark.parametrize("kind, case", CASES, ids=lambda v: v.__name__ if isinstance(v, type) else name(v))
def test_what_a_check_lets_through(kind, case):
    c = kind(case)
    want, types = c.reference(), c.types()
    scales = c.scales(want) if kind is sums.Norm else {}
    for k, units in c.units.items():
        assert want[k].norm() > 0, k
        sums.close(want[k].to(types[k]), want[k], units, k, scales.get(k))
        if k != "mean":
            with pytest.raises(AssertionError):
                sums.close(want[k].to(types[k]) * 0, want[k], units, k, scales.get(k))
            with pytest.raises(AssertionError):
                sums.close(want[k].to(types[k]) * 1.02, want[k], units, k, scales.get(k))
    # the sums over rows, without one of them
    for row in sums.rows_of(c):
        short = kind(case, drop=row).reference()
        for k in c.sums:
            with pytest.raises(AssertionError):
                sums.close(short[k].to(types[k]), want[k], c.units[k], (k, row))
