import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


# Tests that hold a value which the definition (include/rgc.h) does not give.  They stay as they are, run, and have to fail.
HOLD_A_WRONG_VALUE = {
    "test_distillation_entries_left_out_twice_and_masked":
        "its oracle adds up q (ln q - ln p) entry by entry where an index comes twice, and an index stands for the sum of its entries: two "
        "halves on a word that the student is certain of would have the divergence -ln 2 (test_gpu_lm_repeated_entries.py has the same "
        "rows with the sums)",
}


def pytest_collection_modifyitems(items):
    for item in items:
        if item.name in HOLD_A_WRONG_VALUE:
            item.add_marker(pytest.mark.xfail(strict=True, reason=HOLD_A_WRONG_VALUE[item.name]))


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(scope="session")
def oracle():
    import oracle as _oracle
    _oracle.build()
    return _oracle
