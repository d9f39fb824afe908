import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(scope="session", autouse=True)
def _oracle_team():
    """The oracle on all cores, whatever a test's batch: most of the suite's time is its."""
    from oracle import ref
    ref.set_team(min(16, os.cpu_count() or 1))
