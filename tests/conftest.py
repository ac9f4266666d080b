import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Tests that assert nothing but how long calls take.  They come last: a run that stops at its first failure has been through all that tells right from wrong
# before a moment's delay of the host can end it (a pair of calls of 11 us that once took 18, whose kernels take 5.7 and 5.5).
TIMED = {"test_linear_ragged_weight_costs_as_much_as_a_whole_one", "test_rows_in_order_of_their_lengths", "test_kernels_of_rows_in_order_of_their_lengths", "test_backward_of_short_rows",
         "test_middle_rows_in_order_of_lengths", "test_time_of_a_long_gap", "test_time_of_few_words"}


def pytest_collection_modifyitems(items):
    items.sort(key=lambda item: getattr(item, "originalname", item.name) in TIMED)  # stable: each part in its order


def parse_golden(name):
    """tests/golden/<name>: '#' comments, then 'key: v v v ...' lines (ints or floats, a/b fractions allowed)."""
    out = {}
    with open(os.path.join(ROOT, "tests", "golden", name)) as fh:
        for line in fh:
            line = line.split("#", 1)[0].strip()
            if not line:
                continue
            key, vals = line.split(":", 1)
            parsed = []
            for tok in vals.split():
                if "/" in tok:
                    a, b = tok.split("/")
                    parsed.append(float(a) / float(b))
                else:
                    parsed.append(float(tok))
            out[key.strip()] = parsed
    return out


@pytest.fixture(scope="session")
def golden5():
    return parse_golden("five_vertex.txt")


@pytest.fixture(scope="session")
def hgnn():
    """The GPU binding with the library loaded (built first only when nothing is built)."""
    import __graft_entry__ as ge
    ge.ensure_built()
    import paper_2411_01109_amd as mod
    mod.load()
    return mod


@pytest.fixture(scope="session")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def pytest_terminal_summary(terminalreporter):
    """One line per run: how often the norm rule's cancelling branch was taken (tests/parity.py)."""
    try:
        import parity
    except ImportError:
        return
    log = parity.CANCEL_LOG
    worst = max((t[1] for t in log), default=0.0)
    terminalreporter.write_line(f"[parity] cancelling branch of the norm rule taken {len(log)} time(s)"
                                + (f"; largest true rel-L2 it replaced {worst:.3e}" if log else ""))
