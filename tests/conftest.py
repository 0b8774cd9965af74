import collections
import ctypes
import os
import subprocess
import sys
import types

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def _gpu_present():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


def pytest_collection_modifyitems(config, items):
    if _gpu_present():
        return
    skip = pytest.mark.skip(reason="no GPU in this container")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)


Route = collections.namedtuple("Route", "kernels fold nsplit rows columns workspace blocks chunks together two_part pair")


@pytest.fixture(scope="session")
def planner(tmp_path_factory):
    """tests/plan_query.cpp, built."""
    so = str(tmp_path_factory.mktemp("plan") / "plan_query.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-o", so, os.path.join(ROOT, "tests", "plan_query.cpp")],
                   check=True)
    return ctypes.CDLL(so)


@pytest.fixture(scope="session")
def route(planner):
    """route(op, N, C, H, W, K, R, stride, pad, groups=1, dtype=0, workspace=None, S=None): what the planner does with such a
    pass (and a workspace of so many bytes; filters R x S, or R x R), so that a test written for one set of kernels ("fp32",
    "split", "direct" or "window") can assert that it reaches them.  Of the window kernel also the channel blocks per step and
    the chunks; together: a grouped bf16 backward-filter in one launch of each kernel; two_part: a split pass that runs on two
    half-precision parts where its operands' range lets it; pair: one on four-wave tiles."""
    query = planner.plan_query

    def ask(op, N, C, H, W, K, R, stride, pad, groups=1, dtype=0, workspace=None, S=None):
        out = (ctypes.c_longlong * 11)()
        assert query(op, N, C, H, W, K, R, R if S is None else S, stride, pad, groups, dtype,
                     ctypes.c_longlong(-1 if workspace is None else workspace), out) == 0
        return Route(("fp32", "split", "direct", "window")[out[0]], *list(out)[1:])
    return ask


@pytest.fixture(scope="session")
def block_plans(tmp_path_factory):
    """Plans of tests/block_plan_query.cpp as dicts: block_plans.layer_norm(op, N, C, dtype), .kept_grad(N, I, O, dtype) and
    .q4(N, I, O): which kernel takes such a call, its grid and its steps, so that a test written for one of them can assert that it
    reaches it.  A refused call gives its status."""
    so = str(tmp_path_factory.mktemp("plan") / "block_plan_query.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-o", so, os.path.join(ROOT, "tests", "block_plan_query.cpp")],
                   check=True)
    query = ctypes.CDLL(so)

    def ask(name, keys):
        def call(*a):
            out = (ctypes.c_longlong * len(keys))()
            rc = getattr(query, name)(*a, out)
            return rc if rc else dict(zip(keys, out))
        return call

    return types.SimpleNamespace(
        layer_norm=ask("layer_norm_plan", "wide columns apart regs threads blocks lds waves groups rows_per_part part_rows "
                                          "row_blocks join_blocks bytes".split()),
        kept_grad=ask("kept_grad_plan", "slices tile step outputs itiles otiles splits rows_per_split blocks bytes".split()),
        q4=ask("q4_plan", "fused tile steps wide nrows orows bytes".split()))


# Normalised max errors the parity tests measured, printed once at the end of the run (also under -q).
_PARITY = []


@pytest.fixture
def parity_record():
    def record(tag, err, tol):
        _PARITY.append((tag, float(err), float(tol)))
    return record


def pytest_terminal_summary(terminalreporter):
    if not _PARITY:
        return
    terminalreporter.write_line("normalised max error vs the CPU oracle (whole tensors):")
    for tag, err, tol in _PARITY:
        terminalreporter.write_line("  %-44s %.3e  (bar %.1e)" % (tag, err, tol))
