"""Workspaces for captured calls without a GPU: the host-side refusals."""
import ctypes

import pytest

import aq_testutil
import paper_2606_12876_gb300 as aq


@pytest.fixture(scope="module", autouse=True)
def built():
    aq_testutil.ensure_built()


def test_arguments():
    L, p = aq.lib(), ctypes.c_void_p(7)
    assert L.aq_workspace_create(16, None) == aq.AQ_ERR_INVALID_ARG
    assert L.aq_workspace_create(0, ctypes.byref(p)) == aq.AQ_ERR_INVALID_ARG and p.value is None
    assert L.aq_workspace_destroy(None) == aq.AQ_OK
    assert L.aq_capture_id(None, None) == aq.AQ_ERR_INVALID_ARG
