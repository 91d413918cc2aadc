"""Workspaces that the wrappers of the dense calls take by default."""
import torch

import paper_2508_20407_amd as tl
from test_paged_edges import in_two_threads


def test_default_workspaces_are_a_host_threads_own():
    """Partials and their merge are two launches: calls of two host threads on one stream may enqueue them in turn."""
    t = torch.zeros(1)
    a, c = in_two_threads(lambda i: tl._workspace_for(t, None, 0))
    assert a is not c
    assert tl._workspace_for(t, None, 0) is tl._workspace_for(t, None, 0)
    assert tl._workspace_for(t, None, 0) is not tl._workspace_for(t, None, 1)
    assert tl._workspace_for(t, a, 0) is a
