"""The Python side of a step over a growing cache, where it is Python: on which device a kernel is enqueued, numbers that a field of the
C struct cannot hold (CPU only)."""
import contextlib

import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F


def test_a_workspace_is_reset_on_its_own_device(monkeypatch):
    """The null stream is the current device's, so that one has to be the workspace's."""
    current, seen = [0], []

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    class Workspace:
        is_cuda = True
        is_contiguous = lambda self: True
        numel = element_size = data_ptr = lambda self: 4096
        get_device = lambda self: 1

    class Library:
        @staticmethod
        def fairkv_tree_workspace_reset(*args):
            seen.append((current[0], args[-1]))
            return F.FAIRKV_OK

    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(F, "lib", lambda: Library)
    F.fairkv_tree_workspace_reset(Workspace(), 256, stream=Stream)
    assert seen == [(1, 77)] and current == [0]


@pytest.mark.parametrize("kw", [dict(page_rows=(1 << 32) + 16), dict(page_rows=1 << 31), dict(page_rows=-16), dict(expected_rows=1 << 63), dict(expected_rows=(1 << 64) + 5),
                                dict(expected_rows=-1)])
def test_a_cache_refuses_numbers_that_its_fields_do_not_hold(kw):
    k, cap, pages = torch.zeros(16, 64, dtype=torch.bfloat16), torch.ones(1, 1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="bits"):
        F.Cache(k, k, cap, pages=pages, **{**dict(page_rows=16), **kw})
