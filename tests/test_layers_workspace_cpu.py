"""A caller's own workspace object in the calls on a cache: anything with ensure(bytes), as the replay takes it."""
import pytest

from test_layers_cpu import P, cache, lib  # noqa: F401
from paper_2608_30310_b200 import _binding as B
from paper_2608_30310_b200 import _layers as L


class Own:
    def ensure(self, nbytes):
        self.asked = nbytes
        return P, 1 << 20


class Derived(B.Workspace):
    def ensure(self, nbytes):
        return P + 256, nbytes


@pytest.mark.parametrize("count", [0, 5])
def test_ensure_is_what_is_asked(lib, count):  # noqa: F811
    d, own = cache(num_pages=1000), Own()
    keep = L._scratch(lib, d, count, own, None)
    assert keep is own and own.asked == lib.gdn_cache_workspace_size(d, count) > 0
    assert (d.workspace, d.workspace_bytes) == (P, 1 << 20)
    L._scratch(lib, d, count, Derived("cpu"), None)
    assert d.workspace == P + 256
