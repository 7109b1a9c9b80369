"""Which form of the kernels a call takes, by its sizes and the device; nothing is launched."""
import pytest

from paper_2309_01885_gb300 import qe
from tests import cache_host as host


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return host.load(tmp_path_factory.mktemp("host"))


def form(lib, c, at):
    assert host.attend(lib, c, at) == qe.QE_OK
    return lib.fake_kernel().decode()


@pytest.mark.parametrize("dim,group", [(64, 32), (64, 64), (80, 32), (96, 32), (128, 32), (128, 64), (128, 128)])
def test_up_to_32_pairs_are_few(lib, dim, group):
    """(Query row, head) pairs of a kv head: up to 32 the few-rows kernel, more the tiles, in every head dim."""
    lib.fake_device(0, 152)
    for kv in (300, 30000):
        for per_kv, q in ((1, 1), (4, 1), (16, 1), (20, 1), (24, 1), (25, 1), (4, 7), (29, 1), (4, 8), (32, 1), (1, 32)):
            assert "k_attend_rows" in form(lib, host.cache(8, dim, group), host.batch(3, q, kv, 8 * per_kv)), (per_kv, q)
        for per_kv, q in ((33, 1), (1, 33), (4, 9), (71, 1)):
            assert "k_attend_tiles" in form(lib, host.cache(8, dim, group), host.batch(3, q, kv, 8 * per_kv)), (per_kv, q)


@pytest.mark.parametrize("device,sms", [(0, 152), (1, 76), (2, 148)])
def test_forms_for_short_contexts_go_by_the_devices_size(lib, device, sms):
    """A CTA of 8 warps for each item while they fit one an SM, of 4 up to 8 an SM; grids tell the items."""
    lib.fake_device(device, sms)
    c = host.cache(1, 128, 32)
    for items, span, warps in ((sms, 2048, 8), (sms + 1, 1088, 4), (8 * sms, 1088, 4), (8 * sms + 1, 1088, 0), (sms, 2049, 0), (sms + 1, 1089, 0)):
        name = form(lib, c, host.batch(items, 1, span, 4))
        # k_attend_rows<C, GC, NT, warps, WHOLE, HALF>
        assert (f"Li{warps}ELb1E" if warps else "Li2ELb0E") in name, (items, span, name)
        if warps:
            assert lib.fake_grid(0) == items
    lib.fake_device(0, 152)
