"""Properties of the assembly that the kernels of masked and cached attention, of the
cache and of rotary positions compile to, that a run cannot show reliably (CPU)."""
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_sources import _listing, _sgprs


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("score_listings")
    names = ("masked.hip", "kvcache.hip", "rope.hip")
    with ThreadPoolExecutor(len(names)) as ex:
        return dict(zip(names, ex.map(lambda n: _listing(n, tmp), names)))


def _kernels(listings):
    for source, kernels in listings.items():
        for name, k in kernels.items():
            if k.vgprs is not None:      # (functions that are called, not inlined, have no entry of their own)
                yield source, name, k


def test_registers_hold_everything(listings):
    """No kernel keeps registers in memory, and two workgroups of a CU's LDS fit it."""
    found = 0
    for _, name, k in _kernels(listings):
        found += 1
        assert k.spills == 0, (name, k.spills)
        assert 2 * k.lds <= 160 * 1024, (name, k.lds)
    assert found > 50


def test_lds_loads_wait_for_their_base(listings):
    """A vector memory instruction may read a scalar register that a vector
    instruction wrote five wait states later at the earliest; inside inline
    assembly the compiler does not see to it."""
    loads = 0
    for kernels in listings.values():
        for name, k in kernels.items():
            state, written = 0, {}          # wait states passed, scalar register -> state after its vector write
            for c in k.code:
                op, _, args = c.partition(" ")
                if c.endswith(":"):
                    continue
                if op.startswith("global_load_lds"):
                    loads += 1
                    for r in _sgprs(args):
                        assert state - written.get(r, -5) >= 5, (name, c)
                state += 1 + (int(args, 0) if op == "s_nop" else 0)
                if op.startswith("v_"):
                    for r in _sgprs(args.split(",")[0]):
                        written[r] = state
                elif op.startswith("s_"):
                    for r in _sgprs(args.split(",")[0]):
                        written.pop(r, None)
    assert loads > 100


def test_tiles_are_waited_for_before_they_are_read(listings):
    """After a direct-to-LDS load, no read of LDS by a transposing load before a wait for vector memory."""
    found = 0
    for _, name, k in _kernels({"masked.hip": listings["masked.hip"]}):
        if "score_few_kernel" not in name:
            continue
        waiting = False
        for c in k.code:
            if c.startswith("global_load_lds"):
                waiting = True
            elif re.match(r"s_waitcnt.*vmcnt\(0\)", c):
                waiting = False
            elif c.startswith("ds_read_b64_tr"):
                found += 1
                assert not waiting, name
    assert found > 0
