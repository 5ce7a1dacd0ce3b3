"""Page operations of the 4-bit cache refuse int32 arrays that are not aligned to
4 bytes, before any device work (no GPU needed; pointers are fake)."""
import pytest

from paper_2606_00021_amd import sense
from test_kv_abi import FAKE, MISALIGNED, cache

NAMES = {
    "sense_kv_truncate": ("seqs", "lens", "status"),
    "sense_kv_fork": ("src", "dst", "status"),
    "sense_kv_reserve": ("seqs", "counts", "status"),
    "sense_kv_compact": ("seqs", "tails", "keep", "keep_len", "pick", "status"),
}


def call(fn, at):
    lib, c = sense.load_library(), cache()
    a = dict.fromkeys(NAMES[fn], FAKE)
    a.update(at)
    if fn in ("sense_kv_truncate", "sense_kv_fork"):
        first, second = NAMES[fn][:2]
        return getattr(lib, fn)(c, a[first], a[second], 2, a["status"], None)
    if fn == "sense_kv_reserve":
        return lib.sense_kv_reserve(c, a["seqs"], a["counts"], 2, a["status"], FAKE, 1 << 40, None)
    return lib.sense_kv_compact(c, a["seqs"], a["tails"], a["keep"], a["keep_len"], a["pick"], 1, 4,
                                2, a["status"], FAKE, 1 << 40, None)


@pytest.mark.parametrize("fn,name", [(f, n) for f, names in NAMES.items() for n in names])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_int_arrays_must_be_aligned(fn, name, off):
    assert call(fn, {name: FAKE + off}) == MISALIGNED
    assert sense.load_library().sense_last_error_message()
