"""Refusals of the sense_kv_* calls, before any device work (no GPU needed).
Pointers are fake, aligned addresses: every call returns during validation."""
import ctypes

import pytest
import torch

from paper_2606_00021_amd import sense

OK, INVALID, MISALIGNED, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 5
FAKE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return sense.load_library()


def cache(**kw):
    base = dict(codes=FAKE, scales=FAKE, page_table=FAKE, seq_len=FAKE, page_refs=FAKE, n_layers=2,
                n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, n_seqs=4, max_pages=8)
    base.update(kw)
    return sense.KvCacheDesc(**base)


def batch(**kw):
    base = dict(seqs=None, row_start=None, row_len=None, n=2, max_rows=4, n_rows=8)
    base.update(kw)
    return sense.KvBatchDesc(**base)


BAD_CACHE = [
    (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(page_table=None), INVALID),
    (dict(seq_len=None), INVALID), (dict(page_refs=None), INVALID), (dict(n_layers=0), INVALID),
    (dict(n_layers=4097), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=(1 << 26) + 1), INVALID),
    (dict(page_size=8), INVALID), (dict(page_size=48), INVALID), (dict(page_size=256), INVALID),
    (dict(head_dim=32), INVALID), (dict(head_dim=96), INVALID), (dict(head_dim=512), INVALID),
    (dict(n_kv_heads=0), INVALID), (dict(n_kv_heads=1025), INVALID), (dict(n_seqs=0), INVALID),
    (dict(max_pages=0), INVALID), (dict(max_pages=1 << 27), INVALID),
    (dict(codes=FAKE + 8), MISALIGNED), (dict(scales=FAKE + 4), MISALIGNED),
    (dict(seq_len=FAKE + 2), MISALIGNED),
]


def calls(lib, c):
    b = batch()
    return {
        "write": lib.sense_kv_write(c, 0, 1, FAKE, FAKE, 2, 128, 0, b, None),
        "read": lib.sense_kv_read(c, 0, 1, FAKE, FAKE, 2, 128, 0, b, None),
        "attention": lib.sense_kv_attention(c, 0, FAKE, 2, 4, 256, b, None, 0, 0, 0.1, 0, FAKE, 256,
                                            FAKE, 1 << 40, None),
        "truncate": lib.sense_kv_truncate(c, None, None, 2, None, None),
        "fork": lib.sense_kv_fork(c, FAKE, FAKE, 2, None, None),
        "reserve": lib.sense_kv_reserve(c, None, FAKE, 2, None, FAKE, 1 << 40, None),
        "compact": lib.sense_kv_compact(c, None, FAKE, FAKE, FAKE, None, 1, 4, 2, None, FAKE,
                                        1 << 40, None),
    }


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_every_call_refuses_a_bad_cache(lib, kw, status):
    for name, got in calls(lib, ctypes.byref(cache(**kw))).items():
        assert got == status, name
        assert lib.sense_last_error_message()


def test_null_cache(lib):
    assert set(calls(lib, None).values()) == {INVALID}


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(n=65537, seqs=FAKE), INVALID), (dict(n=5), INVALID),
    (dict(max_rows=0), INVALID), (dict(max_rows=(1 << 20) + 1), INVALID), (dict(n_rows=-1), INVALID),
    (dict(seqs=FAKE + 1), MISALIGNED), (dict(row_len=FAKE + 2), MISALIGNED),
    (dict(n=65536, max_rows=1 << 20, seqs=FAKE), UNSUPPORTED),
])
def test_bad_batches(lib, kw, status):
    c, b = ctypes.byref(cache()), ctypes.byref(batch(**kw))
    for fn in (lib.sense_kv_write, lib.sense_kv_read):
        assert fn(c, 0, 1, FAKE, FAKE, 2, 128, 0, b, None) == status
    assert lib.sense_kv_attention(c, 0, FAKE, 2, 4, 256, b, None, 0, 0, 0.1, 0, FAKE, 256, FAKE,
                                  1 << 60, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), INVALID), (dict(layer=2), INVALID), (dict(layer=1, n_layers=2), INVALID),
    (dict(n_layers=0), INVALID), (dict(dtype=3), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(stride=120), INVALID), (dict(k=FAKE + 8), MISALIGNED),
    (dict(v=FAKE + 2), MISALIGNED), (dict(stride=132), MISALIGNED),
    (dict(n_layers=2, layer_stride=100), MISALIGNED),
])
def test_bad_rows(lib, kw, status):
    a = dict(layer=0, n_layers=1, k=FAKE, v=FAKE, dtype=2, stride=128, layer_stride=0)
    a.update(kw)
    for fn in (lib.sense_kv_write, lib.sense_kv_read):
        assert fn(cache(), a["layer"], a["n_layers"], a["k"], a["v"], a["dtype"], a["stride"],
                  a["layer_stride"], batch(), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), INVALID), (dict(dtype=0), INVALID), (dict(dtype=9), INVALID),
    (dict(heads=3), INVALID), (dict(heads=0), INVALID), (dict(heads=4098), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=2.0 ** 127 * 1.25), INVALID), (dict(max_kv=-1), INVALID),
    (dict(mask=FAKE, mask_ld=3), INVALID), (dict(mask=FAKE, mask_ld=4, mask_stride=-1), INVALID),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q_stride=255), INVALID),
    (dict(q_stride=257), MISALIGNED), (dict(q=FAKE + 4), MISALIGNED), (dict(out=FAKE + 8), MISALIGNED),
    (dict(out_stride=260), MISALIGNED), (dict(ws=None, max_kv=2000, pages=1000), WORKSPACE),
    (dict(ws_bytes=64, pages=1000), WORKSPACE), (dict(ws=FAKE + 16, pages=1000), MISALIGNED),
])
def test_bad_attention(lib, kw, status):
    a = dict(layer=0, q=FAKE, dtype=2, heads=4, q_stride=256, mask=None, mask_ld=0, mask_stride=0,
             scale=0.1, max_kv=0, out=FAKE, out_stride=256, ws=FAKE, ws_bytes=1 << 40, pages=8)
    a.update(kw)
    assert lib.sense_kv_attention(
        cache(max_pages=a["pages"]), a["layer"], a["q"], a["dtype"], a["heads"], a["q_stride"],
        batch(), a["mask"], a["mask_ld"], a["mask_stride"], a["scale"], a["max_kv"], a["out"],
        a["out_stride"], a["ws"], a["ws_bytes"], None) == status


def test_bad_page_operations(lib):
    c = cache()
    for n in (-1, 4097):
        assert lib.sense_kv_truncate(c, FAKE, FAKE, n, None, None) == INVALID
        assert lib.sense_kv_fork(c, FAKE, FAKE, n, None, None) == INVALID
        assert lib.sense_kv_reserve(c, FAKE, FAKE, n, None, FAKE, 1 << 40, None) == INVALID
        assert lib.sense_kv_compact(c, FAKE, FAKE, FAKE, FAKE, None, 1, 4, n, None, FAKE, 1 << 40,
                                    None) == INVALID
    assert lib.sense_kv_truncate(c, None, FAKE, 5, None, None) == INVALID      # 4 sequences
    assert lib.sense_kv_reserve(c, None, FAKE, 5, None, FAKE, 1 << 40, None) == INVALID
    assert lib.sense_kv_reserve(c, None, None, 2, None, FAKE, 1 << 40, None) == INVALID
    assert lib.sense_kv_reserve(c, None, FAKE, 2, None, None, 0, None) == WORKSPACE
    assert lib.sense_kv_reserve(c, None, FAKE, 2, None, FAKE, 8, None) == WORKSPACE
    assert lib.sense_kv_reserve(c, None, FAKE, 2, None, FAKE + 64, 1 << 40, None) == MISALIGNED
    assert lib.sense_kv_fork(c, None, FAKE, 2, None, None) == INVALID
    assert lib.sense_kv_fork(c, FAKE, None, 2, None, None) == INVALID

    def compact(tails=FAKE, keep=FAKE, keep_len=FAKE, pick=None, rows=1, ld=4, ws=FAKE, n=2):
        return lib.sense_kv_compact(c, None, tails, keep, keep_len, pick, rows, ld, n, None, ws,
                                    1 << 40, None)
    assert compact(tails=None) == compact(keep=None) == compact(keep_len=None) == INVALID
    assert compact(rows=2) == compact(rows=0) == compact(ld=0) == compact(ld=4097) == INVALID
    assert compact(ws=None) == WORKSPACE
    assert compact(ws=FAKE + 8) == MISALIGNED


def test_empty_calls_do_nothing(lib):
    c, b = cache(), batch(n=0)
    assert lib.sense_kv_write(c, 0, 1, None, None, 2, 128, 0, b, None) == OK
    assert lib.sense_kv_attention(c, 0, None, 2, 4, 256, b, None, 0, 0, 0.1, 0, None, 256, None, 0,
                                  None) == OK
    assert lib.sense_kv_truncate(c, None, None, 0, None, None) == OK
    assert lib.sense_kv_fork(c, None, None, 0, None, None) == OK
    assert lib.sense_kv_reserve(c, None, None, 0, None, None, 0, None) == OK
    assert lib.sense_kv_compact(c, None, None, None, None, None, 1, 4, 0, None, None, 0, None) == OK


def test_workspace_sizes(lib):
    size = ctypes.c_size_t(7)
    c = cache(max_pages=1000)
    assert lib.sense_kv_attention_workspace_size(c, 2, 4, 4, 100, ctypes.byref(size)) == OK
    assert size.value == 0                                   # short: one launch, no partial sums
    assert lib.sense_kv_attention_workspace_size(c, 2, 4, 4, 0, ctypes.byref(size)) == OK
    assert size.value > 0 and size.value % 256 == 0
    assert lib.sense_kv_attention_workspace_size(c, 2, 0, 4, 0, ctypes.byref(size)) == INVALID
    assert lib.sense_kv_attention_workspace_size(c, 2, 4, 5, 0, ctypes.byref(size)) == INVALID
    assert lib.sense_kv_attention_workspace_size(c, 2, 4, 4, 0, None) == INVALID
    assert lib.sense_kv_reserve_workspace_size(c, 3, ctypes.byref(size)) == OK and size.value > 0
    assert lib.sense_kv_compact_workspace_size(3, 8, ctypes.byref(size)) == OK and size.value > 0
    assert lib.sense_kv_compact_workspace_size(3, 0, ctypes.byref(size)) == INVALID


def test_the_binding_refuses_tensors_that_do_not_fit():
    # On the CPU nothing gets as far as the library.
    kv = {"codes": torch.zeros((1, 4, 2, 2, 16, 32), dtype=torch.uint8),
          "scales": torch.zeros((1, 4, 2, 2, 2, 16), dtype=torch.uint8),
          "page_table": torch.full((2, 4), -1, dtype=torch.int32),
          "seq_len": torch.zeros(2, dtype=torch.int32),
          "page_refs": torch.zeros(4, dtype=torch.int32)}
    with pytest.raises(ValueError, match="GPU"):
        sense.sense_kv_truncate(kv)
    for name, t in (("scales", torch.zeros((1, 4, 2, 2, 1, 16), dtype=torch.uint8)),
                    ("codes", torch.zeros((4, 2, 2, 16, 32), dtype=torch.uint8)),
                    ("seq_len", torch.zeros(3, dtype=torch.int32)),
                    ("page_refs", torch.zeros(4, dtype=torch.int64)),
                    ("page_table", torch.full((4, 2), -1, dtype=torch.int32).t())):
        with pytest.raises(ValueError):
            sense.sense_kv_truncate({**kv, name: t})
    with pytest.raises(ValueError):
        sense.sense_build_kv_cache(1, 4, 24, 2, 64, 2, 4, device="cpu")


def test_the_binding_packs_a_cache_as_the_header_lays_it_out():
    fields = sense._KV_CACHE_FIELDS
    assert fields.size == ctypes.sizeof(sense.KvCacheDesc)
    got = sense.KvCacheDesc.from_buffer_copy(fields.pack(*range(1, 13)))
    assert [getattr(got, name) for name, _ in sense.KvCacheDesc._fields_] == list(range(1, 13))
