"""Calls of the window attention and of the cache of 4 bits that the library refuses, with RLHF_EINVAL, before any device work
(no GPU needed): the addresses here are never read."""
import pytest

A, B, C, D, E, F = (i << 32 for i in range(1, 7))      # far apart
BIG = 1 << 30


def _R():
    import paper_2409_13221_amd as R
    return R


PACKED = dict(dtype=0, q=A, ld_q=512, k=B, ld_k=256, v=C, ld_v=256, start=D, q0=D, len=D, out=E, ld_out=512, n_tiles=2, rows=100, window=8, sinks=2,
              hq=4, hkv=2, hd=128, stream=None)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(dtype=-1), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(start=None), dict(q0=None), dict(len=None),
    dict(ld_q=508), dict(ld_k=252), dict(ld_v=252), dict(ld_out=508), dict(ld_q=514), dict(ld_k=257), dict(dtype=2, ld_q=516), dict(q=A + 8), dict(k=B + 4),
    dict(v=C + 2), dict(out=E + 8), dict(n_tiles=-1), dict(rows=-1), dict(rows=BIG + 1), dict(window=0), dict(window=-5), dict(sinks=-1), dict(hq=3),
    dict(hq=0), dict(hkv=0), dict(hd=32), dict(hd=96), dict(hd=256), dict(out=A), dict(out=A + 16), dict(out=B), dict(out=C + 1024),
    dict(hq=1 << 17, hkv=1 << 17, ld_q=1 << 24, ld_k=1 << 24, ld_v=1 << 24, ld_out=1 << 24), dict(ld_k=1 << 25), dict(ld_v=1 << 25),
], ids=str)
def test_window_attention(bad):
    R = _R()
    assert R.lib().rlhf_op_window_attention(*dict(PACKED, **bad).values()) == R.RLHF_EINVAL


@pytest.mark.parametrize("n_tiles", [BIG + 1, 2 ** 31 - 1])
def test_window_attention_of_more_tiles_than_rows_can_have(n_tiles):
    """The count of tiles that launches in turns have done stays within an int."""
    R = _R()
    assert R.lib().rlhf_op_window_attention(*dict(PACKED, n_tiles=n_tiles).values()) == R.RLHF_EINVAL


@pytest.mark.parametrize("empty", [dict(n_tiles=0), dict(rows=0), dict(rows=0, q=None, k=None, v=None, out=None), dict(n_tiles=0, start=None)], ids=str)
def test_window_attention_of_nothing(empty):
    R = _R()
    assert R.lib().rlhf_op_window_attention(*dict(PACKED, **empty).values()) == R.RLHF_OK


DECODE = dict(dtype=0, q=A, ld_q=512, pool=B, n_pages=50, table=C, pt_stride=9, n_samples=8, row=C, ctx=C, out=D, ld_out=512, scratch=E, rows=8,
              layer=0, nsplit=2, window=64, sinks=4, n_layers=2, hq=4, hkv=2, hd=128, stream=None)


@pytest.mark.parametrize("name", ["rlhf_op_window_decode_attention", "rlhf_op_kv4_decode_attention"])
@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(dtype=-1), dict(q=None), dict(pool=None), dict(table=None), dict(row=None), dict(ctx=None), dict(out=None), dict(scratch=None),
    dict(scratch=E + 4), dict(ld_q=508), dict(ld_out=500), dict(ld_q=513), dict(q=A + 4), dict(out=D + 8), dict(pool=B + 8), dict(n_pages=0), dict(n_pages=-1), dict(n_pages=1 << 27),
    dict(pt_stride=0), dict(pt_stride=-1), dict(pt_stride=1 << 27), dict(n_samples=0), dict(n_samples=-1), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(layer=-1), dict(layer=2), dict(nsplit=0),
    dict(nsplit=65), dict(window=0), dict(sinks=-1), dict(hq=3), dict(hkv=0), dict(hd=80), dict(out=A), dict(out=A + 512 * 4), dict(out=B + 16),
    dict(n_layers=1 << 17), dict(n_layers=1 << 16, hq=1 << 14, hkv=1 << 14, ld_q=1 << 21, ld_out=1 << 21, n_pages=1 << 26),
], ids=str)
def test_decode(name, bad):
    R = _R()
    assert getattr(R.lib(), name)(*dict(DECODE, **bad).values()) == R.RLHF_EINVAL


@pytest.mark.parametrize("name", ["rlhf_op_window_decode_attention", "rlhf_op_kv4_decode_attention"])
def test_decode_of_no_rows(name):
    R = _R()
    assert getattr(R.lib(), name)(*dict(DECODE, rows=0, n_pages=0, pt_stride=0, n_samples=0, q=None, pool=None, out=None).values()) == R.RLHF_OK


APPEND = dict(dtype=0, k=A, ld_k=256, v=B, ld_v=256, slot=C, pool=D, n_pages=50, rows=8, layer=1, n_layers=2, hkv=2, hd=128, stream=None)
READ = dict(dtype=0, pool=D, n_pages=50, slot=C, k=A, ld_k=256, v=B, ld_v=256, rows=8, layer=1, n_layers=2, hkv=2, hd=128, stream=None)


@pytest.mark.parametrize("call", ["append", "read"])
@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(dtype=-1), dict(k=None), dict(v=None), dict(slot=None), dict(pool=None), dict(ld_k=252), dict(ld_v=252), dict(ld_k=257), dict(k=A + 4),
    dict(v=B + 8), dict(pool=D + 8), dict(n_pages=0), dict(n_pages=-1), dict(n_pages=1 << 27), dict(rows=-1), dict(rows=BIG + 1), dict(layer=-1), dict(layer=2), dict(hkv=0),
    dict(hd=32), dict(hd=100), dict(k=D + 16), dict(v=D - 1024), dict(n_layers=1 << 17),
    dict(n_layers=1 << 16, hkv=1 << 14, ld_k=1 << 21, ld_v=1 << 21, n_pages=1 << 26),
], ids=str)
def test_kv4(call, bad):
    R = _R()
    base = APPEND if call == "append" else READ
    assert getattr(R.lib(), f"rlhf_op_kv4_{call}")(*dict(base, **bad).values()) == R.RLHF_EINVAL


def test_kv4_read_into_rows_that_overlap():
    R = _R()
    assert R.lib().rlhf_op_kv4_read(*dict(READ, v=A + 16).values()) == R.RLHF_EINVAL


@pytest.mark.parametrize("call", ["append", "read"])
def test_kv4_of_no_rows(call):
    R = _R()
    base = APPEND if call == "append" else READ
    assert getattr(R.lib(), f"rlhf_op_kv4_{call}")(*dict(base, rows=0, n_pages=0, k=None, v=None, slot=None, pool=None).values()) == R.RLHF_OK


def test_sizes():
    R = _R()
    L = R.lib()
    assert L.rlhf_op_kv4_page_bytes(2, 4, 128) == 2 * 4 * 18 * 128 and L.rlhf_op_kv4_page_bytes(1, 1, 64) == 18 * 64
    assert [L.rlhf_op_kv4_page_bytes(*a) for a in ((0, 4, 128), (2, 0, 128), (2, 4, 32))] == [0, 0, 0]
    assert L.rlhf_op_window_decode_scratch_floats(7, 4, 128, 1) == 0
    assert L.rlhf_op_window_decode_scratch_floats(7, 4, 128, 3) == 7 * 4 * 3 * 130
    assert L.rlhf_op_window_decode_scratch_floats(0, 4, 128, 3) == 0


@pytest.mark.parametrize("rows,hq,hkv,ctx,window,sinks", [(1, 32, 32, 1, 1, 0), (1, 8, 1, 131072, 2 ** 31 - 1, 2 ** 31 - 1), (1, 8, 1, 2 ** 31 - 1, 2 ** 31 - 1, 4),
                                                         (64, 32, 32, 4096, 256, 4), (1 << 24, 1 << 16, 1 << 16, 16, 16, 0), (3, 64, 8, 5000, 1, 2 ** 31 - 1)])
def test_nsplit_is_one_that_a_call_takes(rows, hq, hkv, ctx, window, sinks):
    n = _R().lib().rlhf_op_window_decode_nsplit(rows, hq, hkv, ctx, window, sinks)
    visible = min(-(-ctx // 16), -(-sinks // 16) + -(-window // 16) + 1)
    assert 1 <= n <= min(64, visible)


def test_binding_refuses_what_the_library_cannot_see():
    """Types, shapes and strides of tensors, on host tensors: nothing reaches the library."""
    import torch
    R = _R()
    t = R.rlhf_attention_tiles([5, 0, 300], "cpu")
    assert t.rows == 305 and t.n == 4 and t.start.tolist() == [0, 5, 5, 5] and t.q0.tolist() == [0, 0, 128, 256] and t.len.tolist() == [5, 300, 300, 300]
    with pytest.raises(ValueError):
        R.rlhf_attention_tiles([4, -1], "cpu")
    q = torch.zeros(305, 256)
    with pytest.raises(ValueError):                     # fewer rows than the sequences have
        R.rlhf_op_window_attention(q[:304], q[:304], q[:304], t, q[:304], 8, 0, 4, 4, 64)
    with pytest.raises(ValueError):                     # of two types
        R.rlhf_op_window_attention(q, q.half(), q, t, q, 8, 0, 4, 4, 64)
    with pytest.raises(ValueError):                     # in host memory
        R.rlhf_op_window_attention(q, q, q, t, q, 8, 0, 4, 4, 64)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):                     # not whole pages
        R.rlhf_op_window_decode_attention(q[:4], torch.zeros(2, 2, 4, 15, 64), i[None], i, i, q[:4], 0, 1, 4, 4, 64)
    with pytest.raises(ValueError):
        R.rlhf_op_kv4_decode_attention(q[:4], torch.zeros(2, 4, 18 * 64 - 1, dtype=torch.uint8), i[None], i, i, q[:4], 0, 1, 4, 4, 64)
    with pytest.raises(ValueError):                     # pages of another type
        R.rlhf_op_kv4_append(q[:4], q[:4], i, torch.zeros(2, 4, 18 * 64), 0, 1, 4, 64)


@pytest.mark.parametrize("lens", [[1.5], [3, 0.0], [2 ** 62] * 4, [2 ** 64], [2 ** 30, 1], [float("nan")], [[3, 4]], ["3"], [None]], ids=str)
def test_tiles_of_lengths_that_are_none(lens):
    """No length is cut off to a whole number, and no sum of them wraps."""
    with pytest.raises(ValueError):
        _R().rlhf_attention_tiles(lens, "cpu")


def test_tiles_of_whole_numbers_of_any_kind():
    import numpy as np
    import torch
    R = _R()
    for lens in ([3, 130], (3, 130), np.array([3, 130], np.int16), torch.tensor([3, 130]), [np.int64(3), torch.tensor(130)], iter([3, 130])):
        t = R.rlhf_attention_tiles(lens, "cpu")
        assert t.rows == 133 and t.start.tolist() == [0, 3, 3] and t.q0.tolist() == [0, 0, 128] and t.len.tolist() == [3, 130, 130]
    assert R.rlhf_attention_tiles([], "cpu").n == 0 and R.rlhf_attention_tiles([0, 0], "cpu").n == 0


@pytest.mark.parametrize("call", ["append", "read", "decode"])
@pytest.mark.parametrize("bad", ["type", "size", "strides"])
def test_pools_of_4_bits_are_looked_at_first(call, bad):
    """By what they are, whatever else is wrong with a call: here all tensors are in host memory."""
    import torch
    R = _R()
    q, i = torch.zeros(4, 256), torch.zeros(4, dtype=torch.int32)
    pool = {"type": torch.zeros(2, 4, 18 * 64), "size": torch.zeros(2, 4, 18 * 64 - 1, dtype=torch.uint8), "strides": torch.zeros(4, 4, 18 * 64, dtype=torch.uint8)[::2]}[bad]
    with pytest.raises(ValueError, match="uint8"):
        if call == "append":
            R.rlhf_op_kv4_append(q, q, i, pool, 0, 1, 4, 64)
        elif call == "read":
            R.rlhf_op_kv4_read(pool, i, q, q.clone(), 0, 1, 4, 64)
        else:
            R.rlhf_op_kv4_decode_attention(q, pool, i[None], i, i, q, 0, 1, 4, 4, 64)


@pytest.mark.parametrize("call", ["append", "read", "decode", "paged", "packed"])
def test_tensors_in_host_memory(call):
    """All else being right."""
    import torch
    R = _R()
    q, o, i, four = torch.zeros(4, 256), torch.zeros(4, 256), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 4, 18 * 64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device memory"):
        if call == "append":
            R.rlhf_op_kv4_append(q, o, i, four, 0, 1, 4, 64)
        elif call == "read":
            R.rlhf_op_kv4_read(four, i, q, o, 0, 1, 4, 64)
        elif call == "decode":
            R.rlhf_op_kv4_decode_attention(q, four, i[None], i, i, o, 0, 1, 4, 4, 64)
        elif call == "paged":
            R.rlhf_op_window_decode_attention(q, torch.zeros(2, 2, 4, 16, 64), i[None], i, i, o, 0, 1, 4, 4, 64)
        else:
            R.rlhf_op_window_attention(q, q, q, R.rlhf_attention_tiles([4], "cpu"), o, 8, 0, 4, 4, 64)
