"""Calls of the update's operators that the library refuses, with RLHF_EINVAL, before any device work (no GPU needed): the
addresses here are never read."""
import ctypes as C

import pytest

NAN, INF = float("nan"), float("inf")
A, B, D, E = 1 << 30, 2 << 30, 3 << 30, 4 << 30      # far apart


def _R():
    import paper_2409_13221_amd as R
    return R


POLICY = dict(dtype=0, logits=A, ld=100, tokens=B, lp_old=B, lp_ref=B, adv=B, weight=None, lo=0.2, hi=0.2, kl=0.1, scale=1.0,
              lp=B, stats=B, dlogits=D, ld_grad=100, scratch=E, rows=4, vocab=100, stream=None)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(tokens=None), dict(lp_old=None), dict(adv=None), dict(lp=None), dict(stats=None),
    dict(scratch=None), dict(rows=-1), dict(vocab=0), dict(ld=99), dict(ld_grad=99), dict(lo=-0.1), dict(lo=1.5), dict(lo=NAN),
    dict(hi=-0.1), dict(hi=NAN), dict(kl=-1.0), dict(kl=INF), dict(kl=NAN), dict(scale=INF), dict(scale=NAN), dict(lp_ref=None),
    dict(logits=A + 2), dict(dlogits=D + 1), dict(dlogits=A, ld_grad=101), dict(dlogits=A + 4), dict(dlogits=A + 1200),
], ids=str)
def test_policy_loss(bad):
    R = _R()
    assert R.lib().rlhf_op_policy_loss(*dict(POLICY, **bad).values()) == R.RLHF_EINVAL


SIDE_BY_SIDE = "columns of one buffer, side by side, share no element: launched, which fails here for want of a device"


def _launches(rc):
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not memory: only without a device does nothing read them")
    return rc() == _R().RLHF_EDEVICE


@pytest.mark.parametrize("cols,overlap", [(100, False), (101, False), (99, True), (102, True), (150, True), (-100, False), (-101, False), (-99, True), (-102, True), (0, False),
                                          (301, False), (300, True), (700, True)])
def test_policy_loss_side_by_side(cols, overlap):
    """Logits and gradient as columns of one buffer with rows of 201, the gradient `cols` columns behind (0: in place)."""
    R = _R()
    args = dict(POLICY, ld=201, ld_grad=201, dlogits=A + 4 * cols).values()
    rc = lambda: R.lib().rlhf_op_policy_loss(*args)
    if overlap:
        assert rc() == R.RLHF_EINVAL
    else:
        assert _launches(rc), SIDE_BY_SIDE


EMBED = dict(tdt=0, odt=1, table=A, ld=64, tokens=B, scale=1.0, out=D, ld_out=64, rows=8, d=64, vocab=10, stream=None)


@pytest.mark.parametrize("bad", [
    dict(tdt=3), dict(odt=-1), dict(table=None), dict(tokens=None), dict(out=None), dict(ld=63), dict(ld_out=63), dict(rows=-1), dict(d=0),
    dict(vocab=0), dict(table=A + 2), dict(out=D + 1), dict(out=A + 128), dict(out=A - 128),
], ids=str)
def test_embed(bad):
    R = _R()
    assert R.lib().rlhf_op_embed(*dict(EMBED, **bad).values()) == R.RLHF_EINVAL


EGRAD = dict(gdt=0, tdt=0, dout=A, ld=64, tokens=B, scale=1.0, acc=0, dtable=D, ld_table=64, scratch=E, rows=3000, d=64, vocab=10, stream=None)


@pytest.mark.parametrize("bad", [
    dict(gdt=3), dict(tdt=-1), dict(dout=None), dict(tokens=None), dict(dtable=None), dict(scratch=None), dict(scratch=E + 8), dict(ld=63),
    dict(ld_table=63), dict(rows=-1), dict(d=0), dict(vocab=0), dict(dout=A + 2), dict(dtable=D + 2), dict(dtable=A + 256),
], ids=str)
def test_embed_grad(bad):
    R = _R()
    assert R.lib().rlhf_op_embed_grad(*dict(EGRAD, **bad).values()) == R.RLHF_EINVAL


@pytest.mark.parametrize("big", [dict(vocab=1 << 20, d=1 << 22, ld=1 << 22, ld_table=1 << 22), dict(vocab=1 << 20, d=1 << 22, ld=1 << 22, ld_table=1 << 23, rows=100),
                                 dict(rows=1 << 28, d=1 << 20, ld=1 << 20, ld_table=1 << 20, acc=1), dict(rows=(1 << 30) + 1), dict(vocab=(1 << 30) + 1),
                                 dict(d=(1 << 22) + 1, ld=1 << 23, ld_table=1 << 23)], ids=str)
def test_embed_grad_refuses_what_no_launch_holds(big):
    """A launch has fewer than 2^32 threads; of a larger one only the rest beyond 2^32 would run, without an error."""
    R = _R()
    assert R.lib().rlhf_op_embed_grad(*dict(EGRAD, dtable=1 << 60, **big).values()) == R.RLHF_EINVAL


@pytest.mark.parametrize("cols,overlap", [(64, False), (63, True), (-64, False), (-65, True), (193, True), (192, False)])
def test_embedding_side_by_side(cols, overlap):
    """Table and rows as columns of one buffer with rows of 128."""
    R = _R()
    calls = [lambda: R.lib().rlhf_op_embed(*dict(EMBED, odt=0, ld=128, ld_out=128, out=A + 4 * cols).values()),
             lambda: R.lib().rlhf_op_embed_grad(*dict(EGRAD, ld=128, ld_table=128, dtable=A + 4 * cols).values())]
    for rc in calls:
        if overlap:
            assert rc() == R.RLHF_EINVAL
        else:
            assert _launches(rc), SIDE_BY_SIDE


@pytest.mark.parametrize("entry", [(None, D, 4, 0), (A, D, -1, 0), (A, D, 4, 3), (A + 2, D, 4, 0), (A, D + 2, 4, 0), (A, A + 8, 4, 0), (A, None, 4, 0)])
def test_grad_list(entry):
    R = _R()
    good = R.rlhf_tensor(B, B, 100, 1)
    arr = (R.rlhf_tensor * 2)(good, R.rlhf_tensor(*entry))
    assert R.lib().rlhf_op_clip_grads(arr, 2, E, 1.0, None) == R.RLHF_EINVAL
    if entry[1] in (D, None) and entry[0] != A or entry[2] < 0 or entry[3] == 3:     # what the norm reads, too
        assert R.lib().rlhf_op_grad_norm(arr, 2, E, E, None) == R.RLHF_EINVAL
        assert R.lib().rlhf_op_grad_norm_scratch_doubles(arr, 2) == 0


@pytest.mark.parametrize("entries", [
    [(A, A, 100), (A, A, 100)], [(A, A, 100), (B, B, 50), (A + 200, A + 200, 10)], [(A, B, 100), (D, B, 100)], [(A, B, 100), (D, B + 399, 1)],
    [(A, B, 100), (B, D, 100)], [(D, D, 10), (B, A, 100), (A + 396, E, 100)], [(A, A, 100), (A, B, 100)], [(A, A + 400 - 4, 100)],
    [(A + 4, A, 100)], [(B, B, 5)] + [(A + 400 * k, A + 400 * k, 100) for k in range(300)] + [(A + 400 * 200 - 4, E, 1)],
], ids=lambda e: f"{len(e)}")
def test_clipping_refuses_memory_that_two_entries_share(entries):
    """A gradient listed twice in place would be scaled once or twice, as its workgroups happen to run."""
    R = _R()
    arr = (R.rlhf_tensor * len(entries))(*(R.rlhf_tensor(s, d, n, 0) for s, d, n in entries))
    assert R.lib().rlhf_op_clip_grads(arr, len(entries), E + (1 << 20), 1.0, None) == R.RLHF_EINVAL


@pytest.mark.parametrize("n", [1 << 40, 1 << 62, (1 << 63) - 1])
@pytest.mark.parametrize("at", [0, 140, 299])
def test_a_count_beyond_any_memory_is_refused_before_a_launch(at, n):
    """Lists go out 128 tensors a launch: a bad entry behind the first 128 must not leave some of the others clipped."""
    R = _R()
    arr = (R.rlhf_tensor * 300)(*(R.rlhf_tensor(A + 400 * k, A + 400 * k, 100, 0) for k in range(300)))
    arr[at] = R.rlhf_tensor(B, B, n, 0)
    assert R.lib().rlhf_op_clip_grads(arr, 300, E, 1.0, None) == R.RLHF_EINVAL
    assert R.lib().rlhf_op_grad_norm(arr, 300, E, E + 8, None) == R.RLHF_EINVAL
    assert R.lib().rlhf_op_grad_norm_scratch_doubles(arr, 300) == 0


def test_scratch_of_a_long_list_takes_one_pass():
    """A pass over the list for each of its entries would be 4 * 10^10 steps."""
    import time
    R, n = _R(), 200000
    arr = (R.rlhf_tensor * n)(*(R.rlhf_tensor(A, A, 5000, k % 3) for k in range(n)))
    t = time.perf_counter()
    doubles = R.lib().rlhf_op_grad_norm_scratch_doubles(arr, n)
    assert doubles == n and time.perf_counter() - t < 2.0


@pytest.mark.parametrize("entries", [
    [(A, A, 100), (A + 400, A + 400, 100), (A - 400, A - 400, 100)], [(A, B, 100), (A, D, 100), (A + 200, E, 10)], [(A, A, 0), (A, A, 100)],
    [(A, A + 400, 100), (A + 800, A + 1200, 100)],
], ids=str)
def test_clipping_takes_neighbours_and_sources_listed_twice(entries):
    R = _R()
    arr = (R.rlhf_tensor * len(entries))(*(R.rlhf_tensor(s, d, n, 0) for s, d, n in entries))
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not memory: only without a device does nothing read them")
    assert R.lib().rlhf_op_clip_grads(arr, len(entries), E + (1 << 20), 1.0, None) == R.RLHF_EDEVICE


def test_grad_arguments():
    R = _R()
    L, arr = R.lib(), (R.rlhf_tensor * 1)(R.rlhf_tensor(A, A, 100, 0))
    assert L.rlhf_op_grad_norm(arr, 1, None, E, None) == R.RLHF_EINVAL
    assert L.rlhf_op_grad_norm(arr, 1, E, None, None) == R.RLHF_EINVAL
    assert L.rlhf_op_grad_norm(arr, 1, E, E + 4, None) == R.RLHF_EINVAL
    assert L.rlhf_op_grad_norm(arr, -1, E, E, None) == R.RLHF_EINVAL
    assert L.rlhf_op_grad_norm(None, 1, E, E, None) == R.RLHF_EINVAL
    for max_norm in (0.0, -1.0, NAN):
        assert L.rlhf_op_clip_grads(arr, 1, E, max_norm, None) == R.RLHF_EINVAL
    assert L.rlhf_op_clip_grads(arr, 1, None, 1.0, None) == R.RLHF_EINVAL


def test_struct_layout():
    R = _R()
    assert C.sizeof(R.rlhf_tensor) == 3 * 8 + 8


def test_scratch_sizes_of_nothing():
    L = _R().lib()
    assert L.rlhf_op_policy_loss_scratch_floats(0, 100) == 0 and L.rlhf_op_embed_grad_scratch_bytes(0, 8, 8) == 0
    assert L.rlhf_op_embed_grad_scratch_bytes(3000, 8, 8) > 0
    assert L.rlhf_op_policy_loss_scratch_floats(5, 100) >= 15 and L.rlhf_op_grad_norm_scratch_doubles(None, 0) >= 0


def test_binding_refuses_wrong_tensors():
    """Host tensors, and tensors of a wrong shape or type, are ValueErrors; nothing is launched."""
    torch = pytest.importorskip("torch")
    R = _R()
    f, i = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device memory"):
        R.rlhf_op_policy_loss(torch.zeros(4, 8), i, f, f, f, f)
    with pytest.raises(ValueError, match="device memory"):
        R.rlhf_op_embed(torch.zeros(8, 4), i, torch.zeros(4, 4))
    with pytest.raises(ValueError, match="device memory"):
        R.rlhf_op_embed_grad(torch.zeros(4, 4), i, torch.zeros(8, 4))
    with pytest.raises(ValueError, match="one device"):
        R.rlhf_tensor_list([f])
    with pytest.raises(ValueError, match="alike"):
        R.rlhf_tensor_list([f], [f.half()])
    with pytest.raises(ValueError, match="contiguous"):
        R.rlhf_tensor_list([torch.zeros(4, 4)[:, :2]])
    with pytest.raises(ValueError, match="as many"):
        R.rlhf_tensor_list([f], [])
    with pytest.raises(ValueError, match="contiguous rows"):
        R.binding._matrix(torch.zeros(8, 4).t(), 4, 8, "x")
    with pytest.raises(ValueError, match="overlap"):
        R.binding._matrix(torch.zeros(1, 8).expand(4, 8), 4, 8, "x")
    with pytest.raises(ValueError, match="entries"):
        R.binding._vector(torch.zeros(5), 4, torch.float32, "x")
