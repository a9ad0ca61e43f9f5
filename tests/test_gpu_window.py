"""Attention with a sliding window and sinks, packed and paged, and the KV cache of 4 bits, against oracle/window.py in float64.

Tolerances.  E = 2^-24 is the half step of float, U that of the output type.  With S = |q| |k| / sqrt(hd) (a sum of hd products, magnitudes)
the greatest over the keys of a query, and A = the weighted mean of |v|, V the greatest |v|:
  a score is off by at most hd E S by its products and sums, and by 4 E |z| <= 4 E S by scaling and the multiply-add in front of exp2;
  a weight, relative to its like, by twice that and 4 E of exp2 and rescaling: t = E (2 (hd + 4) S + 8);
  a sum of n terms by n / 16 + 32 additions one after the other of E each (pages or tiles of 16 and more keys are joined by trees);
  where weights are rounded to 16 bits for the matrix units, each by W of itself: packed half a step of the type (half 2^-11, bf16 2^-8), paged
  less than 2^-11 (half and bf16 in two terms, 4 bits in half);
so |o - o_exact| <= (2 t + 2 E (n / 16 + 32) + W) A + (U + 2 E)|o|, where 2 t counts numerator and denominator.  A is at most V; where weights round, A
is that of the query itself.  Cache of 4 bits: the same with |k| = |c| + 8 |s|, |v| alike, the values that the cache holds being exact."""
import numpy as np
import pytest
import torch

from oracle import window as W

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TDT = {"fp32": torch.float32, "bf16": torch.bfloat16, "half": torch.float16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "half": 2.0 ** -11}
ROUNDED = {"fp32": 0.0, "bf16": 2.0 ** -11, "half": 2.0 ** -11}        # W, paged
PACKED_ROUNDED = {"fp32": 0.0, "bf16": 2.0 ** -8, "half": 2.0 ** -11}
ALL = 2 ** 31 - 1


def _R():
    import paper_2409_13221_amd as R
    return R


def _np(t):
    return t.detach().double().cpu().numpy()


def _normal(r, *shape, dtype="fp32", std=1.0):
    return torch.from_numpy((r.normal(size=shape) * std).astype(np.float32)).to(TDT[dtype])


def _ints(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _check(got, q, k, v, q_pos, window, sinks, dtype, k_size=None, v_size=None, rounded=ROUNDED):
    """got [T, Hq, hd] against attention of q [T, Hq, hd] over k, v [S, Hkv, hd] (float64)."""
    want = W.attention(q, k, v, q_pos, window, sinks)
    T, Hq, hd = q.shape
    G = Hq // k.shape[1]
    kk, vv = np.abs(k) if k_size is None else k_size, np.abs(v) if v_size is None else v_size
    ones = np.ones((T, Hq, 1))
    for t in range(T):
        at = np.flatnonzero(W.visible([q_pos[t]], len(k), window, sinks)[0])
        for h in range(Hq):
            size = kk[at, h // G] @ np.abs(q[t, h]) / np.sqrt(hd)
            z = k[at, h // G] @ q[t, h] / np.sqrt(hd)
            p = np.exp(z - z.max())
            mean = (p / p.sum()) @ vv[at, h // G]
            tol = (2 * E * (2 * (hd + 4) * size.max() + 8) + 2 * E * (len(at) / 16 + 32) + rounded[dtype]) * mean + (HALF_STEP[dtype] + 2 * E) * np.abs(want[t, h]) + 1e-30
            if dtype == "half":
                tol = tol + 2.0 ** -25
            off = np.abs(got[t, h] - want[t, h])
            assert (off <= tol).all(), (t, h, q_pos[t], float((off / tol).max()), float(off.max()))
    return want


# ------------------------------------------------------------------------------------------------ packed

def _packed(seed, lens, Hq, Hkv, hd, dtype, behind=0, pad=0):
    """q, k, v as columns of one buffer with `pad` more columns of NaN, rows behind the sequences of NaN."""
    r = np.random.default_rng(seed)
    rows, width = sum(lens), (Hq + 2 * Hkv) * hd
    buf = torch.full((rows + behind, width + pad), float("nan"), dtype=TDT[dtype])
    buf[:rows, :width] = _normal(r, rows, width, dtype=dtype)
    buf[:rows, :Hq * hd] *= 2
    buf = buf.cuda()
    return buf[:, :Hq * hd], buf[:, Hq * hd:(Hq + Hkv) * hd], buf[:, (Hq + Hkv) * hd:width]


def _packed_run(q, k, v, lens, window, sinks, Hq, Hkv, hd, out=None):
    R = _R()
    if out is None:
        out = torch.full((q.shape[0], Hq * hd), 7.0, device="cuda", dtype=q.dtype)
    R.rlhf_op_window_attention(q, k, v, R.rlhf_attention_tiles(lens), out, window, sinks, Hq, Hkv, hd)
    torch.cuda.synchronize()
    return out


def _packed_check(out, q, k, v, lens, window, sinks, Hq, Hkv, hd, dtype, rows=None):
    """Every sequence, or of it the given positions."""
    start = 0
    for n in lens:
        s = slice(start, start + n)
        pos = np.arange(n) if rows is None else np.array([i for i in rows if i < n], int)
        if n:
            _check(_np(out[s]).reshape(n, Hq, hd)[pos], _np(q[s]).reshape(n, Hq, hd)[pos], _np(k[s]).reshape(n, Hkv, hd), _np(v[s]).reshape(n, Hkv, hd),
                   pos, window, sinks, dtype, rounded=PACKED_ROUNDED)
        start += n


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("Hq,Hkv,hd", [(2, 2, 64), (2, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 3), (16, 4), (63, 0), (64, 1), (65, 64), (128, 130), (100, 0), (ALL, 0), (3, ALL)])
def test_packed(dtype, Hq, Hkv, hd, window, sinks):
    lens = [1, 17, 128, 0, 129, 64, 200]
    q, k, v = _packed(hd + window % 97, lens, Hq, Hkv, hd, dtype, behind=3, pad=8)
    out = _packed_run(q, k, v, lens, window, sinks, Hq, Hkv, hd)
    _packed_check(out, q, k, v, lens, window, sinks, Hq, Hkv, hd, dtype)
    assert (out[sum(lens):] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (8, 1), (16, 2), (17, 1), (6, 3)])
def test_packed_heads(dtype, Hq, Hkv):
    lens = [40, 150]
    q, k, v = _packed(Hq, lens, Hq, Hkv, 64, dtype)
    _packed_check(_packed_run(q, k, v, lens, 30, 2, Hq, Hkv, 64), q, k, v, lens, 30, 2, Hq, Hkv, 64, dtype, rows=[0, 1, 31, 32, 33, 39, 127, 128, 149])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,sinks", [(700, 5), (ALL, 0), (257, 200), (5, 0)])
def test_packed_long(dtype, hd, window, sinks):
    lens = [1500, 3]
    q, k, v = _packed(hd + sinks, lens, 4, 2, hd, dtype)
    rows = [0, 4, 5, 6, 127, 128, 255, 256, 257, 258, 300, 699, 700, 701, 1023, 1024, 1279, 1280, 1499]
    _packed_check(_packed_run(q, k, v, lens, window, sinks, 4, 2, hd), q, k, v, lens, window, sinks, 4, 2, hd, dtype, rows=rows)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hd", [64, 128])
def test_packed_hidden_keys_reach_nobody(dtype, bad, hd):
    """Key 37 of 200 is not finite: it shows in the queries that see it, 37 to 56, and in no other."""
    lens, window, sinks, Hq, Hkv = [200, 30], 20, 3, 2, 1
    q, k, v = _packed(5, lens, Hq, Hkv, hd, dtype)
    for t in (k, v):
        kk = t.clone()
        kk[37] = bad
        a = (q, kk, v) if t is k else (q, k, kk)
        out = _packed_run(*a, lens, window, sinks, Hq, Hkv, hd)
        clean = _packed_run(q, k, v, lens, window, sinks, Hq, Hkv, hd)
        sees = np.arange(230) // 37 == 1
        sees[57:] = False
        _packed_check(out, *a, lens, window, sinks, Hq, Hkv, hd, dtype, rows=[0, 5, 20, 35, 36, 57, 58, 60, 63, 64, 100, 128, 199])
        if t is v or bad != bad:
            assert not torch.isfinite(out[sees]).any()
        assert torch.isfinite(clean).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hd,long", [(64, 0), (128, 0), (128, 1)])
def test_packed_hidden_keys_change_nothing(dtype, bad, hd, long):
    """Key 37 of 200 (or, with tiles that are mostly full, of 1500) is not finite, in all dims or in one of V: what does not see it keeps its bits."""
    lens, window, sinks, Hq, Hkv = [1500 if long else 200, 30], 20, 3, 4, 2
    q, k, v = _packed(5, lens, Hq, Hkv, hd, dtype)
    clean = _packed_run(q, k, v, lens, window, sinks, Hq, Hkv, hd)
    sees = np.zeros(sum(lens), bool)
    sees[37:57] = True
    for what, dims in ((k, slice(None)), (v, slice(None)), (v, slice(hd + 9, hd + 10))):      # dim 9 of the second KV head
        other = what.clone()
        other[37, dims] = bad
        out = _packed_run(q, *((other, v) if what is k else (k, other)), lens, window, sinks, Hq, Hkv, hd)
        assert torch.equal(out[~sees], clean[~sees])
        if dims != slice(None):
            hit = torch.zeros_like(out, dtype=torch.bool)
            hit.view(-1, Hq, hd)[37:57, 2:, 9] = True
            assert torch.equal(out[~hit], clean[~hit])
            assert (torch.isnan(out[hit]) if bad != bad else out[hit] == bad).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_packed_values_that_are_not_finite(dtype):
    """Per dim: infinities of one sign that a query sees give that infinity, of both or a NaN none, and the other dims are as without them; what a query does not see
    is not there.  The first keys of 300 hold them, seen for a while."""
    lens, hd = [300], 64
    q, k, v = _packed(22, lens, 2, 1, hd, dtype)
    inf = float("inf")
    clean = _packed_run(q, k, v, lens, 100, 0, 2, 1, hd)
    other = v.clone()
    other[2, 5], other[40, 6], other[3, 7], other[90, 7], other[7, 8], other[50, 8], other[60, 63] = inf, -inf, inf, -inf, inf, inf, float("nan")
    out = _packed_run(q, k, other, lens, 100, 0, 2, 1, hd).view(-1, 2, hd)
    want = clean.clone().view(-1, 2, hd)
    want[2:102, :, 5], want[40:140, :, 6], want[3:103, :, 7], want[90:190, :, 7], want[7:107, :, 8] = inf, -inf, inf, -inf, inf
    want[90:103, :, 7], want[50:150, :, 8], want[60:160, :, 63] = float("nan"), inf, float("nan")
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(out.nan_to_num(nan=0.0, posinf=inf, neginf=-inf), want.nan_to_num(nan=0.0, posinf=inf, neginf=-inf))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_packed_queries_keep_their_bits_beside_great_scores(dtype):
    """Every fifth query has scores of some 2^28, too far apart for the references of a tile; the others in its tile keep their bits."""
    lens, hd = [140], 64
    q, k, v = _packed(23, lens, 1, 1, hd, dtype)
    k *= 4096
    q[:] = q / 4096
    clean = _packed_run(q, k, v, lens, 50, 2, 1, 1, hd)
    great = torch.arange(140, device="cuda") % 5 == 0
    q[great] *= 2.0 ** 24
    out = _packed_run(q, k, v, lens, 50, 2, 1, 1, hd)
    assert torch.equal(out[~great], clean[~great]) and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_packed_a_sink_that_is_not_finite_shows_everywhere(dtype):
    lens = [150]
    q, k, v = _packed(6, lens, 2, 2, 64, dtype)
    v[1] = float("nan")
    out = _packed_run(q, k, v, lens, 10, 2, 2, 2, 64)
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1:]).all()
    v[0], v[1] = float("nan"), 0
    assert torch.isfinite(_packed_run(q, k, v, lens, 10, 0, 2, 2, 64)[10:]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_packed_scores_of_great_size(dtype):
    """Scores of 1e20 and more, all far apart and all negative: the greatest takes it all."""
    lens = [140]
    q, k, v = _packed(7, lens, 1, 1, 64, dtype)
    q[:], k[:] = 0, 0
    q[:, 0] = 1e17
    size = 10.0 ** torch.arange(140, device="cuda").remainder(7).add(1).double()
    k[:, 0] = -size.to(k.dtype)
    out = _packed_run(q, k, v, lens, 7, 0, 1, 1, 64)
    for i in (0, 6, 7, 20, 64, 127, 128, 139):
        lo = max(0, i - 6)
        best = lo + int(k[lo:i + 1, 0].float().argmax())
        assert torch.equal(out[i], v[best]), i


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_packed_scores_of_2_to_the_30(dtype, sign):
    """As far as half goes: scores of 2^26 to 2^30, thousands apart; a rounded one may be off by 2^6."""
    lens = [140]
    q, k, v = _packed(14, lens, 1, 1, 64, dtype)
    q[:] = 8192.0
    k[:] = (sign * 32 * (1 + torch.arange(140, device="cuda").mul(37).remainder(140)).double())[:, None].to(k.dtype)
    out = _packed_run(q, k, v, lens, 50, 2, 1, 1, 64)
    for i in range(140):
        seen = [j for j in range(i + 1) if j > i - 50 or j < 2]
        best = seen[int(k[seen, 0].float().argmax())]
        assert torch.equal(out[i], v[best]), i


@pytest.mark.parametrize("dtype", ["bf16", "half"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,sinks", [(2, 0), (3, 1), (40, 4), (700, 5), (ALL, 0)])
def test_packed_equal_values_come_out_as_they_are(dtype, hd, window, sinks):
    """All rows of V of a sequence alike: the weights that multiply V are those that the output is divided by, so it is V.  Products and sums in float are off by
    2 E (n / 16 + 32) <= 2^-16 of it, which no 16-bit rounding of V itself lets through; weights that are summed before they are rounded would be off by
    half a step of their type (half 2^-11, bf16 2^-8) of a weight, more than the 2^-12 (2^-9) that keep an output at V."""
    lens = [1500, 70]
    q, k, v = _packed(21, lens, 4, 2, hd, dtype)
    v[:1500], v[1500:] = v[0].clone(), v[1500].clone()
    out = _packed_run(q, k, v, lens, window, sinks, 4, 2, hd)
    assert torch.equal(out.view(-1, 2, 2, hd), v.reshape(-1, 2, 1, hd).expand(-1, 2, 2, hd))


def test_packed_strides_views_and_streams():
    """Rows of every second one of a buffer, on a stream of its own."""
    lens, Hq, Hkv, hd = [90, 140], 4, 2, 64
    q, k, v = _packed(8, lens, Hq, Hkv, hd, "half")
    want = _packed_run(q, k, v, lens, 50, 2, Hq, Hkv, hd)
    wide = lambda t: torch.full((2 * t.shape[0], t.shape[1] + 24), float("nan"), device="cuda", dtype=t.dtype)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        put = []
        for t in (q, k, v):
            b = wide(t)
            b[::2, 8:8 + t.shape[1]] = t
            put.append(b[::2, 8:8 + t.shape[1]])
        o = wide(want)
        _R().rlhf_op_window_attention(*put, _R().rlhf_attention_tiles(lens), o[::2, 16:16 + Hq * hd], 50, 2, Hq, Hkv, hd)
    s.synchronize()
    assert torch.equal(o[::2, 16:16 + Hq * hd], want)
    assert torch.isnan(o[1::2]).all() and torch.isnan(o[::2, :16]).all() and torch.isnan(o[::2, 16 + Hq * hd:]).all()


def test_packed_tiles_outside_the_rows_are_skipped():
    R = _R()
    q, k, v = _packed(9, [100], 2, 2, 64, "half")
    t = R.rlhf_attention_tiles([40, 60])
    t.tiles[:, 0] = _ints([-1, 0, 40])
    out = torch.full((100, 128), 7.0, device="cuda", dtype=torch.half)
    R.rlhf_op_window_attention(q, k, v, t, out, 9, 0, 2, 2, 64)
    t.tiles[:, 0] = _ints([70, 0, 31])
    R.rlhf_op_window_attention(q, k, v, t, out, 9, 0, 2, 2, 64)
    t.tiles[:, 0] = _ints([0, -128, 40])
    R.rlhf_op_window_attention(q, k, v, t, out, 9, 0, 2, 2, 64)
    t.tiles[:, 0] = _ints([0, 128, 40])
    R.rlhf_op_window_attention(q, k, v, t, out, 9, 0, 2, 2, 64)
    assert (out[:40] == 7).all()
    _check(_np(out[40:]).reshape(60, 2, 64), _np(q[40:]).reshape(60, 2, 64), _np(k[40:]).reshape(60, 2, 64), _np(v[40:]).reshape(60, 2, 64), np.arange(60), 9, 0,
           "half", rounded=PACKED_ROUNDED)


# ------------------------------------------------------------------------------------------------ paged

class Paged:
    """Contexts in a paged pool of garbage, pages in no order, rows in no order of the samples; layer 1 of 3.  Tokens beyond a context,
    and pages of nobody, hold NaN."""

    def __init__(self, seed, ctx, Hq, Hkv, hd, dtype, four=False, extra=3):
        R, r = _R(), np.random.default_rng(seed)
        self.Hq, self.Hkv, self.hd, self.dtype, self.four, self.ctx = Hq, Hkv, hd, dtype, four, ctx
        self.layers, self.layer = 3, 1
        rows, width = len(ctx), max(1, -(-max(ctx) // 16)) + 1
        need = [-(-max(c, 0) // 16) for c in ctx]
        order = r.permutation(sum(need) + extra)
        self.n_pages = len(order)
        self.sample = r.permutation(rows)
        self.table = np.full((rows, width), -1, np.int32)              # entries of no page: never read
        self.k, self.v, self.k_size, self.v_size, first = [], [], [], [], 0
        if four:
            pool = r.integers(0, 256, (self.n_pages, self.layers, Hkv, 18 * hd)).astype(np.uint8)
            pool.view(np.float16)[..., 8 * hd:] = np.nan
        else:
            pool = torch.full((self.n_pages, self.layers, 2, Hkv, 16, hd), float("nan"), dtype=TDT[dtype])
        slots = []
        for i, c in enumerate(ctx):
            pages = order[first:first + need[i]]
            first += need[i]
            self.table[self.sample[i], :need[i]] = pages
            k, v = (_normal(r, max(c, 0), Hkv, hd, dtype=dtype) for _ in range(2))
            if not four:
                for t in range(c):
                    pool[pages[t // 16], self.layer, 0, :, t % 16] = k[t]
                    pool[pages[t // 16], self.layer, 1, :, t % 16] = v[t]
            slots += [int(pages[t // 16]) * 16 + t % 16 for t in range(c)]
            self.k.append(k), self.v.append(v)
        self.q = _normal(r, rows, Hq * hd, dtype=dtype, std=2.0).cuda()
        if four:
            self.pool = torch.from_numpy(pool).cuda()
            k, v = torch.cat(self.k).cuda().flatten(1), torch.cat(self.v).cuda().flatten(1)
            R.rlhf_op_kv4_append(k, v, _ints(slots), self.pool, self.layer, self.layers, Hkv, hd)
            self.k_size, self.v_size = [], []
            for i in range(rows):
                for kv, size in ((self.k, self.k_size), (self.v, self.v_size)):
                    u, p = W.kv4_quantize(kv[i].float().numpy())
                    p = np.abs(p.astype(np.float64))
                    size.append(np.repeat(p[..., 1] + 8 * p[..., 0], 64, -1))
                    kv[i] = W.kv4_values(u, W.kv4_quantize(kv[i].float().numpy())[1])
        else:
            self.pool = pool.cuda()
            self.k, self.v = [_np(t) for t in self.k], [_np(t) for t in self.v]
            self.k_size, self.v_size = [np.abs(t) for t in self.k], [np.abs(t) for t in self.v]
        self.table_d, self.row_d, self.ctx_d = torch.from_numpy(self.table).cuda(), _ints(self.sample), _ints(ctx)

    def run(self, window, sinks, q=None, out=None, **kw):
        R = _R()
        q = self.q if q is None else q
        out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype) if out is None else out
        call = R.rlhf_op_kv4_decode_attention if self.four else R.rlhf_op_window_decode_attention
        call(q, self.pool, self.table_d, self.row_d, self.ctx_d, out, self.layer, self.layers, self.Hq, self.Hkv, self.hd, window, sinks, **kw)
        torch.cuda.synchronize()
        return out

    def check(self, out, window, sinks, rows=None):
        got, q = (_np(t).reshape(len(self.ctx), self.Hq, self.hd) for t in (out, self.q))
        for i, c in enumerate(self.ctx):
            if rows is not None and i not in rows:
                continue
            if c <= 0:
                assert (got[i] == 0).all()
                continue
            _check(got[i:i + 1], q[i:i + 1], self.k[i], self.v[i], np.array([c - 1]), window, sinks, self.dtype, self.k_size[i], self.v_size[i])


EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 255, 256, 257, 300]


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 20), (16, 4), (17, 0), (33, 16), (100, 17), (ALL, 0), (5, ALL)])
def test_decode(four, dtype, hd, window, sinks):
    p = Paged(window % 89 + sinks % 7, EDGES, 2, 2, hd, dtype, four)
    for nsplit in (None, 1, 3):
        p.check(p.run(window, sinks, nsplit=nsplit), window, sinks)


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (8, 1), (16, 1), (17, 1), (40, 2), (6, 3)])
def test_decode_heads(four, dtype, Hq, Hkv):
    p = Paged(Hq, [70, 5, 200], Hq, Hkv, 128, dtype, four)
    for nsplit in (1, 2):
        p.check(p.run(60, 4, nsplit=nsplit), 60, 4)


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("nsplit", [None, 1, 2, 7, 64])
def test_decode_long(four, dtype, nsplit):
    p = Paged(3, [3000, 1, 1777], 4, 2, 64, dtype, four)
    for window, sinks in ((ALL, 0), (1500, 40)):
        p.check(p.run(window, sinks, nsplit=nsplit), window, sinks)


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("dtype", ["fp32", "half"])
def test_decode_many_rows(four, dtype):
    """More rows than the chip holds at once, with and without a bound of the contexts."""
    r = np.random.default_rng(0)
    p = Paged(4, r.integers(0, 60, 700).tolist(), 3, 3, 64, dtype, four)
    a, b = p.run(25, 2), p.run(25, 2, max_ctx=60)
    p.check(a, 25, 2, rows=range(0, 700, 23))
    p.check(b, 25, 2, rows=range(0, 700, 23))


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("Hq,Hkv,hd", [(2, 2, 128), (4, 2, 64), (12, 2, 128), (36, 2, 64), (8, 1, 128)])
def test_decode_many_short_rows(four, dtype, Hq, Hkv, hd):
    """Rows enough to fill the chip with a wave each: contexts of up to 7 pages, of which at most 5 are seen, and all of them."""
    r = np.random.default_rng(1)
    rows = 1030 // Hkv
    p = Paged(17, r.integers(-1, 112, rows).tolist(), Hq, Hkv, hd, dtype, four)
    for window, sinks in ((40, 5), (ALL, 0)):
        p.check(p.run(window, sinks), window, sinks, rows=range(0, rows, 41))


@pytest.mark.parametrize("dtype", ["fp32", "half"])
@pytest.mark.parametrize("Hq,Hkv,hd", [(8, 8, 128), (32, 8, 64), (48, 8, 64), (72, 8, 64)])
def test_four_bits_many_longer_rows(dtype, Hq, Hkv, hd):
    """Rows of up to 40 pages, two waves each."""
    r = np.random.default_rng(2)
    p = Paged(18, (r.integers(0, 640, 128) * (r.random(128) < 0.3)).tolist() + [640], Hq, Hkv, hd, dtype, True)
    for window, sinks in ((600, 5), (ALL, 0)):
        p.check(p.run(window, sinks), window, sinks, rows=[*range(0, 128, 13), 128])


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("nsplit", [1, 2])
def test_decode_pages_without_a_visible_token_are_not_read(four, nsplit):
    """Their entries point outside the pool, or at pages of NaN."""
    p = Paged(5, [200, 90], 2, 1, 64, "half", four)
    want = p.run(40, 18, nsplit=nsplit)
    for bad in (-5, 1 << 30, p.n_pages, None):
        t = p.table.copy()
        t[p.sample[0], 2:10], t[p.sample[1], 2:3] = (bad,) * 2 if bad is not None else (int(np.setdiff1d(np.arange(p.n_pages), p.table)[0]),) * 2
        p.table_d = torch.from_numpy(t).cuda()
        assert torch.equal(p.run(40, 18, nsplit=nsplit), want)


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("nsplit", [1, 3])
def test_decode_hidden_tokens_change_nothing(four, dtype, nsplit):
    """Tokens of pages that are seen in part, before the window, behind the sinks and behind the context: NaN, infinities and numbers of any size in their place leave every bit."""
    ctx, window, sinks, hd = [203, 90, 37], 40, 18, 64
    p = Paged(30, ctx, 4, 2, hd, dtype, four)
    want = p.run(window, sinks, nsplit=nsplit)
    hidden = []
    for i, c in enumerate(ctx):
        last = c + -c % 16
        hidden += [(int(p.table[p.sample[i], t // 16]), t % 16) for t in range(last) if t >= c or (t < c - window and t >= sinks)]
    page, token = (torch.tensor(x, device="cuda") for x in zip(*hidden))
    for bad in (float("nan"), float("inf"), -float("inf"), 60000.0, 0.0):
        if four:
            half = p.pool.view(torch.float16).view(p.n_pages, p.layers, 2, 9 * hd)[..., 8 * hd:].view(p.n_pages, p.layers, 2, 2, 16, 2)       # K | V, token, (s, c)
            half[page, 1, :, :, token] = bad
        else:
            p.pool[page, 1, :, :, token] = bad
        assert torch.equal(p.run(window, sinks, nsplit=nsplit), want), bad


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("nsplit", [1, 3])
@pytest.mark.parametrize("dtype", ["fp32", "half"])
def test_decode_rows_outside_table_or_pool_are_nan(four, nsplit, dtype):
    p = Paged(6, [200, 90, 33, 50, 17, 60], 2, 2, 64, dtype, four)
    want = p.run(ALL, 0, nsplit=nsplit)
    t = p.table.copy()
    t[p.sample[0], 7], t[p.sample[1], 5] = p.n_pages, -1
    p.table_d = torch.from_numpy(t).cuda()
    p.row_d[2], p.row_d[3] = 6, -1
    p.ctx_d[4] = 16 * t.shape[1] + 1
    out = p.run(ALL, 0, nsplit=nsplit)
    assert torch.isnan(out[:5]).all() and torch.equal(out[5], want[5])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("nsplit", [1, 4])
def test_decode_is_the_last_row_of_packed(dtype, nsplit):
    """Same queries, keys and values through both forms."""
    p = Paged(7, [130, 64, 300], 4, 2, 128, dtype)
    dec = p.run(70, 5, nsplit=nsplit)
    rows = sum(p.ctx)
    q = torch.zeros(rows, 4 * 128, dtype=TDT[dtype], device="cuda")
    last = np.cumsum(p.ctx) - 1
    q[last] = p.q
    k, v = (torch.from_numpy(np.concatenate(t)).to(TDT[dtype]).flatten(1).cuda() for t in (p.k, p.v))
    pre = _packed_run(q, k, v, p.ctx, 70, 5, 4, 2, 128)[last]
    bound = 2 * HALF_STEP[dtype] + 2 * PACKED_ROUNDED[dtype]            # of both; values up to 4
    assert (dec.double() - pre.double()).abs().max() <= 4 * bound + 2e-5


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_decode_a_visible_token_that_is_not_finite(four, dtype):
    p = Paged(8, [100, 100], 2, 2, 64, dtype, four)
    page, off = int(p.table[p.sample[0], 5]), 3                          # token 83 of row 0
    if four:
        half = p.pool.view(torch.float16).view(p.n_pages, p.layers, 2, 9 * 64)
        half[page, 1, 0, 8 * 64 + 32 + 2 * off:8 * 64 + 32 + 2 * off + 2] = float("nan")       # scale and center of V, first head
    else:
        p.pool[page, 1, 1, 0, off] = float("inf")
    out = p.run(20, 0)
    assert not torch.isfinite(out[0, :64]).any() and torch.isfinite(out[0, 64:]).all() and torch.isfinite(out[1]).all()
    assert torch.isfinite(p.run(16, 0)).all()                            # hidden, in a page of which tokens 84 on are seen


def _hold(p, i, k, v):
    """Other k, v [ctx, Hkv, hd] in the place of context i of a cache of 4 bits."""
    slots = [int(p.table[p.sample[i], t // 16]) * 16 + t % 16 for t in range(p.ctx[i])]
    k, v = k.to(TDT[p.dtype]), v.to(TDT[p.dtype])
    _R().rlhf_op_kv4_append(k.flatten(1).cuda(), v.flatten(1).cuda(), _ints(slots), p.pool, p.layer, p.layers, p.Hkv, p.hd)
    for kv, to, size in ((k, p.k, p.k_size), (v, p.v, p.v_size)):
        u, par = W.kv4_quantize(kv.float().numpy())
        to[i], par = W.kv4_values(u, par), np.abs(par.astype(np.float64))
        size[i] = np.repeat(par[..., 1] + 8 * par[..., 0], 64, -1)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("Hq", [1, 2])
@pytest.mark.parametrize("great", [2.0 ** 90, 2.0 ** 115, 2.0 ** 127])
def test_four_bits_queries_of_great_size(dtype, Hq, great):
    """One dim of q is so large that the scores, all finite, are far apart: the greatest takes it all."""
    p = Paged(11, [100, 40], Hq, 1, 64, dtype, four=True)
    k = torch.zeros(100, 1, 64)
    k[:, 0, 5] = 2.0 ** -7 * (1 + torch.arange(100).mul(37).remainder(100) / 128)
    _hold(p, 0, k, torch.from_numpy(np.random.default_rng(1).normal(size=(100, 1, 64))))
    q = torch.zeros(2, Hq * 64, device="cuda", dtype=TDT[dtype])
    q[:, 5::64] = great
    out = _np(p.run(50, 3, q=q))[0].reshape(Hq, 64)
    seen = np.r_[0:3, 50:100]
    score = p.k[0][seen, 0, 5]
    best = seen[score == score.max()]                                   # held alike, their values are averaged
    want, size = p.v[0][best, 0].mean(0), p.v_size[0][best, 0].mean(0)
    assert (np.abs(out - want) <= (ROUNDED[dtype] + 8 * E) * size + (HALF_STEP[dtype] + 2 * E) * np.abs(want)).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (6, 1), (12, 1)])
@pytest.mark.parametrize("what", ["grow", "fall", "jump", "equal", "tiny"])
def test_four_bits_values_of_changing_size(dtype, Hq, Hkv, what):
    """V that grows or falls by 2^20 along a context, jumps by 2^15, has scale 0, or the least that half holds."""
    n, r = 400, np.random.default_rng(12)
    p = Paged(13, [n, 33], Hq, Hkv, 128, dtype, four=True)
    t = np.arange(n)[:, None, None]
    size = {"grow": 2.0 ** (t / 20 - 10), "fall": 2.0 ** (10 - t / 20), "jump": np.where(t // 70 % 2, 2.0 ** 10, 2.0 ** -5), "equal": 0.0 * t, "tiny": 2.0 ** -22 + 0 * t}[what]
    v = r.normal(size=(n, Hkv, 128)) * size + (np.where(t < 200, 0.0, 3.0) if what == "equal" else 0.0)
    _hold(p, 0, torch.from_numpy(r.normal(size=(n, Hkv, 128))), torch.from_numpy(v))
    for window, sinks, nsplit in ((ALL, 0, 1), (150, 20, 1), (ALL, 0, 3)):
        p.check(p.run(window, sinks, nsplit=nsplit), window, sinks)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (6, 1), (12, 1)])
@pytest.mark.parametrize("what", ["dims", "first", "heads", "none"])
@pytest.mark.parametrize("apart", [16, 26])
def test_four_bits_values_far_apart(dtype, Hq, Hkv, what, apart):
    """Values 2^apart times as large as others, in the other 64 dims, or of tokens whose weight for a head is nothing, which come first, or are all that other heads see;
    or (none) in a group beside one of equal values.  Every 64 dims of every head are as near as float: 16 times the error of the formula in float32 and 2^-22, beside the
    roundings of 16-bit calls as random numbers add: of a weight times the scale of its token's values, and of the output."""
    n, hd, r = 200, 128, np.random.default_rng(12)
    p = Paged(13, [n, 33], Hq, Hkv, hd, dtype, four=True)
    k, v, q = r.normal(size=(n, Hkv, hd)), r.normal(size=(n, Hkv, hd)) * 2.0 ** (11 - apart), r.normal(size=(2, Hq, hd))
    q[..., 0] = 8
    if what == "dims":
        v[..., 64:] *= 2.0 ** apart
    elif what == "first":
        v[:16] *= 2.0 ** apart
        k[..., 0], k[:16, :, 0] = 1, -84
    elif what == "heads":
        v[:100] *= 2.0 ** apart
        q[..., 0] *= np.where(np.arange(Hq) % 2, 1, -1)
        k[:100, :, 0], k[100:, :, 0] = 40, -40
    else:
        v[..., 64:] = 3
    p.q = torch.from_numpy(q.reshape(2, -1)).to(TDT[dtype]).cuda()
    v = torch.from_numpy(v).to(TDT[dtype])
    _hold(p, 0, torch.from_numpy(k), v)
    center = np.repeat(W.kv4_quantize(v.float().numpy())[1][..., 1].astype(np.float64), 64, -1).repeat(Hq // Hkv, 1)
    q, k, v = _np(p.q)[0].reshape(Hq, hd), p.k[0].repeat(Hq // Hkv, 1), p.v[0].repeat(Hq // Hkv, 1)
    kf, vf, qf = (torch.from_numpy(np.asarray(t, np.float32)) for t in (k, v, q))
    square = lambda t: (t.reshape(Hq, 2, 64) ** 2).sum(-1)
    for window, sinks, nsplit in ((ALL, 0, 1), (150, 20, 1), (ALL, 0, 3)):
        out = _np(p.run(window, sinks, nsplit=nsplit))[0].reshape(Hq, hd)
        at = np.flatnonzero(W.visible([n - 1], n, window, sinks)[0])
        z = (k[at] * q).sum(-1) / np.sqrt(hd)
        w = np.exp(z - z.max(0))
        w /= w.sum(0)
        want = (w[..., None] * v[at]).sum(0)
        wf = torch.softmax((kf[at] * qf).sum(-1) / np.float32(np.sqrt(hd)), 0)
        plain = (wf[..., None] * vf[at]).sum(0).double().numpy()
        rest = ROUNDED[dtype] ** 2 * square(np.sqrt((w[..., None] ** 2 * (v - center)[at] ** 2).sum(0))) + HALF_STEP[dtype] ** 2 * square(want)
        tiny = (2.0 ** -25 if dtype == "half" else 0.0) * 8                 # half a step of half's smallest values, of 64
        bound = 16 * np.sqrt(square(plain - want)) + 2.0 ** -22 * np.sqrt(square(want)) + np.sqrt(rest) + tiny
        assert (np.sqrt(square(out - want)) <= bound).all(), (np.sqrt(square(out - want)) / bound).max()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("great,less", [(2.0 ** 15, 2.0 ** 4), (-2.0 ** 15, 2.0 ** 6), (2.0 ** 60, 1.0), (2.0 ** 100, 2.0 ** 10), (-2.0 ** 60, 1.0)])
@pytest.mark.parametrize("nsplit", [1, 3])
def test_decode_scores_of_great_size(dtype, great, less, nsplit):
    """Finite scores that are far apart: the greatest takes it all."""
    if dtype == "half" and abs(great) > 65504:
        pytest.skip("beyond half")
    p = Paged(15, [200, 40], 2, 1, 64, dtype)
    q = torch.zeros(2, 128, device="cuda", dtype=TDT[dtype])
    q[:, ::64] = great
    for t in range(200):
        x = less * (1 + t * 37 % 200 / 256)
        p.pool[int(p.table[p.sample[0], t // 16]), 1, 0, 0, t % 16, 0] = x
        p.k[0][t, 0, 0] = float(torch.tensor(x).to(TDT[dtype]))
    out = _np(p.run(100, 3, q=q, nsplit=nsplit))[0].reshape(2, 64)
    seen = np.r_[0:3, 100:200]
    score = p.k[0][seen, 0, 0] * np.sign(great)
    want = p.v[0][seen[score == score.max()], 0].mean(0)
    assert (np.abs(out - want) <= (HALF_STEP[dtype] + 8 * E) * np.abs(p.v[0][:, 0]).max(0)).all()


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("Hq,Hkv,hd", [(2, 2, 64), (4, 2, 128), (8, 1, 64), (16, 1, 128)])
def test_decode_in_float_is_as_near_as_float(four, Hq, Hkv, hd):
    """The bounds of _check add magnitudes; roundings add as random numbers do.  A score is a sum of some 16 partial sums, each off by up to a step (2 E) of
    at most 2 S here (codes v = u + 8 are summed, and 8 sum q taken off), so by some 4 * 2 E * 2 S = 16 E S where float products of hd terms in blocks are off by
    E S or so: 16 times the error of the same formula in float32, in the mean over all outputs, with 2^-22 for exp2 and the weights' terms."""
    p = Paged(16, [300, 33, 150], Hq, Hkv, hd, "fp32", four)
    out = _np(p.run(ALL, 0, nsplit=1)).reshape(3, Hq, hd)
    off, plain, size = 0.0, 0.0, 0.0
    for i, c in enumerate(p.ctx):
        q = _np(p.q[i]).reshape(1, Hq, hd)
        want = W.attention(q, p.k[i], p.v[i], np.array([c - 1]), ALL, 0)[0]
        kf, vf, qf = (torch.from_numpy(np.asarray(t, np.float32)) for t in (p.k[i].repeat(Hq // Hkv, 1), p.v[i].repeat(Hq // Hkv, 1), q[0]))
        w = torch.softmax((kf * qf[None]).sum(-1) / np.float32(np.sqrt(hd)), 0)
        off += ((out[i] - want) ** 2).sum()
        plain += (((w[..., None] * vf).sum(0).double().numpy() - want) ** 2).sum()
        size += (want ** 2).sum()
    assert np.sqrt(off) <= 16 * np.sqrt(plain) + 2.0 ** -22 * np.sqrt(size), (np.sqrt(off / size), np.sqrt(plain / size))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("Hq,Hkv,hd", [(2, 2, 64), (4, 2, 128), (8, 1, 64), (16, 1, 128)])
@pytest.mark.parametrize("dim", [4, 35])
def test_four_bits_scores_of_large_terms(dtype, Hq, Hkv, hd, dim):
    """One channel of query and key so large that its term M of a score is some thousands, the same in all scores.  Scores are float all the same.  In float32 the
    formula rounds some hd partial sums of about M; here it is hd / 32 sums of about 2 M (codes v = u + 8, whose 8 sum q comes off again), each of 32 terms that are
    cut off at a step of the greatest: 4 times that error, beside the roundings of 16-bit calls, which add as random numbers do: a weight times the scale of
    its token's values, 2^-11 of it, for the steps s u = v - c that it multiplies, and the output's own half step."""
    p = Paged(19, [300, 150], Hq, Hkv, hd, dtype, four=True)
    r = np.random.default_rng(20)
    q = r.normal(size=(2, Hq, hd))
    q[..., dim] = 100 * np.sign(q[..., dim])
    p.q = torch.from_numpy(q.reshape(2, -1)).to(TDT[dtype]).cuda()
    off, plain, rest, center = 0.0, 0.0, 0.0, []
    for i, n in enumerate(p.ctx):
        k = r.normal(size=(n, Hkv, hd)) * 10
        k[..., dim] = 400
        v = torch.from_numpy(r.normal(size=(n, Hkv, hd))).to(TDT[dtype])
        _hold(p, i, torch.from_numpy(k), v)
        center.append(np.repeat(W.kv4_quantize(v.float().numpy())[1][..., 1].astype(np.float64), 64, -1))
    out = _np(p.run(ALL, 0, nsplit=1)).reshape(2, Hq, hd)
    for i in range(2):
        q = _np(p.q[i]).reshape(Hq, hd)
        k, v, c = (t[i].repeat(Hq // Hkv, 1) for t in (p.k, p.v, center))
        z = (k * q).sum(-1) / np.sqrt(hd)
        w = np.exp(z - z.max(0))
        w /= w.sum(0)
        want = (w[..., None] * v).sum(0)
        kf, vf, qf = (torch.from_numpy(t.astype(np.float32)) for t in (k, v, q))
        wf = torch.softmax((kf * qf).sum(-1) / np.float32(np.sqrt(hd)), 0)
        off += ((out[i] - want) ** 2).sum()
        plain += (((wf[..., None] * vf).sum(0).double().numpy() - want) ** 2).sum()
        rest += ((ROUNDED[dtype] * w[..., None] * (v - c)) ** 2).sum() + (HALF_STEP[dtype] ** 2 * want ** 2).sum()
    assert np.sqrt(off) <= 4 * np.sqrt(plain) + np.sqrt(rest), (np.sqrt(off), np.sqrt(plain), np.sqrt(rest))


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
@pytest.mark.parametrize("nsplit", [1, 3])
def test_decode_strided_and_on_a_stream(four, nsplit):
    p = Paged(9, [40, 300, 0], 2, 2, 64, "half", four)
    want = p.run(50, 3, nsplit=nsplit)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q, o = torch.full((6, 136), float("nan"), device="cuda", dtype=torch.half), torch.full((3, 152), 7.0, device="cuda", dtype=torch.half)
        q[::2, :128] = p.q
        scratch = torch.full((_R().lib().rlhf_op_window_decode_scratch_floats(3, 2, 64, nsplit) + 8,), float("nan"), device="cuda")
        p.run(50, 3, q=q[::2, :128], out=o[:, 8:136], nsplit=nsplit, scratch=scratch)
    s.synchronize()
    assert torch.equal(o[:, 8:136], want) and (o[:, :8] == 7).all() and (o[:, 136:] == 7).all()
    assert torch.isnan(scratch[-8:]).all()


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
def test_decode_numbers_that_do_not_fit_an_argument(four):
    """A layer or number of parts of 2^32 and one is not taken for one, and parts that no call takes need no scratch first."""
    R = _R()
    p = Paged(25, [40, 3], 2, 2, 64, "half", four)
    for bad in (dict(nsplit=2 ** 32 + 1), dict(nsplit=2 ** 32 + 2), dict(nsplit=65), dict(nsplit=2 ** 31 - 1), dict(nsplit=0), dict(nsplit=-1), dict(nsplit=-2 ** 32 + 1)):
        with pytest.raises(R.RlhfError):
            p.run(ALL, 0, **bad)
    for bad in (2 ** 32 + 1, -2 ** 32 + 1, 3, -1):
        p.layer = bad
        with pytest.raises(R.RlhfError):
            p.run(ALL, 0)
        if four:
            k, v = (torch.zeros(2, 128, device="cuda", dtype=torch.half) for _ in range(2))
            with pytest.raises(R.RlhfError):
                R.rlhf_op_kv4_append(k, v, _ints([0, 1]), p.pool, bad, 3, 2, 64)
            with pytest.raises(R.RlhfError):
                R.rlhf_op_kv4_read(p.pool, _ints([0, 1]), k, v, bad, 3, 2, 64)
    torch.cuda.synchronize()


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
def test_decode_offsets_beyond_32_bits(four):
    """The last pages of a pool of more than 2^32 elements (2^33 bytes; of 4 bits 2^32 + bytes)."""
    R = _R()
    Hkv, hd, layers = 8, 128, 64
    page = R.rlhf_op_kv4_page_bytes(layers, Hkv, hd) if four else layers * 2 * Hkv * 16 * hd
    n_pages = ((1 << 32) + (1 << 28)) // page + 2
    p = Paged(10, [40, 17], 8, Hkv, hd, "half", four)
    pool = torch.empty(n_pages * page, dtype=torch.uint8 if four else torch.half, device="cuda")
    shape = (n_pages, layers, Hkv, 18 * hd) if four else (n_pages, layers, 2, Hkv, 16, hd)
    pool = pool.view(shape)
    pool[n_pages - p.n_pages:, layers - 1] = p.pool[:, p.layer]
    p.pool, p.layers, p.layer = pool, layers, layers - 1
    p.table_d += n_pages - p.n_pages
    p.check(p.run(30, 1), 30, 1)
    if four:
        slots = _ints([(n_pages - 1) * 16 + 15, (n_pages - 2) * 16])
        k, v = _normal(np.random.default_rng(0), 2, Hkv * hd).cuda(), _normal(np.random.default_rng(1), 2, Hkv * hd).cuda()
        R.rlhf_op_kv4_append(k, v, slots, pool, layers - 1, layers, Hkv, hd)
        rk, rv = torch.empty_like(k), torch.empty_like(v)
        R.rlhf_op_kv4_read(pool, slots, rk, rv, layers - 1, layers, Hkv, hd)
        np.testing.assert_array_equal(_np(rk), W.kv4_round(k.cpu().numpy().reshape(2, Hkv, hd)).reshape(2, -1).astype(np.float32))
        np.testing.assert_array_equal(_np(rv), W.kv4_round(v.cpu().numpy().reshape(2, Hkv, hd)).reshape(2, -1).astype(np.float32))


# ------------------------------------------------------------------------------------------------ cache of 4 bits

def _blocks(k, v, Hkv, hd, slots, n_pages, layers, layer, start):
    want = start.copy()
    for i, s in enumerate(slots):
        if 0 <= s < 16 * n_pages:
            for h in range(Hkv):
                W.kv4_write(want[s // 16, layer, h], s % 16, k[i, h], v[i, h])
    return want


def _append_case(seed, rows, Hkv, hd, dtype, n_pages):
    r = np.random.default_rng(seed)
    k, v = _normal(r, rows, Hkv, hd, dtype=dtype), _normal(r, rows, Hkv, hd, dtype=dtype, std=5.0)
    start = r.integers(0, 256, (n_pages, 2, Hkv, 18 * hd)).astype(np.uint8)
    return r, k, v, start


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
@pytest.mark.parametrize("rows,Hkv,hd", [(1, 1, 64), (5, 3, 64), (37, 2, 128), (16, 1, 128), (100, 1, 64)])
def test_append_writes_its_tokens_and_nothing_else(dtype, rows, Hkv, hd):
    """Bytes equal to the oracle's, in a pool that held other bytes; slots out of order, some left out."""
    R, n_pages = _R(), 9
    r, k, v, start = _append_case(rows + hd, rows, Hkv, hd, dtype, n_pages)
    slots = r.permutation(16 * n_pages)[:rows]
    if rows >= 5:
        slots[1], slots[3], slots[4] = -1, 16 * n_pages, 2 ** 31 - 1
    pool = torch.from_numpy(start).cuda()
    R.rlhf_op_kv4_append(k.cuda().flatten(1), v.cuda().flatten(1), _ints(slots.tolist()), pool, 1, 2, Hkv, hd)
    want = _blocks(k.float().numpy(), v.float().numpy(), Hkv, hd, slots, n_pages, 2, 1, start)
    np.testing.assert_array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_append_in_order(dtype):
    """Whole pages, and pages that a sequence enters and leaves in the middle."""
    R, n_pages, rows = _R(), 5, 52
    r, k, v, start = _append_case(3, rows, 2, 64, dtype, n_pages)
    for first in (0, 5, 16, 28):
        pool = torch.from_numpy(start).cuda()
        slots = list(range(first, first + rows))
        R.rlhf_op_kv4_append(k.cuda().flatten(1), v.cuda().flatten(1), _ints(slots), pool, 0, 2, 2, 64)
        np.testing.assert_array_equal(pool.cpu().numpy(), _blocks(k.float().numpy(), v.float().numpy(), 2, 64, slots, n_pages, 2, 0, start))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_append_values_at_the_edges_of_the_rounding(dtype):
    """Groups of one value, of two, of whole steps and halves between them, tiny, huge, far from zero, not finite."""
    R, r, hd = _R(), np.random.default_rng(5), 128
    t = TDT[dtype]
    groups = [np.zeros(64), np.full(64, -0.0), np.full(64, 3.7), np.r_[np.full(63, -1.0), 2.0], np.tile(np.arange(16.0) - 3, 4), np.tile(np.arange(32) / 2.0, 2),
              np.tile(np.arange(31) * 0.0625, 3)[:64], r.normal(size=64) * 1e-4, r.normal(size=64) * 1e-7, np.tile([5e-8, 0.0], 32), r.normal(size=64) * 1e4,
              100 + r.normal(size=64) * 1e-3, np.r_[np.full(32, 65504.0), np.full(32, -65504.0)], np.r_[np.nan, np.zeros(63)], np.r_[np.zeros(63), np.inf],
              np.r_[-np.inf, np.ones(63)], np.tile(np.arange(16.0), 4) * 2.0 ** -20, r.integers(-20, 21, 64) / 8.0, r.integers(-7, 9, 64) * 1.0, np.full(64, 1e-7)]
    if dtype != "half":
        groups += [np.r_[np.ones(63), 65600.0], np.r_[np.ones(63), -1e30], r.normal(size=64) * 1e-12]
    groups += [r.integers(-60, 61, 64) / 4.0 for _ in range(8 + len(groups) % 2)]
    x = torch.from_numpy(np.stack(groups).reshape(-1, 2 * 64).astype(np.float32)).to(t)
    rows = x.shape[0]
    n_pages = -(-rows // 16)
    start = np.zeros((n_pages, 2, 1, 18 * hd), np.uint8)
    pool = torch.from_numpy(start).cuda()
    v = x.flip(0)
    R.rlhf_op_kv4_append(x.cuda(), v.cuda(), _ints(list(range(rows))), pool, 1, 2, 1, hd)
    k_oracle, v_oracle = x.float().numpy()[:, None], v.float().numpy()[:, None]
    want = _blocks(k_oracle, v_oracle, 1, hd, range(rows), n_pages, 2, 1, start)
    got = pool.cpu().numpy()
    half = lambda a: a.view(np.float16)[..., 8 * hd:]
    np.testing.assert_array_equal(half(got), half(want))                 # a NaN for a NaN
    np.testing.assert_array_equal(got[..., :16 * hd], want[..., :16 * hd])
    out = [torch.empty(rows, hd, device="cuda") for _ in range(2)]
    R.rlhf_op_kv4_read(pool, _ints(list(range(rows))), *out, 1, 2, 1, hd)
    np.testing.assert_array_equal(_np(out[0]), W.kv4_round(k_oracle)[:, 0].astype(np.float32))
    np.testing.assert_array_equal(_np(out[1]), W.kv4_round(v_oracle)[:, 0].astype(np.float32))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_values_next_to_the_end_of_half(dtype):
    """The nearest step to 65504 may lie at 65536 and more: read back into half, or averaged by decode attention there, it is 65504 and no infinity.  (The other types
    hold it.)"""
    R, hd, r = _R(), 64, np.random.default_rng(24)
    x = np.stack([np.r_[np.full(32, 65504.0), np.full(32, -65504.0)], np.r_[np.full(63, 65504.0), 64000.0], np.r_[np.full(63, -65504.0), 65000.0], np.r_[np.full(63, 65504.0), -60000.0],
                  *np.clip(r.uniform(-1.1, 1.1, (12, 64)), -1, 1) * 65504])
    t = torch.from_numpy(x.astype(np.float32)).to(TDT["half"])
    held = W.kv4_round(t.float().numpy())
    assert (np.abs(held) > 65519).sum() > 100                           # would round to infinity
    pool = torch.zeros(1, 1, 1, 18 * hd, dtype=torch.uint8, device="cuda")
    slots = _ints(list(range(16)))
    R.rlhf_op_kv4_append(t.cuda(), t.cuda(), slots, pool, 0, 1, 1, hd)
    want = torch.from_numpy(held).to(TDT[dtype])
    if dtype == "half":
        want = want.clamp(-65504, 65504)
    out = torch.empty(2, 16, hd, device="cuda", dtype=TDT[dtype])
    R.rlhf_op_kv4_read(pool, slots, out[0], out[1], 0, 1, 1, hd)
    assert torch.equal(out[0].cpu(), want) and torch.equal(out[1].cpu(), want)
    q, o = torch.zeros(16, hd, device="cuda", dtype=TDT[dtype]), torch.empty(16, hd, device="cuda", dtype=TDT[dtype])
    for nsplit in (1, 2):                                                # row i sees token i alone
        R.rlhf_op_kv4_decode_attention(q, pool, _ints([[0]]), _ints([0] * 16), _ints(list(range(1, 17))), o, 0, 1, 1, 1, hd, 1, 0, nsplit=nsplit)
        assert torch.isfinite(o).all()
        off = np.abs(_np(o) - _np(want))
        assert (off <= (HALF_STEP[dtype] + ROUNDED[dtype] + 8 * E) * 2 * np.abs(held).max(1, keepdims=True)).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_codes_of_many_values(dtype):
    """A million values on a coarse grid, where exact halves between steps are frequent, and as many off it."""
    R, hd, Hkv, rows = _R(), 64, 16, 512
    r = np.random.default_rng(6)
    x = torch.from_numpy((r.integers(-120, 121, (rows, Hkv * hd)) / 8.0).astype(np.float32)).to(TDT[dtype])
    y = _normal(r, rows, Hkv * hd, dtype=dtype)
    pool = torch.zeros(rows // 16, 1, Hkv, 18 * hd, dtype=torch.uint8, device="cuda")
    slots = _ints(r.permutation(rows).tolist())
    R.rlhf_op_kv4_append(x.cuda(), y.cuda(), slots, pool, 0, 1, Hkv, hd)
    out = [torch.empty(rows, Hkv * hd, device="cuda") for _ in range(2)]
    R.rlhf_op_kv4_read(pool, slots, *out, 0, 1, Hkv, hd)
    for got, t in zip(out, (x, y)):
        np.testing.assert_array_equal(_np(got), W.kv4_round(t.float().numpy()).astype(np.float32))


def test_scale_and_center_are_rounded_to_float_and_then_to_half():
    """Groups whose scale or center would be another half if it were rounded once."""
    R, r, hd = _R(), np.random.default_rng(8), 64
    lo = (-r.uniform(1, 4, 400000)).astype(np.float32)
    hi = r.uniform(1, 4, 400000).astype(np.float32)
    third = np.float32(np.float32(1) / np.float32(15))
    f = (hi - lo) * third
    s = f.astype(np.float16)
    once = ((hi - lo).astype(np.float64) * np.float64(third)).astype(np.float16) != s
    c = (lo + np.float32(8) * s.astype(np.float32)).astype(np.float16)
    once |= (lo.astype(np.float64) + 8 * s.astype(np.float64)).astype(np.float16) != c
    lo, hi = lo[once], hi[once]
    assert len(lo) >= 16
    rows = len(lo) // 16 * 16
    x = r.uniform(-1, 1, (rows, hd)).astype(np.float32)
    x[:, 5], x[:, 40] = lo[:rows], hi[:rows]
    pool = torch.zeros(rows // 16, 1, 1, 18 * hd, dtype=torch.uint8, device="cuda")
    t = torch.from_numpy(x).cuda()
    R.rlhf_op_kv4_append(t, -t, _ints(list(range(rows))), pool, 0, 1, 1, hd)
    out = [torch.empty(rows, hd, device="cuda") for _ in range(2)]
    R.rlhf_op_kv4_read(pool, _ints(list(range(rows))), *out, 0, 1, 1, hd)
    np.testing.assert_array_equal(_np(out[0]), W.kv4_round(x).astype(np.float32))
    np.testing.assert_array_equal(_np(out[1]), W.kv4_round(-x).astype(np.float32))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "half"])
def test_read(dtype):
    """Any slots, some twice, into strided rows; zeros for a negative slot, NaN beyond the pool; one rounding."""
    R, r, hd, Hkv, n_pages = _R(), np.random.default_rng(7), 128, 3, 6
    pool = r.integers(0, 256, (n_pages, 2, Hkv, 18 * hd)).astype(np.uint8)
    pool.view(np.float16)[..., 8 * hd:] = r.normal(size=(n_pages, 2, Hkv, hd)).astype(np.float16)
    slots = [5, 95, -1, 0, 5, 96, 17, -2 ** 31, 2 ** 31 - 1, 16]
    k, v = (torch.full((len(slots), Hkv * hd + 16), 7.0, device="cuda", dtype=TDT[dtype]) for _ in range(2))
    R.rlhf_op_kv4_read(torch.from_numpy(pool).cuda(), _ints(slots), k[:, 8:8 + Hkv * hd], v[:, :Hkv * hd], 1, 2, Hkv, hd)
    for i, s in enumerate(slots):
        for h in range(Hkv):
            want = [np.zeros(hd)] * 2 if s < 0 else [np.full(hd, np.nan)] * 2 if s >= 96 else [a[s % 16] for a in W.kv4_block_values(pool[s // 16, 1, h], hd)]
            for t, at, w in ((k, 8, want[0]), (v, 0, want[1])):
                # c + s u is exact in float but where the halves are more than 2^9 apart: one rounding there, one to the type
                np.testing.assert_allclose(_np(t[i, at + h * hd:at + (h + 1) * hd]), w, rtol=HALF_STEP[dtype] + 1e-7, atol=1e-7)
    assert (k[:, :8] == 7).all() and (k[:, -8:] == 7).all() and (v[:, Hkv * hd:] == 7).all()


def test_append_and_read_strided():
    R, hd, Hkv, rows = _R(), 64, 2, 40
    q, k, v = _packed(11, [rows], 4, Hkv, hd, "bf16", pad=8)
    pools = [torch.zeros(3, 1, Hkv, 18 * hd, dtype=torch.uint8, device="cuda") for _ in range(2)]
    slots = _ints(list(range(rows)))
    R.rlhf_op_kv4_append(k, v, slots, pools[0], 0, 1, Hkv, hd)
    R.rlhf_op_kv4_append(k.contiguous(), v.contiguous(), slots, pools[1], 0, 1, Hkv, hd)
    assert torch.equal(*pools)


# ------------------------------------------------------------------------------------------------ launches in turns

MANY = 1 << 16                                                           # heads, the most that a call takes: few rows of them fill a launch of 2^32 threads


@pytest.mark.parametrize("dtype,rows", [("half", 260), ("fp32", 130)])
def test_packed_in_turns(dtype, rows):
    """Sequences of one token, more than one launch has workgroups for (half: 248 tiles; float: 120): every output is its token's V."""
    hd, r = 64, np.random.default_rng(27)
    k, v = (_normal(r, rows, hd, dtype=dtype).cuda() for _ in range(2))
    q = torch.empty(rows, MANY * hd, device="cuda", dtype=TDT[dtype]).normal_()
    out = _packed_run(q, k, v, [1] * rows, 1, 0, MANY, 1, hd)
    off = (out.view(rows, MANY, hd) - v[:, None]).abs_().amax(1)
    assert (off <= (0 if dtype == "half" else 4 * E) * v.abs()).all()
    del q, out, off
    torch.cuda.empty_cache()


@pytest.mark.parametrize("four,dtype,rows,width,nsplit", [(False, "half", 10, 4, 32), (True, "half", 10, 4, 32), (True, "fp32", 10, 4, 32), (False, "half", 130, 64, 1)])
def test_decode_in_turns(four, dtype, rows, width, nsplit):
    """More rows than one launch has workgroups for (in 32 parts: 3 rows, over 4 bits 7; in one part 127): every row as in a call of its own, which is one launch, and
    some heads against float64."""
    R, hd, r = _R(), 64, np.random.default_rng(28)
    pages, window = 3, 20 if nsplit > 1 else ALL
    g = torch.Generator(device="cuda").manual_seed(29)
    k, v = (torch.empty(16 * pages, MANY * hd, device="cuda", dtype=torch.half).normal_(generator=g) for _ in range(2))
    if four:
        pool = torch.zeros(pages, 1, MANY, 18 * hd, dtype=torch.uint8, device="cuda")
        R.rlhf_op_kv4_append(k, v, _ints(list(range(16 * pages))), pool, 0, 1, MANY, hd)
    else:
        put = lambda t: t.view(pages, 16, MANY, hd).transpose(1, 2)
        pool = torch.stack([put(k), put(v)], 1)[:, None].contiguous().to(TDT[dtype])
    q = torch.empty(rows, MANY * hd, device="cuda", dtype=TDT[dtype]).normal_(generator=g)
    table = torch.full((1, width), -1, dtype=torch.int32)
    table[0, :pages] = torch.tensor([0, 1, 2])
    table, ctx = table.cuda(), r.integers(1, 16 * pages + 1, rows)
    ctx[rows // 2] = 0
    call = R.rlhf_op_kv4_decode_attention if four else R.rlhf_op_window_decode_attention
    run = lambda a, b, o: call(q[a:b], pool, table, _ints([0] * (b - a)), _ints(ctx[a:b].tolist()), o, 0, 1, MANY, MANY, hd, window, 3, nsplit=nsplit)
    out, one = torch.full_like(q, 7.0), torch.empty_like(q[:1])
    run(0, rows, out)
    for i in range(rows):
        run(i, i + 1, one)
        assert torch.equal(out[i], one[0]), i
    heads = [0, 1, 40000, MANY - 1]
    some = lambda t, n: _np(t.view(n, MANY, hd)[:, heads])
    kk, vv = (some(t, 16 * pages) for t in (k, v))
    size = [None, None]
    if four:
        size = [np.repeat(np.abs(W.kv4_quantize(t.astype(np.float32))[1].astype(np.float64)) @ np.array([8.0, 1.0]), 64, -1) for t in (kk, vv)]
        kk, vv = (W.kv4_round(t.astype(np.float32)) for t in (kk, vv))
    for i in (0, 2, 3, 6, 7, rows - 1):
        n = int(ctx[i])
        if n:
            _check(some(out[i:i + 1], 1), some(q[i:i + 1], 1), kk[:n], vv[:n], np.array([n - 1]), window, 3, dtype, *(t if t is None else t[:n] for t in size))
        else:
            assert (out[i] == 0).all()
    del k, v, pool, q, out, one
    torch.cuda.empty_cache()


def test_append_in_turns():
    """8188 rows of 65536 heads, of which one launch has waves for 8184; all but a few are left out."""
    R, hd, rows = _R(), 64, 8188
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("rows of 69 GB")
    x = torch.empty(rows, MANY * hd, device="cuda", dtype=torch.half)
    at = [0, 8183, 8184, rows - 1]
    slots = torch.full((rows,), -1, dtype=torch.int32)
    for i, row in enumerate(at):
        x[row] = torch.randn(MANY * hd, device="cuda")
        slots[row] = 3 * i + 1
    pool = torch.zeros(1, 1, MANY, 18 * hd, dtype=torch.uint8, device="cuda")
    other = pool.clone()
    R.rlhf_op_kv4_append(x, x, slots.cuda(), pool, 0, 1, MANY, hd)
    few = x[at].contiguous()
    del x
    torch.cuda.empty_cache()
    R.rlhf_op_kv4_append(few, few, _ints([1, 4, 7, 10]), other, 0, 1, MANY, hd)
    assert torch.equal(pool, other) and pool.any()


# ------------------------------------------------------------------------------------------------ together

def test_a_prompt_and_decode_steps():
    """A prompt by packed attention, its K and V into both caches, then steps that append a token and attend, all through a window
    that moves past the prompt; against float64 over the same keys."""
    R = _R()
    Hq, Hkv, hd, lens, window, sinks, steps = 4, 2, 64, [35, 20], 24, 3, 30
    q, k, v = _packed(12, lens, Hq, Hkv, hd, "half")
    _packed_check(_packed_run(q, k, v, lens, window, sinks, Hq, Hkv, hd), q, k, v, lens, window, sinks, Hq, Hkv, hd, "half")
    width = 6
    table = _ints(np.random.default_rng(0).permutation(2 * width).reshape(2, width).tolist())
    pool = torch.full((2 * width, 1, 2, Hkv, 16, hd), float("nan"), device="cuda", dtype=torch.half)
    pool4 = torch.full((2 * width, 1, Hkv, 18 * hd), 255, dtype=torch.uint8, device="cuda")
    slot = lambda s, t: int(table[s, t // 16]) * 16 + t % 16

    def put(kk, vv, slots):
        R.rlhf_op_kv4_append(kk, vv, _ints(slots), pool4, 0, 1, Hkv, hd)
        for i, s in enumerate(slots):
            pool[s // 16, 0, 0, :, s % 16], pool[s // 16, 0, 1, :, s % 16] = kk[i].view(Hkv, hd), vv[i].view(Hkv, hd)

    put(k, v, [slot(s, t) for s in range(2) for t in range(lens[s])])
    keys = [[_np(k[:35]), _np(v[:35])], [_np(k[35:]), _np(v[35:])]]
    r, row = np.random.default_rng(13), _ints([1, 0])
    for step in range(steps):
        nq, nk, nv = (_normal(r, 2, h * hd, dtype="half").cuda() for h in (Hq, Hkv, Hkv))
        ctx = [n + step + 1 for n in lens]
        put(nk, nv, [slot(s, ctx[s] - 1) for s in range(2)])
        outs = [torch.empty_like(nq) for _ in range(2)]
        args = (table, row, _ints([ctx[1], ctx[0]]))
        rows = nq.flip(0).contiguous()
        R.rlhf_op_window_decode_attention(rows, pool, *args, outs[0], 0, 1, Hq, Hkv, hd, window, sinks, max_ctx=max(ctx))
        R.rlhf_op_kv4_decode_attention(rows, pool4, *args, outs[1], 0, 1, Hq, Hkv, hd, window, sinks, max_ctx=max(ctx))
        for s in range(2):
            keys[s] = [np.concatenate([a, _np(t[s:s + 1])]) for a, t in zip(keys[s], (nk, nv))]
            kk, vv = (a.reshape(-1, Hkv, hd) for a in keys[s])
            qq, pos = _np(nq[s]).reshape(1, Hq, hd), np.array([ctx[s] - 1])
            _check(_np(outs[0][1 - s]).reshape(1, Hq, hd), qq, kk, vv, pos, window, sinks, "half")
            k4, v4 = W.kv4_round(kk.astype(np.float32)), W.kv4_round(vv.astype(np.float32))
            size = lambda a: np.repeat(np.abs(W.kv4_quantize(a.astype(np.float32))[1].astype(np.float64)) @ np.array([8.0, 1.0]), 64, -1)
            _check(_np(outs[1][1 - s]).reshape(1, Hq, hd), qq, k4, v4, pos, window, sinks, "half", size(kk), size(vv))


@pytest.mark.parametrize("nsplit", [1, 3])
def test_captured_and_replayed(nsplit):
    """Append and both decode attentions in one graph, replayed on new tokens with eager work in between; and two graphs, each with
    a scratch of its own."""
    R = _R()
    p = Paged(14, [100, 40], 4, 2, 64, "half", True)
    p16 = Paged(14, [100, 40], 4, 2, 64, "half", False)
    k, v = torch.zeros(2, 128, device="cuda", dtype=torch.half), torch.zeros(2, 128, device="cuda", dtype=torch.half)
    slots = _ints([int(p.table[p.sample[i], (c - 1) // 16]) * 16 + (c - 1) % 16 for i, c in enumerate(p.ctx)])
    scratch = [torch.empty(R.lib().rlhf_op_window_decode_scratch_floats(2, 4, 64, nsplit), device="cuda") if nsplit > 1 else None for _ in range(4)]
    outs = [torch.zeros_like(p.q) for _ in range(4)]

    def work(i):
        R.rlhf_op_kv4_append(k, v, slots, p.pool, 1, 3, 2, 64)
        for j, x in ((i, p), (i + 1, p16)):
            call = R.rlhf_op_kv4_decode_attention if x.four else R.rlhf_op_window_decode_attention
            call(x.q, x.pool, x.table_d, x.row_d, x.ctx_d, outs[j], 1, 3, 4, 2, 64, 50, 2, nsplit=nsplit, scratch=scratch[j])

    graphs = []
    for i in (0, 2):
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            work(i)
        torch.cuda.current_stream().wait_stream(side)
        with torch.cuda.graph(g):
            work(i)
        graphs.append(g)
    for step in range(4):
        r = np.random.default_rng(step)
        k.copy_(_normal(r, 2, 128, dtype="half")), v.copy_(_normal(r, 2, 128, dtype="half"))
        p.q.copy_(_normal(r, 2, 256, dtype="half", std=2.0)), p16.q.copy_(p.q)
        for o in outs:
            o.fill_(7.0)
        graphs[step % 2].replay()
        graphs[1 - step % 2].replay()
        torch.cuda.synchronize()
        a, b = p.run(50, 2, nsplit=nsplit), p16.run(50, 2, nsplit=nsplit)
        assert torch.equal(outs[0], a) and torch.equal(outs[2], a) and torch.equal(outs[1], b) and torch.equal(outs[3], b)
        last = torch.empty(2, 128, device="cuda", dtype=torch.half)
        R.rlhf_op_kv4_read(p.pool, slots, last, torch.empty_like(last), 1, 3, 2, 64)
        np.testing.assert_array_equal(_np(last), _np(torch.from_numpy(W.kv4_round(k.float().cpu().numpy().reshape(2, 2, 64)).reshape(2, 128)).half()))


def test_calls_on_two_streams_at_once():
    """Split decode steps of both caches, whose scratch the binding takes, and packed passes, side by side on two streams: as one after the other."""
    ps = [Paged(31 + i, [900, 1200, 64], 8, 2, 128, "half", i == 1) for i in range(2)]
    lens = [700, 33]
    packed = _packed(33, lens, 4, 2, 64, "bf16")
    want = [p.run(ALL, 0, nsplit=8) for p in ps] + [_packed_run(*packed, lens, 60, 2, 4, 2, 64)]
    R = _R()
    tiles, streams = R.rlhf_attention_tiles(lens), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for turn in range(6):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                for j in (turn + i) % 3, (turn + i + 1) % 3:
                    o = torch.full_like(want[j], 7.0)
                    if j == 2:
                        R.rlhf_op_window_attention(*packed, tiles, o, 60, 2, 4, 2, 64)
                    else:
                        p = ps[j]
                        call = R.rlhf_op_kv4_decode_attention if p.four else R.rlhf_op_window_decode_attention
                        call(p.q, p.pool, p.table_d, p.row_d, p.ctx_d, o, p.layer, p.layers, 8, 2, 128, nsplit=8)
                    outs.append((j, o))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[j]) for j, o in outs)


def test_packed_captured_and_replayed():
    R = _R()
    lens = [150, 33]
    q, k, v = _packed(15, lens, 4, 2, 64, "bf16")
    tiles, out = R.rlhf_attention_tiles(lens), torch.zeros(183, 256, device="cuda", dtype=torch.bfloat16)
    R.rlhf_op_window_attention(q, k, v, tiles, out, 60, 2, 4, 2, 64)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.rlhf_op_window_attention(q, k, v, tiles, out, 60, 2, 4, 2, 64)
    for step in range(3):
        q.copy_(torch.randn(q.shape, device="cuda"))
        out.fill_(7.0)
        g.replay()
        assert torch.equal(out, _packed_run(q, k, v, lens, 60, 2, 4, 2, 64))


def test_same_call_same_bits():
    for four in (False, True):
        p = Paged(16, [900, 1200, 64], 8, 2, 128, "bf16", four)
        a = p.run(ALL, 0, nsplit=5)
        for _ in range(3):
            assert torch.equal(p.run(ALL, 0, nsplit=5), a)


# ------------------------------------------------------------------------------------------------ refusals that need tensors of a device

BAD_MATRICES = {"fewer rows": lambda t: t[:-1], "fewer columns": lambda t: t[:, :-8], "flat": lambda t: t.flatten(), "more dims": lambda t: t[None], "columns apart": lambda t: t.t().contiguous().t(),
                "rows that overlap": lambda t: t[:1].expand(t.shape), "rows closer than their length": lambda t: t.as_strided(t.shape, (t.shape[1] - 8, 1)),
                "half": lambda t: t.half(), "host": lambda t: t.cpu()}
BAD_VECTORS = {"int64": lambda t: t.long(), "fewer": lambda t: t[:-1], "apart": lambda t: t.repeat_interleave(2)[::2], "float": lambda t: t.float(), "host": lambda t: t.cpu()}


def _refused(args, at, bad, call):
    args = list(args)
    args[at] = bad(args[at])
    with pytest.raises(ValueError):
        call(*args)


@pytest.mark.parametrize("bad", BAD_MATRICES)
def test_matrices_that_are_refused(bad):
    R = _R()
    f = BAD_MATRICES[bad]
    q, k, v, o = (torch.zeros(6, 128, device="cuda") for _ in range(4))
    tiles = R.rlhf_attention_tiles([4, 1])
    for at in (1, 2, 3) if bad == "fewer rows" else (0, 1, 2, 3):       # rows of q are those of the call
        _refused((q, k, v, o), at, f, lambda q, k, v, o: R.rlhf_op_window_attention(q, k, v, tiles, o, 8, 0, 2, 2, 64))
    pool, four, i = torch.zeros(2, 1, 2, 2, 16, 64, device="cuda"), torch.zeros(2, 2, 18 * 64, device="cuda", dtype=torch.uint8), _ints([0] * 6)
    for name, p in (("rlhf_op_window_decode_attention", pool), ("rlhf_op_kv4_decode_attention", four)):
        for at in (0, 1):
            _refused((q, o), at, f, lambda q, o: getattr(R, name)(q, p, i[None].contiguous(), i, i, o, 0, 1, 2, 2, 64))
    for at in (0, 1):
        _refused((k, v), at, f, lambda k, v: R.rlhf_op_kv4_append(k, v, i, four, 0, 1, 2, 64))
        _refused((k, v), at, f, lambda k, v: R.rlhf_op_kv4_read(four, i, k, v, 0, 1, 2, 64))


@pytest.mark.parametrize("bad", BAD_VECTORS)
def test_vectors_that_are_refused(bad):
    R = _R()
    f = BAD_VECTORS[bad]
    q, k, o = (torch.zeros(6, 128, device="cuda") for _ in range(3))
    pool, four, i = torch.zeros(2, 1, 2, 2, 16, 64, device="cuda"), torch.zeros(2, 2, 18 * 64, device="cuda", dtype=torch.uint8), _ints([0] * 6)
    for name, p in (("rlhf_op_window_decode_attention", pool), ("rlhf_op_kv4_decode_attention", four)):
        for at in (0, 1):
            _refused((i, i), at, f, lambda row, ctx: getattr(R, name)(q, p, _ints([[0, 1]]), row, ctx, o, 0, 1, 2, 2, 64))
    if bad != "fewer":                                                  # as many rows as slots: then k has too many
        _refused((i,), 0, f, lambda s: R.rlhf_op_kv4_append(q, k, s, four, 0, 1, 2, 64))
        _refused((i,), 0, f, lambda s: R.rlhf_op_kv4_read(four, s, q, k, 0, 1, 2, 64))


@pytest.mark.parametrize("four", [False, True], ids=["paged", "four_bits"])
def test_tables_and_scratch_that_are_refused(four):
    R = _R()
    p = Paged(26, [40, 3], 2, 2, 64, "half", four)
    table = p.table_d
    for bad in (table.long(), table.flatten(), table.t(), table[None], table.cpu()):
        p.table_d = bad
        with pytest.raises(ValueError):
            p.run(ALL, 0)
    p.table_d = table
    need = R.lib().rlhf_op_window_decode_scratch_floats(2, 2, 64, 3)
    for bad in (torch.empty(need - 1, device="cuda"), torch.empty(need, device="cuda", dtype=torch.half), torch.empty(2 * need, device="cuda")[::2], torch.empty(need)):
        with pytest.raises(ValueError):
            p.run(ALL, 0, nsplit=3, scratch=bad)
    with pytest.raises(R.RlhfError):                                    # not at 16 bytes
        p.run(ALL, 0, nsplit=3, scratch=torch.empty(need + 4, device="cuda")[1:])
    whole = p.run(ALL, 0, nsplit=3, scratch=torch.empty(need, device="cuda"))
    assert torch.equal(whole, p.run(ALL, 0, nsplit=3))
