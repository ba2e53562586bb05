"""GPU parity of prism_cache_attn against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2602_08426_amd import binding as pb
from tests import serving_util as su

pytestmark = pytest.mark.gpu


class Case:
    """A cache with garbage (NaN) wherever no token lies, a batch and its queries, on the host and on the device."""

    def __init__(self, seed, h, h_kv, d, page, e4m3, lengths, news, behind=0, how="dense", peaked=False, odd_scales=False, wider=1):
        rng = np.random.default_rng(seed)
        self.lengths, self.cu = list(lengths), np.concatenate([[0], np.cumsum(news)]).astype(int)
        self.news, self.rows, self.e4m3 = list(news), int(self.cu[-1]) + behind, e4m3
        self.h, self.h_kv, self.d, self.page = h, h_kv, d, page
        self.table, self.n_pages = su.make_table(rng, lengths, page, wider=wider)
        shape = (self.n_pages, h_kv, page, d)
        k, v = rng.standard_normal(shape) * np.exp(0.4 * rng.standard_normal((1, h_kv, 1, d))), rng.standard_normal(shape)
        self.q = su.bf16(rng.standard_normal((h, self.rows, d)) * (3.0 if peaked else 1.2))
        live = np.zeros((self.n_pages, page), bool)
        for s, n in enumerate(lengths):
            for b in range(-(-max(n, 0) // page)):
                live[self.table[s, b], :min(page, n - b * page)] = True
        if e4m3:
            self.ks, self.vs = (2.0 ** rng.integers(-8, 3, shape[:2]) * (rng.uniform(1, 2, shape[:2]) if odd_scales else 1.0) for _ in range(2))
            self.ks, self.vs = (x.astype(np.float32).astype(np.float64) for x in (self.ks, self.vs))
            k8, v8 = so.to_e4m3(np.clip(k / self.ks[..., None, None], -448, 448)), so.to_e4m3(np.clip(v / self.vs[..., None, None], -448, 448))
            self.k, self.v = k8 * self.ks[..., None, None], v8 * self.vs[..., None, None]
        else:
            k8, v8 = self.k, self.v = su.bf16(k), su.bf16(v)
            self.ks = self.vs = None
        dead = np.broadcast_to(~live[:, None, :, None], shape)
        to = su.e4m3_to_device if e4m3 else su.to_device
        self.kd, self.vd = to(np.where(dead, np.nan, k8)), to(np.where(dead, np.nan, v8))
        self.ksd, self.vsd = ((torch.from_numpy(x.astype(np.float32)).cuda() if e4m3 else None) for x in (self.ks, self.vs))
        self.qd = su.layout_of(su.to_device(self.q), how)
        self.how = how

    def batch(self, uniform=False):
        cu = None if uniform else su.ints(self.cu)
        return pb.make_batch(su.ints(self.lengths), su.ints(self.table), max(max(self.news), 1), cu, self.rows)

    def run(self, window=0, sinks=0, scale=0.0, lse=True, uniform=False, workspace=None, in_place=False):
        cache, batch = pb.make_cache(self.kd, self.vd, self.ksd, self.vsd), self.batch(uniform)
        out = self.qd if in_place else su.layout_of(torch.full((self.h, self.rows, self.d), 7.0, dtype=torch.bfloat16, device="cuda"), self.how)
        sums = torch.full((self.h, self.rows), 7.0, device="cuda") if lse else None
        if workspace is None:
            workspace = pb.alloc_workspace(pb.prism_cache_attn_workspace_bytes(cache, batch, self.h))
            workspace.fill_(0xFF)                  # whatever an earlier use left (NaN)
        pb.prism_cache_attn(cache, batch, self.qd, out, sums, workspace, window, sinks, scale)
        torch.cuda.synchronize()
        return out, sums

    def check(self, window=0, sinks=0, scale=0.0, lse=True, **kw):
        out, sums = self.run(window, sinks, scale, lse, **kw)
        o, l = su.host(out), sums.double().cpu().numpy() if lse else None
        # odd scales: P v_scale is rounded once more in fp32
        mine = su.check_attention(o, l, self.q, self.k, self.v, self.lengths, self.cu, self.table, window, sinks, scale, 1e-6)
        if not kw.get("in_place"):
            assert (o[~mine] == 7.0).all() and (l is None or (l[~mine] == 7.0).all())       # nobody's rows
        if self.how != "dense" and not kw.get("in_place"):
            assert int(torch.isnan(out._base).sum()) == out._base.numel() - out.numel()
        return out, sums


STEPS = [
    # h, h_kv, d, page, lengths
    (1, 1, 128, 64, [1]),
    (32, 8, 128, 64, [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129]),
    (28, 4, 128, 32, [1000, 1, 0, 517, 96]),
    (8, 2, 64, 128, [4097, 128, 700]),
    (7, 1, 64, 64, [333]),
    (16, 16, 128, 128, [250, 129]),
    (16, 1, 128, 64, [777]),
    (40, 2, 128, 64, [300, 45]),                   # 20 q-heads a kv head
    (64, 1, 128, 64, [130, 1]),
    (4, 2, 256, 32, [1, 511, 95]),
    (24, 2, 256, 64, [200, 1023]),
    (2, 2, 128, 64, [20011]),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("h,h_kv,d,page,lengths", STEPS)
def test_steps(h, h_kv, d, page, lengths, e4m3):
    c = Case(len(lengths) + d + h, h, h_kv, d, page, e4m3, lengths, [1] * len(lengths))
    c.check(uniform=True)
    c.check(lse=False, scale=0.37)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 0), (64, 64), (100, 4), (33, 100), (2000, 7), (100000, 3)])
def test_steps_with_window(window, sinks, e4m3):
    for h, h_kv, d, page, lengths in [(8, 2, 128, 64, [1, 2, 64, 65, 99, 1500, 161, 0]), (14, 2, 64, 32, [700, 31, 105]), (4, 4, 256, 128, [600])]:
        Case(window + d, h, h_kv, d, page, e4m3, lengths, [1] * len(lengths)).check(window, sinks, uniform=True)


CHUNKS = [
    # h, h_kv, d, page, lengths, new tokens, rows behind, layout
    (8, 2, 128, 64, [64, 200, 7], [2, 3, 2], 0, "dense"),
    (28, 4, 128, 64, [5, 900, 64], [5, 5, 5], 3, "fused"),
    (4, 1, 64, 32, [70, 333, 1], [33, 1, 1], 0, "gaps"),
    (32, 8, 128, 64, [300, 64, 0, 500, 129], [300, 1, 0, 77, 128], 0, "dense"),
    (6, 2, 128, 128, [1000], [400], 1, "fused"),
    (16, 4, 64, 64, [513, 2], [513, 1], 0, "dense"),
    (2, 2, 256, 64, [333, 90], [200, 90], 0, "dense"),
    (10, 2, 256, 32, [77, 300], [9, 64], 0, "fused"),
    (1, 1, 128, 32, [260], [260], 0, "dense"),
    (20, 1, 128, 64, [90], [47], 0, "dense"),
    (4, 4, 64, 128, [700, 10], [130, 3], 0, "gaps"),
    (3, 1, 128, 64, [2500], [64], 0, "dense"),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("h,h_kv,d,page,lengths,news,behind,how", CHUNKS)
def test_chunks(h, h_kv, d, page, lengths, news, behind, how, e4m3):
    c = Case(sum(news) + d, h, h_kv, d, page, e4m3, lengths, news, behind, how, odd_scales=True)
    c.check()
    c.check(lse=False, scale=0.2)
    c.check(70, 5)
    c.check(17, 0)
    if len(lengths) > 1:                           # tables for 8192 tokens: single tokens apart from chunks, chunks cut by their keys
        Case(sum(news) + d, h, h_kv, d, page, e4m3, lengths, news, behind, how, odd_scales=True, wider=8192 // page).check()


PLANNED = [
    # h, h_kv, d, page, lengths, new tokens: several sequences whose tables have room for 8192 tokens and more
    (8, 2, 128, 64, [9000, 70, 0, 300, 0], [40, 70, 9, 1, 300]),
    (28, 4, 64, 32, [8200, 50, 1], [5, 5, 1]),
    (16, 16, 64, 128, [200, 100, 2500], [129, 100, 20]),
    (6, 3, 128, 64, [1500, 700], [150, 65]),
    (4, 2, 256, 64, [8500, 10, 600], [40, 10, 33]),
    (1, 1, 256, 32, [0, 0], [140, 30]),
    (2, 1, 64, 64, [3000] + [5 * s % 23 for s in range(1100)], [100] + [7 * s % 20 for s in range(1100)]),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("h,h_kv,d,page,lengths,news", PLANNED)
def test_chunks_behind_different_lengths(h, h_kv, d, page, lengths, news, e4m3):
    c = Case(sum(news) + d, h, h_kv, d, page, e4m3, lengths, news, odd_scales=True, wider=8192 // page)
    first, _ = c.check()
    c.check(9000, 3, lse=False)
    c.check(70, 5)
    assert (su.bits(c.run()[0]) == su.bits(first)).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_peaked_rows(e4m3):
    """Large logits: most of a row's weight on a few keys, the maximum moving late."""
    Case(77, 8, 2, 128, 64, e4m3, [900, 300], [1, 1], peaked=True).check()
    Case(78, 8, 2, 128, 64, e4m3, [900, 300], [70, 150], peaked=True).check()


@pytest.mark.parametrize("e4m3", [False, True])
def test_length_smaller_than_new_tokens(e4m3):
    """Queries at positions below zero see nothing."""
    for news in ([6, 40], [2, 1]):
        c = Case(5, 4, 2, 64, 32, e4m3, [3, 33], [1, 1])
        c.news, c.cu = news, np.concatenate([[0], np.cumsum(news)])
        c.lengths, c.rows = [3, min(33, 33)], int(c.cu[-1])
        c.q = su.bf16(np.random.default_rng(1).standard_normal((4, c.rows, 64)))
        c.qd = su.to_device(c.q)
        c.check()
        c.check(2 ** 31 - 1, 2 ** 31 - 1)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("news", [[1, 1], [37, 90]])
def test_pages_that_are_none_are_not_seen(news, e4m3):
    """Entries outside the pool anywhere in a row; a table narrower than a length."""
    c = Case(21, 8, 2, 128, 32, e4m3, [400, 300], news)
    c.table = c.table[:, :12].copy()               # 384 places: the first sequence ends behind them
    c.table[0, [0, 3]], c.table[0, 11] = -1, c.n_pages
    c.table[1, 2:] = 1 << 30
    c.check()
    c.check(60, 4)
    c.table[:] = -5
    c.check()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("news,window,sinks", [([1, 1], 50, 3), ([6, 2], 0, 0), ([6, 2], 20, 2), ([70, 64], 0, 0), ([70, 64], 33, 5)])
def test_infinity_and_nan_outside_a_rows_tokens(news, window, sinks, e4m3):
    """Tokens that some rows of the call see and others do not hold NaN (and infinity): rows that do not see them are as
    without them, rows that do are NaN where the definition is."""
    c = Case(31, 8, 2, 64, 32, e4m3, [200, 131], news)
    if news[0] == 1:
        bad = [(0, 149), (1, 80), (0, 3), (0, 10)]                           # in front of the window, behind the sinks
    elif window == 0:
        bad = [(0, 197), (1, 130)]                                           # among the new tokens
    else:
        bad = [(0, 197), (1, 130), (0, 176), (0, 150), (1, 100), (0, 4)]     # window's edge of some rows, behind the sinks
    for s, j in bad:
        for x, y in ((c.kd, np.nan), (c.vd, np.nan)):
            x.view(torch.uint8 if e4m3 else torch.int16)[c.table[s, j // 32], :, j % 32] = 0x7F if e4m3 else (0x7FC0 if j % 2 else 0x7F80)
    out, lse = c.run(window, sinks)
    o, l = su.host(out), lse.double().cpu().numpy()
    k, v = c.k.copy(), c.v.copy()
    for s, j in bad:                               # the oracle takes only what is seen
        k[c.table[s, j // 32], :, j % 32] = np.nan
    ref, ref_lse, spread, reach = so.attention(c.q, k, v, c.lengths, c.cu, c.table, window, sinks)
    ok = ~np.isnan(ref_lse)
    assert 0 < ok.sum() and (ok.all() if news[0] == 1 else not ok.all())
    assert np.isnan(o[~ok]).all() and np.isnan(l[~ok]).all()
    assert np.isfinite(o[ok]).all()
    keep = [r for r in range(c.rows) if ok[0, r]]
    p_err = su.HALF_STEP + 2 * 70 * 2.0 ** -24 * reach[:, keep] + 1e-5
    su.check_bf16(o[:, keep], ref[:, keep], p_err[..., None] * spread[:, keep])


def test_in_place_and_fused_rows():
    Case(41, 8, 2, 128, 64, False, [300, 5], [1, 1], how="fused").check(in_place=True)
    Case(42, 8, 2, 128, 64, False, [300, 200], [150, 70], how="fused").check(in_place=True)
    Case(43, 2, 2, 128, 64, False, [5000], [1]).check(in_place=True)
    Case(44, 2, 2, 128, 64, True, [5000], [40]).check(in_place=True)


def test_pages_of_k_and_v_in_one_tensor():
    c = Case(51, 8, 2, 128, 64, False, [300, 5, 64], [1, 1, 1])
    a, l = c.run()
    both = torch.stack([c.kd, c.vd], dim=1)
    c.kd, c.vd = both[:, 0], both[:, 1]
    b, m = c.run()
    assert np.array_equal(su.bits(a), su.bits(b)) and torch.equal(l, m)


@pytest.mark.parametrize("news", [[1, 1, 1], [50, 1, 200]])
def test_same_bits_every_time(news):
    c = Case(61, 16, 4, 128, 64, True, [3000, 17, 900], news)
    first = c.run()
    for _ in range(3):
        again = c.run()
        assert np.array_equal(su.bits(first[0]), su.bits(again[0])) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("news", [[1, 1, 1], [40, 40, 40]])
def test_graphs_share_a_workspace_and_follow_the_lengths(news, e4m3):
    """Two captured calls of different shapes and an eager one share a workspace, one after the other; lengths and tables
    change between the replays."""
    c, e = Case(71, 8, 2, 128, 32, e4m3, [600, 300, 50], news), Case(72, 8, 2, 128, 32, e4m3, [90, 2000], [1, 1])
    ws, graphs, args = None, [], []
    for x in (c, e):
        cache = pb.make_cache(x.kd, x.vd, x.ksd, x.vsd)
        batch, out = x.batch(uniform=True), torch.empty_like(x.qd)
        lse = torch.empty((x.h, x.rows), device="cuda")
        need = pb.prism_cache_attn_workspace_bytes(cache, batch, x.h)
        args.append((cache, batch, x.qd, out, lse))
        ws = need if ws is None else max(ws, need)
    ws = pb.alloc_workspace(ws)
    ws.fill_(0xFF)
    for a in args:
        pb.prism_cache_attn(*a, ws, 100, 4)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            pb.prism_cache_attn(*a, ws, 100, 4)
        graphs.append(graph)
    for lengths in ([600, 300, 50], [599, 45, 41], [40, 40, 40], [600, 0, 50]):
        args[0][1]._keep[0].copy_(su.ints(lengths))
        c.lengths = lengths
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for x, a in ((c, args[0]), (e, args[1])):
            su.check_attention(su.host(a[3]), a[4].double().cpu().numpy(), x.q, x.k, x.v, x.lengths, x.cu, x.table, 100, 4)
        e.run(100, 4, workspace=ws)


@pytest.mark.parametrize("window", [0, 300])
def test_graph_of_a_ragged_batch_follows_the_lengths(window):
    """Lengths and offsets change between the replays; tables are wide enough for a plan on the device (window 0)."""
    c = Case(73, 8, 2, 128, 64, False, [1500, 700, 90], [50, 1, 33], behind=44, wider=128)
    cache = pb.make_cache(c.kd, c.vd)
    batch = pb.make_batch(su.ints(c.lengths), su.ints(c.table), 64, su.ints(c.cu), c.rows)
    out, lse = torch.empty_like(c.qd), torch.empty((c.h, c.rows), device="cuda")
    ws = pb.alloc_workspace(pb.prism_cache_attn_workspace_bytes(cache, batch, c.h))
    pb.prism_cache_attn(cache, batch, c.qd, out, lse, ws, window, 4)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        pb.prism_cache_attn(cache, batch, c.qd, out, lse, ws, window, 4)
    for lengths, news in (([1500, 700, 90], [50, 1, 33]), ([1400, 30, 90], [1, 30, 64]), ([64, 699, 0], [64, 60, 0]), ([0, 0, 1], [0, 0, 1])):
        c.lengths, c.cu = lengths, np.concatenate([[0], np.cumsum(news)])
        batch._keep[0].copy_(su.ints(lengths))
        batch._keep[2].copy_(su.ints(c.cu))
        out.fill_(7.0)
        lse.fill_(7.0)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        o, l = su.host(out), lse.double().cpu().numpy()
        mine = su.check_attention(o, l, c.q, c.k, c.v, c.lengths, c.cu, c.table, window, 4)
        assert (o[~mine] == 7.0).all() and (l[~mine] == 7.0).all()


def test_another_stream():
    c = Case(81, 8, 2, 128, 64, False, [700, 1300], [1, 1])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c.check(uniform=True)


def test_more_new_tokens_than_max_tokens_are_left_out():
    """max_tokens bounds the work of a sequence: rows beyond it are not written."""
    c = Case(91, 4, 2, 64, 32, False, [100, 100], [3, 90])
    cache = pb.make_cache(c.kd, c.vd)
    for most in (1, 3, 64):
        batch = pb.make_batch(su.ints(c.lengths), su.ints(c.table), most, su.ints(c.cu), c.rows)
        out = torch.full_like(c.qd, 7.0)
        pb.prism_cache_attn(cache, batch, c.qd, out, None, pb.alloc_workspace(pb.prism_cache_attn_workspace_bytes(cache, batch, 4)))
        torch.cuda.synchronize()
        left = [r for s in range(2) for r in range(c.cu[s] + min(most, c.news[s]), c.cu[s + 1])]
        assert (su.host(out)[:, left] == 7.0).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_offsets_beyond_32_bits(e4m3):
    """A pool of over 4 GiB, a sequence in its last pages."""
    h_kv, page, d = 8, 128, 128
    n_pages = (5 << 30) // (h_kv * page * d * (1 if e4m3 else 2))
    rng = np.random.default_rng(6)
    dt = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    kp, vp = (torch.empty((n_pages, h_kv, page, d), dtype=dt, device="cuda") for _ in range(2))
    ks, vs = ((torch.ones((n_pages, h_kv), device="cuda") for _ in range(2)) if e4m3 else (None, None))
    small = [su.bf16(rng.standard_normal((3, h_kv, page, d))) for _ in range(2)]
    if e4m3:
        small = [so.to_e4m3(x) for x in small]
    ids = [n_pages - 1, 0, n_pages // 2 + 1]
    for i, p in enumerate(ids):
        kp[p], vp[p] = ((su.e4m3_to_device if e4m3 else su.to_device)(x[i]) for x in small)
    table, q = np.array([[0, 1, 2]]), su.bf16(rng.standard_normal((8, 60, d)))
    cache = pb.make_cache(kp, vp, ks, vs)
    for n in (1, 60):
        batch = pb.make_batch(su.ints([300]), su.ints([ids]), n)
        qd = su.to_device(q[:, :n])
        out, lse = torch.empty_like(qd), torch.empty((8, n), device="cuda")
        pb.prism_cache_attn(cache, batch, qd, out, lse, pb.alloc_workspace(pb.prism_cache_attn_workspace_bytes(cache, batch, 8)))
        torch.cuda.synchronize()
        su.check_attention(su.host(out), lse.double().cpu().numpy(), q[:, :n], *small, [300], [0, n], table, 0, 0)


def test_no_tokens():
    c = Case(95, 4, 2, 64, 32, False, [10], [1])
    cache = pb.make_cache(c.kd, c.vd)
    batch = pb.make_batch(su.ints([10]), su.ints(c.table), 1, su.ints([0, 0]), 0)
    none = torch.empty((4, 0, 64), dtype=torch.bfloat16, device="cuda")
    pb.prism_cache_attn(cache, batch, none, none, None, pb.alloc_workspace(256))
    pb.prism_cache_append(cache, batch, None, none[:2], none[:2])
    torch.cuda.synchronize()
