"""GPU parity of prism_cache_append against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2602_08426_amd import binding as pb
from tests import serving_util as su

pytestmark = pytest.mark.gpu

BASE = 5e5


def _rotary(rot, half, **kw):
    return pb.make_rotary(BASE, rot, pb.PRISM_ROPE_HALF if half else pb.PRISM_ROPE_INTERLEAVED, **kw)


def _positions(lengths, cu, rows):
    pos = np.zeros(rows)
    for s, n in enumerate(lengths):
        m = cu[s + 1] - cu[s]
        pos[cu[s]:cu[s + 1]] = n - m + np.arange(m)
    return pos






CASES = [
    # heads, kv heads, d, page, rot (0: as they are), half, lengths after, new tokens, rows behind, layout of the inputs
    (1, 1, 128, 64, 128, False, [1], [1], 0, "dense"),
    (32, 8, 128, 64, 128, True, [300, 64, 65, 1, 128], [1, 1, 1, 1, 1], 0, "dense"),
    (28, 4, 128, 32, 128, True, [500, 77, 0, 33, 200], [500, 13, 0, 1, 199], 5, "fused"),
    (8, 2, 64, 128, 48, False, [130, 257, 3], [2, 129, 3], 0, "gaps"),
    (4, 2, 256, 32, 256, True, [70, 31, 96], [70, 30, 64], 1, "fused"),
    (6, 3, 256, 128, 0, False, [400, 129], [300, 2], 0, "dense"),
    (2, 2, 64, 64, 0, False, [2000], [2000], 0, "fused"),
]


@pytest.mark.parametrize("h,h_kv,d,page,rot,half,lengths,news,behind,how", CASES)
def test_bf16(h, h_kv, d, page, rot, half, lengths, news, behind, how):
    rng = np.random.default_rng(sum(lengths) + d)
    cu = np.concatenate([[0], np.cumsum(news)])
    rows = int(cu[-1]) + behind
    k, v = su.bf16(rng.standard_normal((h_kv, rows, d))), su.bf16(rng.standard_normal((h_kv, rows, d)))
    q = su.bf16(rng.standard_normal((h, rows, d)))
    table, n_pages = su.make_table(rng, lengths, page)
    old = [su.bf16(rng.standard_normal((n_pages, h_kv, page, d))) for _ in range(2)]
    kp, vp = (su.to_device(x) for x in old)
    cache = pb.make_cache(kp, vp)
    batch = pb.make_batch(su.ints(lengths), su.ints(table), max(news), su.ints(cu), rows)
    qd, kd, vd = (su.layout_of(su.to_device(x), how) for x in (q, k, v))
    qo = torch.full((h, rows, d), 9.0, dtype=torch.bfloat16, device="cuda")
    pb.prism_cache_append(cache, batch, _rotary(rot, half) if rot else None, kd, vd, qd, qo)
    torch.cuda.synchronize()
    pos, turned, slack = _positions(lengths, cu, rows), k, np.zeros_like(k)
    mine = np.arange(rows) < cu[-1]
    if rot:
        theta = so.frequencies(BASE, rot)
        turned, slack = so.rotate(k, pos, theta, half), su.TURN * so.pair_magnitude(k, rot, half)
        su.check_bf16(su.host(qo)[:, mine], so.rotate(q, pos, theta, half)[:, mine],
                      su.TURN * so.pair_magnitude(q, rot, half)[:, mine], "q")
    else:
        assert np.array_equal(su.host(qo)[:, mine], q[:, mine])
    assert (su.host(qo)[:, ~mine] == 9.0).all()                           # rows behind the last sequence
    su.check_bf16(su.host(kp), so.append_bf16(old[0], turned, lengths, cu, table),
                  so.append_bf16(np.zeros_like(old[0]), slack, lengths, cu, table), "k")
    assert np.array_equal(su.host(vp), so.append_bf16(old[1], v, lengths, cu, table))


@pytest.mark.parametrize("h,h_kv,d,page,rot,half,lengths,news,behind,how", CASES)
def test_e4m3(h, h_kv, d, page, rot, half, lengths, news, behind, how):
    rng = np.random.default_rng(sum(lengths) + d + 1)
    cu = np.concatenate([[0], np.cumsum(news)])
    rows = int(cu[-1]) + behind
    k, v = su.bf16(2 * rng.standard_normal((h_kv, rows, d))), su.bf16(rng.standard_normal((h_kv, rows, d)))
    k[0, rows // 2], v[0, rows // 2] = 0.0, 0.0
    table, n_pages = su.make_table(rng, lengths, page)
    old = [so.to_e4m3(np.clip(100 * rng.standard_normal((n_pages, h_kv, page, d)), -448, 448)) for _ in range(2)]
    scales = [2.0 ** rng.integers(-12, 2, (n_pages, h_kv)) for _ in range(2)]      # some grow, some are kept
    pools = [su.e4m3_to_device(x) for x in old]
    dev_scales = [torch.from_numpy(x.astype(np.float32)).cuda() for x in scales]
    before = [su.bits(x) for x in pools]
    cache = pb.make_cache(*pools, *dev_scales)
    batch = pb.make_batch(su.ints(lengths), su.ints(table), max(news), su.ints(cu), rows)
    kd, vd = (su.layout_of(su.to_device(x), how) for x in (k, v))
    pb.prism_cache_append(cache, batch, _rotary(rot, half) if rot else None, kd, vd)
    torch.cuda.synchronize()
    pos = _positions(lengths, cu, rows)
    turned = so.rotate(k, pos, so.frequencies(BASE, rot), half) if rot else k
    slack = su.TURN * so.pair_magnitude(k, rot, half) if rot else np.zeros_like(k)
    for i, (x, off) in enumerate(((turned, slack), (v, np.zeros_like(v)))):
        ref, s, new, moved = so.append_e4m3(old[i], scales[i], x, lengths, cu, table)
        at = so.append_bf16(np.zeros_like(ref), off, lengths, cu, table) / s[..., None, None]
        got_s = dev_scales[i].double().cpu().numpy()
        assert np.array_equal(got_s, s), np.argwhere(got_s != s)
        got = su.host(pools[i])
        # half a step: 2^-4 of the value, 2^-10 among the smallest
        bound = np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10) * 1.000001 + 1.07 * at
        assert (np.abs(got - ref) <= np.where((new | moved)[..., None], bound, 0.0)).all()
        same = ~(new | moved)
        assert np.array_equal(su.bits(pools[i]).reshape(before[i].shape)[same], before[i].reshape(before[i].shape)[same])
        exact = so.to_e4m3(ref)                                           # apart from what the rotation moves
        assert (got != exact)[new | moved].mean() < (1e-3 if rot and i == 0 else 1e-12)


def test_e4m3_step_by_step_is_as_good_as_at_once():
    """A page filled token by token, magnitudes growing: the final scale is that of one call; a value that moved k times
    is off by its first rounding, 2^-4 of it, and where it gets among the smallest magnitudes by half a step, 2^-10 of the
    scale, for each move: 2^-10 * (1 + 1/2 + ...) of the last scale."""
    rng = np.random.default_rng(3)
    d, page, n = 64, 32, 40
    x = su.bf16(rng.standard_normal((1, n, d)) * np.exp(np.linspace(-3, 3, n))[None, :, None])
    table = np.array([[1, 0]])
    dev, scales = [], []
    for news in ([n], [1] * n, [7, 20, 13]):
        kp, vp, ks, vs = pb.alloc_cache(2, 1, page, d, pb.PRISM_CACHE_E4M3)
        for t in (kp, vp):
            t.view(torch.uint8).fill_(0x7F)
        ks.fill_(float("inf")), vs.fill_(float("inf"))                     # of an earlier use: must not matter
        cache, at = pb.make_cache(kp, vp, ks, vs), 0
        for m in news:
            part = su.to_device(x[:, at:at + m])
            at += m
            pb.prism_cache_append(cache, pb.make_batch(su.ints([at]), su.ints(table), m), None, part, part)
        torch.cuda.synchronize()
        assert torch.equal(ks, vs) and np.array_equal(su.bits(kp), su.bits(vp))
        dev.append(su.host(kp)[[1, 0], 0].reshape(2 * page, d)[:n])
        scales.append(ks.cpu().numpy()[[1, 0], 0])
    s = np.repeat(scales[0], page)[:n, None].astype(np.float64)
    for values, sc in zip(dev, scales):
        assert np.array_equal(sc, scales[0])
        assert (np.abs(values * s - x[0]) <= 2.0 ** -4 * np.abs(x[0]) + 2.0 ** -9 * s).all()


def test_e4m3_infinity_nan_and_zeros():
    x = torch.ones((1, 32, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 3, 5], x[0, 4, 6], x[0, 5, 7] = float("inf"), float("nan"), 300.0
    z = torch.zeros_like(x)
    kp, vp, ks, vs = pb.alloc_cache(1, 1, 32, 64, pb.PRISM_CACHE_E4M3)
    pb.prism_cache_append(pb.make_cache(kp, vp, ks, vs), pb.make_batch(su.ints([32]), su.ints([[0]]), 32), None, x, z)
    torch.cuda.synchronize()
    assert ks.item() == 1.0 and vs.item() == 2.0 ** -120
    k = su.host(kp)[0, 0]
    assert np.isnan(k[3, 5]) and np.isnan(k[4, 6]) and k[5, 7] == so.to_e4m3(np.array([300.0]))[0]
    assert np.isnan(k).sum() == 2 and (su.host(vp) == 0).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_are_none_are_left_out(e4m3):
    """Entries outside the pool and positions outside the table: nothing is stored for them, the rest is."""
    rng = np.random.default_rng(9)
    d, page, n_pages = 64, 32, 4
    table = np.array([[0, -1, 2], [n_pages, 1, -7]])
    lengths, news = [96, 140], [96, 140]                                   # the second is longer than its table
    cu = np.array([0, 96, 236])
    x = su.bf16(rng.standard_normal((2, 236, d)))
    kp, vp, ks, vs = pb.alloc_cache(n_pages, 2, page, d, pb.PRISM_CACHE_E4M3 if e4m3 else pb.PRISM_CACHE_BF16)
    for t in (kp, vp):
        t.view(torch.uint8).fill_(0x11)
    if e4m3:
        ks.fill_(1.0), vs.fill_(1.0)
    xd = su.to_device(x)
    pb.prism_cache_append(pb.make_cache(kp, vp, ks, vs), pb.make_batch(su.ints(lengths), su.ints(table), 140, su.ints(cu), 236),
                          None, xd, xd)
    torch.cuda.synchronize()
    for p in (0, 1, 2):
        src = x[:, {0: slice(0, 32), 2: slice(64, 96), 1: slice(96 + 32, 96 + 64)}[p]]
        got = su.host(kp)[p] * (ks.cpu().numpy()[p][:, None, None] if e4m3 else 1.0)
        assert (np.abs(got - src) <= (2.0 ** -4 * np.abs(src) + 1e-2 if e4m3 else 0.0)).all()
    assert (su.bits(kp)[3] == 0x11).all() and (su.bits(vp)[3] == 0x11).all()


def test_length_smaller_than_new_tokens():
    """Positions below zero are not stored; the others are."""
    kp, vp, _, _ = pb.alloc_cache(2, 1, 32, 64)
    kp.fill_(5.0)
    x = torch.arange(6, device="cuda").to(torch.bfloat16)[None, :, None].expand(1, 6, 64).contiguous()
    pb.prism_cache_append(pb.make_cache(kp, vp), pb.make_batch(su.ints([4]), su.ints([[1]]), 6), None, x, x)
    torch.cuda.synchronize()
    assert su.host(kp)[1, 0, :5, 0].tolist() == [2.0, 3.0, 4.0, 5.0, 5.0] and (su.host(kp)[0] == 5.0).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_of_k_and_v_in_one_tensor(e4m3):
    """page_stride: K and V pages side by side; the same bits as in two tensors."""
    rng = np.random.default_rng(12)
    n_pages, h_kv, page, d = 5, 2, 32, 128
    x, y = (su.to_device(rng.standard_normal((h_kv, 70, d))) for _ in range(2))
    table, lengths = su.ints([[4, 0, 2]]), su.ints([70])
    kp, vp, ks, vs = pb.alloc_cache(n_pages, h_kv, page, d, pb.PRISM_CACHE_E4M3 if e4m3 else pb.PRISM_CACHE_BF16)
    both = torch.zeros((n_pages, 2, h_kv, page, d), dtype=kp.dtype, device="cuda")
    kp.view(torch.uint8).zero_(), vp.view(torch.uint8).zero_()
    for a, b in ((kp, vp), (both[:, 0], both[:, 1])):
        pb.prism_cache_append(pb.make_cache(a, b, ks, vs), pb.make_batch(lengths, table, 70), _rotary(64, True), x, y)
    torch.cuda.synchronize()
    assert np.array_equal(su.bits(both[:, 0]), su.bits(kp)) and np.array_equal(su.bits(both[:, 1]), su.bits(vp))


def test_q_in_place_and_offset():
    rng = np.random.default_rng(13)
    q, k = su.bf16(rng.standard_normal((4, 3, 128))), su.bf16(rng.standard_normal((2, 3, 128)))
    kp, vp, _, _ = pb.alloc_cache(4, 2, 64, 128)
    qd, kd = su.layout_of(su.to_device(q), "fused"), su.to_device(k)
    lengths, table = [10, 1, 64], [[0], [1], [2]]
    pb.prism_cache_append(pb.make_cache(kp, vp), pb.make_batch(su.ints(lengths), su.ints(table)),
                          _rotary(128, True, position_offset=1000), kd, kd, qd, qd)
    torch.cuda.synchronize()
    pos, theta = np.array(lengths) - 1 + 1000, so.frequencies(BASE, 128)
    su.check_bf16(su.host(qd), so.rotate(q, pos, theta, True), su.TURN * so.pair_magnitude(q, 128, True))
    for s in range(3):
        su.check_bf16(su.host(kp)[table[s][0], :, lengths[s] - 1], so.rotate(k, pos, theta, True)[:, s],
                      su.TURN * so.pair_magnitude(k, 128, True)[:, s])


@pytest.mark.parametrize("e4m3", [False, True])
def test_graph_replays_follow_the_lengths(e4m3):
    """A step captured once and replayed while the sequences grow gives what eager calls give."""
    rng = np.random.default_rng(14)
    d, page, h_kv, seqs, steps = 128, 32, 2, 3, 6
    table = su.ints(np.arange(seqs * 3).reshape(seqs, 3))
    start = np.array([30, 0, 61])
    x = [su.to_device(rng.standard_normal((h_kv, seqs, d)) * (1 + i)) for i in range(steps)]
    pools = []
    for captured in (False, True):
        kp, vp, ks, vs = pb.alloc_cache(seqs * 3, h_kv, page, d, pb.PRISM_CACHE_E4M3 if e4m3 else pb.PRISM_CACHE_BF16)
        kp.view(torch.uint8).zero_(), vp.view(torch.uint8).zero_()
        if e4m3:
            ks.fill_(2.0 ** -9), vs.fill_(2.0 ** -9)
        lengths, k = su.ints(start), torch.empty_like(x[0])
        cache, batch = pb.make_cache(kp, vp, ks, vs), pb.make_batch(lengths, table)
        call = lambda: pb.prism_cache_append(cache, batch, _rotary(128, False), k, k)
        graph = None
        if captured:
            k.copy_(x[0])
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                call()
        for i in range(steps):
            k.copy_(x[i])
            lengths.copy_(su.ints(start + i + 1))
            graph.replay() if captured else call()
            torch.cuda.synchronize()
        pools.append((su.bits(kp), su.bits(vp), None if ks is None else su.bits(ks)))
    assert np.array_equal(pools[0][0], pools[1][0]) and np.array_equal(pools[0][1], pools[1][1])
    assert not e4m3 or np.array_equal(pools[0][2], pools[1][2])
