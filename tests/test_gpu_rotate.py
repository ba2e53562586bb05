"""GPU parity of prism_rotate against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2602_08426_amd import binding as pb
from paper_2602_08426_amd import workloads as wl
from tests import gpu_util as gu
from tests import serving_util as su

pytestmark = pytest.mark.gpu

YARN = (32768, 4.0, 1.0, 32.0)
LLAMA = (8192, 8.0, 1.0, 4.0)


def _rotary(base, rot, half, yarn=None, offset=0, magnitude=1.0):
    y = yarn or (0, 1.0, 1.0, 32.0)
    return pb.make_rotary(base, rot, pb.PRISM_ROPE_HALF if half else pb.PRISM_ROPE_INTERLEAVED, offset, magnitude, *y)


def _check(got, x, pos, base, rot, half, yarn=None, magnitude=1.0, backward=False):
    ref = so.rotate(x, pos, so.frequencies(base, rot, yarn), half, magnitude, backward)
    slack = su.TURN * magnitude * so.pair_magnitude(x, rot, half)
    su.check_bf16(su.host(got), ref, slack, "rotated")
    if rot < x.shape[-1]:
        assert np.array_equal(su.host(got)[..., rot:], x[..., rot:])


@pytest.mark.parametrize("h,h_kv,tokens,d,rot,half,yarn,offset,given,how", [
    (1, 1, 1, 128, 128, False, None, 0, False, "dense"),
    (32, 8, 1, 128, 128, True, None, 131071, False, "dense"),
    (28, 4, 333, 128, 128, True, YARN, 0, False, "fused"),
    (8, 2, 65, 64, 64, False, LLAMA, 1000, False, "gaps"),
    (7, 1, 130, 64, 32, True, None, 0, True, "dense"),
    (4, 4, 77, 256, 256, True, None, 0, True, "fused"),
    (5, 5, 31, 256, 240, False, YARN, 7, True, "gaps"),
    (3, 1, 259, 128, 16, False, None, 0, False, "fused"),
    (2, 1, 4097, 128, 112, True, LLAMA, 120000, False, "dense"),
])
def test_forward_and_backward(h, h_kv, tokens, d, rot, half, yarn, offset, given, how):
    rng = np.random.default_rng(tokens + d)
    q, k = su.bf16(rng.standard_normal((h, tokens, d))), su.bf16(3 * rng.standard_normal((h_kv, tokens, d)))
    pos = rng.integers(0, 1 << 20, tokens) if given else np.arange(tokens)
    positions = su.ints(pos) if given else None
    for flags, magnitude in ((0, 1.0), (pb.PRISM_ROTATE_BACKWARD, 1.25)):
        qd, kd = su.layout_of(su.to_device(q), how), su.layout_of(su.to_device(k), how)
        qo, ko = (su.layout_of(torch.full_like(su.to_device(x), 7.0), how) for x in (q, k))
        pb.prism_rotate(_rotary(5e5, rot, half, yarn, offset, magnitude), qd, kd, qo, ko, positions, flags)
        torch.cuda.synchronize()
        _check(qo, q, pos + offset, 5e5, rot, half, yarn, magnitude, flags != 0)
        _check(ko, k, pos + offset, 5e5, rot, half, yarn, magnitude, flags != 0)
        for x in (qo, ko):                         # nothing beside the rows is written
            base = x._base if x._base is not None else x
            if how != "dense":
                assert int(torch.isnan(base).sum()) == base.numel() - x.numel()
        # in place
        pb.prism_rotate(_rotary(5e5, rot, half, yarn, offset, magnitude), qd, kd, qd, kd, positions, flags)
        torch.cuda.synchronize()
        assert np.array_equal(su.bits(qd), su.bits(qo)) and np.array_equal(su.bits(kd), su.bits(ko))


def test_negative_and_large_positions():
    rng = np.random.default_rng(5)
    pos = np.array([-1, -100000, 0, (1 << 30), 16777217, 2 ** 31 - 1])
    q = su.bf16(rng.standard_normal((2, 6, 128)))
    qd = su.to_device(q)
    out = torch.empty_like(qd)
    pb.prism_rotate(_rotary(1e4, 128, True), qd, None, out, None, su.ints(pos))
    torch.cuda.synchronize()
    # 2^31 positions at 0.16 turns: 2^-53 of 3.4e8 turns is 4e-8 turns, 2.4e-7 radians more
    ref = so.rotate(q, pos, so.frequencies(1e4, 128), True)
    su.check_bf16(su.host(out), ref, 2 * su.TURN * so.pair_magnitude(q, 128, True))


def test_one_side_only_and_no_tokens():
    rng = np.random.default_rng(6)
    k = su.bf16(rng.standard_normal((2, 40, 64)))
    kd = su.to_device(k)
    out = torch.empty_like(kd)
    pb.prism_rotate(_rotary(1e4, 64, False), None, kd, None, out)
    torch.cuda.synchronize()
    _check(out, k, np.arange(40), 1e4, 64, False)
    none = torch.empty((2, 0, 64), dtype=torch.bfloat16, device="cuda")
    pb.prism_rotate(_rotary(1e4, 64, False), none, None, none, None)


def test_infinity_and_nan_stay_in_their_pairs():
    x = torch.ones((1, 3, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 1, 4], x[0, 2, 40] = float("inf"), float("nan")
    out = torch.empty_like(x)
    pb.prism_rotate(_rotary(1e4, 32, True), x, None, out, None, su.ints([3, 3, 3]))
    torch.cuda.synchronize()
    o = su.host(out)
    assert np.flatnonzero(~np.isfinite(o[0, 1])).tolist() == [4, 20]
    assert np.flatnonzero(np.isnan(o[0, 2])).tolist() == [40]          # behind the turning dims: as it was
    assert np.isfinite(o[0, 0]).all()


def test_full_interleaved_rotation_is_that_of_the_estimate():
    """prism_rope_estimate rotates on its way; apart from its fp32 recurrence the tensors are the same."""
    w = wl.small_variant(wl.WORKLOADS["c2_llama_8k"], 1024, 4, 2)
    Qb, Kb, _ = wl.generate(w, rotate=False)
    q, k = pb.bf16_bits_to_device(Qb), pb.bf16_bits_to_device(Kb)
    params = gu.params_for(w)
    outs = pb.alloc_estimate_outputs(params)
    ws = pb.alloc_workspace(pb.prism_estimate_workspace_bytes(params))
    q1, k1, q2, k2 = (torch.empty_like(x) for x in (q, k, q, k))
    pb.prism_rope_estimate(params, pb.make_rope(w.rope_base, 17), None, q, k, q1, k1, *outs[:3], outs[2].numel(), outs[3], ws)
    pb.prism_rotate(_rotary(w.rope_base, 128, False, None, 17), q, k, q2, k2)
    torch.cuda.synchronize()
    for a, b in ((q1, q2), (k1, k2)):
        assert (a != b).float().mean().item() < 2e-3
        pair = so.pair_magnitude(su.host(q if a is q1 else k), 128, False)
        assert (np.abs(su.host(a) - su.host(b)) <= 2 * su.HALF_STEP * np.abs(su.host(b)) + 4e-6 * pair).all()


def test_graph_replays_follow_the_positions():
    rng = np.random.default_rng(8)
    q = su.bf16(rng.standard_normal((4, 9, 128)))
    qd, pos = su.to_device(q), su.ints(np.zeros(9))
    out = torch.empty_like(qd)
    rot = _rotary(1e4, 128, True)
    pb.prism_rotate(rot, qd, None, out, None, pos)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        pb.prism_rotate(rot, qd, None, out, None, pos)
    for start in (0, 5000, 99):
        at = np.arange(start, start + 9)
        pos.copy_(su.ints(at))
        graph.replay()
        torch.cuda.synchronize()
        _check(out, q, at, 1e4, 128, True)
