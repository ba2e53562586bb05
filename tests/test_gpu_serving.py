"""The serving operators together, and with the prefill path: prompts stored after prism_sparse_attn, steps, chunks."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2602_08426_amd import binding as pb
from tests import gpu_util as gu
from tests import serving_util as su

pytestmark = pytest.mark.gpu


def _attend(cache, batch, q, window=0, sinks=0):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = pb.alloc_workspace(pb.prism_cache_attn_workspace_bytes(cache, batch, q.shape[0]))
    pb.prism_cache_attn(cache, batch, q, out, lse, ws, window, sinks)
    return out, lse


@pytest.mark.parametrize("layout,rot,e4m3", [(pb.PRISM_ROPE_INTERLEAVED, 128, False), (pb.PRISM_ROPE_HALF, 64, True)])
def test_prompt_chunk_and_steps_are_attention_over_everything(layout, rot, e4m3):
    """Two conversations: a prompt in one call, a chunk behind it, then steps through one captured graph.  Every output is the
    oracle's over the tokens rotated by their positions, read back from the cache for 8 bits."""
    rng = np.random.default_rng(11)
    h, h_kv, d, page, seqs = 8, 2, 128, 32, 2
    prompt, chunk, steps = [150, 37], [70, 33], 5
    total = [p + c + steps for p, c in zip(prompt, chunk)]
    table, n_pages = su.make_table(rng, total, page)
    kp, vp, ks, vs = pb.alloc_cache(n_pages, h_kv, page, d, pb.PRISM_CACHE_E4M3 if e4m3 else pb.PRISM_CACHE_BF16)
    for t in (kp, vp):
        t.view(torch.uint8).fill_(0x7F)                                       # what is not stored is NaN (e4m3) or 3e38
    cache, rotary = pb.make_cache(kp, vp, ks, vs), pb.make_rotary(1e4, rot, layout)
    x = {n: [su.bf16(rng.standard_normal((hn, t, d))) for t in total] for n, hn in (("q", h), ("k", h_kv), ("v", h_kv))}
    dtable = su.ints(table)
    theta, half = so.frequencies(1e4, rot), layout == pb.PRISM_ROPE_HALF

    def turned(n, s, at):
        return so.rotate(x[n][s][:, at], at, theta, half)

    def check(q, out, lse, lengths, news):
        cu = np.concatenate([[0], np.cumsum(news)])
        ref_q = np.concatenate([turned("q", s, np.arange(lengths[s] - news[s], lengths[s])) for s in range(seqs)], axis=1)
        given = np.concatenate([x["q"][s][:, lengths[s] - news[s]:lengths[s]] for s in range(seqs)], axis=1)
        su.check_bf16(su.host(q), ref_q, su.TURN * so.pair_magnitude(given, rot, half), "q")
        kc, vc = su.host(kp), su.host(vp)
        if e4m3:
            kc, vc = kc * ks.double().cpu().numpy()[..., None, None], vc * vs.double().cpu().numpy()[..., None, None]
        for s in range(seqs):                     # what is stored is what was given, to half a step (and 2^-9 of a scale that grew)
            j = np.arange(lengths[s])
            for c, ref, sc in ((kc, turned("k", s, j), ks), (vc, x["v"][s][:, j], vs)):
                got = c[table[s, j // page], :, j % page].transpose(1, 0, 2)
                tol = su.HALF_STEP * np.abs(ref) + 5e-6
                if e4m3:
                    tol = 2.0 ** -4 * np.abs(ref) + 2.0 ** -9 * sc.double().cpu().numpy()[table[s, j // page]].T[..., None] + 5e-6
                assert (np.abs(got - ref) <= tol).all()
        su.check_attention(su.host(out), lse.double().cpu().numpy(), su.host(q), kc, vc, lengths, cu, table, 0, 0)

    def call(lengths, news, q, k, v, batch):
        pb.prism_cache_append(cache, batch, rotary, k, v, q, q)
        return _attend(cache, batch, q)

    done = [0, 0]
    for news in (prompt, chunk):
        lengths = [a + b for a, b in zip(done, news)]
        q, k, v = (torch.cat([su.to_device(x[n][s][:, done[s]:lengths[s]]) for s in range(seqs)], dim=1) for n in "qkv")
        cu = np.concatenate([[0], np.cumsum(news)])
        out, lse = call(lengths, news, q, k, v, pb.make_batch(su.ints(lengths), dtable, max(news), su.ints(cu), sum(news)))
        torch.cuda.synchronize()
        check(q, out, lse, lengths, news)
        done = lengths

    q, k, v = (torch.empty((hn, seqs, d), dtype=torch.bfloat16, device="cuda") for hn in (h, h_kv, h_kv))
    lengths_dev = su.ints(done)
    batch = pb.make_batch(lengths_dev, dtable)
    out, lse = torch.empty_like(q), torch.empty((h, seqs), device="cuda")
    ws = pb.alloc_workspace(pb.prism_cache_attn_workspace_bytes(cache, batch, h))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        pb.prism_cache_append(cache, batch, rotary, k, v, q, q)
        pb.prism_cache_attn(cache, batch, q, out, lse, ws)
    for i in range(steps):
        lengths = [n + 1 for n in done]
        for t, n in ((q, "q"), (k, "k"), (v, "v")):
            t.copy_(torch.cat([su.to_device(x[n][s][:, done[s]:lengths[s]]) for s in range(seqs)], dim=1))
        lengths_dev.copy_(su.ints(lengths))
        graph.replay()
        torch.cuda.synchronize()
        check(q, out, lse, lengths, [1] * seqs)
        done = lengths


@pytest.mark.parametrize("L", [1024, 1500])
def test_chunk_over_a_stored_prompt_is_the_prefills_dense_attention(L):
    """The attention of a whole prompt through the cache is prism_sparse_attn over the all-ones lists: two kernels, each a
    bf16 rounding of P and one of the output off."""
    h, h_kv, d, B, page = 8, 2, 128, 128, 64
    gen = torch.Generator(device="cuda").manual_seed(L)
    q, k, v = (torch.randn((n, L, d), generator=gen, device="cuda").to(torch.bfloat16) for n in (h, h_kv, h_kv))
    rotary = pb.make_rotary(5e5, d)
    pb.prism_rotate(rotary, q, k, q, k)
    params = pb.make_params(h, h_kv, L, B)
    N = params.n_blocks
    row_ptr = torch.empty(h * N + 1, dtype=torch.int32, device="cuda")
    col_idx = torch.empty(h * N * (N + 1) // 2, dtype=torch.int32, device="cuda")
    pb.prism_causal_csr(params, row_ptr, col_idx, col_idx.numel())
    ref, ref_lse = gu.gpu_sparse_attn(params, q, k, v, row_ptr, col_idx, col_idx.numel())
    pages = -(-L // page)
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)[None]
    kp, vp, _, _ = pb.alloc_cache(pages, h_kv, page, d)
    cache, batch = pb.make_cache(kp, vp), pb.make_batch(su.ints([L]), table, L)
    pb.prism_cache_append(cache, batch, None, k, v)
    out, lse = _attend(cache, batch, q)
    torch.cuda.synchronize()
    a, b = su.host(out), su.host(ref)
    assert (np.abs(a - b) <= 2 * su.HALF_STEP * np.abs(b) + 2 * su.HALF_STEP * 0.8 + 1e-3).all()      # sum of P |v|: about 0.8 of v's deviation
    assert (lse - ref_lse).abs().max().item() < 1e-4


@pytest.mark.parametrize("news", [1, 3])
def test_many_sequences(news):
    """More sequences than a workgroup scans at a time, many of them empty."""
    rng = np.random.default_rng(20)
    n, h, h_kv, d, page = 700, 4, 2, 64, 32
    lengths = np.where(rng.random(n) < 0.3, 0, rng.integers(1, 90, n))
    table, n_pages = su.make_table(rng, lengths, page)
    k, v = (su.bf16(rng.standard_normal((n_pages, h_kv, page, d))) for _ in range(2))
    q = su.bf16(rng.standard_normal((h, n * news, d)))
    cache, batch = pb.make_cache(su.to_device(k), su.to_device(v)), pb.make_batch(su.ints(lengths), su.ints(table), news)
    out, lse = _attend(cache, batch, su.to_device(q), 40, 2)
    torch.cuda.synchronize()
    su.check_attention(su.host(out), lse.double().cpu().numpy(), q, k, v, lengths, np.arange(n + 1) * news, table, 40, 2)


def test_many_ragged_sequences_of_steps_and_chunks():
    rng = np.random.default_rng(21)
    n, h, h_kv, d, page = 300, 8, 2, 64, 32
    news = np.where(rng.random(n) < 0.1, rng.integers(2, 60, n), np.where(rng.random(n) < 0.1, 0, 1))
    lengths = news + rng.integers(0, 60, n)
    cu = np.concatenate([[0], np.cumsum(news)])
    table, n_pages = su.make_table(rng, lengths, page)
    old = [su.bf16(rng.standard_normal((n_pages, h_kv, page, d))) for _ in range(2)]
    x, q = su.bf16(rng.standard_normal((h_kv, cu[-1], d))), su.bf16(rng.standard_normal((h, cu[-1], d)))
    kp, vp = (su.to_device(t) for t in old)
    cache = pb.make_cache(kp, vp)
    batch = pb.make_batch(su.ints(lengths), su.ints(table), int(news.max()), su.ints(cu), int(cu[-1]))
    pb.prism_cache_append(cache, batch, None, su.to_device(x), su.to_device(x))
    out, lse = _attend(cache, batch, su.to_device(q))
    torch.cuda.synchronize()
    k, v = (so.append_bf16(t, x, lengths, cu, table) for t in old)
    assert np.array_equal(su.host(kp), k) and np.array_equal(su.host(vp), v)
    su.check_attention(su.host(out), lse.double().cpu().numpy(), q, k, v, lengths, cu, table, 0, 0)


@pytest.mark.parametrize("e4m3", [False, True])
def test_long_tables(e4m3):
    """More pages than a wave holds entries of, with sinks far from the window."""
    rng = np.random.default_rng(22)
    h, h_kv, d, page, lengths = 4, 2, 64, 32, [7000, 4500]
    table, n_pages = su.make_table(rng, lengths, page)
    k, v = (su.bf16(rng.standard_normal((n_pages, h_kv, page, d))) for _ in range(2))
    ks = vs = None
    kd, vd = su.to_device(k), su.to_device(v)
    if e4m3:
        k, v = so.to_e4m3(k), so.to_e4m3(v)
        kd, vd, ks = su.e4m3_to_device(k), su.e4m3_to_device(v), torch.full((n_pages, h_kv), 0.5, device="cuda")
        k, v, vs = 0.5 * k, 0.5 * v, ks.clone()
    cache = pb.make_cache(kd, vd, ks, vs)
    for news in (1, 50):
        q = su.bf16(rng.standard_normal((h, 2 * news, d)))
        batch = pb.make_batch(su.ints(lengths), su.ints(table), news)
        for window, sinks in ((0, 0), (2900, 100)):
            out, lse = _attend(cache, batch, su.to_device(q), window, sinks)
            torch.cuda.synchronize()
            su.check_attention(su.host(out), lse.double().cpu().numpy(), q, k, v, lengths, [0, news, 2 * news], table, window, sinks)
