"""Performance cases of the serving operators: rotary positions, appending to a paged cache, attention over it.

A pass is one call as a serving program makes it for one layer.  Buffers, workspaces, the cache and its page table are made
once; lengths and tables live on the device and no call waits for it.  `own` is set from outside: the operators' plain forms
(elementary torch operations in 32 bits, angles in 64) where it is false, the library's entry points where it is true.

Kinds
  rotate  rotary positions applied to Q and K, or (backward) to their gradients
  append  new keys and values, rotated on the way or as they are, into the pages; Q of the same tokens rotated too if asked
  attn    attention of the new tokens of every sequence over its cache: single tokens (steps) and chunks of prompts
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0
MIN_EXPONENT = -120                     # of a scale: an all-zero page and head
# NTK-by-parts frequencies: native length, scale, alpha, beta
YARN = (32768, 4.0, 1.0, 32.0)


def _rotate_case(h, h_kv, tokens, *, head_dim=128, rot=128, half=False, yarn=False, base=5.0e5, backward=False,
                 given=False, strided=False):
    return dict(kind="rotate", h=h, h_kv=h_kv, tokens=tokens, head_dim=head_dim, rot=rot, half=half, yarn=yarn,
                base=base, backward=backward, given=given, strided=strided)


def _append_case(h, h_kv, lens, news, *, head_dim=128, page=64, e4m3=False, rot=128, half=False, yarn=False, base=5.0e5,
                 with_q=False):
    return dict(kind="append", h=h, h_kv=h_kv, lens=lens, news=news, head_dim=head_dim, page=page, e4m3=e4m3, rot=rot,
                half=half, yarn=yarn, base=base, with_q=with_q)


def _attn_case(h, h_kv, lens, news, *, head_dim=128, page=64, e4m3=False, window=0, sinks=0, lse=False):
    return dict(kind="attn", h=h, h_kv=h_kv, lens=lens, news=news, head_dim=head_dim, page=page, e4m3=e4m3,
                window=window, sinks=sinks, lse=lse)


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


def listed():
    prompts = "8192,1500,4096,77,12288,3001,640,5000"
    # 64 conversations of a serving batch: lengths spread over their logarithm
    talk = [round(500 * 2 ** (6.03 * ((i * 37) % 64) / 63)) for i in range(64)]
    short = [round(20 * 2 ** (5.0 * ((i * 29) % 64) / 63)) for i in range(64)]
    return [
        # one token of one sequence: latency is all there is
        dict(_rotate_case(32, 8, 1), name="rotate_1_token"),
        # a 32K prompt of a 28 / 4 head decoder, pairs (j, j + d/2), frequencies stretched for long contexts
        dict(_rotate_case(28, 4, 32768, half=True, yarn=True, base=1.0e6), name="rotate_32k_half_yarn"),
        # gradients of a packed batch (positions given) rotated back; half of each head carries positions, heads inside
        # one fused projection
        dict(_rotate_case(32, 8, 20011, rot=64, half=True, backward=True, given=True, strided=True),
             name="rotate_back_20011_partial"),
        # a step of 64 sequences: one new token each, Q rotated with it
        dict(_append_case(32, 8, _text(short), _text([1] * 64), half=True, with_q=True), name="append_step_64"),
        # the keys that the prefill path has rotated already, and the values of its prompt, stored
        dict(_append_case(32, 8, "32768", "32768", rot=0), name="append_prompt_32k"),
        # a packed batch of prompts into an 8-bit cache, some behind what is there
        dict(_append_case(32, 8, "8192,1700,4096,77,12288,3001,777,5000", prompts, e4m3=True, half=True, with_q=True),
             name="append_8_prompts_e4m3"),
        # the smallest step: one sequence of 2K tokens
        dict(_attn_case(32, 8, "2048", "1"), name="attn_step_1_2k"),
        # an ordinary serving batch
        dict(_attn_case(32, 8, _text(talk), _text([1] * 64)), name="attn_step_64"),
        # the longest contexts, in 8 bits
        dict(_attn_case(32, 8, _text([131072 - 1111 * i for i in range(8)]), _text([1] * 8), page=128, e4m3=True),
             name="attn_step_8_128k_e4m3"),
        # a window of 4096 tokens and four sinks in contexts of 64K; pages behind the window are gone
        dict(_attn_case(28, 4, _text([65536 - 999 * i for i in range(16)]), _text([1] * 16), window=4096, sinks=4,
                        lse=True), name="attn_step_16_window"),
        # a chunk of a long prompt
        dict(_attn_case(32, 8, "32768", "2048", lse=True), name="attn_chunk_2k_at_32k"),
        # steps and chunks in one batch, 8 bits, the smaller head size, a window with sinks
        dict(_attn_case(16, 4, "5000,333,9777,12000,2048,64,31000,1300", "1,1,777,1,2048,64,1,300", head_dim=64, page=32,
                        e4m3=True, window=1024, sinks=4), name="attn_mixed_window_e4m3"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: operator, heads, head size, page, type, options, and lengths spread over their logarithm."""
    kind = rng.choice(["rotate", "append", "attn", "attn"])
    h, h_kv = rng.choice([(1, 1), (8, 2), (7, 1), (16, 4), (28, 4), (32, 8), (16, 16)])
    head_dim = rng.choice([64, 128, 128, 256])
    rot = rng.choice([head_dim, head_dim, head_dim // 2, head_dim - 16])
    half, yarn, base = rng.random() < 0.5, rng.random() < 0.3, rng.choice([1.0e4, 5.0e5, 1.0e6])
    if kind == "rotate":
        return _rotate_case(h, h_kv, _log_uniform(rng, 1, 32768 * 128 // head_dim * 32 // max(h, 32)), head_dim=head_dim,
                            rot=rot, half=half, yarn=yarn, base=base, backward=rng.random() < 0.4,
                            given=rng.random() < 0.5, strided=rng.random() < 0.4)
    page, e4m3 = rng.choice([32, 64, 64, 128]), rng.random() < 0.5
    step = rng.random() < 0.6
    if kind == "append":
        n = _log_uniform(rng, 1, 64) if step else rng.randint(1, 6)
        news = [1 if step else _log_uniform(rng, 2, 8192) for _ in range(n)]
        lens = [m + (_log_uniform(rng, 1, 700) if rng.random() < 0.7 else 0) for m in news]
        return _append_case(h, h_kv, _text(lens), _text(news), head_dim=head_dim, page=page, e4m3=e4m3,
                            rot=rng.choice([0, rot, rot]), half=half, yarn=yarn, base=base, with_q=rng.random() < 0.6)
    window = rng.choice([0, 0, 512, 4096])
    sinks = rng.choice([0, 4, 64]) if window else 0
    if step:                                    # single tokens, or a few of them (drafts to be verified)
        n = _log_uniform(rng, 1, 64)
        most = max(256, min(131072, (1 << 20) // n * 8 // max(h_kv, 8) * 128 // head_dim))
        lens = [_log_uniform(rng, 16, most) for _ in range(n)]
        m = rng.choice([1, 1, 1, 2, 5])
        news = [min(m, x) for x in lens]
    else:
        n = rng.randint(1, 4)
        news = [_log_uniform(rng, 2, 2048 // n) for _ in range(n)]
        lens = [m + _log_uniform(rng, 1, 30000 // n) for m in news]
    return _attn_case(h, h_kv, _text(lens), _text(news), head_dim=head_dim, page=page, e4m3=e4m3, window=window,
                      sinks=sinks, lse=rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------------
def _heads_of(gen, h, tokens, d, scale=1.0):
    """[h, tokens, d] bf16 with the outlier channels that projections of trained models have."""
    x = torch.randn((h, tokens, d), generator=gen, device="cuda")
    channel = torch.exp(0.5 * torch.randn((h, 1, d), generator=gen, device="cuda"))
    return (x * (channel * scale)).to(torch.bfloat16)


def _fused_heads(gen, h, h_kv, tokens, d):
    """Q and K as views of one projection [tokens, (h + 2 h_kv) * d]."""
    x = torch.randn((tokens, h + 2 * h_kv, d), generator=gen, device="cuda").to(torch.bfloat16).transpose(0, 1)
    return x[:h], x[h:h + h_kv]


def _pages(case, gen, table_lens):
    """Page table [sequences, widest] of pages in no order, -1 where there is none, and the number of pages."""
    page = case["page"]
    counts = [max(1, -(-n // page)) for n in table_lens]
    n_pages, widest = sum(counts) + 3, max(counts)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(counts), widest), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    return table, n_pages


def _to_e4m3(x):
    """[pages, heads, page, d] values as e4m3 with a power-of-two scale for each page and head."""
    mant, exp = torch.frexp(x.float().abs().amax(dim=(2, 3)))
    e = torch.where(mant > 0, exp - 9 + (mant > 0.875).to(exp.dtype), torch.full_like(exp, MIN_EXPONENT))
    scale = torch.ldexp(torch.ones_like(mant), e.clamp(min=MIN_EXPONENT))
    return (x.float() / scale[:, :, None, None]).to(torch.float8_e4m3fn), scale


def _positions(case, gen):
    """Positions of a packed batch: each of its sequences counts from where it stands."""
    t = case["tokens"]
    cuts = torch.sort(torch.randint(0, t, (5,), generator=gen, device="cuda")).values
    at = torch.arange(t, device="cuda")
    start = torch.where(cuts[None] <= at[:, None], cuts[None], torch.zeros_like(cuts[None])).amax(1)
    return (at - start + torch.randint(0, 100000, (1,), generator=gen, device="cuda")).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))
    h, h_kv, d = case["h"], case["h_kv"], case["head_dim"]
    st = {"case": case}
    if case["kind"] == "rotate":
        t = case["tokens"]
        if case["strided"]:
            st["q"], st["k"] = _fused_heads(gen, h, h_kv, t, d)
        else:
            st["q"], st["k"] = _heads_of(gen, h, t, d), _heads_of(gen, h_kv, t, d)
        st["q_out"] = torch.empty((h, t, d), dtype=torch.bfloat16, device="cuda")
        st["k_out"] = torch.empty((h_kv, t, d), dtype=torch.bfloat16, device="cuda")
        st["positions"] = _positions(case, gen) if case["given"] else None
        return st
    lens, news = _ints(case["lens"]), _ints(case["news"])
    total = sum(news)
    st["table"], n_pages = _pages(case, gen, lens)
    st["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
    shape = (n_pages, h_kv, case["page"], d)
    channel = torch.exp(0.5 * torch.randn((1, h_kv, 1, d), generator=gen, device="cuda")).to(torch.bfloat16)
    k_pages = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16).mul_(channel)
    v_pages = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    st["k_scale"] = st["v_scale"] = None
    if case["e4m3"]:
        k_pages, st["k_scale"] = _to_e4m3(k_pages)
        v_pages, st["v_scale"] = _to_e4m3(v_pages)
    st["k_pages"], st["v_pages"] = k_pages, v_pages
    if case["kind"] == "append":
        st["k"], st["v"] = _heads_of(gen, h_kv, total, d, 1.3), _heads_of(gen, h_kv, total, d)
        st["q"] = _heads_of(gen, h, total, d) if case["with_q"] else None
        st["q_out"] = torch.empty_like(st["q"]) if case["with_q"] else None
        return st
    if case["window"]:                          # pages that no query of the call sees any more are given back
        first = torch.arange(st["table"].shape[1], device="cuda")[None] * case["page"]
        oldest = (st["lengths"] - torch.tensor(news, device="cuda", dtype=torch.int32) - case["window"] + 1)[:, None]
        gone = (first + case["page"] <= oldest) & (first >= case["sinks"])
        st["table"] = torch.where(gone, torch.full_like(st["table"], -1), st["table"])
    # logits of a standard deviation of about 2, and a strong first token
    st["q"] = _heads_of(gen, h, total, d, 1.2)
    st["out"] = torch.empty_like(st["q"])
    st["lse"] = torch.empty((h, total), dtype=torch.float32, device="cuda") if case["lse"] else None
    return st


# ---- plain forms ------------------------------------------------------------------------------------
def _frequencies(case):
    rot = case["rot"]
    theta = torch.pow(torch.tensor(case["base"], dtype=torch.float64),
                      -2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    if case["yarn"]:
        native, s, alpha, beta = YARN
        keep = ((native * theta / (2.0 * math.pi) - alpha) / (beta - alpha)).clamp(0.0, 1.0)
        theta = (1.0 - keep) * theta / s + keep * theta
    return theta.to("cuda")


def _turn(case, x, positions, backward=False):
    """x [heads, tokens, d] turned by its positions, in 32 bits (angles in 64)."""
    rot = case["rot"]
    x = x.float()
    if rot == 0:
        return x
    a = positions.double()[:, None] * _frequencies(case)[None]
    c, s = torch.cos(a).float(), torch.sin(a).float()
    s = -s if backward else s
    if case["half"]:
        u, v = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([u * c - v * s, u * s + v * c, x[..., rot:]], dim=-1)
    u, v = x[..., 0:rot:2], x[..., 1:rot:2]
    both = torch.stack([u * c - v * s, u * s + v * c], dim=-1).flatten(-2)
    return torch.cat([both, x[..., rot:]], dim=-1)


def _plain_rotate(st):
    case = st["case"]
    at = st["positions"] if case["given"] else torch.arange(case["tokens"], device="cuda")
    return [_turn(case, st[n], at, case["backward"]).to(torch.bfloat16) for n in ("q", "k")]


def _token_places(st):
    """Sequence and position of every new token."""
    cu, lengths = st["cu"].long(), st["lengths"].long()
    i = torch.arange(sum(_ints(st["case"]["news"])), device="cuda")
    s = torch.searchsorted(cu[1:], i, right=True)
    return s, lengths[s] - (cu[s + 1] - cu[s]) + i - cu[s]


def _store_e4m3(case, pages, scales, ids, offs, fresh, x):
    """x [tokens, heads, d] into pages of e4m3; ids [tokens] pages, offs places; fresh [pages]: nothing in it counts."""
    page = case["page"]
    need = torch.zeros_like(scales).index_reduce_(0, ids, x.abs().amax(-1), "amax")
    touched = torch.zeros(scales.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, ids, True)
    mant, exp = torch.frexp(need)
    e = torch.where(mant > 0, exp - 9 + (mant > 0.875).to(exp.dtype), torch.full_like(exp, MIN_EXPONENT))
    need = torch.ldexp(torch.ones_like(mant), e.clamp(min=MIN_EXPONENT))
    new = torch.where(fresh[:, None], need, torch.maximum(need, scales))
    new = torch.where(touched[:, None], new, scales)
    grown = torch.nonzero((touched & ~fresh)[:, None].expand_as(new) & (new > scales))
    if grown.shape[0]:                          # what is there already moves to the new scale
        first = torch.full((scales.shape[0],), page, dtype=torch.long, device="cuda").index_reduce_(0, ids, offs, "amin")
        p, hd = grown[:, 0], grown[:, 1]
        old = pages[p, hd].float()
        moved = (old * (scales[p, hd] / new[p, hd])[:, None, None]).to(torch.float8_e4m3fn).float()
        live = torch.arange(page, device="cuda")[None] < first[p][:, None]
        pages[p, hd] = torch.where(live[..., None], moved, old).to(torch.float8_e4m3fn)
    scales.copy_(new)
    pages[ids, :, offs] = (x / new[ids][..., None]).to(torch.float8_e4m3fn)


def _plain_append(st):
    case = st["case"]
    s, pos = _token_places(st)
    ids, offs = st["table"][s, pos // case["page"]].long(), pos % case["page"]
    k = _turn(case, st["k"], pos).transpose(0, 1)
    v = st["v"].float().transpose(0, 1)
    if case["e4m3"]:
        first = torch.full((st["k_pages"].shape[0],), case["page"], dtype=torch.long, device="cuda")
        fresh = first.index_reduce_(0, ids, offs, "amin") == 0
        _store_e4m3(case, st["k_pages"], st["k_scale"], ids, offs, fresh, k)
        _store_e4m3(case, st["v_pages"], st["v_scale"], ids, offs, fresh, v)
    else:
        st["k_pages"][ids, :, offs] = k.to(torch.bfloat16)
        st["v_pages"][ids, :, offs] = v.to(torch.bfloat16)
    q = _turn(case, st["q"], pos).to(torch.bfloat16) if case["with_q"] else None
    return [st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], q]


def _cached(case, pages, scales, table):
    """[sequences, heads, tokens, d] in 32 bits, zeros where there is no page."""
    x = pages[table.clamp(min=0).long()].float()
    if scales is not None:
        x = x * scales[table.clamp(min=0).long()][..., None, None]
    x = torch.where((table >= 0)[:, :, None, None, None], x, torch.zeros((), device="cuda"))
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attn(st):
    case = st["case"]
    h, h_kv, d, page = case["h"], case["h_kv"], case["head_dim"], case["page"]
    most, g = max(_ints(case["news"])), h // h_kv
    cu, lengths = st["cu"].long(), st["lengths"].long()
    n = cu[1:] - cu[:-1]
    seqs = n.shape[0]
    i = torch.arange(most, device="cuda")
    rows = (cu[:-1, None] + i).clamp(max=st["q"].shape[1] - 1)                       # [sequences, most]
    q = st["q"].float()[:, rows].view(h_kv, g, seqs, most, d).permute(2, 0, 1, 3, 4).reshape(seqs, h_kv, g * most, d)
    keys = _cached(case, st["k_pages"], st["k_scale"], st["table"])
    scores = torch.matmul(q, keys.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(seqs, h_kv, g, most, -1)
    del keys
    j = torch.arange(scores.shape[-1], device="cuda")
    pos = (lengths - n)[:, None] + i                                                 # [sequences, most]
    sees = j <= pos[..., None]
    if case["window"]:
        sees &= (j > pos[..., None] - case["window"]) | (j < case["sinks"])
    sees &= (st["table"] >= 0).repeat_interleave(page, dim=1)[:, None]
    scores.masked_fill_(~sees[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    values = _cached(case, st["v_pages"], st["v_scale"], st["table"])
    o = torch.matmul(p.view(seqs, h_kv, g * most, -1), values).view(seqs, h_kv, g, most, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    s, _ = _token_places(st)
    at = torch.arange(s.shape[0], device="cuda") - cu[s]
    out = o[s, :, :, at].flatten(1, 2).transpose(0, 1).to(torch.bfloat16).contiguous()
    if not case["lse"]:
        return [out]
    lse = (total.log() + top)[..., 0][s, :, :, at].flatten(1, 2).transpose(0, 1).contiguous()
    return [out, lse]


# ---- the library's calls ----------------------------------------------------------------------------
def _own(st):
    from paper_2602_08426_amd import binding as pb
    case = st["case"]
    if "call" not in st:                        # descriptors and workspace, made once as a program would
        yarn = YARN if case.get("yarn") else (0, 1.0, 1.0, 32.0)
        if case.get("rot"):
            st["rotary"] = pb.make_rotary(case["base"], case["rot"], yarn_native_len=yarn[0], yarn_scale=yarn[1],
                                          yarn_alpha=yarn[2], yarn_beta=yarn[3],
                                          layout=pb.PRISM_ROPE_HALF if case["half"] else pb.PRISM_ROPE_INTERLEAVED)
        else:
            st["rotary"] = None
        if case["kind"] != "rotate":
            news = _ints(case["news"])
            same = all(m == news[0] for m in news)
            st["cache"] = pb.make_cache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
            st["batch"] = pb.make_batch(st["lengths"], st["table"], max_tokens=max(news),
                                        cu_tokens=None if same else st["cu"], n_tokens=sum(news))
        if case["kind"] == "attn":
            st["workspace"] = pb.alloc_workspace(pb.prism_cache_attn_workspace_bytes(st["cache"], st["batch"], case["h"]))
        st["call"] = True
    if case["kind"] == "rotate":
        pb.prism_rotate(st["rotary"], st["q"], st["k"], st["q_out"], st["k_out"], positions=st["positions"],
                        flags=pb.PRISM_ROTATE_BACKWARD if case["backward"] else 0)
        return [st["q_out"], st["k_out"]]
    if case["kind"] == "append":
        pb.prism_cache_append(st["cache"], st["batch"], st["rotary"], st["k"], st["v"], st["q"], st["q_out"])
        return [st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], st["q_out"]]
    pb.prism_cache_attn(st["cache"], st["batch"], st["q"], st["out"], st["lse"], st["workspace"],
                        window=case["window"], sinks=case["sinks"])
    return [st["out"], st["lse"]] if case["lse"] else [st["out"]]


def run(st):
    if own:
        return _own(st)
    kind = st["case"]["kind"]
    return _plain_rotate(st) if kind == "rotate" else _plain_append(st) if kind == "append" else _plain_attn(st)


# ---- what a pass cannot do without -------------------------------------------------------------------
def _visible(length, new, window, sinks):
    """(cached tokens that some query sees, pairs of a query and a token that it sees)"""
    pos = np.arange(length - new, length, dtype=np.int64)
    if not window:
        return length, int((pos + 1).sum())
    low = np.maximum(pos - window + 1, 0)
    pairs = int((pos - low + 1 + np.minimum(low, sinks)).sum())
    low0 = int(low[0])
    return length - low0 + min(low0, sinks), pairs


def work(case):
    h, h_kv, d = case["h"], case["h_kv"], case["head_dim"]
    if case["kind"] == "rotate":
        values = (h + h_kv) * case["tokens"] * d
        return {"bytes": 4.0 * values + (4.0 * case["tokens"] if case["given"] else 0), "flops": 3.0 * values}
    lens, news = _ints(case["lens"]), _ints(case["news"])
    total, size = sum(news), 1 if case["e4m3"] else 2
    if case["kind"] == "append":
        bytes_ = 2.0 * h_kv * total * d * (2 + size) + (4.0 * h * total * d if case["with_q"] else 0)
        return {"bytes": bytes_, "flops": 3.0 * (h_kv + (h if case["with_q"] else 0)) * total * d}
    seen = [_visible(n, m, case["window"], case["sinks"]) for n, m in zip(lens, news)]
    bytes_ = 2.0 * h_kv * d * size * sum(t for t, _ in seen) + 4.0 * h * total * d + (4.0 * h * total if case["lse"] else 0)
    return {"bytes": bytes_, "flops": 4.0 * d * h * sum(p for _, p in seen)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------
def _exact_turn(case, x, positions, sign=1.0):
    """Pairs as complex numbers, times e^(i angle)."""
    rot, half = case["rot"], case["half"]
    x = x.double().clone()
    if rot == 0:
        return x
    j = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
    w = torch.exp(-(2.0 * j / rot) * math.log(case["base"]))
    if case["yarn"]:
        native, s, alpha, beta = YARN
        g = torch.clamp((native * w / (2 * math.pi) - alpha) / (beta - alpha), 0, 1)
        w = w * ((1 - g) / s + g)
    turn = torch.polar(torch.ones_like(w)[None].expand(len(positions), -1).contiguous(), sign * positions.double()[:, None] * w)
    re = slice(0, rot // 2) if half else slice(0, rot, 2)
    im = slice(rot // 2, rot) if half else slice(1, rot, 2)
    z = torch.complex(x[..., re], x[..., im]) * turn
    x[..., re], x[..., im] = z.real, z.imag
    return x


def _exact_places(case, table):
    """(token, page, place, position) of all new tokens, counted on the host."""
    rows = table.cpu().numpy()
    found, t = [], 0
    for s, (n, m) in enumerate(zip(_ints(case["lens"]), _ints(case["news"]))):
        for pos in range(n - m, n):
            found.append((t, int(rows[s, pos // case["page"]]), pos % case["page"], pos))
            t += 1
    return torch.tensor(found, device="cuda").T


def _exact_append(case, st):
    _, ids, offs, pos = _exact_places(case, st["table"])
    new = {"k": _exact_turn(case, st["k"], pos), "v": st["v"].double()}
    pools, scales = [], []
    for n in ("k", "v"):
        pool = st[n + "_pages"].to(torch.float64)
        x = new[n].permute(1, 0, 2)
        if not case["e4m3"]:
            pool[ids, :, offs] = x
            pools.append(pool)
            scales.append(None)
            continue
        scale = st[n + "_scale"].double()
        for p in torch.unique(ids).tolist():
            mine = ids == p
            need = x[mine].abs().amax(dim=(0, 2))
            e = torch.ceil(torch.log2((need / 448.0).clamp(min=2.0 ** MIN_EXPONENT)))
            s_new = torch.exp2(e)
            begin = int(offs[mine].min())
            if begin > 0:
                s_new = torch.maximum(s_new, scale[p])
                pool[p, :, :begin] *= (scale[p] / s_new)[:, None, None]
            scale[p] = s_new
        pool[ids, :, offs] = x / scale[ids][..., None]
        pools.append(pool)
        scales.append(scale)
    q = _exact_turn(case, st["q"], pos) if case["with_q"] else None
    return pools + scales + [q]


def _exact_attn(case, st):
    h, h_kv, d, page = case["h"], case["h_kv"], case["head_dim"], case["page"]
    g = h // h_kv
    total = st["q"].shape[1]
    out = torch.zeros((h, total, d), dtype=torch.float64, device="cuda")
    lse = torch.full((h, total), -math.inf, dtype=torch.float64, device="cuda")
    t = 0
    for s, (n, m) in enumerate(zip(_ints(case["lens"]), _ints(case["news"]))):
        j = torch.arange(n, device="cuda")
        ids = st["table"][s].long()[j // page]
        there = ids >= 0
        j, ids = j[there], ids[there]
        for kv in range(h_kv):
            k, v = st["k_pages"][ids, kv, j % page].double(), st["v_pages"][ids, kv, j % page].double()
            if case["e4m3"]:
                k = k * st["k_scale"][ids, kv].double()[:, None]
                v = v * st["v_scale"][ids, kv].double()[:, None]
            at = torch.arange(n - m, n, device="cuda")[:, None]
            ok = j[None] <= at
            if case["window"]:
                ok = ok & ((at - j[None] < case["window"]) | (j[None] < case["sinks"]))
            for head in range(kv * g, kv * g + g):
                logits = (st["q"][head, t:t + m].double() @ k.T) / math.sqrt(d)
                logits = torch.where(ok, logits, -math.inf)
                lse[head, t:t + m] = torch.logsumexp(logits, -1)
                out[head, t:t + m] = torch.softmax(logits, -1) @ v
        t += m
    return [out, lse] if case["lse"] else [out]


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rotate":
        at = st["positions"] if case["given"] else torch.arange(case["tokens"], device="cuda")
        return [_exact_turn(case, st[n], at, -1.0 if case["backward"] else 1.0) for n in ("q", "k")]
    return _exact_append(case, st) if case["kind"] == "append" else _exact_attn(case, st)
