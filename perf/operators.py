"""The operators of generating with a trained model, and what they cost.

A step of generation rotates the new tokens' queries (positions with one axis for text, several for images and video), rotates
their keys and appends them with the values to a paged cache, and attends from the one new token of every sequence over its
cached keys. With `own` false `run` computes an operator from its formula in elementary torch operations; with `own` true it
calls the library. Lengths come from the training workloads' own mixes: one document of 256K tokens, a packed 32K micro-batch,
many documents of 64 to 512 tokens; heads are the library's two models (192 / 128 with K and V per head, 128 / 128 shared).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D_V = 128
THETA = 10000.0
LARGEST_BYTES = 2.7e9           # the largest listed case reads 2.68 GB
MAX_PADDED = 1.5e9              # elements of K and V of a batch padded to its longest sequence (the plain form's layout)


# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------
def _decode(mix, seqs, longest, heads, kv_heads, d_qk, page, length_seed=34318):
    return dict(op="decode", mix=mix, seqs=seqs, longest=longest, heads=heads, kv_heads=kv_heads, d_qk=d_qk, page=page,
                length_seed=length_seed)


def _append(form, mix, seqs, new, cached, heads, d_qk, page, axes, length_seed=34318):
    return dict(op="append", form=form, mix=mix, seqs=seqs, new=new, cached=cached, heads=heads, d_qk=d_qk, page=page,
                axes=axes, length_seed=length_seed)


def _rope(tokens, heads, d, offset, axes, inverse, fused, length_seed=34318):
    return dict(op="rope", tokens=tokens, heads=heads, d=d, offset=offset, axes=axes, inverse=inverse, fused=fused,
                length_seed=length_seed)


def listed():
    return [
        # one user, a short context: launches and a chain of dependent loads are what it costs
        dict(_decode("one", 1, 1000, 16, 16, 192, 64), name="decode_1k"),
        # the sequences of a packed 32K micro-batch generated from at once: lengths of 64 to some thousands
        dict(_decode("lognormal", 19, 8192, 16, 16, 192, 64), name="decode_packed32k"),
        # many short conversations, pages of 16 tokens, 32 heads
        dict(_decode("short", 230, 512, 32, 32, 192, 16), name="decode_short64k"),
        # one document of 256K tokens: everything hangs on splitting its length over the GPU
        dict(_decode("one", 1, 262144, 16, 16, 192, 64), name="decode_256k"),
        # the grouped-query model: heads of 128, eight query heads per key / value head, one 48K document among shorter ones
        dict(_decode("skewed", 24, 49152, 16, 2, 128, 16), name="decode_gqa128_skewed"),
        # one new token of each of 230 conversations into the cache
        dict(_append("mla", "one_each", 230, 1, 300, 32, 192, 16, 1), name="append_one_token_each"),
        # the prompts of a packed 32K micro-batch into the cache, MLA heads
        dict(_append("mla", "lognormal", 19, 32768, 0, 16, 192, 64, 1), name="append_prefill_packed32k"),
        # a video of 64K patches: (time, height, width) positions, two KV heads, k and v slices of a fused projection
        dict(_append("gqa", "even", 4, 65536, 0, 2, 128, 64, 3), name="append_prefill_video64k"),
        # the queries of one new token of each of 230 conversations
        dict(_rope(230, 32, 192, 128, 1, False, False), name="rope_one_token_each"),
        # the queries of the video, all columns rotary, a slice of the fused projection
        dict(_rope(65536, 16, 128, 0, 3, False, True), name="rope_video64k"),
        # training on images: the gradient of the rotated queries (height, width), an odd number of patches
        dict(_rope(8191, 16, 192, 128, 2, True, False), name="rope_image_backward"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw(rng)
        if work(case)["bytes"] > LARGEST_BYTES:
            continue
        if case["op"] == "decode" and case["seqs"] * case["longest"] * case["kv_heads"] * (case["d_qk"] + D_V) > MAX_PADDED:
            continue
        return case


def _draw(rng):
    seed = rng.randrange(1 << 30)
    op = rng.choice(["decode", "decode", "decode", "append", "append", "rope"])
    d_qk = rng.choice([128, 192])
    page = rng.choice([8, 16, 16, 32, 48, 64, 64, 128])
    if op == "decode":
        mix = rng.choice(["one", "even", "lognormal", "short", "skewed"])
        heads = rng.choice([4, 8, 16, 32, 64])
        kv_heads = rng.choice([heads, heads, heads // 4, max(1, heads // 8), max(1, heads // 16)])
        seqs = 1 if mix == "one" else _log_uniform(rng, 2, 256)
        return _decode(mix, seqs, _log_uniform(rng, 1, 262144), heads, kv_heads, d_qk, page, seed)
    if op == "append":
        form, kv_heads = rng.choice([("mla", rng.choice([4, 16, 32])), ("gqa", rng.choice([1, 2, 8]))])
        mix = rng.choice(["one_each", "even", "lognormal"])
        seqs = _log_uniform(rng, 1, 256) if mix == "one_each" else rng.randint(1, 24)
        new = 1 if mix == "one_each" else _log_uniform(rng, 32, 65536)
        return _append(form, mix, seqs, new, _log_uniform(rng, 1, 4096) - 1, kv_heads, 192 if form == "mla" else d_qk, page,
                       rng.choice([1, 2, 3]), seed)
    offset = rng.choice([0, d_qk - 64])
    return _rope(_log_uniform(rng, 1, 131072), rng.choice([1, 4, 8, 16, 32]), d_qk, offset, rng.choice([1, 2, 3, 4]),
                 rng.random() < 0.5, rng.random() < 0.5, seed)


def _lengths(case):
    """Cached tokens of every sequence, the new one among them (decode), or new tokens of every sequence (append)."""
    gen, n, mix = np.random.default_rng(case["length_seed"]), case["seqs"], case["mix"]
    if mix == "one_each":
        return [1] * n
    if case["op"] == "append":
        total = case["new"]
        share = np.ones(n) if mix == "even" else np.exp(gen.normal(0.0, 1.0, n))
        lengths = np.maximum(1, np.floor(total * share / share.sum()).astype(np.int64))
        lengths[-1] = max(1, int(lengths[-1]) + total - int(lengths.sum()))
        return [int(x) for x in lengths]
    longest = case["longest"]
    if mix == "one":
        return [longest] * n
    if mix == "even":
        return [max(1, longest - int(x)) for x in gen.integers(0, 1 + longest // 8, n)]
    if mix == "lognormal":
        return [int(x) for x in np.clip(np.round(np.exp(gen.normal(math.log(max(2.0, longest / 8)), 1.0, n))), 1, longest)]
    lengths = [int(x) for x in gen.integers(max(1, longest // 8), longest + 1, n)]
    if mix == "skewed":                             # one long document, the others up to a twelfth of it
        lengths = [max(1, x // 12) for x in lengths]
        lengths[n // 2] = longest
    return lengths


def _rope_dim(case):
    return case["d"] - case["offset"] if case["op"] == "rope" else 64 if case["form"] == "mla" else case["d_qk"]


def _axis_pairs(case):
    """Rotary pairs of every axis: a quarter for the first of several (time), the rest split evenly."""
    pairs, axes = _rope_dim(case) // 2, case["axes"]
    if axes == 1:
        return [pairs]
    rest = [pairs // 4] + [(pairs - pairs // 4) // (axes - 1)] * (axes - 1)
    rest[-1] += pairs - sum(rest)
    return rest


def work(case):
    if case["op"] == "decode":
        tokens, h, d = sum(_lengths(case)), case["heads"], case["d_qk"]
        pages = sum(-(-x // case["page"]) for x in _lengths(case))
        rows = case["seqs"] * h
        return {"bytes": 2.0 * tokens * case["kv_heads"] * (d + D_V) + rows * (2.0 * (d + D_V) + 4.0) + 4.0 * (pages + case["seqs"]),
                "flops": 2.0 * tokens * h * (d + D_V)}
    if case["op"] == "append":
        tokens, h, d = sum(_lengths(case)), case["heads"], case["d_qk"]
        read = h * (128 + D_V) + 64 if case["form"] == "mla" else h * (d + D_V)
        return {"bytes": tokens * (2.0 * read + 2.0 * h * (d + D_V) + 4.0 * case["axes"]),
                "flops": 3.0 * tokens * _rope_dim(case) * (1 if case["form"] == "mla" else h)}
    elements = case["tokens"] * case["heads"] * case["d"]
    return {"bytes": 4.0 * elements + 4.0 * case["axes"] * case["tokens"],
            "flops": 3.0 * case["tokens"] * case["heads"] * _rope_dim(case)}


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _pages(lengths, page, gen):
    """A page table whose pages lie scattered over a cache with a tenth of it free; entries past a sequence's end are -1."""
    need = [-(-x // page) for x in lengths]
    n_pages = sum(need) + max(2, sum(need) // 10)
    ids = torch.randperm(n_pages, generator=gen, device="cuda")[:sum(need)].to(torch.int32)
    counts = torch.tensor(need, device="cuda")
    col = torch.arange(max(need), device="cuda")
    table = torch.full((len(need), max(need)), -1, dtype=torch.int32, device="cuda")
    table[col[None, :] < counts[:, None]] = ids
    return table, n_pages


def _positions(case, lengths, cached):
    """[axes, tokens] int32: the index in the sequence for one axis; frame, row, column of 16 x 16 patches for several."""
    counts = torch.tensor(lengths, device="cuda")
    first = torch.cumsum(counts, 0) - counts
    index = torch.arange(sum(lengths), device="cuda") - torch.repeat_interleave(first, counts) + cached
    axes = [index] if case["axes"] == 1 else [index // 256, index // 16 % 16, index % 16, index % 7][:case["axes"]]
    return torch.stack(axes).to(torch.int32).contiguous()


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1 + int(seed))
    s = {"op": case["op"]}
    if case["op"] == "rope":
        tokens, h, d = case["tokens"], case["heads"], case["d"]
        x = _normal(gen, tokens, h + 4, d)[:, :h] if case["fused"] else _normal(gen, tokens, h, d)
        s.update(x=x, y=torch.empty((tokens, h, d), dtype=torch.bfloat16, device="cuda"), offset=case["offset"],
                 inverse=case["inverse"], positions=_positions(case, [tokens], int(seed) % 1000),
                 axis_pairs=_axis_pairs(case))
        if own:
            import paper_2609_34318_b200 as P
            s["rope"] = P.rope_spec(THETA, _rope_dim(case), case["offset"], s["axis_pairs"])
        return s
    lengths, page, d = _lengths(case), case["page"], case["d_qk"]
    if case["op"] == "decode":
        h, hk = case["heads"], case["kv_heads"]
        table, n_pages = _pages(lengths, page, gen)
        s.update(q=_normal(gen, len(lengths), h, d), scale=d ** -0.5, heads=h,
                 out=torch.empty((len(lengths), h, D_V), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty((h, len(lengths)), dtype=torch.float32, device="cuda"))
        held = lengths
    else:
        hk, cached = case["heads"], case["cached"]
        held = [x + cached for x in lengths]
        table, n_pages = _pages(held, page, gen)
        tokens = sum(lengths)
        s.update(form=case["form"], tokens=tokens, positions=_positions(case, lengths, cached), axis_pairs=_axis_pairs(case),
                 offset=d - _rope_dim(case), one_each=case["mix"] == "one_each",
                 cu_new=torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda"))
        if case["form"] == "mla":
            s.update(kv_up=_normal(gen, tokens, hk, 128 + D_V), k_pe=_normal(gen, tokens, 64))
        else:                                       # slices of a projection whose rows hold 16 query heads before them
            fused = _normal(gen, tokens, 16 * d + hk * (d + D_V))
            s.update(k=fused[:, 16 * d:16 * d + hk * d].unflatten(1, (hk, d)),
                     v=fused[:, 16 * d + hk * d:].unflatten(1, (hk, D_V)))
    s.update(k_pages=_normal(gen, n_pages, hk, page, d), v_pages=_normal(gen, n_pages, hk, page, D_V), table=table,
             seq_lens=torch.tensor(held, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2609_34318_b200 as P
        s["cache"] = P.paged_cache(s["k_pages"], s["v_pages"], s["table"], s["seq_lens"])
        if case["op"] == "decode":
            s["workspace"] = torch.zeros(P.hydra_workspace_bytes_decode(s["heads"], hk), dtype=torch.uint8, device="cuda")
        else:
            s["rope"] = P.rope_spec(THETA, _rope_dim(case), s["offset"], s["axis_pairs"])
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "decode":
        return _plain_decode(s)
    if s["op"] == "append":
        return _plain_append(s)
    return _plain_rotate(s["x"], s["positions"], s["offset"], s["axis_pairs"], s["inverse"])


def _run_own(s):
    import paper_2609_34318_b200 as P
    if s["op"] == "decode":
        P.hydra_attn_decode(s["q"], s["cache"], s["heads"], s["scale"], s["out"], s["lse"], s["workspace"])
        return s["out"], s["lse"]
    if s["op"] == "append":
        cu_new = None if s["one_each"] else s["cu_new"]
        if s["form"] == "mla":
            P.hydra_mla_kv_append(s["kv_up"], s["k_pe"], s["positions"], cu_new, s["tokens"], s["rope"], s["cache"])
        else:
            P.hydra_kv_append(s["k"], s["v"], s["positions"], cu_new, s["tokens"], s["rope"], s["cache"])
        return s["k_pages"], s["v_pages"]
    tokens, h, d = s["x"].shape
    P.hydra_rope_axes(s["x"], s["positions"], tokens, h, d, s["rope"], s["inverse"], s["y"])
    return s["y"]


def _angles(positions, axis_pairs):
    """[tokens, pairs] float64: pair i turns by the position on its axis times theta^(-2i / dim)."""
    pairs = sum(axis_pairs)
    axis = torch.repeat_interleave(torch.arange(len(axis_pairs), device=positions.device),
                                   torch.tensor(axis_pairs, device=positions.device), output_size=pairs)
    rate = THETA ** (-torch.arange(pairs, dtype=torch.float64, device=positions.device) / pairs)
    return positions[axis].T.double() * rate


def _plain_rotate(x, positions, offset, axis_pairs, inverse):
    """x [tokens, heads, d]: the pairs (2i, 2i + 1) of the columns from `offset` on, turned by their angles."""
    dim = 2 * sum(axis_pairs)
    angle = _angles(positions, axis_pairs)[:, None, :]
    c, s = angle.cos().float(), angle.sin().float() * (-1.0 if inverse else 1.0)
    y = x.float()
    a, b = y[..., offset:offset + dim:2], y[..., offset + 1:offset + dim:2]
    turned = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    return torch.cat((y[..., :offset], turned, y[..., offset + dim:]), -1).to(x.dtype)


def _plain_append(s):
    if s["form"] == "mla":
        nope = s["kv_up"].shape[2] - D_V
        turned = _plain_rotate(s["k_pe"][:, None, :], s["positions"], 0, s["axis_pairs"], False)
        k = torch.cat((s["kv_up"][..., :nope], turned.expand(-1, s["kv_up"].shape[1], -1)), -1)
        v = s["kv_up"][..., nope:]
    else:
        k, v = _plain_rotate(s["k"], s["positions"], s["offset"], s["axis_pairs"], False), s["v"]
    page = s["k_pages"].shape[2]
    cu = s["cu_new"].long()
    t = torch.arange(s["tokens"], device=k.device)
    b = torch.searchsorted(cu, t, right=True) - 1
    at = s["seq_lens"].long()[b] - (cu[b + 1] - t)          # its place in the sequence; all of these have a page
    to = s["table"].long()[b, at // page]
    s["k_pages"][to, :, at % page] = k
    s["v_pages"][to, :, at % page] = v
    return s["k_pages"], s["v_pages"]


def _plain_decode(s):
    """Over the batch padded to its longest sequence; a position counts where it lies before the end and has a page."""
    n, h, d = s["q"].shape
    hk, page = s["k_pages"].shape[1:3]
    table = s["table"].long()
    there = (table >= 0) & (table < s["k_pages"].shape[0])
    at = torch.where(there, table, 0)
    k = s["k_pages"][at].transpose(1, 2).reshape(n, hk, -1, d).float()
    v = s["v_pages"][at].transpose(1, 2).reshape(n, hk, -1, D_V).float()
    seen = there.repeat_interleave(page, 1) & (torch.arange(k.shape[2], device=k.device) < s["seq_lens"][:, None])
    v = v.masked_fill(~seen[:, None, :, None], 0.0)
    scores = (s["q"].float().view(n, hk, h // hk, d) @ k.transpose(2, 3)) * s["scale"]
    scores = scores.masked_fill(~seen[:, None, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (scores - top).exp()
    total = p.sum(-1, keepdim=True)
    out = torch.where(total > 0, (p @ v) / total, 0.0).to(s["q"].dtype)
    return out.view(n, h, D_V), (top + total.log()).view(n, h).T.contiguous()


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_rotate(x, positions, offset, axis_pairs, inverse):
    """As products of complex numbers; positions are whole, x [tokens, heads, d] is turned where its pairs stand."""
    dim = 2 * sum(axis_pairs)
    y = x.double().clone()
    first = 0
    for axis, count in enumerate(axis_pairs):
        for i in range(first, first + count):
            angle = positions[axis].double() * math.exp(-2.0 * i / dim * math.log(THETA))
            turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle)[:, None]
            z = torch.complex(y[..., offset + 2 * i], y[..., offset + 2 * i + 1]) * turn
            y[..., offset + 2 * i], y[..., offset + 2 * i + 1] = z.real, z.imag
        first += count
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rotate(s["x"], s["positions"], s["offset"], s["axis_pairs"], s["inverse"])
    lengths, page = _lengths(case), case["page"]
    if case["op"] == "append":
        if case["form"] == "mla":
            pe = _exact_rotate(s["k_pe"][:, None, :], s["positions"], 0, s["axis_pairs"], False)
            up = s["kv_up"].double()
            k, v = torch.cat((up[..., :128], pe.repeat(1, case["heads"], 1)), 2), up[..., 128:]
        else:
            k = _exact_rotate(s["k"], s["positions"], s["offset"], s["axis_pairs"], False)
            v = s["v"].double()
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        t0 = 0
        for b, n in enumerate(lengths):
            places = torch.arange(case["cached"], case["cached"] + n, device="cuda")
            to, row = s["table"][b].long()[places // page], places % page
            for a in range(case["heads"]):
                k_pages[to, a, row], v_pages[to, a, row] = k[t0:t0 + n, a], v[t0:t0 + n, a]
            t0 += n
        return k_pages, v_pages
    h, hk = case["heads"], case["kv_heads"]
    out = torch.zeros((case["seqs"], h, D_V), dtype=torch.float64, device="cuda")
    lse = torch.full((h, case["seqs"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths):
        places = torch.arange(n, device="cuda")
        to, row = s["table"][b].long()[places // page], places % page
        for a in range(hk):
            k, v = s["k_pages"][to, a, row].double(), s["v_pages"][to, a, row].double()
            heads = slice(a * (h // hk), (a + 1) * (h // hk))
            scores = s["q"][b, heads].double() @ k.T * s["scale"]
            lse[heads, b] = torch.logsumexp(scores, 1)
            out[b, heads] = torch.softmax(scores, 1) @ v
    return out, lse
