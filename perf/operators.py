"""Operators over a paged key-value cache: what is measured of them, and their plain forms.

A case is a dict of plain values.  ``kind`` names the operator:

* ``rotate``   apack_rotary: rotary positions of the heads of packed token rows
* ``append``   apack_rotary_append: rotary positions of new tokens' queries and keys, keys and values
               written to the pages of their sequences
* ``attend``   apack_paged_decode_attention: one decode token per sequence over its pages
* ``compact``  apack_paged_compact: the kept rows of every sequence moved to pages of their own
* ``copy``     apack_copy_pages: pages copied over all layers (a forked sequence's own pages)

Where ``own`` is false ``run`` computes them with elementary torch operations.
"""

import math
import random

import torch

own = False

BASE = 1000000.0


def listed():
    return [
        # The query rows of one question at a pruning layer, rotated before they score the cache: small.
        dict(name="rotate_question", kind="rotate", n=256, heads=32, spare=4, d=128, dtype="bf16", layout="half",
             rdim=128, axes=3, scaling="none", factor=1.0, far=135000, transpose=False),
        # The gradient with respect to the unrotated rows of a one-minute clip's prompt.
        dict(name="rotate_minute_gradient", kind="rotate", n=8780, heads=18, spare=2, d=128, dtype="fp16",
             layout="half", rdim=128, axes=1, scaling="none", factor=1.0, far=8780, transpose=True),
        # One decode step of a batch: a token each, at the end of caches of any length; neighbouring
        # elements rotated together, half of each head, stretched to a longer context.
        dict(name="append_step61", kind="append", n=61, heads="32/8", d=128, dtype="fp16", layout="pairs", rdim=64,
             axes=1, scaling="yarn", factor=8.0, far=200000, page=16, order="hnd", prompt=False, shape=1),
        # The whole prompt of a two-minute clip, three position axes, into pages of 64 tokens.
        dict(name="append_prompt_2min", kind="append", n=27144, heads="28/4", d=128, dtype="bf16", layout="half",
             rdim=128, axes=3, scaling="none", factor=1.0, far=27144, page=64, order="nhd", prompt=True, shape=2),
        # The smallest call: the pruned cache of a ten-second clip.
        dict(name="attend_10s", kind="attend", heads="28/4", d=128, dtype="bf16", seqs=1, len_lo=473, len_hi=473,
             page=16, order="nhd", shape=3),
        # The unpruned ten-minute sequence.
        dict(name="attend_10min", kind="attend", heads="28/4", d=128, dtype="bf16", seqs=1, len_lo=135272,
             len_hi=135272, page=64, order="nhd", shape=4),
        # A serving batch over pruned caches of clips of many lengths.
        dict(name="attend_batch16", kind="attend", heads="28/4", d=128, dtype="bf16", seqs=16, len_lo=600,
             len_hi=12000, page=16, order="nhd", shape=5),
        # Many short conversations, a KV head per query head, narrow heads.
        dict(name="attend_many_short", kind="attend", heads="8/8", d=64, dtype="fp16", seqs=96, len_lo=1, len_hi=3000,
             page=32, order="hnd", shape=6),
        # A prefill's contiguous caches of 24 layers sliced into pages at the first pruning layer.
        dict(name="compact_prompt_2min", kind="compact", heads="28/4", d=128, dtype="bf16", layers=24, seqs=1,
             len_lo=27144, len_hi=27144, keep=0.436, page=64, source="slab", shape=7),
        # A later pruning step of a serving batch, from pages to pages.
        dict(name="compact_batch", kind="compact", heads="16/2", d=128, dtype="bf16", layers=6, seqs=13, len_lo=300,
             len_hi=9000, keep=0.7, page=16, source="pages", shape=8),
        # One sequence forked: its last, partly filled page in every layer.
        dict(name="copy_fork", kind="copy", heads="28/4", d=128, dtype="bf16", layers=28, pairs=1, page=16,
             order="nhd"),
        # A batch of sequences moved to pages of their own.
        dict(name="copy_batch", kind="copy", heads="28/4", d=128, dtype="bf16", layers=28, pairs=257, page=16,
             order="nhd"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rotation(rng, d):
    rdim = rng.choice((d, d, d // 2))
    scaling = rng.choice(("none", "none", "linear", "ntk", "yarn"))
    return dict(layout=rng.choice(("half", "pairs")), rdim=rdim, axes=rng.choice((1, 3)), scaling=scaling,
                factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)))


def draw(rng):
    """Another case of the same ranges; costs stay below the largest listed ones."""
    kind = rng.choice(("rotate", "append", "append", "attend", "attend", "attend", "compact", "copy"))
    shape = rng.randrange(1 << 20)
    dtype = rng.choice(("bf16", "bf16", "fp16"))
    d = rng.choice((128, 128, 64))
    page = rng.choice((16, 16, 32, 64, 128))
    order = rng.choice(("nhd", "nhd", "hnd"))
    heads = rng.choice(("28/4", "28/4", "16/2", "32/8", "8/8", "12/2", "8/1"))
    hq, hkv = map(int, heads.split("/"))
    if kind == "rotate":
        return dict(kind=kind, n=_log_uniform(rng, 1, 16000), heads=hq + hkv, spare=hkv, d=d, dtype=dtype,
                    far=_log_uniform(rng, 500, 1000000), transpose=rng.random() < 0.4, **_rotation(rng, d))
    if kind == "append":
        prompt = rng.random() < 0.5
        return dict(kind=kind, n=_log_uniform(rng, 2, 20000) if prompt else _log_uniform(rng, 1, 256), heads=heads,
                    d=d, dtype=dtype, far=_log_uniform(rng, 500, 1000000), page=page, order=order, prompt=prompt,
                    shape=shape, **_rotation(rng, d))
    if kind == "attend":
        seqs = rng.choice((1, 1, rng.randint(2, 16), rng.randint(17, 128)))
        hi = _log_uniform(rng, 16, min(135000, 300000 // seqs))
        return dict(kind=kind, heads=heads, d=d, dtype=dtype, seqs=seqs, len_lo=hi if seqs == 1 else 1, len_hi=hi,
                    page=page, order=order, shape=shape)
    row = 2 * d * hkv
    if kind == "compact":
        seqs = rng.choice((1, rng.randint(2, 16)))
        hi = _log_uniform(rng, 60, 30000 // seqs)
        layers = rng.randint(1, max(1, min(28, int(6e8 // (seqs * hi * row)))))
        return dict(kind=kind, heads=heads, d=d, dtype=dtype, layers=layers, seqs=seqs,
                    len_lo=hi if seqs == 1 else max(1, hi // 8), len_hi=hi, keep=round(rng.uniform(0.1, 0.95), 3),
                    page=page, source=rng.choice(("slab", "pages")), shape=shape)
    layers = rng.randint(1, 28)
    most = max(1, min(400, int(2e8 // (layers * page * row))))
    return dict(kind=kind, heads=heads, d=d, dtype=dtype, layers=layers, pairs=_log_uniform(rng, 1, most), page=page,
                order=order)


# ---------------------------------------------------------------- inputs


DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _heads(case):
    hq, hkv = case["heads"].split("/")
    return int(hq), int(hkv)


def _lengths(case):
    r = random.Random(case["shape"])
    return [_log_uniform(r, case["len_lo"], case["len_hi"]) for _ in range(case["seqs"])]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, dtype, *shape, scale=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=g)


def _pool(g, case, layers, pages, scale=1.0):
    """[layers, pages, page, heads, d] of a pool whose pages hold their tokens, or their heads, outermost."""
    hkv = _heads(case)[1] if "/" in str(case["heads"]) else case["heads"]
    if case.get("order", "nhd") == "hnd":
        return _normal(g, DTYPES[case["dtype"]], layers, pages, hkv, case["page"], case["d"], scale=scale).permute(0, 1, 3, 2, 4)
    return _normal(g, DTYPES[case["dtype"]], layers, pages, case["page"], hkv, case["d"], scale=scale)


def _tables(g, lens, page, spare=0):
    """Pages of every sequence, in random order; -1 behind a sequence's last page.  Also the number of
    pages of the pool."""
    need = [-(-n // page) for n in lens]
    total = sum(need) + spare
    perm = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, total


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _frequencies(case):
    """Radians per position of every pair, and the factor on cos and sin, in 64 bits on the host."""
    r, factor, scaling = case["rdim"], case["factor"], case["scaling"]
    base = BASE * factor ** (r / (r - 2)) if scaling == "ntk" else BASE
    freq = base ** -(torch.arange(0, r, 2, dtype=torch.float64) / r)
    if scaling == "linear":
        return freq / factor, 1.0
    if scaling == "yarn":
        turns = 32768 * freq / (2 * math.pi)          # over the context that the model was trained on
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        return freq * keep + freq / factor * (1 - keep), 0.1 * math.log(factor) + 1.0
    return freq, 1.0


def _sections(case):
    """Pairs per position axis: all, or a quarter and two halves of the rest."""
    pairs = case["rdim"] // 2
    if case["axes"] == 1:
        return [pairs]
    return [pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8]


def _positions(g, case, n):
    """Rising positions with the gaps that pruning leaves, up to `far`; the other axes near the first."""
    first = torch.randint(0, max(1, case["far"]), (n,), generator=g, device="cuda").sort().values
    rows = [first] + [(first - torch.randint(0, 60, (n,), generator=g, device="cuda")).clamp(min=0)
                      for _ in range(case["axes"] - 1)]
    return torch.stack(rows).to(torch.int32)


def _rotary_handle(case):
    import paper_2608_08794_gb300 as ap
    return ap.Rotary(case["rdim"], base=BASE, interleaved=case["layout"] == "pairs", scaling=case["scaling"],
                     factor=case["factor"], original_len=32768,
                     sections=_sections(case) if case["axes"] > 1 else None)


def _workspace(nbytes):
    raw = torch.zeros(nbytes + 256, dtype=torch.uint8, device="cuda")
    off = (-raw.data_ptr()) % 256
    return raw[off:off + nbytes]


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    dtype = DTYPES[case["dtype"]]
    s = dict(case=case)
    if kind == "rotate":
        n, h = case["n"], case["heads"]
        rows = _normal(g, dtype, n, h + case["spare"], case["d"])     # a projection's output: values behind the heads
        s.update(x=rows[:, :h], positions=_positions(g, case, n),
                 out=torch.empty(n, h, case["d"], dtype=dtype, device="cuda"))
        s["freq"] = _frequencies(case)[0].cuda()
        if own:
            s["rotary"] = _rotary_handle(case)
    elif kind == "append":
        hq, hkv = _heads(case)
        n, page = case["n"], case["page"]
        r = random.Random(case["shape"])
        if case["prompt"]:
            lens, seqs = [n], torch.zeros(n, dtype=torch.int32, device="cuda")
            rows = torch.arange(n, dtype=torch.int32, device="cuda")
        else:
            lens = [_log_uniform(r, 1, 3000) for _ in range(n)]
            seqs, rows = torch.arange(n, dtype=torch.int32, device="cuda"), _int32([x - 1 for x in lens])
        table, pages = _tables(g, lens, page, spare=2)
        qkv = _normal(g, dtype, n, hq + 2 * hkv, case["d"])
        s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], positions=_positions(g, case, n),
                 rows=rows, seqs=seqs, table=table, k_pool=_pool(g, case, 1, pages), v_pool=_pool(g, case, 1, pages),
                 q_out=torch.empty(n, hq, case["d"], dtype=dtype, device="cuda"))
        s["freq"] = _frequencies(case)[0].cuda()
        if own:
            import paper_2608_08794_gb300 as ap
            s["rotary"] = _rotary_handle(case)
            s["cache"] = ap.PagedCache(s["k_pool"], s["v_pool"], table)
    elif kind == "attend":
        hq, hkv = _heads(case)
        lens = _lengths(case)
        table, pages = _tables(g, lens, case["page"], spare=2)
        s.update(q=_normal(g, dtype, len(lens), hq, case["d"]), k_pool=_pool(g, case, 1, pages, scale=1.5),
                 v_pool=_pool(g, case, 1, pages), table=table, lens=_int32(lens), longest=max(lens),
                 out=torch.empty(len(lens), hq, case["d"], dtype=dtype, device="cuda"),
                 lse=torch.empty(len(lens), hq, dtype=torch.float32, device="cuda"))
        if own:
            import paper_2608_08794_gb300 as ap
            s["cache"] = ap.PagedCache(s["k_pool"], s["v_pool"], table)
            s["ws"] = _workspace(ap.apack_paged_decode_workspace_size(s["cache"], hq))
    elif kind == "compact":
        hkv, layers, page = _heads(case)[1], case["layers"], case["page"]
        lens = _lengths(case)
        kept = [max(1, int(case["keep"] * n)) for n in lens]
        at, picks = 0, []
        for n, k in zip(lens, kept):
            picks.append(torch.randperm(n, generator=g, device="cuda")[:k].sort().values + at)
            at += n
        s.update(keep=torch.cat(picks).to(torch.int32), n_out=sum(kept),
                 cu_src=_int32([sum(lens[:b]) for b in range(len(lens) + 1)]),
                 cu_dst=_int32([sum(kept[:b]) for b in range(len(kept) + 1)]))
        if case["source"] == "slab":              # one contiguous slab per layer: a single page of all tokens
            shape = (layers, 1, sum(lens), hkv, case["d"])
            s.update(k_src=_normal(g, dtype, *shape), v_src=_normal(g, dtype, *shape),
                     src_table=torch.zeros(len(lens), 1, dtype=torch.int32, device="cuda"))
        else:
            s["src_table"], pages = _tables(g, lens, page, spare=2)
            s.update(k_src=_pool(g, case, layers, pages), v_src=_pool(g, case, layers, pages))
        s["dst_table"], pages = _tables(g, kept, page, spare=2)
        s.update(k_dst=_pool(g, case, layers, pages), v_dst=_pool(g, case, layers, pages))
        if own:
            import paper_2608_08794_gb300 as ap
            s["src"] = ap.PagedCache(s["k_src"], s["v_src"], s["src_table"])
            s["dst"] = ap.PagedCache(s["k_dst"], s["v_dst"], s["dst_table"])
    else:
        n = case["pairs"]
        pages = 2 * n + 3
        s.update(k_pool=_pool(g, case, case["layers"], pages), v_pool=_pool(g, case, case["layers"], pages),
                 pairs=torch.randperm(pages, generator=g, device="cuda")[:2 * n].view(n, 2).to(torch.int32))
        if own:
            import paper_2608_08794_gb300 as ap
            s["cache"] = ap.PagedCache(s["k_pool"], s["v_pool"], torch.zeros(1, 1, dtype=torch.int32, device="cuda"))
    return s


# ---------------------------------------------------------------- plain forms


def _rotated(case, x, positions, freq, transpose=False):
    """Each pair (a, b) of a row becomes m (a cos - b sin, b cos + a sin); the transpose turns the other way."""
    axis = torch.repeat_interleave(torch.arange(case["axes"], device=x.device),
                                   torch.tensor(_sections(case), device=x.device))
    angle = positions[axis].double().T * freq          # far positions: the angle needs 64 bits
    m = 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "yarn" else 1.0
    cos, sin = (m * angle.cos()).float()[:, None], (m * angle.sin()).float()[:, None]
    if transpose:
        sin = -sin
    r, y = case["rdim"], x.float()
    if case["layout"] == "pairs":
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, y[..., r:]), -1).to(x.dtype)


def _plain_attend(s):
    case = s["case"]
    hq, hkv = _heads(case)
    page, longest, scale = case["page"], s["longest"], 1.0 / math.sqrt(case["d"])
    t = torch.arange(longest, device="cuda")
    pages = s["table"][:, t // page].long().clamp(min=0)
    k = s["k_pool"][0][pages, t % page].float()                       # [B, T, Hkv, D], padded to the longest
    v = s["v_pool"][0][pages, t % page].float()
    there = (t < s["lens"][:, None])[:, None, None]                     # [B, 1, 1, T]
    q = s["q"].float().view(-1, hkv, hq // hkv, case["d"])
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) * scale                  # [B, Hkv, G, T]
    x = x.masked_fill(~there, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - top).exp()
    total = p.sum(-1, keepdim=True)
    v = v.masked_fill(~there[:, 0, 0, :, None, None], 0.0)
    out = torch.matmul(p / total, v.permute(0, 2, 1, 3))
    lse = (top + total.log())[..., 0]
    return [out.reshape(-1, hq, case["d"]).to(s["q"].dtype), lse.reshape(-1, hq)]


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "rotate":
        return [_rotated(case, s["x"], s["positions"], s["freq"], case["transpose"])]
    if kind == "append":
        page = case["page"]
        q_out = _rotated(case, s["q"], s["positions"], s["freq"])
        at = s["table"][s["seqs"].long(), (s["rows"] // page).long()].long()
        s["k_pool"][0][at, (s["rows"] % page).long()] = _rotated(case, s["k"], s["positions"], s["freq"])
        s["v_pool"][0][at, (s["rows"] % page).long()] = s["v"]
        return [q_out, s["k_pool"], s["v_pool"]]
    if kind == "attend":
        return _plain_attend(s)
    if kind == "compact":
        j = torch.arange(s["n_out"], device="cuda")
        seq = torch.searchsorted(s["cu_dst"], j, right=True) - 1
        to = j - s["cu_dst"][seq]
        page = case["page"]
        if case["source"] == "slab":
            source = torch.zeros_like(j), s["keep"].long()
        else:
            row = s["keep"] - s["cu_src"][seq]
            source = s["src_table"][seq, (row // page).long()].long(), (row % page).long()
        dest = s["dst_table"][seq, to // page].long(), to % page
        s["k_dst"][:, dest[0], dest[1]] = s["k_src"][:, source[0], source[1]]
        s["v_dst"][:, dest[0], dest[1]] = s["v_src"][:, source[0], source[1]]
        return [s["k_dst"], s["v_dst"]]
    src, dst = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    s["k_pool"][:, dst] = s["k_pool"][:, src]
    s["v_pool"][:, dst] = s["v_pool"][:, src]
    return [s["k_pool"], s["v_pool"]]


def _own(s):
    import paper_2608_08794_gb300 as ap
    case, kind = s["case"], s["case"]["kind"]
    if kind == "rotate":
        ap.apack_rotary(s["rotary"], s["x"], s["positions"], s["out"], transpose=case["transpose"])
        return [s["out"]]
    if kind == "append":
        ap.apack_rotary_append(s["rotary"], s["cache"], 0, s["q"], s["k"], s["v"], s["q_out"], s["positions"],
                               s["rows"], seqs=s["seqs"])
        return [s["q_out"], s["k_pool"], s["v_pool"]]
    if kind == "attend":
        ap.apack_paged_decode_attention(s["cache"], 0, s["lens"], s["q"], s["out"], s["ws"], lse=s["lse"])
        return [s["out"], s["lse"]]
    if kind == "compact":
        ap.apack_paged_compact(s["src"], s["dst"], s["cu_dst"], s["n_out"], keep_idx=s["keep"],
                               cu_src=None if case["source"] == "slab" else s["cu_src"])
        return [s["k_dst"], s["v_dst"]]
    ap.apack_copy_pages(s["cache"], s["pairs"])
    return [s["k_pool"], s["v_pool"]]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind = case["kind"]
    size = 2 * case["d"]
    if kind == "rotate":
        cells = case["n"] * case["heads"]
        return {"bytes": 2 * cells * size + 4 * case["n"] * case["axes"], "flops": 3 * cells * case["rdim"]}
    hq, hkv = _heads(case)
    if kind == "append":
        n = case["n"]
        return {"bytes": 2 * n * (hq + 2 * hkv) * size + 4 * n * (case["axes"] + 2), "flops": 3 * n * (hq + hkv) * case["rdim"]}
    if kind == "attend":
        lens = _lengths(case)
        total = sum(lens)
        return {"bytes": 2 * total * hkv * size + len(lens) * hq * (2 * size + 4) + 4 * sum(-(-n // case["page"]) for n in lens),
                "flops": 4 * total * hq * case["d"]}
    if kind == "compact":
        rows = sum(max(1, int(case["keep"] * n)) for n in _lengths(case))
        return {"bytes": 4 * rows * hkv * size * case["layers"] + 4 * rows, "flops": 0}
    return {"bytes": 4 * case["pairs"] * case["page"] * hkv * size * case["layers"] + 8 * case["pairs"], "flops": 0}


# ---------------------------------------------------------------- from the definitions, in 64 bits


def _turned64(case, x, positions, back=False):
    """The pairs as complex numbers times m e^(i angle)."""
    freq, m = _frequencies(case)
    axis = []
    for a, count in enumerate(_sections(case)):
        axis += [a] * count
    angle = positions.double().cpu()[axis].T * freq
    factor = torch.polar(torch.full_like(angle, m), -angle if back else angle).to(x.device)[:, None]
    y, r = x.double(), case["rdim"]
    out = y.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if case["layout"] == "pairs" else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * factor
    out[..., first], out[..., second] = z.real, z.imag
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind not in ("rotate", "append", "attend"):
        return None                    # rows are moved, nothing is computed
    s = prepare(case, seed)
    if kind == "rotate":
        return [_turned64(case, s["x"], s["positions"], case["transpose"])]
    if kind == "append":
        rows, seqs = s["rows"].tolist(), s["seqs"].tolist()
        table = s["table"].cpu()
        page = [int(table[b, r // case["page"]]) for b, r in zip(seqs, rows)]
        slot = [r % case["page"] for r in rows]
        k, v = s["k_pool"].double(), s["v_pool"].double()
        k[0, page, slot] = _turned64(case, s["k"], s["positions"])
        v[0, page, slot] = s["v"].double()
        return [_turned64(case, s["q"], s["positions"]), k, v]
    hq, hkv = _heads(case)
    outs, lses = [], []
    for b, n in enumerate(s["lens"].tolist()):
        pages = s["table"][b, :-(-n // case["page"])].long()
        k = s["k_pool"][0, pages].double().flatten(0, 1)[:n]
        v = s["v_pool"][0, pages].double().flatten(0, 1)[:n]
        out, lse = [], []
        for h in range(hq):
            x = k[:, h // (hq // hkv)] @ s["q"][b, h].double() / math.sqrt(case["d"])
            z = torch.logsumexp(x, 0)
            lse.append(z)
            out.append((x - z).exp() @ v[:, h // (hq // hkv)])
        outs.append(torch.stack(out))
        lses.append(torch.stack(lse))
    return [torch.stack(outs), torch.stack(lses)]
