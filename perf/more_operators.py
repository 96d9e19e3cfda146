"""Operators of a serving batch over paged caches: what is measured of them, and their plain forms.

A case is a dict of plain values.  ``kind`` names the operator:

* ``share``   apack_paged_group_plan once and apack_paged_group_attention per layer: attention of one or more new
              tokens per sequence over its pages, where groups of sequences share their first pages (questions about
              one video), each group's shared rows read once
* ``step``    apack_pages_release, then apack_pages_extend: the rows that a step gives up, and room for the next ones:
              page tables, lengths and the map from new rows to slots, kept on the GPU
* ``fork``    apack_pages_release, apack_pages_fork, apack_pages_extend: the last questions about cached videos leave,
              new ones share their pages, and get pages of their own where they write

Where ``own`` is false ``run`` computes them with elementary torch operations.
"""

import math
import random

import torch

own = False


def listed():
    return [
        # Two follow-up questions about a ten-second clip, one token each: the smallest call.
        dict(name="share_pair_10s", kind="share", heads="28/4", d=128, dtype="bf16", layers=1, groups=1, members=2,
             pre_lo=473, pre_hi=473, own_lo=9, own_hi=40, new_lo=1, new_hi=1, page=16, order="nhd", shape=1),
        # 64 conversations about one ten-minute video, pruned: a decode step of four layers.
        dict(name="share_decode64", kind="share", heads="28/4", d=128, dtype="bf16", layers=4, groups=1, members=64,
             pre_lo=22772, pre_hi=22772, own_lo=20, own_hi=400, new_lo=1, new_hi=1, page=64, order="nhd", shape=2),
        # Several videos, some with one conversation and some with many, few heads.
        dict(name="share_videos", kind="share", heads="16/2", d=128, dtype="fp16", layers=2, groups=7, members=24,
             pre_lo=300, pre_hi=12000, own_lo=1, own_hi=900, new_lo=1, new_hi=1, page=16, order="nhd", shape=3),
        # Many short prompts of one kind each, a KV head per query head, narrow heads, a few drafted tokens.
        dict(name="share_short_drafts", kind="share", heads="8/8", d=64, dtype="fp16", layers=1, groups=12, members=14,
             pre_lo=100, pre_hi=3000, own_lo=1, own_hi=120, new_lo=1, new_hi=5, page=32, order="hnd", shape=4),
        # The tokens of 16 new questions about one pruned ten-minute video.
        dict(name="share_questions16", kind="share", heads="28/4", d=128, dtype="bf16", layers=1, groups=1, members=16,
             pre_lo=22772, pre_hi=22772, own_lo=0, own_hi=0, new_lo=12, new_hi=60, page=64, order="nhd", shape=5),
        # The last 2,048 tokens of a two-minute clip's prompt: nothing is shared, causal among themselves.
        dict(name="share_prompt_chunk", kind="share", heads="28/4", d=128, dtype="bf16", layers=1, groups=1, members=1,
             pre_lo=25096, pre_hi=25096, own_lo=0, own_hi=0, new_lo=2048, new_hi=2048, page=16, order="nhd", shape=6),
        # Eight questions about the unpruned ten-minute video: the largest.
        dict(name="share_questions_unpruned", kind="share", heads="28/4", d=128, dtype="bf16", layers=1, groups=1,
             members=8, pre_lo=135272, pre_hi=135272, own_lo=0, own_hi=0, new_lo=25, new_hi=60, page=64, order="nhd",
             shape=7),
        # One decode step of a batch: a row each.
        dict(name="step_decode61", kind="step", seqs=61, len_lo=300, len_hi=23000, drop_lo=1, drop_hi=1, page=16,
             pages=60000, shape=8),
        # Drafted tokens, of which some were rejected: rows go and rows come.
        dict(name="step_drafts256", kind="step", seqs=256, len_lo=100, len_hi=9000, drop_lo=0, drop_hi=8, page=16,
             pages=40000, shape=9),
        # Prompts of clips of up to two minutes enter.
        dict(name="step_prompts16", kind="step", seqs=16, len_lo=1298, len_hi=27144, drop_lo=1298, drop_hi=27144,
             page=64, pages=9000, shape=10),
        # A thousand prompts at once: the largest slot map.
        dict(name="step_prompts1000", kind="step", seqs=1000, len_lo=100, len_hi=2000, drop_lo=50, drop_hi=2000,
             page=16, pages=150000, shape=11),
        # Questions about a few cached videos: every one shares a video's pages and copies its last.
        dict(name="fork_questions64", kind="fork", seqs=64, parents=5, len_lo=4644, len_hi=22772, new_lo=12, new_hi=60,
             page=16, pages=9000, shape=12),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges; costs stay below the largest listed ones."""
    kind = rng.choice(("share", "share", "share", "step", "step", "fork"))
    shape = rng.randrange(1 << 20)
    page = rng.choice((16, 16, 32, 64, 128))
    if kind == "step":
        seqs = _log_uniform(rng, 1, 1000)
        hi = _log_uniform(rng, 40, min(30000, 1500000 // seqs))
        drop = rng.choice((1, 9, hi))
        return dict(kind=kind, seqs=seqs, len_lo=max(1, hi // 20), len_hi=hi, drop_lo=min(drop, rng.choice((0, 1))),
                    drop_hi=drop, page=page, pages=seqs * (hi // page + 2) + 100, shape=shape)
    if kind == "fork":
        seqs, parents = _log_uniform(rng, 1, 400), rng.randint(1, 9)
        hi = _log_uniform(rng, 100, 25000)
        return dict(kind=kind, seqs=seqs, parents=parents, len_lo=max(1, hi // 8), len_hi=hi, new_lo=1,
                    new_hi=_log_uniform(rng, 1, 100), page=page, pages=parents * (hi // page + 2) + seqs * 110 + 100,
                    shape=shape)
    d = rng.choice((128, 128, 128, 64))
    heads = rng.choice(("28/4", "28/4", "16/2", "32/8", "8/8", "12/2", "8/1"))
    groups = rng.choice((1, 1, rng.randint(2, 16)))
    members = _log_uniform(rng, 1, 64 if groups == 1 else 24)
    hi = _log_uniform(rng, 64, 135000 if groups == 1 else 60000 // groups)
    layers = rng.choice((1, 1, 2))
    mine, new = _log_uniform(rng, 1, 600), rng.choice((1, 1, 1, 6, 64, 2048))
    cost = 4.0 * layers * groups * members * (hi + mine + new) * int(heads.split("/")[0]) * d     # per new token each
    new = max(1, min(new, int(6e11 / cost)))
    return dict(kind=kind, heads=heads, d=d, dtype=rng.choice(("bf16", "bf16", "fp16")), layers=layers,
                groups=groups, members=members, pre_lo=hi if groups == 1 else max(1, hi // 20), pre_hi=hi,
                own_lo=rng.choice((0, 1)), own_hi=mine, new_lo=1 if new <= 64 else new // 2, new_hi=new, page=page,
                order=rng.choice(("nhd", "nhd", "hnd")), shape=shape)


# ---------------------------------------------------------------- inputs


DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _heads(case):
    hq, hkv = case["heads"].split("/")
    return int(hq), int(hkv)


def _between(r, lo, hi):
    """From lo to hi, over the logarithm where that spans more than a factor of ten."""
    return r.randint(lo, hi) if lo == 0 or hi <= 10 * lo else _log_uniform(r, lo, hi)


def _batch(case):
    """Per group: the rows of its prompt, and the (own rows before this step, new rows) of its members."""
    r = random.Random(case["shape"])
    out = []
    for _ in range(case["groups"]):
        pre = _between(r, case["pre_lo"], case["pre_hi"])
        count = case["members"] if case["groups"] == 1 else r.randint(1, case["members"])
        out.append((pre, [(_between(r, case["own_lo"], case["own_hi"]), _between(r, case["new_lo"], case["new_hi"]))
                          for _ in range(count)]))
    return out


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(g, case, pages, scale):
    """[layers, pages, page, heads, d] of a pool whose pages hold their tokens, or their heads, outermost."""
    hkv, d, page = _heads(case)[1], case["d"], case["page"]
    hnd = case["order"] == "hnd"
    shape = (case["layers"], pages) + ((hkv, page) if hnd else (page, hkv)) + (d,)
    x = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(0.0, scale, generator=g)
    return x.permute(0, 1, 3, 2, 4) if hnd else x


def _workspace(nbytes):
    raw = torch.zeros(nbytes + 256, dtype=torch.uint8, device="cuda")
    off = (-raw.data_ptr()) % 256
    return raw[off:off + nbytes]


def _prepare_share(case, seed):
    g = _generator(seed)
    hq, hkv = _heads(case)
    page = case["page"]
    batch = _batch(case)
    lens, new, prefix, cu_groups, tables, total = [], [], [], [0], [], 0
    for pre, members in batch:
        common = pre // page                       # whole pages; the prompt's last rows were copied to each member
        shared = list(range(total, total + common))
        total += common
        for mine, fresh in members:
            n = pre + mine + fresh
            need = -(-n // page) - common
            tables.append(shared + list(range(total, total + need)))
            total += need
            lens.append(n)
            new.append(fresh)
        prefix.append(common * page)
        cu_groups.append(len(lens))
    perm = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed))).tolist()
    width = max(len(t) for t in tables)
    # the batch's sequences are rows of the page table in another order
    order = list(range(len(lens)))
    random.Random(case["shape"] + 1).shuffle(order)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = [0] * len(lens)
    for i, t in enumerate(tables):
        table[order[i], :len(t)] = torch.tensor([perm[p] for p in t], dtype=torch.int32)
        at[order[i]] = lens[i]
    cu_q = [0]
    for m in new:
        cu_q.append(cu_q[-1] + m)
    n_q, dtype = cu_q[-1], DTYPES[case["dtype"]]
    s = dict(case=case, lens_h=lens, new_h=new, seqs_h=order, table=table.cuda(), lens=_int32(at), seqs=_int32(order),
             cu_q=_int32(cu_q), cu_groups=_int32(cu_groups), prefix=_int32(prefix), n_q=n_q,
             k=_pool(g, case, total, 1.5), v=_pool(g, case, total, 1.0),
             q=torch.empty(case["layers"], n_q, hq, case["d"], dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g),
             out=torch.empty(case["layers"], n_q, hq, case["d"], dtype=dtype, device="cuda"),
             lse=torch.empty(case["layers"], n_q, hq, dtype=torch.float32, device="cuda"))
    if own:
        import paper_2608_08794_gb300 as ap
        s["cache"] = ap.PagedCache(s["k"], s["v"], s["table"])
        s["ws"] = _workspace(ap.apack_paged_group_workspace_size(s["cache"], hq, len(lens), n_q))
    return s


def _pages_sizes(case):
    """Lengths before the call, rows kept by its release, and rows that its extension adds."""
    r = random.Random(case["shape"])
    if case["kind"] == "step":
        lens = [_between(r, case["len_lo"], case["len_hi"]) for _ in range(case["seqs"])]
        drop = [min(n, _between(r, case["drop_lo"], case["drop_hi"])) for n in lens]
        return lens, [n - m for n, m in zip(lens, drop)], drop
    parents = [_between(r, case["len_lo"], case["len_hi"]) for _ in range(case["parents"])]
    return parents, [r.randrange(case["parents"]) for _ in range(case["seqs"])], [
        _between(r, case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]


def _prepare_pages(case, seed):
    """Page tables of a running server: pages in any order, some sequences of which the call does not speak."""
    a, b, grow = _pages_sizes(case)
    page, pages = case["page"], case["pages"]
    host = torch.Generator().manual_seed(int(seed))
    perm = torch.randperm(pages, generator=host).to(torch.int32)
    fork = case["kind"] == "fork"
    rows = len(a) + (len(grow) if fork else 3)
    place = torch.randperm(rows, generator=host).tolist()
    longest = max(a) + (max(grow) if fork else 0)
    width = -(-longest // page) + 2
    table = torch.full((rows, width), -1, dtype=torch.int32)
    lengths, refs, at = torch.zeros(rows, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32), 0
    for i, n in enumerate(a):
        need = -(-n // page)
        table[place[i], :need] = perm[at:at + need]
        refs[perm[at:at + need].long()] = 1
        lengths[place[i]] = n
        at += need
    free = torch.full((pages,), -1, dtype=torch.int32)
    free[:pages - at] = perm[at:]
    cap = sum(grow) + 5                         # a captured batch has room to spare
    n = len(grow)
    s = dict(case=case, table=table.cuda(), lengths=lengths.cuda(), refs=refs.cuda(), free=free.cuda(),
             count=_int32([pages - at]), grow=_int32(grow), cu=torch.empty(n + 1, dtype=torch.int32, device="cuda"),
             rows=torch.empty(cap, dtype=torch.int32, device="cuda"),
             row_seqs=torch.empty(cap, dtype=torch.int32, device="cuda"),
             slots=torch.empty(cap, dtype=torch.int64, device="cuda"),
             pairs=torch.empty(n, 2, dtype=torch.int32, device="cuda"))
    if fork:
        s.update(parents=_int32([place[p] for p in b]), seqs=_int32(place[len(a):]),
                 keep=torch.zeros(n, dtype=torch.int32, device="cuda"))
    else:
        s.update(seqs=_int32(place[:n]), keep=_int32(b))
    if own:
        import paper_2608_08794_gb300 as ap
        s["tables"] = ap.PageTables(s["table"], s["lengths"], s["refs"], s["free"], s["count"], page)
        s["ws"] = _workspace(1024)
    return s


def prepare(case, seed):
    return _prepare_share(case, seed) if case["kind"] == "share" else _prepare_pages(case, seed)


# ---------------------------------------------------------------- plain forms


def _plain_share(s):
    case = s["case"]
    hq, hkv = _heads(case)
    g, d, page = hq // hkv, case["d"], case["page"]
    for layer in range(case["layers"]):
        at = 0
        for seq, n, m in zip(s["seqs_h"], s["lens_h"], s["new_h"]):
            t = torch.arange(n, device="cuda")
            pages, slot = s["table"][seq][t // page].long(), t % page
            k = s["k"][layer][pages, slot].float().transpose(0, 1)                   # [Hkv, n, D]
            v = s["v"][layer][pages, slot].float().transpose(0, 1)
            q = s["q"][layer, at:at + m].float().view(m, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, m * g, d)
            x = torch.matmul(q, k.transpose(1, 2)).view(hkv, m, g, n) * (1.0 / math.sqrt(d))
            behind = t[None, :] > (n - m + torch.arange(m, device="cuda"))[:, None]   # [m, n]: later than the token
            if m > 1:
                x.masked_fill_(behind[None, :, None], -math.inf)
            top = x.amax(-1, keepdim=True)
            x.sub_(top).exp_()
            total = x.sum(-1, keepdim=True)
            o = torch.matmul(x.view(hkv, m * g, n), v).view(hkv, m, g, d) / total
            s["out"][layer, at:at + m] = o.permute(1, 0, 2, 3).reshape(m, hq, d).to(s["out"].dtype)
            s["lse"][layer, at:at + m] = (top + total.log())[..., 0].permute(1, 0, 2).reshape(m, hq)
            at += m
    return [s["out"], s["lse"]]


def _plain_release(s, page):
    """Pages behind the kept rows are given up; those that nobody holds any more go to the free list, the first of them
    on top (in the order of the entries, then of their rows), each at its first mention."""
    seqs, keep = s["seqs"].long(), s["keep"]
    mine = s["table"][seqs]
    column = torch.arange(mine.shape[1], device="cuda")
    gone = (column >= ((keep + page - 1) // page)[:, None]) & (column < ((s["lengths"][seqs] + page - 1) // page)[:, None])
    at = mine.long().clamp(min=0).flatten()
    s["refs"].index_add_(0, at, -gone.flatten().to(torch.int32))
    order = torch.arange(at.numel(), device="cuda")
    first = torch.full_like(s["refs"], at.numel(), dtype=torch.int64)
    first.scatter_reduce_(0, at, torch.where(gone.flatten(), order, at.numel()), "amin")
    back = gone.flatten() & (s["refs"][at] == 0) & (first[at] == order)
    count = s["count"] + back.sum()
    place = torch.where(back, count - back.cumsum(0), s["free"].numel())
    room = torch.cat((s["free"], s["free"][:1]))
    room.index_copy_(0, place, mine.flatten())            # what is no page to give back lands behind the end
    s["free"].copy_(room[:-1])
    s["count"].copy_(count)
    s["table"][seqs] = torch.where(gone, -1, mine)
    s["lengths"][seqs] = keep


def _plain_extend(s, page):
    seqs, grow, table = s["seqs"].long(), s["grow"], s["table"]
    n, cap = seqs.numel(), s["rows"].numel()
    old = s["lengths"][seqs]
    new = old + grow
    held, want = (old + page - 1) // page, (new + page - 1) // page
    last = torch.where((old % page != 0) & (grow > 0), table[seqs, (held - 1).clamp(min=0).long()], -1)
    earlier = torch.tril(last[:, None] == last[None, :], -1).sum(1)
    copied = (last >= 0) & (s["refs"][last.long().clamp(min=0)] - earlier > 1)
    take = want - held + copied
    end = take.cumsum(0)
    pages = torch.where(torch.arange(s["free"].numel(), device="cuda") >= s["count"], -1, s["free"])
    # entry i's column c holds taken page number c - held + copied + what the entries before it take
    column = torch.arange(table.shape[1], device="cuda")
    fresh = (column >= (held - copied.long())[:, None]) & (column < want[:, None])
    number = (end - take)[:, None] + column - (held - copied.long())[:, None]
    got = pages[(s["count"].long() - 1 - number).clamp(0, pages.numel() - 1)]
    own_page = got.gather(1, (held - 1).clamp(min=0).long()[:, None])[:, 0]
    s["pairs"].copy_(torch.where(copied[:, None], torch.stack((last, own_page), 1), 0))
    s["refs"].index_add_(0, last.long().clamp(min=0), -copied.to(torch.int32))
    s["refs"].index_add_(0, got.long().clamp(min=0).flatten(), fresh.flatten().to(torch.int32))
    table[seqs] = torch.where(fresh, got, table[seqs])
    s["count"].sub_(end[-1:])
    s["lengths"][seqs] = new.to(torch.int32)
    s["cu"].zero_()
    s["cu"][1:] = grow.cumsum(0)
    j = torch.arange(cap, device="cuda")
    entry = torch.searchsorted(s["cu"][1:].contiguous(), j.to(torch.int32), right=True)
    real = entry < n
    entry = entry.clamp(max=n - 1)
    row = old[entry] + j - s["cu"][entry]
    s["rows"].copy_(torch.where(real, row, -1))
    s["row_seqs"].copy_(torch.where(real, seqs[entry], -1))
    page_of = table[seqs[entry], (row // page).clamp(max=table.shape[1] - 1).long()].long()
    s["slots"].copy_(torch.where(real, page_of * page + row % page, -1))


def _pages_outputs(s):
    return [s["cu"], s["rows"], s["row_seqs"], s["slots"], s["pairs"], s["table"], s["lengths"], s["refs"], s["count"],
            s["free"]]


def _plain_pages(s):
    page = s["case"]["page"]
    _plain_release(s, page)
    if s["case"]["kind"] == "fork":
        parents, seqs = s["parents"].long(), s["seqs"].long()
        s["table"][seqs] = s["table"][parents]
        s["lengths"][seqs] = s["lengths"][parents]
        shared = s["table"][parents]
        s["refs"].index_add_(0, shared.long().clamp(min=0).flatten(), (shared >= 0).flatten().to(torch.int32))
    _plain_extend(s, page)
    return _pages_outputs(s)


def _own(s):
    import paper_2608_08794_gb300 as ap
    case = s["case"]
    if case["kind"] == "share":
        ap.apack_paged_group_plan(s["cache"], s["lens"], _heads(case)[0], s["n_q"], s["ws"], cu_q=s["cu_q"],
                                  seqs=s["seqs"], cu_groups=s["cu_groups"], prefix=s["prefix"])
        for layer in range(case["layers"]):
            ap.apack_paged_group_attention(s["cache"], layer, s["q"][layer], s["out"][layer], s["ws"],
                                           lse=s["lse"][layer])
        return [s["out"], s["lse"]]
    ap.apack_pages_release(s["tables"], s["keep"], seqs=s["seqs"], ws=s["ws"])
    if case["kind"] == "fork":
        ap.apack_pages_fork(s["tables"], s["parents"], s["seqs"], ws=s["ws"])
    ap.apack_pages_extend(s["tables"], s["grow"], s["cu"], s["rows"], seqs=s["seqs"], row_seqs=s["row_seqs"],
                          slots=s["slots"], pairs=s["pairs"], ws=s["ws"])
    return _pages_outputs(s)


def run(state):
    if own:
        return _own(state)
    return _plain_share(state) if state["case"]["kind"] == "share" else _plain_pages(state)


def work(case):
    if case["kind"] == "share":
        hq, hkv = _heads(case)
        rows = pairs = n_q = pages = 0
        for pre, members in _batch(case):
            rows += pre // case["page"] * case["page"]              # shared rows are read once
            for mine, m in members:
                n = pre + mine + m
                rows += n - pre // case["page"] * case["page"]
                pairs += m * n - m * (m - 1) // 2
                n_q += m
                pages += -(-n // case["page"])
        size = 2 * case["d"]
        return {"bytes": case["layers"] * (2 * rows * hkv * size + n_q * hq * (2 * size + 4)) + 4 * pages,
                "flops": case["layers"] * 4 * pairs * hq * case["d"]}
    a, b, grow = _pages_sizes(case)
    page, new, n = case["page"], sum(grow), len(grow)
    if case["kind"] == "step":
        moved = sum(-(-x // page) - -(-y // page) for x, y in zip(a, b))
    else:
        moved = sum(-(-a[p] // page) + -(-(a[p] + m) // page) for p, m in zip(b, grow))
    # maps of the new rows; an entry of the table, the free list and the counts per page that comes or goes
    return {"bytes": 16 * new + 2 * 12 * moved + 40 * n, "flops": 0}


# ---------------------------------------------------------------- from the definitions


def _exact_share(s):
    case = s["case"]
    hq, hkv = _heads(case)
    d, page = case["d"], case["page"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    for layer in range(case["layers"]):
        at = 0
        for seq, n, m in zip(s["seqs_h"], s["lens_h"], s["new_h"]):
            pages = s["table"][seq, :-(-n // page)].long()
            k = s["k"][layer, pages].flatten(0, 1)[:n]
            v = s["v"][layer, pages].flatten(0, 1)[:n]
            for h in range(hq):
                kh, vh = (x[:, h // (hq // hkv)].double() for x in (k, v))
                x = s["q"][layer, at:at + m, h].double() @ kh.T / math.sqrt(d)
                for i in range(m - 1):
                    x[i, n - m + 1 + i:] = -math.inf
                z = torch.logsumexp(x, 1)
                out[layer, at:at + m, h] = (x - z[:, None]).exp_() @ vh
                lse[layer, at:at + m, h] = z
            at += m
    return [out, lse]


def _exact_pages(s):
    """The same bookkeeping with lists, one sequence after the other."""
    case, page = s["case"], s["case"]["page"]
    table, lengths, refs = s["table"].tolist(), s["lengths"].tolist(), s["refs"].tolist()
    free, count = s["free"].tolist(), s["count"].item()
    seqs, keep, grow = s["seqs"].tolist(), s["keep"].tolist(), s["grow"].tolist()
    back = []
    for b, n in zip(seqs, keep):
        for c in range(-(-n // page), -(-lengths[b] // page)):
            back.append(table[b][c])
            refs[table[b][c]] -= 1
            table[b][c] = -1
        lengths[b] = n
    back = [p for p in dict.fromkeys(back) if refs[p] == 0]
    free[count:count + len(back)] = back[::-1]
    count += len(back)
    if case["kind"] == "fork":
        for p, b in zip(s["parents"].tolist(), seqs):
            table[b], lengths[b] = list(table[p]), lengths[p]
            for c in table[p]:
                if c >= 0:
                    refs[c] += 1
    cu, rows, owners, slots, pairs = [0], [], [], [], []
    for b, m in zip(seqs, grow):
        n = lengths[b]
        pair = [0, 0]
        if m and n % page and refs[table[b][n // page]] > 1:
            count -= 1
            pair = [table[b][n // page], free[count]]
            refs[pair[0]] -= 1
            refs[pair[1]] = 1
            table[b][n // page] = pair[1]
        pairs.append(pair)
        for c in range(-(-n // page), -(-(n + m) // page)):
            count -= 1
            table[b][c] = free[count]
            refs[free[count]] = 1
        lengths[b] = n + m
        cu.append(cu[-1] + m)
        rows += range(n, n + m)
        owners += [b] * m
        slots += [table[b][r // page] * page + r % page for r in range(n, n + m)]
    pad = [-1] * (s["rows"].numel() - len(rows))
    return [torch.tensor(x, dtype=y.dtype, device="cuda") for x, y in zip(
        (cu, rows + pad, owners + pad, slots + pad, pairs, table, lengths, refs, [count], free), _pages_outputs(s))]


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_share(s) if case["kind"] == "share" else _exact_pages(s)
