"""Operators on a cache of keys and values in 8 bits and on beams, as cases that can be timed and compared.

cache   rows appended to a paged cache in 8 bits (a scale for each page and head) and attention of their queries over it
window  the same where a row sees the last positions and a few first ones
pages   sequences that share pages: forking, growing with copies of shared last pages, giving back, moving together
beams   the best continuations over beams and vocabulary, with the beams' histories in their new order

With `own` false `run` computes them from elementary tensor operations, else through the library.  A user's program keeps
the cache's arrays and its handle, a workspace for the selection and the arrays that results go to; rows, queries, parents,
logits and scores come with each call.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CODE = {"f32": 0, "bf16": 1, "f16": 2}  # bild.h: BILD_DT_*
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _bild():
    import paper_2302_07863_amd as bild
    return bild


# ------------------------------------------------------------------------------------------------ cases
def _cache(name, op="cache", layers=1, page=64, sinks=0, window=0, lengths="same", prompts=0, **more):
    return dict(name=name, op=op, layers=layers, page=page, sinks=sinks, window=window, lengths=lengths, prompts=prompts, **more)


def listed():
    return [
        # a single-token step of one short sequence of a small model: microseconds, latency counts
        _cache("cache-step-small", seqs=1, rows=1, length=513, heads=8, group=1, d_head=64, dtype="bf16", layers=6, page=32),
        # one token far into a long context, a key head for every query head
        _cache("cache-step-long", seqs=1, rows=1, length=65537, heads=32, group=1, d_head=128, dtype="f16"),
        # a step of a server's batch: lengths far apart, four query heads a key head
        _cache("cache-batch", seqs=64, rows=1, length=16384, heads=8, group=4, d_head=128, dtype="bf16", lengths="spread"),
        # a review of ten drafts by a model that keeps its activations in fp32
        _cache("cache-review", seqs=1, rows=11, length=777, heads=16, group=1, d_head=64, dtype="f32", layers=2),
        # the second part of a long prompt
        _cache("cache-prompt", seqs=1, rows=2000, length=5001, heads=8, group=4, d_head=128, dtype="bf16"),
        # a step of a batch of long chats that look back a few thousand tokens
        _cache("window-step", op="window", seqs=16, rows=1, length=50001, heads=8, group=4, d_head=128, dtype="bf16", sinks=4, window=4096),
        # a whole prompt through a layer with a short window, heads of 80
        _cache("window-prompt", op="window", seqs=1, rows=4001, length=4001, heads=16, group=1, d_head=80, dtype="f16", sinks=4, window=512, page=32),
        # a beam step of a small model: parents, one more token, copies of shared last pages
        dict(name="pages-beams-small", op="pages", what="beams", beams=4, length=71, layers=6, heads=8, d_head=64, page=32),
        # the same for many beams of a large model behind a common prompt
        dict(name="pages-beams", op="pages", what="beams", beams=32, length=285, layers=24, heads=16, d_head=64, page=32),
        # a pool half of whose pages are free, packed together
        dict(name="pages-compact", op="pages", what="compact", pages=600, layers=8, heads=4, d_head=64, page=64, seqs=24),
        # a beam step over one sentence
        dict(name="beams-step", op="beams", batch=1, beams=4, vocab=32128, choices=4, dtype="f32", penalty=0.0, steps=17),
        # a beam step over a batch and a large vocabulary, twice as many choices as beams
        dict(name="beams-batch", op="beams", batch=16, beams=8, vocab=250112, choices=16, dtype="bf16", penalty=0.6, steps=120),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cache", "cache", "window", "pages", "beams"])
    if op in ("cache", "window"):
        while True:
            c = dict(op=op, layers=rng.choice([1, 2, 3]), page=rng.choice([32, 64, 128]), heads=rng.choice([1, 2, 4, 8, 12, 16, 32]), group=rng.choice([1, 1, 2, 4, 7, 8]),
                     d_head=rng.choice([32, 64, 72, 80, 96, 128, 128, 256]), dtype=rng.choice(["f32", "bf16", "f16"]), sinks=0, window=0, prompts=0,
                     seqs=rng.choice([1, 1, _log(rng, 1, 64), _log(rng, 1, 64)]), rows=rng.choice([1, 1, _log(rng, 1, 32), _log(rng, 1, 3000)]))
            c["length"] = c["rows"] + _log(rng, 1, 65536) - 1
            c["lengths"] = "spread" if c["seqs"] > 1 and rng.random() < 0.6 else "same"
            if c["seqs"] > 2 and c["rows"] == 1 and rng.random() < 0.4:  # a few prompts between single tokens
                c["prompts"] = _log(rng, 2, 600)
                c["length"] = max(c["length"], c["prompts"])
            if op == "window":
                c["sinks"], c["window"] = rng.choice([0, 1, 4, 33]), _log(rng, 1, 8192)
            w = work(c)
            if w["bytes"] <= 6e8 and w["flops"] <= 1.4e11 and c["seqs"] * c["length"] * c["heads"] * c["d_head"] * 2 * c["layers"] <= 8e9:
                return c
    if op == "pages":
        while True:
            c = dict(op=op, layers=_log(rng, 1, 32), heads=rng.choice([1, 2, 4, 8, 16]), d_head=rng.choice([32, 64, 80, 128]), page=rng.choice([32, 64, 128]))
            if rng.random() < 0.7:
                c.update(what="beams", beams=_log(rng, 1, 64), length=_log(rng, 1, 2000))
                pages = c["length"] // c["page"] + 2 * c["beams"] + 4
            else:
                c.update(what="compact", pages=_log(rng, 4, 3000), seqs=_log(rng, 1, 60))
                pages = c["pages"]
            if pages * c["layers"] * 2 * c["heads"] * c["page"] * c["d_head"] <= 2.6e8:
                return c
    beams, batch = _log(rng, 1, 32), _log(rng, 1, 64)
    vocab, dtype = _log(rng, 1000, 260000), rng.choice(["f32", "bf16", "f16"])
    batch = max(1, min(batch, 16 * 8 * 250112 * 2 // (beams * vocab * BYTES[dtype])))
    return dict(op=op, batch=batch, beams=beams, vocab=vocab, choices=rng.choice([beams, min(64, 2 * beams)]), dtype=dtype,
                penalty=rng.choice([0.0, 0.6, 1.0]), steps=_log(rng, 1, 500))


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _sizes(c):
    """Lengths of the sequences, the new rows among them, and how many new rows each has."""
    n, top = c["seqs"], c["length"]
    rows = [c["rows"]] * n
    for i in range(0, n, 3) if c["prompts"] else ():
        rows[i] = max(1, c["prompts"] - i)
    if c["lengths"] == "same" or n == 1:
        lengths = [top] * n
    else:  # from 1 to the longest, evenly over their logarithm, in an order of its own
        lengths = [int(round(top ** ((i * 37 % n) / (n - 1)))) if math.gcd(37, n) == 1 else int(round(top ** (i / (n - 1)))) for i in range(n)]
    return [max(a, b) for a, b in zip(lengths, rows)], rows


def _cache_inputs(c, seed):
    g = _generator(seed)
    lengths, rows = _sizes(c)
    n, page, heads, d = c["seqs"], c["page"], c["heads"], c["d_head"]
    most = max(-(-length // page) for length in lengths)
    counts = torch.tensor([-(-length // page) for length in lengths], device="cuda")
    total = sum(-(-length // page) for length in lengths)
    pages = total + 3
    at = torch.arange(most, device="cuda")[None, :] < counts[:, None]
    table = torch.full((n, most), -1, device="cuda", dtype=torch.int32)
    table[at] = torch.randperm(pages, device="cuda", generator=g)[:total].to(torch.int32)
    refs = torch.zeros(pages, device="cuda", dtype=torch.int32)
    refs[table[at].long()] = 1
    codes = torch.empty(pages, c["layers"], 2, heads, page, d, device="cuda", dtype=torch.int8)
    flat = codes.view(-1)
    for i in range(0, flat.numel(), 1 << 28):  # values of a spread of a third of the largest
        part = flat[i:i + (1 << 28)]
        part.copy_((torch.randn(part.numel(), device="cuda", generator=g) * 42).round_().clamp_(-127, 127))
    scales = 3.0 * (0.5 + torch.rand(pages, c["layers"], 2, heads, device="cuda", generator=g))
    tokens = sum(rows)
    dt = TORCH[c["dtype"]]
    q = (1.5 * torch.randn(tokens, heads * c["group"], d, device="cuda", generator=g)).to(dt)
    kv = torch.randn(2, tokens, heads, d, device="cuda", generator=g)
    kv *= torch.where(torch.rand(d, device="cuda", generator=g) < 0.02, 4.0, 1.0)  # a few wide features
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    return dict(codes=codes, scales=scales, table=table, refs=refs, lengths=torch.tensor(lengths, device="cuda", dtype=torch.int32),
                starts=torch.tensor(starts, device="cuda", dtype=torch.int32), q=q, k=kv[0].to(dt), v=kv[1].to(dt), layer=c["layers"] - 1,
                host=(lengths, rows, starts))


def _pages_inputs(c, seed):
    g = _generator(seed)
    if c["what"] == "beams":  # as many sequences again are empty: there the new beams go
        n, whole = c["beams"], (c["length"] - 1) // c["page"]
        pages = whole + 2 * n + 2
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        table = torch.full((2 * n, whole + 2), -1, device="cuda", dtype=torch.int32)
        table[:n, :whole] = order[:whole]
        table[:n, whole] = order[whole:whole + n]  # (each beam has its own last page)
        refs = torch.zeros(pages, device="cuda", dtype=torch.int32)
        refs[order[:whole].long()] = n
        refs[order[whole:whole + n].long()] = 1
        lengths = torch.tensor([c["length"]] * n + [0] * n, device="cuda", dtype=torch.int32)
        # beams of the next step: the better ones go on more than once
        parents = (n * torch.rand(n, device="cuda", generator=g) ** 2).to(torch.int32).clamp_(max=n - 1)
        more = dict(parents=torch.cat((torch.arange(n, device="cuda", dtype=torch.int32), parents)),
                    new=torch.arange(n, 2 * n, device="cuda", dtype=torch.int32))
    else:
        n, pages = c["seqs"], c["pages"]
        used = pages // 2
        most = -(-used // n)
        held = torch.randperm(pages, device="cuda", generator=g)[:used].to(torch.int32)
        table = torch.full((n * most,), -1, device="cuda", dtype=torch.int32)
        table[:used] = held
        table = table.view(most, n).t().contiguous()
        lengths = ((table >= 0).sum(dim=1) * c["page"]).to(torch.int32)
        lengths -= (torch.rand(n, device="cuda", generator=g) * c["page"]).to(torch.int32) * (lengths > 0)
        refs = torch.zeros(pages, device="cuda", dtype=torch.int32)
        refs[held.long()] = 1
        more = {}
    codes = torch.randint(-127, 128, (pages, c["layers"], 2, c["heads"], c["page"], c["d_head"]), device="cuda", generator=g, dtype=torch.int8)
    scales = torch.rand(pages, c["layers"], 2, c["heads"], device="cuda", generator=g)
    return dict(codes=codes, scales=scales, table=table, refs=refs, lengths=lengths, **more)


def _beams_inputs(c, seed):
    g = _generator(seed)
    rows = c["batch"] * c["beams"]
    out = dict(logits=(2.5 * torch.randn(rows, c["vocab"], device="cuda", generator=g)).to(TORCH[c["dtype"]]))
    lengths = torch.full((rows,), c["steps"], device="cuda", dtype=torch.int32)
    finished = torch.rand(rows, device="cuda", generator=g) < 0.15
    finished[::c["beams"]] = False  # (the best beam of each goes on)
    lengths = torch.where(finished, (lengths * torch.rand(rows, device="cuda", generator=g)).to(torch.int32), lengths)
    out["scores"] = -1.2 * lengths.float() - 2.0 * torch.rand(rows, device="cuda", generator=g)
    out["lengths"], out["finished"] = lengths, finished.to(torch.int32)
    out["history"] = torch.randint(0, c["vocab"], (rows, c["steps"] + 8), device="cuda", generator=g, dtype=torch.int32)
    return out


EOS, PAD = 1, 0


def prepare(case, seed):
    c = case
    state = dict(case=c)
    if c["op"] == "beams":
        state.update(_beams_inputs(c, seed))
        n = c["batch"] * c["choices"]
        i32 = dict(device="cuda", dtype=torch.int32)
        state["out"] = dict(scores=torch.empty(n, device="cuda"), parents=torch.empty(n, **i32), tokens=torch.empty(n, **i32), lengths=torch.empty(n, **i32),
                            finished=torch.empty(n, **i32), history=torch.zeros(n, c["steps"] + 1, **i32))
        if own:
            state["beams"] = _bild().Beams(c["vocab"], c["batch"], c["beams"])
        return state
    state.update(_pages_inputs(c, seed) if c["op"] == "pages" else _cache_inputs(c, seed))
    if c["op"] == "pages":
        if c["what"] == "compact":
            state["saved"] = tuple(state[name].clone() for name in ("table", "refs", "lengths"))
            state["used"] = torch.zeros(1, device="cuda", dtype=torch.int32)
    else:
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(state["q"].shape[:2], device="cuda")
    if own:
        torch.cuda.synchronize()
        state["cache"] = _bild().Cache(state["codes"].shape[0], c["page"], c["layers"], c["heads"], c["d_head"], state["table"].shape[0], state["table"].shape[1],
                                       codes=state["codes"].data_ptr(), scales=state["scales"].data_ptr(), table=state["table"].data_ptr(),
                                       lengths=state["lengths"].data_ptr(), refs=state["refs"].data_ptr())
    return state


# ------------------------------------------------------------------------------------------------ the library's calls
def _own_cache(s, c, stream):
    cache, dt, (lengths, rows, starts) = s["cache"], CODE[c["dtype"]], s["host"]
    n, tokens = c["seqs"], starts[-1]
    which = dict(starts=s["starts"].data_ptr(), tokens=tokens) if c["prompts"] else {}
    most = max(rows)
    cache.append(s["layer"], dt, n, most, s["k"].data_ptr(), s["v"].data_ptr(), stream=stream, **which)
    cache.attend(s["layer"], dt, n, most, c["heads"] * c["group"], s["q"].data_ptr(), s["out"].data_ptr(), c["d_head"] ** -0.5, lse=s["lse"].data_ptr(),
                 window=c["window"], sinks=c["sinks"], stream=stream, **which)
    return s["out"], s["lse"], s["scales"]


def _own_pages(s, c, stream):
    cache = s["cache"]
    if c["what"] == "beams":
        n = c["beams"]
        cache.fork(2 * n, s["parents"].data_ptr(), stream=stream)
        cache.extend(n, 1, sequences=s["new"].data_ptr(), stream=stream)
    else:
        _go_back(s)
        cache.compact(used=s["used"].data_ptr(), stream=stream)
    return _pages_outputs(s, c)


def _go_back(s):
    """The sequences as they were saved: what is packed then."""
    for name, was in zip(("table", "refs", "lengths"), s["saved"]):
        s[name].copy_(was)


def _pages_outputs(s, c):
    out = {name: s[name] for name in ("table", "lengths", "refs", "codes", "scales")}
    if c["what"] == "compact":
        out["used"] = s["used"]
    return out


def _own_beams(s, c, stream):
    out = s["out"]
    s["beams"].select(s["logits"].data_ptr(), CODE[c["dtype"]], c["batch"], c["choices"], s["scores"].data_ptr(), out["scores"].data_ptr(), out["parents"].data_ptr(),
                      out["tokens"].data_ptr(), lengths=s["lengths"].data_ptr(), finished=s["finished"].data_ptr(), out_lengths=out["lengths"].data_ptr(),
                      out_finished=out["finished"].data_ptr(), eos=EOS, pad=PAD, penalty=c["penalty"], history=s["history"].data_ptr(),
                      history_stride=s["history"].stride(0), out_history=out["history"].data_ptr(), out_history_stride=out["history"].stride(0), steps=c["steps"],
                      stream=stream)
    return out


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_append(s, c):
    lengths, rows, starts = s["host"]
    page, layer = c["page"], s["layer"]
    counts = s["starts"][1:] - s["starts"][:-1]
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), counts.long(), output_size=starts[-1])
    row = torch.arange(starts[-1], device="cuda")
    pos = s["lengths"][seq] - counts[seq] + row - s["starts"][seq]
    held = s["table"][seq, (pos // page).long()].long()
    first = (row == s["starts"][seq]) | (pos % page == 0)
    touched = sum((length - 1) // page - (length - r) // page + 1 for length, r in zip(lengths, rows))
    which = torch.cumsum(first, 0) - 1  # the touched page of each row
    pages = torch.zeros(touched, device="cuda", dtype=torch.long).index_put_((which,), held)
    before = torch.full((touched,), page, device="cuda", dtype=torch.long).scatter_reduce_(0, which, (pos % page).long(), "amin")  # rows that were there
    for i, x in enumerate((s["k"], s["v"])):
        new = torch.zeros(touched, page, c["heads"], c["d_head"], device="cuda")
        new[which, (pos % page).long()] = x.float()
        new = new.transpose(1, 2)
        was = torch.where(before[:, None] > 0, s["scales"][pages, layer, i], 0.0)
        scale = torch.maximum(was, new.abs().amax(dim=(2, 3)))  # what code 127 stands for
        safe = torch.where(scale > 0, scale, 1.0)[:, :, None, None]
        old = s["codes"][pages, layer, i]
        there = torch.arange(page, device="cuda")[None, :] < before[:, None]
        moved = torch.where((scale > was)[:, :, None, None], (old.float() * was[:, :, None, None] / safe).round(), old.float())
        filled = torch.zeros(touched, page, device="cuda", dtype=torch.bool)
        filled[which, (pos % page).long()] = True
        now = torch.where(there[:, None, :, None], moved, torch.where(filled[:, None, :, None], (new * 127 / safe).round(), old.float()))
        s["codes"][pages, layer, i] = now.to(torch.int8)
        s["scales"][pages, layer, i] = scale


def _held(s, c, i, first, last, which):
    """Keys (which 0) or values of sequence i from position first on, [heads][positions][d_head]."""
    page = c["page"]
    b0, b1 = first // page, (last - 1) // page + 1
    pages = s["table"][i, b0:b1].long()
    x = s["codes"][pages, s["layer"], which].float() * (s["scales"][pages, s["layer"], which] / 127)[:, :, None, None]
    return x.transpose(0, 1).reshape(c["heads"], -1, c["d_head"])[:, first - b0 * page:last - b0 * page]


def _plain_cache(s, c):
    _plain_append(s, c)
    lengths, rows, starts = s["host"]
    heads, group, d = c["heads"], c["group"], c["d_head"]
    outs, lses = [], []
    for i, (length, r) in enumerate(zip(lengths, rows)):
        step = max(1, (1 << 28) // (heads * group * length))
        if c["window"]:
            step = min(step, max(256, c["window"]))
        for r0 in range(0, r, step):
            r1 = min(r0 + step, r)
            pos = length - r + torch.arange(r0, r1, device="cuda")
            last = length - r + r1
            spans = [(0, last)]
            if c["window"]:
                low = max(0, length - r + r0 - c["window"] + 1)
                spans = [(low, last)]
                if c["sinks"] and low > 0:
                    spans.insert(0, (0, min(c["sinks"], low)))
            k = torch.cat([_held(s, c, i, a, b, 0) for a, b in spans], 1)
            v = torch.cat([_held(s, c, i, a, b, 1) for a, b in spans], 1)
            at = torch.cat([torch.arange(a, b, device="cuda") for a, b in spans])
            q = s["q"][starts[i] + r0:starts[i] + r1].float().view(-1, heads, group, d).permute(1, 2, 0, 3).reshape(heads, -1, d)
            z = torch.matmul(q, k.transpose(1, 2)) * d ** -0.5
            z = z.view(heads, group, r1 - r0, -1)
            seen = at[None, :] <= pos[:, None]
            if c["window"]:
                seen &= (at[None, :] > pos[:, None] - c["window"]) | (at[None, :] < c["sinks"])
            z = torch.where(seen, z, -math.inf)
            top = z.amax(dim=3, keepdim=True)
            p = torch.exp(z - top)
            total = p.sum(dim=3, keepdim=True)
            o = torch.matmul(p.view(heads, -1, p.shape[3]), v).view(heads, group, r1 - r0, d) / total
            outs.append(o.permute(2, 0, 1, 3).reshape(r1 - r0, heads * group, d).to(TORCH[c["dtype"]]))
            lses.append((top + torch.log(total))[..., 0].permute(2, 0, 1).reshape(r1 - r0, heads * group))
    return torch.cat(outs), torch.cat(lses), s["scales"]


def _plain_pages(s, c):
    table, lengths, refs, page = s["table"], s["lengths"], s["refs"], c["page"]
    pages = refs.shape[0]
    if c["what"] == "beams":
        n = c["beams"]
        table[:] = table[s["parents"].long()]
        lengths[:] = lengths[s["parents"].long()]
        held = table.clamp(min=0).long().view(-1)
        refs.copy_(torch.zeros_like(refs).scatter_add_(0, held, (table >= 0).to(torch.int32).view(-1)))
        # one more token each: a new page where the last one is full, a copy where others hold it too
        new = s["new"].long()
        at = (lengths[new] // page).long()
        part = (lengths[new] % page).long()
        last = table[new, at]
        asked = torch.zeros_like(refs).scatter_add_(0, last.clamp(min=0).long(), ((last >= 0) & (part > 0)).to(torch.int32))
        place = torch.arange(n, device="cuda")
        latest = torch.full((pages,), -1, device="cuda", dtype=torch.long).scatter_reduce_(0, last.clamp(min=0).long(), torch.where(last >= 0, place, -1), "amax")
        old = last.clamp(min=0).long()
        keeps = (asked[old] == refs[old]) & (latest[old] == place)  # (the last of those that grow, where nobody else is left)
        copies = (part > 0) & (refs[old] > 1) & ~keeps
        needs = copies | (part == 0)
        free = torch.argsort((refs != 0).to(torch.int32), stable=True)  # the free ones first, lowest first
        fresh = free[(torch.cumsum(needs, 0) - 1).clamp(min=0)]
        mine = torch.where(needs, fresh, old)
        counts = torch.where(copies, part, 0)[:, None] > torch.arange(page, device="cuda")[None, :]
        for j in range(0, n, 16):  # (sixteen pages at a time are read in one piece)
            to, of = mine[j:j + 16], old[j:j + 16]
            s["codes"][to] = torch.where(counts[j:j + 16, None, None, None, :, None], s["codes"][of], s["codes"][to])
        s["scales"][mine] = torch.where(copies[:, None, None, None], s["scales"][old], s["scales"][mine])
        table[new, at] = mine.to(torch.int32)
        refs.scatter_add_(0, old, -copies.to(torch.int32))
        refs.scatter_add_(0, mine, needs.to(torch.int32))
        lengths[new] += 1
        return _pages_outputs(s, c)
    _go_back(s)
    used = (refs > 0).sum()
    s["used"][0] = used
    place = torch.arange(pages, device="cuda")
    hole, mover = (refs == 0) & (place < used), (refs > 0) & (place >= used)
    to = torch.argsort((~hole).to(torch.int32), stable=True)  # the holes first, lowest first
    moved = torch.where(mover, to[(torch.cumsum(mover, 0) - 1).clamp(min=0)], place)
    # the page that comes to lie in each place: the one that moves there (movers alone write, each into a hole of its own), else itself
    source = place.clone()
    source[moved[mover]] = place[mover]
    for name in ("codes", "scales"):
        s[name].copy_(s[name][source])
    refs.copy_(torch.where(place < used, refs[source], 0))
    table.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()].to(torch.int32), table))
    return _pages_outputs(s, c)


def _ranked(c, scores, lse, z, lengths, finished):
    """Sums and ranks [batch][beams * vocab] in 64 bits of what each beam can go on with."""
    rows, vocab = z.shape
    total = (scores.double() - lse)[:, None] + z.double()
    over = lengths.double()
    total = torch.where(finished[:, None] != 0, -math.inf, total)
    total[:, PAD] = torch.where(finished != 0, scores.double(), total[:, PAD])
    over = torch.where(finished != 0, over, over + 1).clamp(min=1) ** c["penalty"]
    return total.view(c["batch"], -1), (total / over[:, None]).view(c["batch"], -1)


def _plain_beams(s, c):
    batch, beams, k, vocab = c["batch"], c["beams"], c["choices"], c["vocab"]
    z = s["logits"].double()
    top = z.amax(dim=1, keepdim=True)
    lse = (top + torch.log(torch.exp(z - top).sum(dim=1, keepdim=True)))[:, 0]
    total, rank = _ranked(c, s["scores"], lse, z, s["lengths"], s["finished"])
    out = {name: [] for name in s["out"]}
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :k]  # (equal ranks: the lowest index)
    row = torch.arange(batch, device="cuda")[:, None] * beams + order // vocab
    token = (order % vocab).to(torch.int32)
    was = s["finished"][row]
    history = s["history"][row][:, :, :c["steps"]]
    return dict(scores=total.gather(1, order).float().view(-1), parents=(order // vocab).to(torch.int32).view(-1), tokens=token.view(-1),
                lengths=(s["lengths"][row] + (was == 0)).to(torch.int32).view(-1), finished=((was != 0) | (token == EOS)).to(torch.int32).view(-1),
                history=torch.cat((history, token[:, :, None]), 2).view(batch * k, -1))


def run(state):
    c = state["case"]
    if own:
        stream = torch.cuda.current_stream().cuda_stream
        return {"cache": _own_cache, "window": _own_cache, "pages": _own_pages, "beams": _own_beams}[c["op"]](state, c, stream)
    return {"cache": _plain_cache, "window": _plain_cache, "pages": _plain_pages, "beams": _plain_beams}[c["op"]](state, c)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] in ("cache", "window"):
        lengths, rows = _sizes(c)
        flops = keys = pages = 0
        for length, r in zip(lengths, rows):
            first = length - r
            window = c["window"] or length
            low = max(0, first - window + 1)
            keys += length - low + min(c["sinks"], low)
            pages += (length - low + c["page"] - 1) // c["page"]
            for r0 in range(0, r, max(1, r // 64)):  # (of 64 places of a sequence's rows)
                each = min(max(1, r // 64), r - r0)
                pos = first + r0 + each // 2
                flops += each * (min(pos + 1, window) + min(c["sinks"], max(0, pos + 1 - window)))
        width, tokens = c["heads"] * c["d_head"], sum(rows)
        return dict(bytes=2 * keys * width + 8 * pages * c["heads"] + 2 * tokens * width * (c["group"] + 1) * BYTES[c["dtype"]] + 2 * tokens * width
                    + 4 * tokens * c["heads"] * c["group"], flops=4 * flops * width * c["group"])
    if c["op"] == "pages":
        token = c["layers"] * 2 * c["heads"] * c["d_head"]
        scales = 4 * c["layers"] * 2 * c["heads"]
        if c["what"] == "beams":
            n = c["beams"]
            entries = c["length"] // c["page"] + 1
            copied = c["length"] % c["page"] * token + scales if c["length"] % c["page"] else 0
            return dict(bytes=2 * n * copied + 12 * n * entries, flops=n)
        return dict(bytes=2 * (c["pages"] // 4) * (c["page"] * token + scales) + 8 * c["pages"], flops=c["pages"])
    rows = c["batch"] * c["beams"]
    return dict(bytes=rows * (c["vocab"] * BYTES[c["dtype"]] + 12) + c["batch"] * c["choices"] * (20 + 8 * c["steps"]), flops=6 * rows * c["vocab"])


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_cache(c, seed):
    s = _cache_inputs(c, seed)
    lengths, rows, starts = s["host"]
    heads, group, d, page, layer = c["heads"], c["group"], c["d_head"], c["page"], s["layer"]
    if work(c)["flops"] > 2e11:
        return None
    held = s["scales"].double()
    out = torch.zeros(sum(rows), heads * group, d, device="cuda", dtype=torch.float64)
    lse = torch.zeros(sum(rows), heads * group, device="cuda", dtype=torch.float64)
    for i, (length, r) in enumerate(zip(lengths, rows)):
        low = max(0, length - r - c["window"] + 1) if c["window"] else 0  # (what lies between the sinks and here nobody sees)
        near, far = low // page, -(-c["sinks"] // page) if c["window"] else 0
        blocks = sorted(set(range(min(far, near))) | set(range(near, -(-length // page))))
        at = torch.cat([torch.arange(b * page, min((b + 1) * page, length), device="cuda") for b in blocks])
        pages = s["table"][i][torch.tensor(blocks, device="cuda")].long()
        for h in range(heads):
            both = []
            for which, new in ((0, s["k"]), (1, s["v"])):
                codes, scales = s["codes"][pages, layer, which, h].double(), s["scales"][pages, layer, which, h].double()
                fresh = new[starts[i]:starts[i + 1], h].double()
                for b in range((length - r) // page, -(-length // page)):  # the pages that new rows go to
                    j = blocks.index(b)
                    t0, t1 = max(length - r - b * page, 0), min(length - b * page, page)
                    x = fresh[b * page + t0 - (length - r):b * page + t1 - (length - r)]
                    was = scales[j].clone() if t0 else torch.zeros((), device="cuda", dtype=torch.float64)
                    scales[j] = torch.maximum(was, x.abs().max())
                    codes[j, :t0] = torch.round(codes[j, :t0] * was / scales[j])
                    codes[j, t0:t1] = torch.round(127 * x / scales[j])
                    held[pages[j], layer, which, h] = scales[j]
                both.append((codes * scales[:, None, None] / 127).reshape(-1, d)[:len(at)])
            k, v = both
            for r0 in range(0, r, 512):
                r1 = min(r0 + 512, r)
                pos = length - r + torch.arange(r0, r1, device="cuda")
                hidden = at[None, :] > pos[:, None]
                if c["window"]:
                    hidden |= (pos[:, None] - at[None, :] >= c["window"]) & (at[None, :] >= c["sinks"])
                for e in range(group):
                    head = h * group + e
                    z = (s["q"][starts[i] + r0:starts[i] + r1, head].double() @ k.t()) / math.sqrt(d)
                    z.masked_fill_(hidden, -math.inf)
                    total = torch.logsumexp(z, dim=1)
                    lse[starts[i] + r0:starts[i] + r1, head] = total
                    out[starts[i] + r0:starts[i] + r1, head] = torch.exp(z - total[:, None]) @ v
    return out, lse, held


def _exact_pages(c, seed):
    """Page by page on the host; the codes and scales follow the moves."""
    s = _pages_inputs(c, seed)
    table, lengths, refs = s["table"].tolist(), s["lengths"].tolist(), s["refs"].tolist()
    codes, scales, page = s["codes"], s["scales"], c["page"]
    if c["what"] == "beams":
        n = c["beams"]
        old = [list(row) for row in table]
        for i, p in enumerate(s["parents"].tolist()):
            table[i], lengths[i] = list(old[p]), lengths[p] if p < n else 0
        refs = [0] * len(refs)
        for row in table:
            for p in row:
                if p >= 0:
                    refs[p] += 1
        copies = []
        for i in range(n, 2 * n):  # one after the other: who is alone on a page by then keeps it
            b, part = lengths[i] // page, lengths[i] % page
            if part == 0 or refs[table[i][b]] > 1:
                to = min(j for j, r in enumerate(refs) if r == 0 and j not in {a for _, a, _ in copies})
                if part:
                    copies.append((table[i][b], to, part))
                    refs[table[i][b]] -= 1
                refs[to], table[i][b] = 1, to
            lengths[i] += 1
        was, were = codes.clone(), scales.clone()
        for a, b, part in copies:
            codes[b, ..., :part, :], scales[b] = was[a, ..., :part, :], were[a]
        more = {}
    else:
        used = sum(r > 0 for r in refs)
        holes = [p for p in range(used) if refs[p] == 0]
        moves = dict(zip([p for p in range(used, len(refs)) if refs[p] > 0], holes))
        for a, b in moves.items():
            codes[b], scales[b] = codes[a].clone(), scales[a].clone()
            refs[b], refs[a] = refs[a], 0
        table = [[moves.get(p, p) for p in row] for row in table]
        more = dict(used=torch.tensor([used], dtype=torch.int32))
    as_ints = [torch.tensor(x, device="cuda", dtype=torch.int32) for x in (table, lengths, refs)]
    return dict(table=as_ints[0], lengths=as_ints[1], refs=as_ints[2], codes=codes, scales=scales, **{k: v.cuda() for k, v in more.items()})


def _exact_beams(c, seed):
    s = _beams_inputs(c, seed)
    beams, k, vocab = c["beams"], c["choices"], c["vocab"]
    out = {name: [] for name in ("scores", "parents", "tokens", "lengths", "finished", "history")}
    lengths, finished = s["lengths"].tolist(), s["finished"].tolist()
    for b in range(c["batch"]):
        found = []
        for j in range(beams):
            row = b * beams + j
            score = float(s["scores"][row])
            if finished[row]:
                found.append((-(score / max(lengths[row], 1) ** c["penalty"]), j, PAD, score))
                continue
            logp = score + torch.log_softmax(s["logits"][row].double(), dim=0)
            # (the best of a row by their logits, where equal ones are equal)
            best = torch.sort(s["logits"][row].double(), descending=True, stable=True).indices[:k]
            over = (lengths[row] + 1) ** c["penalty"]
            found += [(-(v / over), j, t, v) for t, v in zip(best.tolist(), logp[best].tolist())]
        for _, j, t, v in sorted(found)[:k]:
            row = b * beams + j
            out["scores"].append(v)
            out["parents"].append(j)
            out["tokens"].append(t)
            out["lengths"].append(lengths[row] + (not finished[row]))
            out["finished"].append(int(bool(finished[row]) or t == EOS))
            out["history"].append(s["history"][row, :c["steps"]].tolist() + [t])
    return {name: torch.tensor(v, device="cuda", dtype=torch.float64 if name == "scores" else torch.int32) for name, v in out.items()}


def exact(case, seed):
    return {"cache": _exact_cache, "window": _exact_cache, "pages": _exact_pages, "beams": _exact_beams}[case["op"]](case, seed)
