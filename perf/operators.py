"""Cases of the paged cache operators, for timing and comparing builds.

A paged cache holds the keys and values of many sequences in pages of a few slots each.
Four operators work on it: appending token rows with the position rotation applied on the
way, to pages of 16-bit values and to pages of 4-bit values (MXFP4: e2m1 elements with
one power-of-two scale per 32 channels), and attention over either, each token row seeing
a range of its sequence's slots: all slots up to its own, its group and the one before
(the decoder's own mask), its document, a common prefix, or a window.

Where `own` is false the operators are computed in elementary torch operations; where it
is true, by the library.  Lengths come from the case, values and the order of the pages
from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda"
ROPE_BASE = 1e5
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one user's decode step: three committed bytes of one layer of the d = 1024 model
        dict(name="append_step_b1", op="append", cache="f16", q="f32", seqs=1, heads=16, kv_heads=16, dim=64, page=64,
             before=4096, rows=3, ragged=0, shape=1),
        # a full server takes in its prompts: 64 of up to 2048 bytes, one layer
        dict(name="append_prompt_b64", op="append", cache="f16", q="f32", seqs=64, heads=16, kv_heads=16, dim=64, page=64,
             before=0, rows=2048, ragged=1, shape=2),
        # the step of 64 users with five bytes each, into a 4-bit cache
        dict(name="append_fp4_step_b64", op="append", cache="mxfp4", q="f32", seqs=64, heads=16, kv_heads=16, dim=64, page=64,
             before=2048, rows=5, ragged=1, shape=3),
        # prompts of a model with grouped heads, 16-bit activations, into a 4-bit cache
        dict(name="append_fp4_prompt_b8", op="append", cache="mxfp4", q="bf16", seqs=8, heads=32, kv_heads=8, dim=128, page=16,
             before=0, rows=4096, ragged=1, shape=4),
        # the smallest attention: one byte of one user
        dict(name="attend_step_b1", op="attend", cache="f16", q="f32", seqs=1, heads=16, kv_heads=16, dim=64, page=64,
             before=1024, rows=1, ragged=0, mask="causal", shape=5),
        # one byte for each of 64 users with ragged contexts
        dict(name="attend_step_b64", op="attend", cache="f16", q="f32", seqs=64, heads=16, kv_heads=16, dim=64, page=64,
             before=2048, rows=1, ragged=1, mask="causal", shape=6),
        # verification of seven drafts at d = 2048 over 8192-byte contexts
        dict(name="attend_verify_b16", op="attend", cache="bf16", q="bf16", seqs=16, heads=32, kv_heads=32, dim=64, page=128,
             before=8192, rows=7, ragged=0, mask="causal", shape=7),
        # a whole sequence under the group mask, as the MB layers see it
        dict(name="attend_groups_t4096", op="attend", cache="f16", q="f32", seqs=1, heads=16, kv_heads=16, dim=64, page=64,
             before=0, rows=4096, ragged=0, mask="groups", shape=8),
        # packed documents of a model with grouped heads: the largest
        dict(name="attend_documents_b4", op="attend", cache="bf16", q="bf16", seqs=4, heads=32, kv_heads=8, dim=128, page=32,
             before=0, rows=4096, ragged=0, mask="documents", shape=9),
        # 4-bit: one user with a very long context
        dict(name="attend_fp4_long_b1", op="attend", cache="mxfp4", q="bf16", seqs=1, heads=32, kv_heads=8, dim=128, page=64,
             before=131071, rows=1, ragged=0, mask="causal", shape=10),
        # 4-bit: a full server's step over ragged contexts
        dict(name="attend_fp4_step_b64", op="attend", cache="mxfp4", q="f32", seqs=64, heads=16, kv_heads=16, dim=64, page=64,
             before=8192, rows=3, ragged=1, mask="causal", shape=11),
        # 4-bit: two prompts continue after 8192 slots, their next 1500 bytes at once
        dict(name="attend_fp4_prompt_b2", op="attend", cache="mxfp4", q="f16", seqs=2, heads=16, kv_heads=4, dim=64, page=16,
             before=8192, rows=1500, ragged=1, mask="prefix", shape=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend"])
    cache = rng.choice(["bf16", "f16", "mxfp4", "mxfp4"])
    c = dict(op=op, cache=cache, q=rng.choice(["f32", rng.choice(["bf16", "f16"]) if cache == "mxfp4" or op == "append" else cache]),
             page=rng.choice([16, 32, 64, 128, 256]), ragged=rng.randint(0, 1), shape=rng.randint(100, 1 << 30))
    c["dim"] = rng.choice([32, 64, 64, 128])
    c["kv_heads"] = rng.choice([1, 2, 4, 5, 8, 16])
    c["heads"] = c["kv_heads"] * rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8) if g * c["kv_heads"] <= 40])
    prompt = rng.random() < 0.4
    c["seqs"] = _log_int(rng, 1, 8 if prompt else 64)
    most = max(32, min(8192 if prompt else 40000, (1 << 20) // (c["seqs"] * c["kv_heads"] * c["dim"] // 64)))
    c["rows"] = _log_int(rng, 17, min(3000, most)) if prompt else rng.randint(1, 8)
    if op == "append":
        c["before"] = rng.choice([0, _log_int(rng, 1, most)])
        return c
    c["before"] = rng.choice([0, _log_int(rng, 1, most), _log_int(rng, 1, most)])
    c["mask"] = rng.choice(["causal", "causal", "groups", "documents", "prefix", "window"])
    while c["seqs"] * c["rows"] * (c["before"] + c["rows"]) * c["heads"] * c["dim"] > 4 * 4096 * 4096 * 32 * 128:
        c["before"], c["rows"] = 2 * c["before"] // 3, 2 * c["rows"] // 3
    return c


def _lengths(case):
    """(slots held before, new rows) of every sequence."""
    r = random.Random(case["shape"])
    out = []
    for _ in range(case["seqs"]):
        before, rows = case["before"], case["rows"]
        if case["ragged"]:
            before, rows = r.randint(before // 2, before), r.randint((rows + 1) // 2, rows)
        out.append((before, rows))
    return out


def _ranges(case):
    """Visible slots [lo, hi) of every row, in row order; some rows of a document mask
    belong to no document and see nothing."""
    r = random.Random(case["shape"] + 1)
    lo, hi = [], []
    for before, rows in _lengths(case):
        kind, n = case["mask"], before + rows
        if kind == "causal":
            lo += [0] * rows
            hi += range(before + 1, n + 1)
        elif kind == "window":
            w = max(1, n // 3)
            lo += [max(0, s + 1 - w) for s in range(before, n)]
            hi += range(before + 1, n + 1)
        elif kind == "prefix":
            p = (before + n) // 2
            lo += [0] * rows
            hi += [max(s + 1, p) for s in range(before, n)]
        else:  # segments: words of up to 16 bytes, or documents
            start, prev, end, skip = 0, 0, 0, False
            for s in range(n):
                if s == end:
                    prev, start = start, s
                    end = s + (min(16, 1 + int(r.expovariate(1 / 6))) if kind == "groups" else r.randint(1, max(2, n // 2)))
                    skip = kind == "documents" and r.random() < 0.05 and s > 0
                    end = min(end, s + 9) if skip else end
                if s >= before:
                    lo.append(prev if kind == "groups" else start)
                    hi.append(start if skip else s + 1)
    return lo, hi


def _page_bytes(case):
    """Bytes of one page of one head."""
    if case["cache"] == "mxfp4":
        return case["page"] * (case["dim"] // 2 + case["dim"] // 32)
    return case["page"] * case["dim"] * 2


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    lens = _lengths(case)
    total = sum(rows for _, rows in lens)
    page, heads, kvh, dim = case["page"], case["heads"], case["kv_heads"], case["dim"]
    counts = [-(-(b + r) // page) for b, r in lens]
    width = max(counts)
    n_pages = sum(counts) + 3
    order = torch.randperm(n_pages, generator=g, device=DEVICE, dtype=torch.int32)
    count = torch.tensor(counts, device=DEVICE)
    at = torch.arange(width, device=DEVICE)
    place = (count.cumsum(0) - count)[:, None] + at
    pages = torch.where(at < count[:, None], order[place.clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    starts = [0]
    for _, rows in lens:
        starts.append(starts[-1] + rows)
    s = dict(case=case, total=total, page=page, heads=heads, kvh=kvh, dim=dim, n_pages=n_pages, pages=pages,
             row_start=torch.tensor(starts, dtype=torch.int32, device=DEVICE),
             first_slot=torch.tensor([b for b, _ in lens], dtype=torch.int32, device=DEVICE),
             max_rows=max(r for _, r in lens), max_slots=max(b + r for b, r in lens))

    def values(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    qt = _TYPES[case["q"]]
    s["q"] = (2.0 * values(total, heads, dim)).to(qt)
    if case["op"] == "append":
        s["k"], s["v"] = values(total, kvh, dim).to(qt), values(total, kvh, dim).to(qt)
        s["q_out"] = torch.zeros_like(s["q"])
        j = torch.arange(dim // 2, dtype=torch.float64, device=DEVICE)
        angle = torch.arange(s["max_slots"], dtype=torch.float64, device=DEVICE)[:, None] * ROPE_BASE ** (-2 * j / dim)
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
    if case["cache"] == "mxfp4":
        shape, tall = (n_pages, kvh, _page_bytes(case)), page * dim // 2
        make = lambda: torch.zeros(shape, dtype=torch.uint8, device=DEVICE)  # noqa: E731
        if case["op"] == "attend":
            def make():  # codes of normal values with amax near 2: scales 2^-2 .. 2^-1
                p = torch.empty(shape, dtype=torch.uint8, device=DEVICE)
                p[..., :tall] = torch.randint(0, 256, (n_pages, kvh, tall), generator=g, device=DEVICE, dtype=torch.uint8)
                p[..., tall:] = torch.randint(125, 127, (n_pages, kvh, shape[2] - tall), generator=g, device=DEVICE, dtype=torch.uint8)
                return p
    else:
        shape, kt = (n_pages, kvh, page, dim), _TYPES[case["cache"]]
        make = lambda: torch.zeros(shape, dtype=kt, device=DEVICE) if case["op"] == "append" else values(*shape).to(kt)  # noqa: E731
    s["kp"], s["vp"] = make(), make()
    if case["op"] == "attend":
        s["scale"] = 1.0 / math.sqrt(dim)
        s["out"] = torch.zeros_like(s["q"])
        if case["mask"] == "causal":
            s["lo"] = s["hi"] = None
        else:
            lo, hi = _ranges(case)
            s["lo"] = torch.tensor(lo, dtype=torch.int32, device=DEVICE)
            s["hi"] = torch.tensor(hi, dtype=torch.int32, device=DEVICE)
            s["max_slots"] = max(s["max_slots"], max(hi))
    if own:  # what a program keeps: the cache over its pools, and the step's rows
        import paper_2608_15454_amd as mbp

        dtype = {"bf16": mbp.BF16, "f16": mbp.F16, "mxfp4": mbp.MXFP4}[case["cache"]]
        s["paged"] = mbp.PagedCache(dtype, kvh, dim, page, pages=pages, k=s["kp"], v=s["vp"])
        s["batch"] = mbp.PagedRows(s["row_start"], s["first_slot"], total, s["max_rows"], s["max_slots"])
    return s


# ------------------------------------------------------------------ the plain forms
def _rows(s):
    """Sequence, index in its run, and slot of every row."""
    r = torch.arange(s["total"], device=DEVICE, dtype=torch.int32)
    seq = torch.searchsorted(s["row_start"][1:], r, right=True)
    j = r - s["row_start"][seq]
    return seq, j.long(), (s["first_slot"][seq] + j).long()


def _rotated(x, table, pos):
    x = x.unflatten(-1, (-1, 2))
    cs = table[pos].to(x.dtype)[:, None]
    a, b, c, sn = x[..., 0], x[..., 1], cs[..., 0], cs[..., 1]
    return torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2)


def _to_mxfp4(x):
    """(codes of float64 x, scale bytes, the values that they stand for)."""
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(amax)[1] - 3).clamp(-127, 127)
    e = torch.where(amax > 0, e, -127)
    y = torch.ldexp(b, -e)
    a = y.abs()
    # nearest value of e2m1, ties to the even code
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(a.dtype)
    near = ((a / step).round() * step).clamp(max=6.0)
    code = torch.searchsorted(torch.tensor(E2M1, dtype=a.dtype, device=a.device), near) + 8 * (torch.signbit(b)).long()
    return code.flatten(-2).to(torch.uint8), (e + 127).squeeze(-1).to(torch.uint8), torch.ldexp(torch.copysign(near, b), e).flatten(-2)


def _plain_append(s):
    seq, _, slot = _rows(s)
    page, at = s["pages"][seq, slot // s["page"]].long(), slot % s["page"]
    s["q_out"].copy_(_rotated(s["q"].float(), s["rope"], slot))
    if s["case"]["cache"] != "mxfp4":
        s["kp"][page, :, at] = _rotated(s["k"].float(), s["rope"], slot).to(s["kp"].dtype)
        s["vp"][page, :, at] = s["v"].float().to(s["vp"].dtype)
        return s["q_out"], s["kp"], s["vp"]
    tall, out = s["page"] * s["dim"] // 2, [s["q_out"]]
    # float64: a value next to the middle of two codes goes to the right one
    ck, ek, vk = _to_mxfp4(_rotated(s["k"].double(), s["rope"], slot))
    cv, ev, vv = _to_mxfp4(s["v"].double())
    codes_k, scales_k = s["kp"][..., :tall].unflatten(-1, (s["page"], -1)), s["kp"][..., tall:].unflatten(-1, (s["page"], -1))
    codes_v, scales_v = s["vp"][..., :tall].unflatten(-1, (s["page"], -1)), s["vp"][..., tall:].unflatten(-1, (s["page"], -1))
    codes_k[page, :, at], scales_k[page, :, at] = ck[..., 0::2] | (ck[..., 1::2] << 4), ek
    codes_v[page, :, at], scales_v[page, :, at] = cv[..., 0::2] | (cv[..., 1::2] << 4), ev
    return out + [vk.to(torch.bfloat16), vv.to(torch.bfloat16)]


def _dense(s, pool):
    """Every sequence's slots in order, float32 [seqs, kv heads, slots, dim]."""
    t = torch.arange(s["max_slots"], device=DEVICE)
    page, at = s["pages"][:, t // s["page"]].clamp(min=0).long(), t % s["page"]
    if s["case"]["cache"] != "mxfp4":
        return pool[page, :, at].float().transpose(1, 2).contiguous()
    tall = s["page"] * s["dim"] // 2
    codes = pool[..., :tall].unflatten(-1, (s["page"], -1))[page, :, at]
    e = pool[..., tall:].unflatten(-1, (s["page"], -1))[page, :, at].float() - 127.0
    table = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=DEVICE)
    x = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()]
    return (x.unflatten(-1, (-1, 32)) * torch.exp2(e)[..., None]).flatten(-2).transpose(1, 2).contiguous()


def _plain_attend(s):
    seq, j, slot = _rows(s)
    seqs, group = s["case"]["seqs"], s["heads"] // s["kvh"]
    k, v = _dense(s, s["kp"]), _dense(s, s["vp"])
    lo = torch.zeros(seqs, s["max_rows"], dtype=torch.int32, device=DEVICE)
    hi = torch.zeros_like(lo)
    hi[seq, j] = (slot + 1).int() if s["hi"] is None else s["hi"]
    if s["lo"] is not None:
        lo[seq, j] = s["lo"]
    q = torch.zeros(seqs, s["max_rows"], s["heads"], s["dim"], device=DEVICE)
    q[seq, j] = s["q"].float()
    q = q.unflatten(2, (s["kvh"], group)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [seqs, kv heads, rows * group, dim]
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * s["scale"]
    t = torch.arange(s["max_slots"], device=DEVICE)
    seen = ((t >= lo[..., None]) & (t < hi[..., None])).repeat_interleave(group, 1)[:, None]
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    o = o.unflatten(2, (s["max_rows"], group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s["out"].copy_(o[seq, j])
    return s["out"]


def run(s):
    if not own:
        return _plain_append(s) if s["case"]["op"] == "append" else _plain_attend(s)
    if s["case"]["op"] == "attend":
        return s["paged"].attend(s["batch"], s["q"], out=s["out"], lo=s["lo"], hi=s["hi"], scale=s["scale"])
    s["paged"].append(s["batch"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rope"])
    if s["case"]["cache"] != "mxfp4":
        return s["q_out"], s["kp"], s["vp"]
    return [s["q_out"], *s["paged"].read(s["batch"], dtype=torch.bfloat16)]


def work(case):
    lens = _lengths(case)
    rows = sum(r for _, r in lens)
    width = {"f32": 4, "bf16": 2, "f16": 2}[case["q"]]
    slot = case["kv_heads"] * _page_bytes(case) / case["page"]  # bytes of one slot's keys, or values
    q = rows * case["heads"] * case["dim"] * width
    if case["op"] == "append":
        new = 2 * rows * case["kv_heads"] * case["dim"]
        back = new * 2 + 2 * rows * slot if case["cache"] == "mxfp4" else 0  # read back as 16-bit values
        return {"bytes": 2 * q + new * width + 2 * rows * slot + back + max(b + r for b, r in lens) * case["dim"] * 4,
                "flops": 3 * rows * (case["heads"] + case["kv_heads"]) * case["dim"]}
    lo, hi = _ranges(case)
    pairs = sum(max(0, b - a) for a, b in zip(lo, hi))
    at, seen = 0, 0
    for _, r in lens:  # slots that some row of the sequence sees
        ends, last = sorted(zip(lo[at:at + r], hi[at:at + r])), 0
        for a, b in ends:
            seen += max(0, b - max(a, last))
            last = max(last, b)
        at += r
    return {"bytes": 2 * q + 2 * seen * slot, "flops": 4 * case["heads"] * case["dim"] * pairs}


# ------------------------------------------------------------------ in 64 bits, row by row of the definition
def _exact_slots(pool, case, page_ids, n):
    """Values of slots 0 .. n-1 behind page_ids: float64 [kv heads, n, dim]."""
    x = pool[page_ids.long()]  # [pages, kv heads, ...]
    if case["cache"] != "mxfp4":
        return x.double().transpose(0, 1).flatten(1, 2)[:, :n]
    tall = case["page"] * case["dim"] // 2
    code = x[..., :tall].transpose(0, 1).reshape(case["kv_heads"], -1, case["dim"] // 2)[:, :n].int()
    byte = x[..., tall:].transpose(0, 1).reshape(case["kv_heads"], -1, case["dim"] // 32)[:, :n].int()
    code = torch.stack((code % 16, code // 16), 3).reshape(case["kv_heads"], n, case["dim"])
    mag = code % 8
    value = torch.where(mag < 2, mag / 2.0, (1.0 + (mag % 2) / 2.0) * 2.0 ** (mag // 2 - 1).double()).double()
    value = torch.where(code >= 8, -value, value)
    return value * (2.0 ** (byte.double() - 127.0)).repeat_interleave(32, 2)


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    lens = _lengths(case)
    kvh, dim, page = case["kv_heads"], case["dim"], case["page"]
    if case["op"] == "attend":
        lo, hi = _ranges(case)
        out = torch.zeros(s["total"], case["heads"], dim, dtype=torch.float64, device=DEVICE)
        at = 0
        for i, (before, rows) in enumerate(lens):
            n = max(hi[at:at + rows])
            keys = _exact_slots(s["kp"], case, s["pages"][i, : -(-n // page)], n)
            vals = _exact_slots(s["vp"], case, s["pages"][i, : -(-n // page)], n)
            first = torch.tensor(lo[at:at + rows], device=DEVICE)[:, None]
            end = torch.tensor(hi[at:at + rows], device=DEVICE)[:, None]
            where = torch.arange(n, device=DEVICE)
            hidden = (where < first) | (where >= end)
            for h in range(case["heads"]):
                logit = s["q"][at:at + rows, h].double() @ keys[h * kvh // case["heads"]].T / math.sqrt(dim)
                weight = torch.exp(logit - logit.amax(1, keepdim=True)).masked_fill(hidden, 0.0)
                norm = weight.sum(1, keepdim=True)
                o = weight @ vals[h * kvh // case["heads"]] / norm
                out[at:at + rows, h] = torch.where((end > first), o, 0.0)
            at += rows
        return out
    pos = torch.cat([torch.arange(b, b + r, device=DEVICE) for b, r in lens])
    turn = torch.view_as_complex(s["rope"].double())[pos][:, None]
    q = torch.view_as_real(torch.view_as_complex(s["q"].double().reshape(s["total"], -1, dim // 2, 2)) * turn).reshape(s["total"], -1, dim)
    k = torch.view_as_real(torch.view_as_complex(s["k"].double().reshape(s["total"], -1, dim // 2, 2)) * turn).reshape(s["total"], -1, dim)
    v = s["v"].double()
    if case["cache"] == "mxfp4":
        grid = torch.tensor(E2M1, dtype=torch.float64, device=DEVICE)
        middle = (grid[1:] + grid[:-1]) / 2
        back = []
        for x in (k, v):
            block = x.reshape(s["total"], kvh, dim // 32, 32)
            unit = 2.0 ** (torch.floor(torch.log2(block.abs().amax(-1, keepdim=True).clamp(min=1e-300))) - 2).clamp(min=-127)
            y = block / unit
            size = y.abs()
            code = torch.bucketize(size, middle)  # the smaller of two equally near values
            odd_tie = (code < 7) & (size == middle[code.clamp(max=6)]) & (code % 2 == 1)
            back.append((grid[code + odd_tie.long()] * torch.sign(y) * unit).reshape(s["total"], kvh, dim))
        return [q, *back]
    pools = []
    for x, pool in ((k, s["kp"]), (v, s["vp"])):
        p = pool.double()
        at = 0
        for i, (before, rows) in enumerate(lens):
            where = torch.arange(before, before + rows, device=DEVICE)
            p[s["pages"][i, where // page].long(), :, where % page] = x[at:at + rows]
            at += rows
        pools.append(p)
    return [q, *pools]
