"""The operators of decoding over a paged key-value cache, as cases that can be timed and compared.

  rope    norm of every query and key head with the position rotation in the same pass (`jot.head_norm_rope`), with or
          without the rotated keys and the values going straight into the cache's pages
  write   rows of keys and values into the pages (`jot.kv_write`)
  copy    whole pages to other pages, in every layer at once (`jot.kv_copy_pages`): what forking a sequence and
          compacting a pool come down to
  attend  attention of a few new rows per sequence over its pages (`jot.paged_attention`): one row (a token), a block's
          rows, or a stretch of a canvas

Pages are [layers, pages, kv heads, page size, head dimension], keys and values apart.  Attention is bidirectional: every
query sees all keys of its sequence.  Head counts, canvas lengths and block sizes are those of the models that this
repository decodes (32 heads of 128; 28 query over 4 key heads of 128; 4 heads of 64).
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _rope(name, seqs, rows, nq, nkv, hd, *, rotary=None, interleaved=False, dtype="bf16", norm=False, first=0, theta=500000.0,
          factor=1.0, page=0):
    return {"op": "rope", "name": name, "seqs": seqs, "rows": rows, "nq": nq, "nkv": nkv, "hd": hd, "rotary": rotary or hd,
            "interleaved": interleaved, "dtype": dtype, "norm": norm, "first": first, "theta": theta, "factor": factor,
            "page": page}


def _write(name, seqs, rows, nkv, hd, page, *, dtype="bf16"):
    return {"op": "write", "name": name, "seqs": seqs, "rows": rows, "nkv": nkv, "hd": hd, "page": page, "dtype": dtype}


def _copy(name, n, layers, nkv, hd, page, *, dtype="bf16"):
    return {"op": "copy", "name": name, "n": n, "layers": layers, "nkv": nkv, "hd": hd, "page": page, "dtype": dtype}


def _attend(name, seqs, rows, nq, nkv, hd, shortest, longest, page, *, dtype="bf16"):
    return {"op": "attend", "name": name, "seqs": seqs, "rows": rows, "nq": nq, "nkv": nkv, "hd": hd, "shortest": shortest,
            "longest": longest, "page": page, "dtype": dtype}


def listed():
    return [
        # one new token of one sequence, far into a context that was stretched four times
        _rope("rope_token", 1, 1, 28, 4, 128, norm=True, first=90001, theta=1e6, factor=4.0),
        # a block's rows of 16 sequences, keys and values into the pages: what a block pass does in every layer
        _rope("rope_block_pages", 16, 32, 32, 32, 128, norm=True, first=671, page=64),
        # the whole canvas of 16 sequences, queries and keys as they stand in the QKV projection's output
        _rope("rope_canvas", 16, 704, 32, 32, 128),
        # half of each head rotated, neighbours paired, in half precision, odd lengths
        _rope("rope_partial_fp16", 8, 753, 28, 4, 128, rotary=64, interleaved=True, dtype="fp16", norm=True, first=131,
              theta=10000.0),
        # a block's rows of eight sequences, small pages
        _write("write_block", 8, 32, 4, 128, 16),
        # whole canvases after a pass over everything
        _write("write_canvas", 16, 704, 32, 128, 64),
        # a fork: the last, partly filled page of five sequences
        _copy("copy_fork", 5, 28, 4, 128, 16),
        # compaction of a pool: the pages behind its new end into the holes before it
        _copy("copy_compact", 512, 28, 4, 128, 64),
        # one token of one short sequence: latency
        _attend("attend_token_short", 1, 1, 28, 4, 128, 129, 129, 16),
        # one token of four long sequences of unequal length: the cache is read once
        _attend("attend_token_long", 4, 1, 28, 4, 128, 40007, 131072, 64),
        # blocks of 32 rows of 16 sequences, every query head with keys of its own
        _attend("attend_block", 16, 32, 32, 32, 128, 384, 704, 64),
        # blocks of 32 rows of eight ragged sequences, seven query heads to a key head, pages that end inside tiles
        _attend("attend_block_shared_fp16", 8, 32, 28, 4, 128, 2001, 9001, 24, dtype="fp16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    nq, nkv, hd = rng.choice([(32, 32, 128), (28, 4, 128), (4, 4, 64), (4, 2, 64), (32, 8, 128), (2, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    op = rng.choice(["rope", "write", "copy", "attend", "attend"])
    if op == "rope":
        total = _log(rng, 1, 11264)
        seqs = _log(rng, 1, min(16, total))
        case = _rope("", seqs, max(1, total // seqs), nq, nkv, hd, rotary=rng.choice([hd, hd, hd // 2, hd // 4]),
                     interleaved=rng.random() < 0.4, dtype=dtype, norm=rng.random() < 0.6, first=_log(rng, 1, 120000),
                     theta=rng.choice([10000.0, 500000.0, 1e6]), factor=rng.choice([1.0, 1.0, 2.0, 8.0]),
                     page=rng.choice([0, 0, 16, 24, 64, 100]))
    elif op == "write":
        total = _log(rng, 1, 11264)
        seqs = _log(rng, 1, min(16, total))
        case = _write("", seqs, max(1, total // seqs), nkv, hd, rng.choice([1, 16, 24, 64, 100, 128]), dtype=dtype)
    elif op == "copy":
        layers, page = rng.choice([1, 2, 28, 32]), rng.choice([1, 16, 24, 64, 100, 128])
        most = min(512, 7 * 2 ** 26 // (layers * nkv * hd * page))
        case = _copy("", _log(rng, 1, max(1, most)), layers, nkv, hd, page, dtype=dtype)
    else:
        rows = rng.choice([1, 1, 1, 2, 5, 16, 32, 32, 61, 200, 384])
        # what a case may read and compute is bounded by the listed ones'
        seqs = _log(rng, 1, 32)
        longest = _log(rng, 1, max(1, min(131072, 2 ** 29 // (seqs * nkv * hd * 2), 2 ** 26 // (seqs * nq * rows))))
        case = _attend("", seqs, rows, nq, nkv, hd, rng.randint(1, longest), longest, rng.choice([1, 16, 24, 64, 100, 128]), dtype=dtype)
    del case["name"]
    return case


def _lengths(case):
    """Key counts of the sequences, spread evenly from the shortest to the longest."""
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def work(case):
    elem, hd = 2, case["hd"]
    if case["op"] == "rope":
        n = case["seqs"] * case["rows"]
        heads = case["nq"] + case["nkv"] + (case["nkv"] if case["page"] else 0)
        return {"bytes": 2 * n * heads * hd * elem + n * (8 if case["page"] else 4), "flops": n * (case["nq"] + case["nkv"]) * hd * 8}
    if case["op"] == "write":
        n = case["seqs"] * case["rows"]
        return {"bytes": 4 * n * case["nkv"] * hd * elem + 4 * n, "flops": 0}
    if case["op"] == "copy":
        return {"bytes": 4 * case["n"] * case["layers"] * case["nkv"] * case["page"] * hd * elem, "flops": 0}
    keys, q = sum(_lengths(case)), case["seqs"] * case["rows"] * case["nq"]
    return {"bytes": 2 * keys * case["nkv"] * hd * elem + q * (2 * hd * elem + 4), "flops": 4 * keys * case["rows"] * case["nq"] * hd}


def _normal(gen, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def _inverse_frequencies(case):
    """theta^(-2 i / rotary), positions divided by the factor by which the context was stretched."""
    i = torch.arange(case["rotary"] // 2, dtype=torch.float64)
    return (case["theta"] ** (-2.0 * i / case["rotary"]) / case["factor"]).float().cuda()


def prepare(case, seed):
    rng = random.Random(seed * 7919 + 17)
    gen = torch.Generator("cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    nkv, hd, page = case["nkv"], case["hd"], case["page"]
    if case["op"] == "copy":
        n = case["n"]
        pages = list(range(2 * n + 3))
        rng.shuffle(pages)
        shape = (case["layers"], 2 * n + 3, nkv, page, hd)
        return {"case": case, "k": _normal(gen, shape, dtype), "v": _normal(gen, shape, dtype), "src": pages[:n], "dst": pages[n:2 * n]}
    if case["op"] == "attend":
        lens = _lengths(case)
        rng.shuffle(lens)
        counts = [(n + page - 1) // page for n in lens]
        width = max(counts) + 2
        ids = list(range(sum(counts) + 3))
        rng.shuffle(ids)
        table, at = [], 0
        for c in counts:                                    # a table is as wide as a sequence may become: the rest is unused
            table.append(ids[at:at + c] + [-1] * (width - c))
            at += c
        shape = (1, len(ids), nkv, page, hd)
        return {"case": case, "k": _normal(gen, shape, dtype), "v": _normal(gen, shape, dtype),
                "q": _normal(gen, (case["seqs"], case["rows"], case["nq"], hd), dtype),
                "table": torch.tensor(table, dtype=torch.int32, device="cuda"),
                "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    seqs, rows = case["seqs"], case["rows"]
    n, nq = seqs * rows, case.get("nq", 0)
    qkv = _normal(gen, (n, (nq + 2 * nkv), hd), dtype)       # the projection's output: queries, keys, values of a row
    state = {"case": case, "q": qkv[:, :nq], "k": qkv[:, nq:nq + nkv], "v": qkv[:, nq + nkv:]}
    if case["op"] == "rope":
        first = [case["first"] + rng.randrange(64) for _ in range(seqs)]
        state["positions"] = (torch.tensor(first, device="cuda")[:, None] + torch.arange(rows, device="cuda")).flatten().int()
        state["inv_freq"] = _inverse_frequencies(case)
        state["magnitude"] = 0.1 * math.log(case["factor"]) + 1.0
        gain = (lambda: (1.0 + 0.1 * _normal(gen, (hd,), torch.float32)).to(dtype)) if case["norm"] else (lambda: None)
        state["q_gain"], state["k_gain"] = gain(), gain()
    if page:
        each = (rows + page - 1) // page + 1                 # rows start somewhere in their first page
        ids = list(range(seqs * each + 2))
        rng.shuffle(ids)
        table = torch.tensor(ids[:seqs * each], device="cuda").view(seqs, each)
        at = torch.tensor([rng.randrange(page) for _ in range(seqs)], device="cuda")[:, None] + torch.arange(rows, device="cuda")
        state["slots"] = (table.gather(1, at // page) * page + at % page).flatten().int()
        shape = (1, len(ids), nkv, page, hd)
        state["pk"], state["pv"] = _normal(gen, shape, dtype), _normal(gen, shape, dtype)
    return state


def _norm_rotate(x, gain, s, eps=1e-6):
    """Norm (where there is a gain) and rotation of heads [rows, heads, hd], in 32 bits; angles in 64."""
    y = x.float()
    if gain is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * gain.float()
    half = s["inv_freq"].numel()
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    c, z = (angle.cos() * s["magnitude"]).float(), (angle.sin() * s["magnitude"]).float()
    if s["case"]["interleaved"]:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack([a * c - b * z, b * c + a * z], -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat([a * c - b * z, b * c + a * z], -1)
    return torch.cat([turned, y[..., 2 * half:]], -1).to(x.dtype)


def _put(pages, rows, slots):
    page = pages.shape[3]
    slots = slots.long()
    pages[0][slots // page, :, slots % page] = rows


def _attention(s):
    k, v, q, table, lens = s["k"][0], s["v"][0], s["q"].float(), s["table"], s["lens"]
    nkv, page, hd = k.shape[1:]
    seqs, rows, nq = q.shape[:3]
    keys = table.shape[1] * page
    at = table.clamp(min=0).long()
    real = torch.arange(keys, device=q.device) < lens[:, None]
    kk = k[at].transpose(1, 2).reshape(seqs, nkv, keys, hd).float()
    vv = v[at].transpose(1, 2).reshape(seqs, nkv, keys, hd).float()
    vv = torch.where(real[:, None, :, None], vv, 0.0)
    qq = q.view(seqs, rows, nkv, nq // nkv, hd).transpose(1, 2).reshape(seqs, nkv, -1, hd)
    score = (qq @ kk.transpose(-1, -2)) / math.sqrt(hd)
    score = torch.where(real[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    back = lambda t: t.view(seqs, nkv, rows, nq // nkv, -1).transpose(1, 2).reshape(seqs, rows, nq, -1)
    return back((p @ vv) / total).to(s["q"].dtype), back(top + total.log())[..., 0]


def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        from paper_2602_11133_b200 import jot
        if op == "rope":
            rope = jot.Rope(s["inv_freq"], s["case"]["interleaved"], s["magnitude"])
            if "slots" in s:
                q, _ = jot.head_norm_rope(s["q"], s["k"], s["positions"], rope, s["q_gain"], s["k_gain"], 1e-6, v=s["v"],
                                          pages=jot.KVPages(s["pk"], s["pv"]), slots=s["slots"])
                return q, s["pk"], s["pv"]
            return jot.head_norm_rope(s["q"], s["k"], s["positions"], rope, s["q_gain"], s["k_gain"], 1e-6)
        if op == "write":
            jot.kv_write(jot.KVPages(s["pk"], s["pv"]), s["k"], s["v"], s["slots"])
            return s["pk"], s["pv"]
        if op == "copy":
            jot.kv_copy_pages(jot.KVPages(s["k"], s["v"]), s["src"], s["dst"])
            return s["k"], s["v"]
        lse = torch.empty(s["q"].shape[:3], dtype=torch.float32, device="cuda")
        return jot.paged_attention(s["q"], jot.KVPages(s["k"], s["v"]), s["table"], s["lens"], lse=lse), lse
    if op == "rope":
        q, k = _norm_rotate(s["q"], s["q_gain"], s), _norm_rotate(s["k"], s["k_gain"], s)
        if "slots" not in s:
            return q, k
        _put(s["pk"], k, s["slots"])
        _put(s["pv"], s["v"], s["slots"])
        return q, s["pk"], s["pv"]
    if op == "write":
        _put(s["pk"], s["k"], s["slots"])
        _put(s["pv"], s["v"], s["slots"])
        return s["pk"], s["pv"]
    if op == "copy":
        src, dst = (torch.tensor(s[x], device="cuda") for x in ("src", "dst"))
        s["k"][:, dst] = s["k"][:, src]
        s["v"][:, dst] = s["v"][:, src]
        return s["k"], s["v"]
    return _attention(s)


def exact(case, seed):
    """From the definitions, in 64 bits: complex rotation of the pairs; attention sequence by sequence."""
    if case["op"] in ("write", "copy"):                       # nothing is computed
        return None
    s = prepare(case, seed)
    if case["op"] == "attend":
        out, lse = [], []
        for b in range(case["seqs"]):
            n = int(s["lens"][b])
            ids = s["table"][b, :(n + case["page"] - 1) // case["page"]].long()
            k, v = (s[x][0, ids].permute(1, 0, 2, 3).flatten(1, 2)[:, :n].double() for x in ("k", "v"))
            group = case["nq"] // case["nkv"]
            o, l = [], []
            for h in range(case["nkv"]):
                q = s["q"][b, :, h * group:(h + 1) * group].double().flatten(0, 1)
                a = q @ k[h].T * case["hd"] ** -0.5
                l.append(torch.logsumexp(a, 1).view(-1, group))
                o.append((torch.softmax(a, 1) @ v[h]).view(-1, group, case["hd"]))
            out.append(torch.cat(o, 1))
            lse.append(torch.cat(l, 1))
        return torch.stack(out), torch.stack(lse)

    def turned(x, gain):
        x = x.double()
        if gain is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["hd"] + 1e-6) * gain.double()
        half = case["rotary"] // 2
        pair = torch.stack([2 * torch.arange(half), 2 * torch.arange(half) + 1] if case["interleaved"]
                           else [torch.arange(half), torch.arange(half) + half]).cuda()
        z = torch.complex(x[..., pair[0]], x[..., pair[1]])
        z = z * torch.polar(torch.full_like(s["inv_freq"], s["magnitude"], dtype=torch.float64).expand(x.shape[0], half),
                            torch.outer(s["positions"].double(), s["inv_freq"].double()))[:, None]
        x = x.clone()
        x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
        return x

    q, k = turned(s["q"], s["q_gain"]), turned(s["k"], s["k_gain"])
    if "slots" not in s:
        return q, k
    pk, pv = s["pk"].double(), s["pv"].double()
    for i, slot in enumerate(s["slots"].tolist()):
        pk[0, slot // case["page"], :, slot % case["page"]] = k[i]
        pv[0, slot // case["page"], :, slot % case["page"]] = s["v"][i].double()
    return q, pk, pv
