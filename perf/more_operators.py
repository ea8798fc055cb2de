"""What a decoder of answers keeps and checks: its keys and values in 4 bits,
attention over them, and the tokens that a smaller model drafted for it.

`run` computes the operators in plain torch operations, or with `own` set
through the library's entry points.  Keys and values are held in pages: of
`page` tokens each, for every key head the codes of the keys and of the values
(4-bit floats 1.2.1, feature 2i in the low half of byte i), then one byte for
each 32 features of a key or value, their scale's exponent + 127.  A table
names the pages of each sequence.

Every case is a dict of plain values.  The lengths of its sequences come from
the case, their order, the pages and every value from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
TINY = 2.0 ** -100  # the least largest magnitude that 32 values' scale is made for
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # One decoding step's keys and values of 64 answers (large shape's
        # heads), written and read back: latency.
        {"name": "write_step", "kind": "store", "seqs": 64, "rows": 1, "kv": 96, "kv_heads": 16,
         "dh": 64, "page": 16, "ragged": True, "write": True},
        # The keys and values of a SuperBatch's texts (bge lengths and heads),
        # written once and read back.
        {"name": "write_states", "kind": "store", "seqs": 4000, "rows": 48, "kv": 48, "kv_heads": 12,
         "dh": 64, "page": 32, "ragged": True, "write": True},
        # The last tokens of seven short answers, narrow heads.
        {"name": "read_tails", "kind": "store", "seqs": 7, "rows": 13, "kv": 301, "kv_heads": 2,
         "dh": 32, "page": 16, "ragged": True, "write": False},
        # One long document's states taken back to 16 bits.
        {"name": "read_long", "kind": "store", "seqs": 1, "rows": 100_003, "kv": 100_003,
         "kv_heads": 8, "dh": 128, "page": 64, "ragged": False, "write": False},
        # One decoding step of 64 short answers, a key head for each head.
        {"name": "attend_step", "kind": "attend", "seqs": 64, "rows": 1, "kv": 96, "heads": 16,
         "kv_heads": 16, "dh": 64, "page": 16, "ragged": True, "causal": True},
        # One token over one long document: a stream of the cache.
        {"name": "attend_long", "kind": "attend", "seqs": 1, "rows": 1, "kv": 100_003, "heads": 32,
         "kv_heads": 8, "dh": 128, "page": 64, "ragged": False, "causal": True},
        # One decoding step of a batch of long answers, the ordinary call.
        {"name": "attend_batch", "kind": "attend", "seqs": 48, "rows": 1, "kv": 8000, "heads": 32,
         "kv_heads": 8, "dh": 128, "page": 128, "ragged": True, "causal": True},
        # Four drafted tokens and the one before them, for 16 answers.
        {"name": "attend_drafts", "kind": "attend", "seqs": 16, "rows": 5, "kv": 3001, "heads": 16,
         "kv_heads": 4, "dh": 128, "page": 32, "ragged": True, "causal": True},
        # Four prompts' later chunks, over what is in the cache of them.
        {"name": "attend_prompts", "kind": "attend", "seqs": 4, "rows": 1500, "kv": 6000,
         "heads": 16, "kv_heads": 4, "dh": 128, "page": 64, "ragged": True, "causal": True},
        # One answer's four drafts against the encoders' vocabulary.
        {"name": "verify_one", "kind": "verify", "seqs": 1, "drafts": 4, "vocab": 30_522,
         "ragged": False, "draft_probs": True},
        # Drafts without probabilities (looked up in the text), some answers
        # without any.
        {"name": "verify_lookup", "kind": "verify", "seqs": 64, "drafts": 4, "vocab": 30_522,
         "ragged": True, "draft_probs": False},
        # A large batch and a large vocabulary.
        {"name": "verify_batch", "kind": "verify", "seqs": 256, "drafts": 6, "vocab": 100_003,
         "ragged": False, "draft_probs": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["store", "attend", "attend", "verify"])
    if kind == "verify":
        vocab = _log_int(rng, 100, 260_000)
        drafts = rng.randint(1, 12)
        most = min(1024, 256 * 7 * 100_003 // ((drafts + 1) * vocab))
        return {"kind": kind, "seqs": _log_int(rng, 1, max(1, most)), "drafts": drafts,
                "vocab": vocab, "ragged": rng.random() < 0.5, "draft_probs": rng.random() < 0.7}
    heads, kv_heads, dh = rng.choice([(12, 12, 32), (12, 12, 64), (16, 16, 64), (16, 4, 64),
                                      (8, 1, 128), (16, 4, 128), (32, 8, 128), (6, 2, 32)])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "store":
        kv = _log_int(rng, 1, 20_000)
        rows = rng.choice([1, kv, _log_int(rng, 1, kv)])
        most = 4000 * 48 * 12 * 64 // (max(kv, page) * kv_heads * dh)
        return {"kind": kind, "seqs": _log_int(rng, 1, max(1, min(4000, most))), "rows": rows,
                "kv": kv, "kv_heads": kv_heads, "dh": dh, "page": page,
                "ragged": rng.random() < 0.8, "write": rng.random() < 0.5}
    rows = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 1, 2000)])
    kv = _log_int(rng, 1, 20_000)
    pairs = 0.4 * 4 * 1500 * 6000 * 16 * 128 / (rows * kv * heads * dh)
    held = 48 * 8000 * 8 * 128 / (max(kv, page) * kv_heads * dh + rows * heads * dh)
    return {"kind": kind, "seqs": _log_int(rng, 1, max(1, int(min(2000, pairs, held)))),
            "rows": rows, "kv": kv, "heads": heads, "kv_heads": kv_heads, "dh": dh, "page": page,
            "ragged": rng.random() < 0.8, "causal": rng.random() < 0.8}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _lengths(case, which):
    """int64 [seqs]: the case's median length, spread log-normally up to half
    more where the case is ragged."""
    n, median = case["seqs"], case[which]
    if not case["ragged"] or median <= 4:
        return np.full(n, median, np.int64)
    z = np.random.default_rng([n, median]).standard_normal(n)
    return np.clip(np.rint(median * np.exp(0.5 * z)), 1, median + median // 2).astype(np.int64)


def _ordered(case, which, seed):
    order = np.random.default_rng([seed, 1]).permutation(case["seqs"])
    return _lengths(case, which)[order]


def _device(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def _cache_inputs(case, seed):
    """A cache's pages with the sequences' tokens in them, table and lengths,
    and the rows of a call: which positions of which sequence they are."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    kv = _ordered(case, "kv", seed)
    rows = np.minimum(_ordered(case, "rows", seed), kv)
    page, hk, dh = case["page"], case["kv_heads"], case["dh"]
    need = -(-kv // page)
    width, total = int(need.max()), int(need.sum())
    perm = np.random.default_rng([seed, 2]).permutation(total + 1 + total // 8)[:total]
    table = np.full((case["seqs"], width), -1, np.int64)
    table[np.arange(width) < need[:, None]] = perm
    st = {"case": case, "n_pages": total + 1 + total // 8, "max_length": int(kv.max()),
          "max_rows": int(rows.max()), "n_rows": int(rows.sum()),
          "table": _device(table), "lengths": _device(kv),
          "cu": _device(np.concatenate([[0], np.cumsum(rows)]))}
    st["pages"] = torch.randint(0, 256, (st["n_pages"], hk, page * dh * 17 // 16), generator=g,
                                dtype=torch.uint8, device=DEV)
    all_rows = _rows_at(_device(np.concatenate([[0], np.cumsum(kv)])), st["lengths"], int(kv.sum()))
    shift = torch.randn(hk * dh, generator=g, device=DEV)
    for a in range(0, int(kv.sum()), 1 << 17):
        at = [x[a:a + (1 << 17)] for x in all_rows]
        x = torch.randn(len(at[0]), 2 * hk * dh, generator=g, device=DEV)
        x[:, :hk * dh] += 2 * shift * (shift.abs() > 2)  # a few features are far from 0 in all keys
        _plain_store(st, at, x[:, :hk * dh].bfloat16(), x[:, hk * dh:].bfloat16())
    return st, g


def _verify_inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, k, v = case["seqs"], case["drafts"], case["vocab"]
    logits = 3 * torch.randn(n, k + 1, v, generator=g, device=DEV)
    st = {"case": case, "p": torch.softmax(logits, 2)}
    logits[:, :k] += torch.randn(n, k, v, generator=g, device=DEV)
    q = torch.softmax(logits[:, :k], 2)
    if case["draft_probs"]:
        st["q"] = q
        noise = torch.rand(n, k, v, generator=g, device=DEV).clamp_min(1e-30)
        st["drafts"] = (q / -torch.log(noise)).argmax(2).int()  # drawn from q
    else:
        st["drafts"] = q.argmax(2).int()
    st["u"] = torch.rand(n, k + 1, generator=g, device=DEV)
    count = np.full(n, k, np.int64)
    if case["ragged"]:
        count = np.random.default_rng([n, k]).integers(0, k + 1, n)
    st["n_drafts"] = _device(count[np.random.default_rng([seed, 1]).permutation(n)])
    st["tokens"] = torch.empty(n, k + 1, dtype=torch.int32, device=DEV)
    st["accepted"] = torch.empty(n, dtype=torch.int32, device=DEV)
    return st


def _inputs(case, seed):
    if case["kind"] == "verify":
        return _verify_inputs(case, seed)
    st, g = _cache_inputs(case, seed)
    w = case["kv_heads"] * case["dh"]
    if case["kind"] == "store":
        if case["write"]:
            kv = torch.randn(st["n_rows"], 2 * w, generator=g, device=DEV).bfloat16()
            st["k"], st["v"] = kv[:, :w], kv[:, w:]  # one projection's output
        st["k_out"], st["v_out"] = (torch.empty(st["n_rows"], w, dtype=torch.bfloat16, device=DEV)
                                    for _ in range(2))
    else:
        hd = case["heads"] * case["dh"]
        st["q"] = torch.randn(st["n_rows"], hd, generator=g, device=DEV).bfloat16()
        st["out"] = torch.empty(st["n_rows"], hd, dtype=torch.bfloat16, device=DEV)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:  # what a program keeps over its steps: the cache's description and a workspace
        from paper_2605_01060_amd import surge as S
        need = 0
        if case["kind"] == "verify":
            need = S.surge_verify_workspace(case["seqs"], case["vocab"])
        else:
            st["cache"] = S.KVCache(st["pages"], st["n_pages"], case["page"], case["kv_heads"],
                                    case["dh"], st["table"], st["table"].shape[1], case["seqs"],
                                    st["lengths"], st["max_length"])
        if case["kind"] == "attend":
            need = S.surge_cache_attention_workspace(st["cache"], st["max_rows"], case["heads"])
        st["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _rows_at(cu, lengths, n):
    """(sequence, position) of each of n rows: a sequence's rows are its last
    positions."""
    count = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(len(lengths), device=DEV), count.long(),
                                  output_size=n)
    return seq, (lengths - cu[1:])[seq] + torch.arange(n, device=DEV)


def _fields(st):
    """The pages' parts: codes of keys and of values [pages, heads, tokens,
    dh / 2], their scales [pages, heads, tokens, dh / 32]."""
    page, dh = st["case"]["page"], st["case"]["dh"]
    out, at = [], 0
    for width in (dh // 2, dh // 2, dh // 32, dh // 32):
        out.append(st["pages"][:, :, at:at + page * width].unflatten(2, (page, width)))
        at += page * width
    return out


def _plain_quantized(x):
    """Codes (two a byte) and scale bytes of rows [T, heads, dh] in 32 bits."""
    x = x.unflatten(2, (-1, 32))
    a = x.abs().amax(3, keepdim=True)
    m, e = torch.frexp(a.clamp_min(TINY))
    e = (e - 3 + (m > 0.875).int()).clamp_max(125)  # the least with a <= 7 2^e
    y = torch.ldexp(x.abs(), -e)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = (torch.round(y / step) * step).clamp_max(6)
    code = torch.where(y < 2, 2 * y, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.uint8)
    code = (code | (x < 0).to(torch.uint8) << 3).flatten(2)
    return code[:, :, 0::2] | code[:, :, 1::2] << 4, (e[..., 0] + 127).to(torch.uint8)


def _plain_store(st, rows, k, v):
    page, hk = st["case"]["page"], st["case"]["kv_heads"]
    seq, pos = rows
    at, slot = st["table"][seq, pos // page].long(), pos % page
    k_codes, v_codes, k_scales, v_scales = _fields(st)
    k_codes[at, :, slot], k_scales[at, :, slot] = _plain_quantized(k.float().unflatten(1, (hk, -1)))
    v_codes[at, :, slot], v_scales[at, :, slot] = _plain_quantized(v.float().unflatten(1, (hk, -1)))


def _plain_values(codes, scales):
    """Codes [..., dh / 2] and scales [..., dh / 32] as values in 32 bits."""
    table = torch.tensor(VALUES + [-v for v in VALUES], device=DEV)
    x = table[torch.stack([codes & 15, codes >> 4], -1).int()].flatten(-2).unflatten(-1, (-1, 32))
    return torch.ldexp(x, scales.int()[..., None] - 127).flatten(-2)


def _plain_load(st, rows):
    page = st["case"]["page"]
    seq, pos = rows
    at, slot = st["table"][seq, pos // page].long(), pos % page
    k_codes, v_codes, k_scales, v_scales = _fields(st)
    return (_plain_values(k_codes[at, :, slot], k_scales[at, :, slot]).flatten(1),
            _plain_values(v_codes[at, :, slot], v_scales[at, :, slot]).flatten(1))


def _run_plain_store(st):
    rows = _rows_at(st["cu"], st["lengths"], st["n_rows"])
    if st["case"]["write"]:
        _plain_store(st, rows, st["k"], st["v"])
    k, v = _plain_load(st, rows)
    return {"k": k.bfloat16(), "v": v.bfloat16()}


def _run_plain_attend(st):
    case = st["case"]
    h, hk, dh = case["heads"], case["kv_heads"], case["dh"]
    b, longest, lq = case["seqs"], st["max_length"], st["max_rows"]
    at = torch.arange(longest, device=DEV)
    some = at < st["lengths"][:, None]  # [b, longest]
    seq = torch.arange(b, device=DEV)[:, None].expand(b, longest).flatten()
    pos = torch.minimum(at, st["lengths"][:, None] - 1).flatten()
    k, v = (x.view(b, longest, hk, dh).permute(0, 2, 1, 3) for x in _plain_load(st, (seq, pos)))
    beg, count = st["cu"][:-1], st["cu"][1:] - st["cu"][:-1]
    j = torch.arange(lq, device=DEV)
    rows = (beg[:, None] + j).clamp_max(st["n_rows"] - 1)
    q = st["q"][rows].float().view(b, lq, hk, h // hk, dh).permute(0, 2, 3, 1, 4)
    q = q.reshape(b, hk, h // hk * lq, dh)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(dh))
    seen = some[:, None, :].expand(b, lq, longest)
    if case["causal"]:
        seen = seen & (at <= (st["lengths"] - count)[:, None, None] + j[:, None])
    seen = seen[:, None, None].expand(b, 1, h // hk, lq, longest).reshape(b, 1, -1, longest)
    s = torch.where(seen, s, -1e30)
    p = torch.exp(s - s.amax(3, keepdim=True)) * seen
    o = torch.matmul(p, v.contiguous()) / p.sum(3, keepdim=True).clamp_min(1e-30)
    o = o.view(b, hk, h // hk, lq, dh).permute(0, 3, 1, 2, 4).reshape(b, lq, h * dh)
    return o[j < count[:, None]].bfloat16()


def _run_plain_verify(st):
    n, k, v = st["case"]["seqs"], st["case"]["drafts"], st["case"]["vocab"]
    x, u, count = st["drafts"].long(), st["u"].double(), st["n_drafts"]
    j, every = torch.arange(k, device=DEV), torch.arange(n, device=DEV)
    px = st["p"][:, :k].gather(2, x[..., None])[..., 0].double()
    qx = st["q"].gather(2, x[..., None])[..., 0].double() if "q" in st else 1.0
    ok = (u[:, :k] * qx < px) & (j < count[:, None])
    a = torch.cumprod(ok.int(), 1).sum(1)
    p = st["p"][every, a].double()
    rejected, last = (a < count)[:, None], a.clamp_max(k - 1)
    if "q" in st:
        q = torch.where(rejected, st["q"][every, last].double(), 0.0)
        r = (p - q).clamp_min(0)
    else:
        r = torch.where(rejected & (torch.arange(v, device=DEV) == x[every, last][:, None]), 0.0, p)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, p)
    c = r.cumsum(1)
    token = (c <= u[:, k:] * c[:, -1:]).sum(1).int()
    tokens = torch.where(torch.arange(k + 1, device=DEV) < a[:, None],
                         torch.cat([st["drafts"], st["drafts"][:, :1]], 1), -1)
    tokens[every, a] = token
    return {"tokens": tokens, "accepted": a.int()}


def run(st):
    case = st["case"]
    if not own:
        return {"store": _run_plain_store, "attend": _run_plain_attend,
                "verify": _run_plain_verify}[case["kind"]](st)
    from paper_2605_01060_amd import surge as S
    stream = torch.cuda.current_stream()
    if case["kind"] == "verify":
        v = case["vocab"]
        S.surge_op_verify_drafts(case["seqs"], case["drafts"], v, st["n_drafts"], st["drafts"],
                                 st["p"], v, st.get("q"), v, st["u"], st["workspace"],
                                 st["tokens"], st["accepted"], stream)
        return {"tokens": st["tokens"], "accepted": st["accepted"]}
    if case["kind"] == "store":
        w = case["kv_heads"] * case["dh"]
        if case["write"]:
            S.surge_op_cache_write(st["cache"], st["n_rows"], st["cu"], st["k"], 2 * w, st["v"],
                                   2 * w, stream)
        S.surge_op_cache_read(st["cache"], st["n_rows"], st["cu"], st["k_out"], w, st["v_out"], w,
                              stream)
        return {"k": st["k_out"], "v": st["v_out"]}
    hd = case["heads"] * case["dh"]
    S.surge_op_cache_attention(st["cache"], st["n_rows"], st["cu"], st["max_rows"], case["heads"],
                               case["causal"], 1.0 / math.sqrt(case["dh"]), st["q"], hd,
                               st["workspace"], st["out"], hd, stream)
    return st["out"]


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    if case["kind"] == "verify":  # of each answer one row of either's probabilities
        n = case["seqs"] * case["vocab"]
        return {"bytes": n * (8 if case["draft_probs"] else 4), "flops": 3 * n}
    kv = _lengths(case, "kv").astype(np.float64)
    rows = np.minimum(_lengths(case, "rows"), kv)
    w, cached = case["kv_heads"] * case["dh"], 2 * case["kv_heads"] * case["dh"] * 17 / 32
    if case["kind"] == "store":
        t = rows.sum()
        b = t * (4 * w + cached) + (t * (4 * w + cached) if case["write"] else 0)
        return {"bytes": float(b), "flops": float(4 * t * w)}
    hd = case["heads"] * case["dh"]
    pairs = rows * kv - (rows * (rows - 1) / 2 if case["causal"] else 0)
    return {"bytes": float(4 * rows.sum() * hd + kv.sum() * cached),
            "flops": float(4 * pairs.sum() * hd)}


# ---------------------------------------------------------------------------
# The same results in 64 bits
# ---------------------------------------------------------------------------

def _nearest(x):
    """The values in 64 bits that rows [T, w] stand for in the cache: the
    nearest of sixteen, the even code of two."""
    x = x.double().view(len(x), -1, 32)
    a = x.abs().max(2, keepdim=True).values.clamp(min=TINY)
    scale = torch.pow(2.0, torch.ceil(torch.log2(a / 7)).clamp(max=125))
    y = x.abs() / scale
    code = torch.zeros_like(y, dtype=torch.int64)
    for i in range(7):
        middle = (VALUES[i] + VALUES[i + 1]) / 2
        code += (y > middle) | ((y == middle) & (i % 2 == 1))
    v = torch.tensor(VALUES, dtype=torch.float64, device=DEV)[code] * scale * torch.sign(x)
    return v.view(len(x), -1)


def _held(st, i, first, last):
    """Keys and values [positions first .. last - 1, heads, dh] of sequence i."""
    case = st["case"]
    page, hk, dh = case["page"], case["kv_heads"], case["dh"]
    pos = np.arange(first, last)
    at = st["table"].cpu().numpy()[i][pos // page]
    slot = torch.from_numpy(pos % page).to(DEV)
    body = st["pages"][torch.from_numpy(at).to(DEV).long()]
    sign = torch.tensor([1.0, -1.0], dtype=torch.float64, device=DEV)
    size = torch.tensor(VALUES, dtype=torch.float64, device=DEV)
    found = []
    for which in range(2):
        start = which * page * dh // 2 + slot * (dh // 2)
        idx = (start[:, None] + torch.arange(dh // 2, device=DEV))[:, None].expand(-1, hk, -1)
        byte = body.gather(2, idx)
        start = page * dh + which * page * dh // 32 + slot * (dh // 32)
        idx = (start[:, None] + torch.arange(dh // 32, device=DEV))[:, None].expand(-1, hk, -1)
        scale = torch.pow(2.0, body.gather(2, idx).double() - 127).repeat_interleave(32, 2)
        x = torch.empty(last - first, hk, dh, dtype=torch.float64, device=DEV)
        for half, code in ((0, byte % 16), (1, byte // 16)):
            x[:, :, half::2] = size[(code % 8).long()] * sign[(code // 8).long()]
        found.append(x * scale)
    return found


def _exact_store(st):
    case = st["case"]
    if case["write"]:
        return {x: torch.cat([_nearest(r) for r in st[x].split(1 << 15)]) for x in ("k", "v")}
    cu, lengths = st["cu"].tolist(), st["lengths"].tolist()
    parts = []
    for i, n in enumerate(lengths):
        first = n - (cu[i + 1] - cu[i])
        parts += [_held(st, i, a, min(n, a + (1 << 14))) for a in range(first, n, 1 << 14)]
    return {x: torch.cat([p[w] for p in parts]).flatten(1) for w, x in enumerate("kv")}


def _exact_attend(st):
    case = st["case"]
    h, hk, dh = case["heads"], case["kv_heads"], case["dh"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    cu, lengths = st["cu"].tolist(), st["lengths"].tolist()
    for i, n in enumerate(lengths):
        a, b = cu[i], cu[i + 1]
        k, v = _held(st, i, 0, n)
        k, v = k.permute(1, 2, 0).contiguous(), v.permute(1, 0, 2).contiguous()
        step = max(1, (1 << 28) // (n * h))
        for c in range(a, b, step):
            d = min(b, c + step)
            q = st["q"][c:d].double().view(d - c, hk, h // hk, dh).permute(1, 2, 0, 3)
            s = (q.reshape(hk, -1, dh) @ k / math.sqrt(dh)).view(hk, h // hk, d - c, n)
            if case["causal"]:
                after = torch.arange(n, device=DEV) > torch.arange(n - b + c, n - b + d, device=DEV)[:, None]
                s.masked_fill_(after, -math.inf)
            o = torch.softmax(s, 3).view(hk, -1, n) @ v
            out[c:d] = o.view(h, d - c, dh).permute(1, 0, 2).reshape(d - c, h * dh)
    return out


def _exact_verify(st):
    n, k = st["case"]["seqs"], st["case"]["drafts"]
    x, count = st["drafts"].tolist(), st["n_drafts"].tolist()
    u = st["u"].double().tolist()
    idx = st["drafts"].long()[..., None]
    px = st["p"][:, :k].gather(2, idx)[..., 0].double().tolist()
    qx = st["q"].gather(2, idx)[..., 0].double().tolist() if "q" in st else None
    tokens = torch.full((n, k + 1), -1, dtype=torch.int32)
    accepted = torch.zeros(n, dtype=torch.int32)
    for i in range(n):
        a = 0
        while a < count[i] and px[i][a] > u[i][a] * (qx[i][a] if qx else 1.0):
            tokens[i, a] = x[i][a]
            a += 1
        r = st["p"][i, a].double()
        if a < count[i]:
            less = r.clone()
            if qx:
                less -= st["q"][i, a]
            else:
                less[x[i][a]] = 0
            less[less < 0] = 0
            r = less if less.sum() > 0 else r
        c = torch.cumsum(r, 0)
        tokens[i, a] = int(torch.searchsorted(c, c[-1] * u[i][k], right=True))
        accepted[i] = a
    return {"tokens": tokens.to(DEV), "accepted": accepted.to(DEV)}


def exact(case, seed):
    return {"store": _exact_store, "attend": _exact_attend,
            "verify": _exact_verify}[case["kind"]](_inputs(case, seed))
