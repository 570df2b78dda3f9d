"""The operators of a 4-bit paged cache and of cache pages, as cases to time
and to compare.

A case is a dict of plain values; ``what`` names the operator:

* ``append``   rows of keys and values quantized into the pages of a 4-bit
               cache (keys rotated first where ``rope``), and read back from
               them as the values that the pages hold;
* ``attend``   causal grouped-query attention of query rows over such pages:
               one row of each sequence (a decode step), or several (a prompt,
               or a part of one behind ``past`` cached positions);
* ``copy``     pages of a cache copied to other pages in every layer: whole
               streams (``sources`` == ``pairs``), or a few pages that many new
               streams get their own copies of (a fork's last, partly filled
               page);
* ``compact``  the live pages of a pool moved to its lowest ids and the page
               tables rewritten.

Sequences hold pages in no order, as a free list deals them.  Keys, values and
queries are N(0, 1), as normalised projections are; heads have 64 dimensions,
pages 16 positions, and the head counts are those of the models of the
workload table (32 query heads on 8 kv heads, 4 on 2) and their neighbours.
``pad`` sequences of a batch are padding: their one row has position -1.
"""
import math

import torch

own = False

PAGE, HEAD, BLOCK = 16, 64, 1152  # positions a page, dimensions a head, bytes a (page, kv head)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------ cases

def listed():
    return [
        # The step of a lockstep batch: one new row of each of 32 streams.
        dict(name="append 32 x 1", what="append", hkv=8, dtype="bf16", seqs=32, rows=1, past=700, rope=True, pad=0),
        # A long prompt's keys and values as the QKV product leaves them.
        dict(name="append 8192", what="append", hkv=8, dtype="f32", seqs=1, rows=8192, past=0, rope=True, pad=0),
        # The first answer tokens of one short request: latency.
        dict(name="token 1 x 300", what="attend", hq=32, hkv=8, dtype="f16", seqs=1, rows=1, past=300, rope=False, pad=0),
        # The small model's step, in its 32-bit type, in a padded batch.
        dict(name="tokens 6 x 200 f32", what="attend", hq=4, hkv=2, dtype="f32", seqs=6, rows=1, past=200, rope=True, pad=2),
        # A lockstep batch of ragged streams around 4,000 positions.
        dict(name="tokens 32 x 4000", what="attend", hq=32, hkv=8, dtype="bf16", seqs=32, rows=1, past=4000, rope=True, pad=0),
        # One stream at the longest context the runtime takes.
        dict(name="token 1 x 131072", what="attend", hq=32, hkv=8, dtype="f16", seqs=1, rows=1, past=131071, rope=True, pad=0),
        # Second turns of three conversations, one prefill pass.
        dict(name="turns 3 x 150 at 5000", what="attend", hq=32, hkv=8, dtype="f32", seqs=3, rows=150, past=5000, rope=False, pad=0),
        # The workload table's long prompt.
        dict(name="prompt 8192", what="attend", hq=32, hkv=8, dtype="bf16", seqs=1, rows=8192, past=0, rope=True, pad=0),
        # A prompt shared by 63 new streams: their own copies of its last page.
        dict(name="fork 63", what="copy", layers=16, page_bytes=32768, pages=1024, pairs=63, sources=1),
        # A stream's whole context copied: 1,500 pages of a 4-bit cache.
        dict(name="copy 1500", what="copy", layers=16, page_bytes=9216, pages=4096, pairs=1500, sources=1500),
        # The small model's pool after some of its streams ended.
        dict(name="compact 500", what="compact", layers=2, page_bytes=16384, pages=500, streams=9, filled=0.45, shared=0.1),
        # A serving pool of 4-bit pages, half of it live.
        dict(name="compact 6000", what="compact", layers=16, page_bytes=9216, pages=6000, streams=40, filled=0.5, shared=0.2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["append", "attend", "attend", "attend", "copy", "compact"])
    c = dict(what=what)
    if what == "copy":
        c["layers"] = _log_int(rng, 1, 32)
        c["page_bytes"] = rng.choice([1152, 2304, 9216, 16384, 32768])
        c["pages"] = _log_int(rng, 64, max(128, min(8192, (1 << 29) // (c["layers"] * c["page_bytes"]))))
        c["pairs"] = _log_int(rng, 1, c["pages"] // 2)
        c["sources"] = rng.choice([c["pairs"], _log_int(rng, 1, c["pairs"])])
        return c
    if what == "compact":
        c["layers"] = _log_int(rng, 1, 32)
        c["page_bytes"] = rng.choice([1152, 2304, 9216, 16384, 32768])
        c["pages"] = _log_int(rng, 64, max(128, min(32768, (1 << 29) // (c["layers"] * c["page_bytes"]))))
        c["streams"] = _log_int(rng, 1, 64)
        c["filled"], c["shared"] = round(rng.uniform(0.1, 0.95), 2), round(rng.uniform(0.0, 0.4), 2)
        return c
    c["hkv"] = rng.choice([1, 2, 4, 8, 8])
    c["dtype"] = rng.choice(["f32", "f16", "bf16"])
    c["rope"], c["pad"] = rng.random() < 0.5, rng.choice([0, 0, 1, 3])
    if what == "append":
        c["seqs"] = _log_int(rng, 1, 64)
        c["rows"], c["past"] = _log_int(rng, 1, 8192 // c["seqs"]), _log_int(rng, 1, 6000)
        return c
    c["hq"] = c["hkv"] * rng.choice([1, 2, 4, 4, 8])
    if rng.random() < 0.6:
        c["rows"], c["seqs"] = 1, _log_int(rng, 1, 128)
        c["past"] = _log_int(rng, 1, 131071 // c["seqs"])
    else:
        c["seqs"] = _log_int(rng, 1, 16)
        c["rows"] = _log_int(rng, 2, int(6000 * min(1.0, 32 / c["hq"]) ** 0.5) // c["seqs"])
        most = min(30000, 8192 * 8192 * 32 // (c["seqs"] * c["hq"] * 2 * c["rows"]))
        c["past"] = _log_int(rng, 1, max(1, most - 2 * c["rows"]))
    return c


# ------------------------------------------------------------------ the case's sequences

def _spread(n, mid):
    """n counts from 0.6 to 1.4 times ``mid`` (one: ``mid`` itself)."""
    return [mid if n == 1 else max(1, int(round(mid * (0.6 + 0.8 * ((7 * i + 3) % n) / (n - 1))))) for i in range(n)]


def _sequences(case):
    """(rows, first position) of every sequence, the padding ones last."""
    n = case["seqs"]
    past = [min(p, 131072 - 2 * case["rows"]) if case["rows"] > 1 else min(p, 131071) for p in _spread(n, case["past"])] if case["past"] else [0] * n
    rows = _spread(n, case["rows"]) if case["rows"] > 1 else [1] * n
    return list(zip(rows, past)) + [(1, -1)] * case["pad"]


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(shape, dtype, g):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)


def _perm(n, g):
    return torch.randperm(n, generator=g, device="cuda")


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rope_table(n):
    """cos and sin of position x pair, base 5e5, as the runtime's table holds them."""
    ang = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 5e5 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32.0)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


def _cache_inputs(case, seed):
    g = _gen(seed)
    seqs = _sequences(case)
    need = [(p + r + PAGE - 1) // PAGE for r, p in seqs]
    wide, used = max(need), sum(need)
    n_pages = used + 5
    ids = _perm(n_pages, g)[:used].to(torch.int32)
    table = torch.zeros((len(seqs), wide), dtype=torch.int32, device="cuda")
    held = torch.arange(wide, device="cuda")[None, :] < torch.tensor(need, device="cuda")[:, None]
    table[held] = ids
    start = [0]
    for r, _ in seqs:
        start.append(start[-1] + r)
    dt = TYPES[case["dtype"]]
    s = dict(case=case, table=table, start=_ints(start), first=_ints([p for _, p in seqs]), n_pages=n_pages, rows=start[-1],
             most=max(r for r, _ in seqs), rope=_rope_table(wide * PAGE) if case["rope"] else None)
    if case["what"] == "append":
        # The rows stand in the fused rows of the QKV product (4 query heads a kv head).
        fused = _normal((start[-1], 6 * case["hkv"], HEAD), dt, g)
        s["k"], s["v"] = fused[:, 4 * case["hkv"]:5 * case["hkv"]], fused[:, 5 * case["hkv"]:]
        s["pool"] = torch.zeros((n_pages, case["hkv"], BLOCK), dtype=torch.uint8, device="cuda")
        s["k_back"], s["v_back"] = (torch.empty((start[-1], case["hkv"], HEAD), dtype=dt, device="cuda") for _ in "kv")
    else:
        s["pool"] = _random_pages(n_pages, case["hkv"], g)
        s["q"] = _normal((start[-1], case["hq"], HEAD), dt, g)
        s["out"] = torch.empty_like(s["q"])
    return s


def _pool_inputs(case, seed):
    g = _gen(seed)
    shape = (case["layers"], case["pages"], case["page_bytes"])
    s = dict(case=case, pool=torch.empty(shape, dtype=torch.uint8, device="cuda").random_(0, 256, generator=g))
    order = _perm(case["pages"], g)
    if case["what"] == "copy":
        n, k = case["pairs"], case["sources"]
        src = order[n:n + k][torch.arange(n, device="cuda") % k]
        s["src"], s["dst"] = src.to(torch.int32).cpu().numpy(), order[:n].to(torch.int32).cpu().numpy()
        return s
    # Streams of ragged lengths over the live part of the pool; the first pages
    # of a stream may be another's too (a fork's shared prompt).
    n, live = case["streams"], max(case["streams"], int(case["filled"] * case["pages"]))
    each = [max(1, x) for x in _spread(n, live // n)]
    lead = [0 if i == 0 else min(int(case["shared"] * e), each[0]) for i, e in enumerate(each)]
    wide = max(each) + 3
    table = torch.zeros((n, wide), dtype=torch.int32, device="cuda")
    at, lens = 0, []
    for i in range(n):
        mine = each[i] - lead[i]
        mine = min(mine, case["pages"] - at)
        table[i, :lead[i]] = table[0, :lead[i]]
        table[i, lead[i]:lead[i] + mine] = order[at:at + mine].to(torch.int32)
        at += mine
        lens.append(max(0, (lead[i] + mine) * PAGE - (5 * i) % PAGE))
    s["table"], s["lengths"] = table, _ints(lens)
    s["out_table"], s["live"] = torch.empty_like(table), torch.empty(1, dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    return _pool_inputs(case, seed) if case["what"] in ("copy", "compact") else _cache_inputs(case, seed)


# ------------------------------------------------------------------ plain forms

def _quantize(x):
    """Codes (with 8 added) and scales of the groups of 32 of fp32 rows [..., 64].
    The quotients are the format's correctly rounded ones: a division in 32 bits
    that is not would move values next to a border."""
    g = x.reshape(*x.shape[:-1], 2, 32).double()
    a = (g.abs().amax(-1) / torch.full((), 7.0, device=x.device, dtype=torch.float64)).float()
    s = torch.where(a < 2.0 ** -17, torch.round(a * 2.0 ** 24) * 2.0 ** -24, a.bfloat16().float().clamp(max=2720.0))
    c = torch.where(s[..., None] > 0, (g / s[..., None].double()).float().round().clamp(-7, 7), torch.zeros((), device=x.device))
    return (c + 8).to(torch.uint8).reshape(x.shape), s.half()


def _code_bytes(k, v):
    """The code bytes of key and value rows (codes [rows, heads, 64]) of one position
    each: 32 bytes as [4][8] and 16 pairs."""
    k = k.reshape(*k.shape[:-1], 2, 4, 2, 2, 2)  # step, quarter, byte, nibble, half
    k = (k[..., 0, :] | k[..., 1, :] << 4).permute(0, 1, 3, 2, 5, 4)  # quarter, step, half, byte
    v = v.reshape(*v.shape[:-1], 16, 2, 2)
    return k.reshape(*k.shape[:2], 4, 8), v[..., 0] | v[..., 1] << 4


def _put(pool, page, slot, k, v):
    """Rows of fp32 keys and values into the slots of a pool's pages."""
    kc, ks = _quantize(k)
    vc, vs = _quantize(v)
    kb, vb = _code_bytes(kc, vc)
    n, h = k.shape[0], k.shape[1]
    d = k.device
    quarter, eight, row16, two = (torch.arange(i, device=d) for i in (4, 8, 16, 2))
    slot = slot[:, None, None]
    at = torch.cat([((quarter[:, None] * 16 + slot) * 8 + eight).reshape(n, 32),
                    (512 + ((slot // 4 * 16 + row16[:, None]) * 4 + slot % 4) * 2 + two).reshape(n, 32),
                    (1024 + slot * 4 + torch.arange(4, device=d)).reshape(n, 4),
                    (1088 + two[:, None] * 32 + slot * 2 + two).reshape(n, 4)], 1)
    data = torch.cat([kb.reshape(n, h, 32), vb.reshape(n, h, 32), ks.view(torch.uint8), vs.view(torch.uint8)], 2)
    pool[page[:, None, None], torch.arange(h, device=d)[None, :, None], at[:, None, :]] = data


def _random_pages(n, h, g):
    pool = torch.empty((n, h, BLOCK), dtype=torch.uint8, device="cuda")
    page = torch.arange(n, device="cuda").repeat_interleave(PAGE)
    slot = torch.arange(PAGE, device="cuda").repeat(n)
    _put(pool, page, slot, _normal((n * PAGE, h, HEAD), torch.float32, g), _normal((n * PAGE, h, HEAD), torch.float32, g))
    return pool


def _values(blocks):
    """fp32 keys and values [..., 16, heads, 64] of page blocks [..., heads, 1152]."""
    lead, h = blocks.shape[:-2], blocks.shape[-2]

    def nibbles(b):
        return torch.stack([b & 15, b >> 4], -1).float() - 8.0

    n = len(lead)
    k = nibbles(blocks[..., :512].reshape(*lead, h, 4, 16, 2, 2, 2))  # quarter, slot, step, half, byte, nibble
    k = k.permute(*range(n), n + 2, n, n + 3, n + 1, n + 5, n + 6, n + 4).reshape(*lead, PAGE, h, 2, 32)
    v = nibbles(blocks[..., 512:1024].reshape(*lead, h, 4, 16, 2, 2, 2))  # slot / 4, dims / 4, pair, half, byte, nibble
    v = v.permute(*range(n), n + 1, n + 3, n + 4, n, n + 2, n + 5, n + 6).reshape(*lead, PAGE, h, 2, 32)
    s = blocks[..., 1024:].contiguous().view(torch.float16).float()
    ks = s[..., :32].reshape(*lead, h, PAGE, 2).transpose(-3, -2)
    vs = s[..., 32:].reshape(*lead, h, 2, PAGE).permute(*range(n), n + 2, n, n + 1)
    return (k * ks[..., None]).reshape(*lead, PAGE, h, HEAD), (v * vs[..., None]).reshape(*lead, PAGE, h, HEAD)


def _rotate(x, rope, pos):
    """Rotation of pairs (i, i + 32) of rows at their positions, in 64 bits,
    since keys next to a code's border are quantized after it."""
    c, s = rope[pos].double().unbind(-1)
    c, s = c[:, None], s[:, None]
    a, b = x[..., :32].double(), x[..., 32:].double()
    return torch.cat([a * c - b * s, b * c + a * s], -1).float()


def _row_places(state):
    """Each row's sequence and position."""
    start = state["start"].long()
    row = torch.arange(state["rows"], device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), row, right=True)
    return seq, state["first"].long()[seq] + row - start[seq]


def _append_plain(state):
    seq, pos = _row_places(state)
    k, v = state["k"].float(), state["v"].float()
    if state["rope"] is not None:
        k = _rotate(k, state["rope"], pos.clamp(min=0))
    real = pos >= 0
    at = pos.clamp(min=0)
    page, slot = state["table"].long()[seq, at // PAGE], at % PAGE
    _put(state["pool"], page[real], slot[real], k[real], v[real])
    kb, vb = _values(state["pool"][page])
    row = torch.arange(state["rows"], device="cuda")
    none = torch.zeros((), device="cuda")
    dt = state["k"].dtype
    return tuple(torch.where(real[:, None, None], x[row, slot], none).to(dt) for x in (kb, vb))


def _attend_plain(state):
    case = state["case"]
    hq, hkv, n, most = case["hq"], case["hkv"], state["first"].numel(), state["most"]
    seq, pos = _row_places(state)
    q = state["q"].float()
    if state["rope"] is not None:
        q = _rotate(q, state["rope"], pos.clamp(min=0))
    k, v = _values(state["pool"][state["table"].long()])  # [n, pages, 16, hkv, 64]
    keys = k.shape[1] * PAGE
    k = k.reshape(n, keys, hkv, HEAD).permute(0, 2, 3, 1).reshape(n * hkv, HEAD, keys)
    v = v.reshape(n, keys, hkv, HEAD).transpose(1, 2).reshape(n * hkv, keys, HEAD)
    at = torch.arange(state["rows"], device="cuda") - state["start"].long()[seq]
    padded = torch.zeros((n, most, hq, HEAD), device="cuda")
    padded[seq, at] = q
    limit = torch.full((n, most), -1, dtype=torch.int64, device="cuda")
    limit[seq, at] = pos
    group = hq // hkv
    padded = padded.reshape(n, most, hkv, group, HEAD).permute(0, 2, 3, 1, 4).reshape(n * hkv, group * most, HEAD)
    w = torch.bmm(padded, k).mul_(0.125).view(n, hkv, group, most, keys)
    hidden = torch.arange(keys, device="cuda") > limit[..., None]
    w.masked_fill_(hidden[:, None, None], -math.inf)
    w.sub_(w.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.bmm(w.view(n * hkv, group * most, keys), v).view(n, hkv, group, most, HEAD)
    o = torch.where(total > 0, o / total, torch.zeros((), device="cuda"))
    return o.permute(0, 3, 1, 2, 4).reshape(n, most, hq, HEAD)[seq, at].to(state["q"].dtype)


def _copy_plain(state):
    src, dst = (torch.from_numpy(state[k]).long().to("cuda") for k in ("src", "dst"))
    state["pool"][:, dst] = state["pool"][:, src]
    return state["pool"]


def _compact_plain(state):
    pool, table = state["pool"], state["table"].long()
    n = pool.shape[1]
    held = torch.arange(table.shape[1], device="cuda")[None, :] < ((state["lengths"].long() + PAGE - 1) // PAGE)[:, None]
    used = torch.zeros(n, dtype=torch.bool, device="cuda")
    used[table[held]] = True
    page = torch.arange(n, device="cuda")
    live = used.sum()
    src, dst = page[used & (page >= live)], page[~used & (page < live)]
    pool[:, dst] = pool[:, src]
    page[src] = dst
    return pool, torch.where(held, page[table], table).to(torch.int32), live.to(torch.int32).reshape(1)


# ------------------------------------------------------------------ a pass

def _plan(state):
    """What a program of the framework keeps beside its cache: the descriptions
    of pool and rows, and the workspace."""
    from paper_2606_12154_amd import hh
    case = state["case"]
    plan = dict(hh=hh)
    if case["what"] == "compact":
        plan["ws"] = torch.empty(hh.hh_kv_compact_workspace(case["pages"]), dtype=torch.uint8, device="cuda")
    elif case["what"] != "copy":
        pool, table = state["pool"], state["table"]
        plan["type"] = {"f32": hh.HH_F32, "bf16": hh.HH_BF16, "f16": hh.HH_F16}[case["dtype"]]
        plan["pool"] = hh.hh_kv4_pool(pool.data_ptr(), table.data_ptr(), state["n_pages"], case["hkv"], table.shape[1], table.shape[0])
        plan["rows"] = hh.hh_kv4_rows(state["start"].data_ptr(), state["first"].data_ptr(), None, state["first"].numel(), state["rows"], state["most"])
        plan["rope"] = (None, 0) if state["rope"] is None else (state["rope"].data_ptr(), state["rope"].shape[0])
        if case["what"] == "attend":
            plan["ws"] = torch.empty(hh.hh_kv4_attention_workspace(plan["pool"], plan["rows"], case["hq"]), dtype=torch.uint8, device="cuda")
    return plan


def _own(state):
    plan = state.get("plan")
    if plan is None:
        plan = state["plan"] = _plan(state)
    hh, case = plan["hh"], state["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if case["what"] == "append":
        k, v, kb, vb = state["k"], state["v"], state["k_back"], state["v_back"]
        hh.hh_kv4_append(plan["pool"], plan["rows"], k.data_ptr(), v.data_ptr(), plan["type"], k.stride(0), v.stride(0), *plan["rope"], stream)
        hh.hh_kv4_read(plan["pool"], plan["rows"], kb.data_ptr(), vb.data_ptr(), plan["type"], kb.stride(0), vb.stride(0), stream)
        return kb, vb
    if case["what"] == "attend":
        q, o, ws = state["q"], state["out"], plan["ws"]
        hh.hh_kv4_attention(plan["pool"], plan["rows"], q.data_ptr(), plan["type"], q.stride(0), case["hq"], 0.125, *plan["rope"],
                            o.data_ptr(), plan["type"], o.stride(0), ws.data_ptr(), ws.numel(), stream)
        return o
    pool = state["pool"]
    if case["what"] == "copy":
        hh.hh_kv_copy_pages(pool.data_ptr(), pool.shape[0], pool.stride(0), pool.shape[2], pool.shape[1], state["src"], state["dst"], stream)
        return pool
    table = state["out_table"].copy_(state["table"])
    hh.hh_kv_compact(pool.data_ptr(), pool.shape[0], pool.stride(0), pool.shape[2], pool.shape[1], table.data_ptr(), table.shape[0], table.shape[1],
                     state["lengths"].data_ptr(), state["live"].data_ptr(), plan["ws"].data_ptr(), plan["ws"].numel(), stream)
    return pool, table, state["live"]


def run(state):
    if own:
        return _own(state)
    what = state["case"]["what"]
    return {"append": _append_plain, "attend": _attend_plain, "copy": _copy_plain, "compact": _compact_plain}[what](state)


# ------------------------------------------------------------------ cost

def work(case):
    if case["what"] == "copy":
        each = case["layers"] * case["page_bytes"]
        return dict(bytes=(case["sources"] + case["pairs"]) * each, flops=0)
    if case["what"] == "compact":
        # Moved pages: those past the live count; about the live share of the rest.
        n = case["streams"]
        each = [max(1, x) for x in _spread(n, max(n, int(case["filled"] * case["pages"])) // n)]
        live = min(case["pages"], each[0] + sum(e - min(int(case["shared"] * e), each[0]) for e in each[1:]))
        moved = live * (case["pages"] - live) / case["pages"]
        return dict(bytes=2 * moved * case["layers"] * case["page_bytes"] + 8 * sum(each) + 4 * n, flops=0)
    seqs = _sequences(case)
    rows, keys = sum(r for r, _ in seqs), sum(r + p for r, p in seqs)
    size = 4 if case["dtype"] == "f32" else 2
    rope = 256 * rows if case["rope"] else 0
    if case["what"] == "append":
        # Rows in, pages out and in again, values out.
        return dict(bytes=rows * case["hkv"] * (4 * HEAD * size + 2 * 72) + rope, flops=rows * case["hkv"] * HEAD * 8)
    attended = sum(r * p + r * (r + 1) // 2 for r, p in seqs)
    return dict(bytes=keys * (case["hkv"] * 72 + 4 / PAGE) + 2 * rows * case["hq"] * HEAD * size + rope, flops=4 * HEAD * case["hq"] * attended)


# ------------------------------------------------------------------ 64-bit results

def _exact_group(x):
    """The 64-bit values that groups of 32 of rows [..., 64] are held as: the
    format divides in 32 bits, and a quotient rounded from 64 bits is the same."""
    g = x.double().unflatten(-1, (2, 32))
    top = (g.abs().amax(-1, keepdim=True) / torch.full_like(g[..., :1], 7.0)).float()
    e = torch.frexp(top.double())[1].long()
    step = ((e - 8).clamp(min=-24) + 1023 << 52).view(torch.float64)  # a power of two, exactly
    s = (torch.round(top.double() / step) * step).clamp(max=2720.0)
    c = (g / s).float().double().round().clamp(-7.0, 7.0)
    return torch.where(s > 0, c * s, torch.zeros_like(c)).flatten(-2)


def _exact_pages(pool):
    """64-bit keys and values [pages, heads, 16, 64] of a pool, by looking up where
    each element's nibble and scale stand."""
    d = pool.device
    slot, dim = torch.arange(16, device=d)[:, None], torch.arange(64, device=d)[None, :]
    e = dim % 8
    k_at = ((dim % 32 // 8) * 16 + slot) * 8 + dim // 32 * 4 + e % 2 * 2 + e // 4
    v_at = 512 + (slot // 4 * 16 + dim // 4) * 8 + slot % 4 * 2 + dim % 4 // 2
    scales = pool[..., 1024:].contiguous().view(torch.float16).double()
    k = (pool[..., k_at].int() >> (e // 2 % 2 * 4) & 15) - 8
    v = (pool[..., v_at].int() >> (dim % 2 * 4) & 15) - 8
    return k.double() * scales[..., slot * 2 + dim // 32], v.double() * scales[..., 32 + dim // 32 * 16 + slot]


def _exact_turn(x, rope, pos):
    z = torch.complex(x[..., :32].double(), x[..., 32:].double())
    w = torch.view_as_complex(rope[pos].double().contiguous())[:, None]
    z = torch.complex(z.real * w.real - z.imag * w.imag, z.imag * w.real + z.real * w.imag)
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    if case["what"] in ("copy", "compact"):
        return None  # copies and whole numbers
    state = prepare(case, seed)
    seqs, r0, parts = _sequences(case), 0, []
    if case["what"] == "append":
        pos = torch.cat([torch.arange(p, p + r, device="cuda") for r, p in seqs])
        k = state["k"].double()
        if case["rope"]:
            k = _exact_turn(state["k"], state["rope"], pos.clamp(min=0)).float()
        real = (pos >= 0)[:, None, None]
        return tuple(torch.where(real, _exact_group(x), torch.zeros((), dtype=torch.float64, device="cuda")) for x in (k, state["v"]))
    group = case["hq"] // case["hkv"]
    for s, (r, p) in enumerate(seqs):
        q = state["q"][r0:r0 + r].double()
        r0 += r
        if p < 0:
            parts.append(torch.zeros_like(q))
            continue
        pos = torch.arange(p, p + r, device="cuda")
        if case["rope"]:
            q = _exact_turn(q, state["rope"], pos)
        k, v = _exact_pages(state["pool"][state["table"][s, :(p + r + PAGE - 1) // PAGE].long()])
        hidden = torch.arange(k.shape[0] * PAGE, device="cuda")[None, :] > pos[:, None]
        o = torch.empty_like(q)
        for j in range(case["hq"]):
            kj, vj = (x[:, j // group].reshape(-1, HEAD) for x in (k, v))
            a = (q[:, j].contiguous() @ kj.T.contiguous() / 8.0).masked_fill_(hidden, -math.inf)
            o[:, j] = torch.softmax(a, -1) @ vj
        parts.append(o)
    return torch.cat(parts)
