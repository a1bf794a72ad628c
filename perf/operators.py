"""Performance cases of the paged-cache operators: page tables kept on the GPU,
the write into the paged cache, the selection of pages by their block keys and
the attention over the selected pages, as a serving loop calls them through
``PageTables`` and ``PagedKV``.

A case is one of four operators (``op``):

``pages``
    ``append`` of new tokens to the requests of a batch: page tables, slot map,
    positions.  With ``admit`` the batch's slots are released first and new
    prompts take their place; without, every request grows by one token.
``write``
    Keys and values of the batch's rows into their pages, and the block keys
    of the pages that become full.
``select``
    For each row and KV head the pages that its attention reads.
``attend``
    The attention of each row over its selected pages.

Shapes are the repository's own: the draft layers of the tiny fp32, the 8B and
the 70B models, pages of 16 tokens.  Lengths come from the case alone; page
placement and values from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
MODELS = {
    "tiny": dict(n_q=4, n_kv=2, hd=64, fmt="f32"),
    "8b": dict(n_q=32, n_kv=8, hd=128, fmt="bf16"),
    "70b": dict(n_q=64, n_kv=8, hd=128, fmt="bf16"),
}
GROW = 2048        # tokens a standing batch grows by before it starts over


def _case(op, model, requests, lo, hi, seed, **more):
    """``requests`` of lo..hi tokens each, the newest ``rows`` of each (1..rows,
    ragged) being the call's rows, and ``pad`` empty rows behind them."""
    c = dict(op=op, model=model, requests=requests, lo=lo, hi=hi, lens_seed=seed, rows=1, pad=0, admit=False,
             top_k=64, sink=1, local=4, gate=False)
    c.update(more)
    return c


def listed():
    return [
        # a full decode instance: one token for each of 512 requests, in a batch padded for a captured graph
        _case("pages", "8b", 509, 256, 8192, 0, name="pages-step-512", pad=3),
        # a saturated prefill instance: a batch of prompts takes the place of the last one
        _case("pages", "70b", 64, 64, 16384, 1, name="pages-admit-64", admit=True),
        # the step's rows: 512 single tokens, some of which fill a page
        _case("write", "8b", 509, 256, 8192, 0, name="write-step-512", pad=3),
        # a prompt batch of a prefill instance, ragged lengths
        _case("write", "8b", 32, 32, 2000, 2, name="write-prefill-32", rows=4096),
        # the smallest call: the fp32 layer, a few requests, latency
        _case("select", "tiny", 4, 40, 400, 3, name="select-tiny-4", top_k=8, sink=1, local=2),
        # the full decode instance
        _case("select", "8b", 509, 256, 8192, 0, name="select-step-512", pad=3),
        # a few requests with very long caches
        _case("select", "70b", 6, 60000, 131072, 4, name="select-long-6", top_k=128),
        # the newest rows of long prompts, each with its own selection
        _case("select", "8b", 4, 20000, 32768, 5, name="select-chunk-4", rows=130, top_k=96),
        # the smallest call
        _case("attend", "tiny", 4, 40, 400, 3, name="attend-tiny-4", top_k=8, sink=1, local=2),
        # the full decode instance
        _case("attend", "8b", 509, 256, 8192, 0, name="attend-step-512", pad=3),
        # a few requests with very long caches, with the output gate
        _case("attend", "70b", 6, 60000, 131072, 4, name="attend-long-6", top_k=128, gate=True),
        # the newest rows of long prompts
        _case("attend", "8b", 4, 20000, 32768, 5, name="attend-chunk-4", rows=130, top_k=96),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pages", "write", "select", "select", "attend", "attend"])
    seed = rng.randrange(1 << 30)
    model = rng.choice(["tiny", "8b", "8b", "70b"])
    pad = rng.randint(0, 9) if rng.random() < 0.3 else 0
    if op == "pages":
        n, hi = _log(rng, 1, 512), _log(rng, 20, 16384)
        admit = rng.random() < 0.5
        if admit:
            n = min(n, max(1, 500000 // hi))
        return _case(op, model, n, rng.randint(1, hi), hi, seed, pad=pad, admit=admit)
    if op == "write":
        if rng.random() < 0.5:
            return _case(op, model, _log(rng, 1, 512), 1, _log(rng, 16, 8192), seed, pad=pad)
        hi = _log(rng, 16, 4096)
        n = max(1, min(_log(rng, 1, 32), 30000 // hi))
        return _case(op, model, n, rng.randint(1, hi), hi, seed, rows=rng.randint(2, 4096), pad=pad)
    top_k = _log(rng, 4, 160)
    sink = rng.randint(0, 2)
    local = rng.randint(1, min(8, top_k - sink - 1))
    least = 20 * top_k         # the longest request has pages to choose from
    kind = rng.choice(["step", "step", "long", "rows"])
    if model == "tiny":
        kind = "step"
    more = dict(top_k=top_k, sink=sink, local=local, pad=pad, gate=op == "attend" and rng.random() < 0.3)
    if kind == "step":
        hi = _log(rng, least, 8192)
        n = min(_log(rng, 1, 64 if model == "tiny" else 500), 28000 // top_k)
        return _case(op, model, n, rng.randint(1, hi), hi, seed, **more)
    if kind == "long":
        hi = _log(rng, 8192, 131072)
        return _case(op, model, rng.randint(1, 6), rng.randint(hi // 4, hi), hi, seed, **more)
    hi = _log(rng, least, 32768)
    return _case(op, model, rng.randint(1, 4), rng.randint(hi // 2, hi), hi, seed, rows=_log(rng, 2, 60),
                 **more)


# ---------------------------------------------------------------- inputs

def _lengths(case):
    """(tokens, new rows) of each request."""
    r = random.Random(case["lens_seed"])
    lens = [case["hi"]] + [r.randint(case["lo"], case["hi"]) for _ in range(case["requests"] - 1)]
    rows = [n if case["rows"] > n else max(1, round(case["rows"] * r.uniform(0.6, 1.0))) for n in lens]
    return lens, rows


def _generator(case, seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1_000_003 + case["lens_seed"] * 101 + stream) & 0x7FFFFFFFFFFF)
    return g


def _normal(shape, dtype, g, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    x.normal_(0.0, scale, generator=g)
    return x


def _i32(values):
    return torch.as_tensor(np.asarray(values, dtype=np.int32), device="cuda")


def _dtype(case):
    return torch.float32 if MODELS[case["model"]]["fmt"] == "f32" else torch.bfloat16


def _placement(case, seed, lens, spare):
    """Page table [slots, width] and the number of pages: the requests' pages
    scattered over a pool with `spare` others."""
    need = [(n + PAGE - 1) // PAGE for n in lens]
    total = sum(need)
    num_pages = total + spare
    r = np.random.default_rng((int(seed), case["lens_seed"]))
    ids = r.permutation(num_pages)[:total].astype(np.int32)
    return need, ids, num_pages, r


def _layout(case, seed, spare=8):
    lens, rows = _lengths(case)
    need, ids, num_pages, r = _placement(case, seed, lens, spare)
    table = np.full((len(lens) + 2, max(need) + 1), -1, dtype=np.int32)
    slots = r.permutation(len(lens) + 2)[:len(lens)]
    at = 0
    for s, n in zip(slots, need):
        table[s, :n] = ids[at:at + n]
        at += n
    row_slot = np.concatenate([np.full(t, s) for s, t in zip(slots, rows)] + [np.full(case["pad"], -1)])
    pos = np.concatenate([np.arange(n - t, n) for n, t in zip(lens, rows)] + [np.full(case["pad"], -1)])
    return table, row_slot.astype(np.int32), pos.astype(np.int32), num_pages


def _prepare_pages(case, seed):
    lens, _ = _lengths(case)
    n, pad = len(lens), case["pad"]
    grow = 0 if case["admit"] else GROW
    width = (max(lens) + grow + PAGE - 1) // PAGE
    need, ids, num_pages, r = _placement(case, seed, lens, n * (grow // PAGE + 1) + 200)
    free = np.ones(-(-num_pages // 32) * 32, dtype=bool)
    free[num_pages:] = False
    free[ids] = False
    slots = r.permutation(n + 4)[:n]
    table = np.full((n + 4, width), -1, dtype=np.int32)
    seq = np.zeros(n + 4, dtype=np.int32)
    at = 0
    for s, m, length in zip(slots, need, lens):
        table[s, :m] = ids[at:at + m]
        seq[s] = length
        at += m
    bits = np.packbits(free.reshape(-1, 32), axis=1, bitorder="little").view(np.int32).reshape(-1)
    # one element more than the table has, for the plain form's unused writes
    flat = torch.as_tensor(np.append(table.reshape(-1), np.int32(-1)), device="cuda")
    s = dict(case=case, slots=_i32(np.append(slots, [-1] * pad)),
             new=_i32((lens if case["admit"] else [1] * n) + [0] * pad), flat=flat,
             table=flat[:-1].view(n + 4, width), seq=_i32(seq), free=torch.as_tensor(bits, device="cuda"),
             num_pages=num_pages, rows=sum(lens) if case["admit"] else n + pad, max_seq=width * PAGE, left=grow)
    s["start"] = [s[k].clone() for k in ("flat", "seq", "free")]
    if own:
        from paper_2609_01068_amd.paged import PageTables
        s["pt"] = PageTables(num_pages, n + 4, s["max_seq"],
                             buffers=dict(page_table=s["table"], seq_len=s["seq"], free_bits=s["free"]))
    return s


def _kv(s, num_pages, width, **buffers):
    """The framework's cache over the case's memory."""
    from paper_2609_01068_amd.paged import PagedKV, PageTables
    m = MODELS[s["case"]["model"]]
    tables = PageTables(num_pages, s["table"].shape[0], width * PAGE, buffers=dict(page_table=s["table"]))
    return PagedKV(tables, m["n_kv"], m["hd"], m["fmt"], buffers=buffers)


def prepare(case, seed):
    if case["op"] == "pages":
        return _prepare_pages(case, seed)
    m, dt = MODELS[case["model"]], _dtype(case)
    n_q, n_kv, hd = m["n_q"], m["n_kv"], m["hd"]
    table, row_slot, pos, num_pages = _layout(case, seed)
    n, width = len(pos), table.shape[1]
    s = dict(case=case, table=torch.as_tensor(table, device="cuda"), row_slot=_i32(row_slot), pos=_i32(pos),
             num_pages=num_pages)
    if case["op"] == "write":
        # only the pages that the rows touch, renumbered: the rest of the pool does not matter
        live = pos >= 0
        page = table[np.maximum(row_slot, 0), np.maximum(pos, 0) // PAGE]
        used = np.unique(page[live])
        s["num_pages"] = num_pages = len(used) + 8
        where = np.random.default_rng((int(seed), 7)).permutation(num_pages)
        slot_map = where[np.searchsorted(used, page).clip(0, len(used) - 1)] * PAGE + pos % PAGE
        s["slot_map"] = _i32(np.where(live, slot_map, -1))
        # one page more than the pool has, for the plain form's unused writes
        s["k_all"] = _normal((num_pages + 1, n_kv, PAGE, hd), dt, _generator(case, seed, 1))
        s["v_all"] = _normal((num_pages + 1, n_kv, hd, PAGE), dt, _generator(case, seed, 2))
        s["key_all"] = _normal((num_pages + 1, n_kv, hd), dt, _generator(case, seed, 3), 0.25)
        s["k_pool"], s["v_pool"], s["keys"] = s["k_all"][:-1], s["v_all"][:-1], s["key_all"][:-1]
        # keys and values as a projection leaves them: columns of one wide row
        s["qkv"] = _normal((n, (n_q + 2 * n_kv) * hd), dt, _generator(case, seed, 4))
        s["k"] = s["qkv"][:, n_q * hd:(n_q + n_kv) * hd].view(n, n_kv, hd)
        s["v"] = s["qkv"][:, (n_q + n_kv) * hd:].view(n, n_kv, hd)
        s["fills"] = sum((t + PAGE - 1) // PAGE for t in _lengths(case)[1])     # pages that the rows can fill
        if own:
            s["kv"] = _kv(s, num_pages, width, k_pool=s["k_pool"], v_pool=s["v_pool"], block_keys=s["keys"])
        return s
    s["qkv"] = _normal((n, (n_q + 2 * n_kv + n_q) * hd), dt, _generator(case, seed, 4))
    s["q"] = s["qkv"][:, :n_q * hd].view(n, n_q, hd)
    if case["op"] == "select":
        s["keys"] = _normal((num_pages, n_kv, hd), dt, _generator(case, seed, 3), 0.25)
        if own:
            s["kv"] = _kv(s, num_pages, width, block_keys=s["keys"])
        return s
    s["gate"] = s["qkv"][:, (n_q + 2 * n_kv) * hd:].view(n, n_q, hd) if case["gate"] else None
    s["k_pool"] = _normal((num_pages, n_kv, PAGE, hd), dt, _generator(case, seed, 1))
    s["v_pool"] = _normal((num_pages, n_kv, hd, PAGE), dt, _generator(case, seed, 2))
    # selections: the first and the last pages, and others that the rows of a
    # request mostly share
    g = _generator(case, seed, 5)
    base = torch.rand((table.shape[0], n_kv, width), generator=g, device="cuda")
    score = base[s["row_slot"].clamp(min=0).long()]
    score += 0.1 * torch.rand(score.shape, generator=g, device="cuda")
    s["sel"] = _pick(case, s["pos"], score)
    if own:
        s["kv"] = _kv(s, num_pages, width, k_pool=s["k_pool"], v_pool=s["v_pool"])
    return s


# ---------------------------------------------------------------- the plain forms

def _pick(case, pos, score):
    """Pages of each row and KV head in ascending order, -1 behind them: all
    visible ones, or the first `sink`, the last `local` and those of the
    largest score (ties to the lowest index)."""
    k, sink, local = case["top_k"], case["sink"], case["local"]
    width = score.shape[-1]
    nb = torch.where(pos >= 0, pos // PAGE + 1, torch.zeros_like(pos))[:, None, None]
    idx = torch.arange(width, device=pos.device, dtype=torch.int32)
    fixed = (idx < sink) | (idx >= nb - local)
    score = score.masked_fill(fixed | (idx >= nb), -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :k - sink - local]
    chosen = torch.zeros(score.shape, dtype=torch.bool, device=pos.device)
    chosen.scatter_(-1, order, True)
    chosen = torch.where(nb <= k, torch.ones_like(chosen), chosen | fixed) & (idx < nb)
    out = torch.sort(torch.where(chosen, idx, torch.full_like(idx, 1 << 30)), dim=-1).values[..., :k]
    out = torch.where(out == 1 << 30, torch.full_like(out, -1), out)
    return torch.nn.functional.pad(out, (0, k - out.shape[-1]), value=-1).to(torch.int32).contiguous()


def _plain_release(s):
    live = s["slots"] >= 0
    slot = torch.where(live, s["slots"], torch.zeros_like(s["slots"])).long()
    width = s["table"].shape[1]
    held = s["table"][slot]
    mine = (held >= 0) & live[:, None]
    flags = _flags(s)
    spare = len(flags) - 1
    flags[torch.where(mine, held.long(), torch.full_like(held, spare).long())] = True
    _pack(s, flags)
    at = slot[:, None] * width + torch.arange(width, device=slot.device)
    s["flat"][torch.where(mine, at, torch.full_like(at, len(s["flat"]) - 1))] = -1
    hit = torch.zeros_like(s["seq"]).index_add_(0, slot, live.int())
    s["seq"].masked_fill_(hit > 0, 0)


def _flags(s):
    """The free bits as truth values, and one more for unused writes."""
    shift = torch.arange(32, device="cuda", dtype=torch.int32)
    bits = ((s["free"][:, None] >> shift) & 1).bool().reshape(-1)
    return torch.cat([bits, bits.new_zeros(1)])


def _pack(s, flags):
    shift = torch.arange(32, device="cuda", dtype=torch.int64)
    word = (flags[:-1].view(-1, 32).long() << shift).sum(dim=1)
    s["free"].copy_(torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32))


def _plain_append(s):
    slots, rows, width = s["slots"], s["rows"], s["table"].shape[1]
    live = slots >= 0
    slot = torch.where(live, slots, torch.zeros_like(slots)).long()
    t = torch.where(live, s["new"], torch.zeros_like(s["new"])).long()
    old = s["seq"][slot].long()
    have = (old + PAGE - 1) // PAGE
    need = (old + t + PAGE - 1) // PAGE - have
    cu, pages = torch.cumsum(t, 0), torch.cumsum(need, 0)
    flags = _flags(s)
    count = flags.sum()
    ids = torch.argsort((~flags[:-1]).to(torch.int8), stable=True)
    # the new pages, by rank
    cap = min(rows, len(ids))
    rank = torch.arange(cap, device="cuda")
    req = torch.searchsorted(pages, rank, right=True).clamp(max=len(slots) - 1)
    used = rank < pages[-1]
    at = slot[req] * width + have[req] + rank - (pages - need)[req]
    s["flat"][torch.where(used, at, torch.full_like(at, len(s["flat"]) - 1))] = torch.where(
        used, ids[:cap], torch.full_like(ids[:cap], -1)).to(torch.int32)
    flags[torch.where(used, ids[:cap], torch.full_like(ids[:cap], len(flags) - 1))] = False
    _pack(s, flags)
    s["seq"].index_add_(0, slot, t.to(torch.int32))
    # the rows
    r = torch.arange(rows, device="cuda")
    req = torch.searchsorted(cu, r, right=True).clamp(max=len(slots) - 1)
    there = r < cu[-1]
    pos = old[req] + r - (cu - t)[req]
    page = s["table"].reshape(-1)[torch.where(there, slot[req] * width + pos // PAGE, torch.zeros_like(pos))].long()
    none = torch.full_like(pos, -1)
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    status = torch.cat([zero, cu[-1:], pages[-1:], (count - pages[-1])[None]])
    return dict(cu=torch.cat([zero, cu]).int(), slot_map=torch.where(there, page * PAGE + pos % PAGE, none).int(),
                positions=torch.where(there, pos, none).int(),
                row_slot=torch.where(there, slot[req], none).int(), status=status.int())


def _plain_write(s):
    slot_map, dt = s["slot_map"].long(), s["k_all"].dtype
    n, spare = len(slot_map), s["num_pages"]
    live = slot_map >= 0
    page = torch.where(live, slot_map // PAGE, torch.full_like(slot_map, spare))
    off = torch.where(live, slot_map % PAGE, torch.zeros_like(slot_map))
    s["k_all"][page, :, off] = s["k"]
    s["v_all"][page, :, :, off] = s["v"]
    full = live & (off == PAGE - 1)
    pick = torch.argsort((~full).to(torch.int8), stable=True)[:s["fills"]]
    done = torch.where(full[pick], page[pick], torch.full_like(pick, spare))
    s["key_all"][done] = s["k_all"][done].double().mean(dim=2).to(dt)


def _plain_select(s):
    case, out = s["case"], []
    m = MODELS[case["model"]]
    n_kv, G, hd, width = m["n_kv"], m["n_q"] // m["n_kv"], m["hd"], s["table"].shape[1]
    step = max(1, (1 << 27) // (width * n_kv * hd))
    for a in range(0, len(s["pos"]), step):
        pos = s["pos"][a:a + step]
        ids = s["table"][s["row_slot"][a:a + step].clamp(min=0).long()].clamp(min=0).long()
        key = s["keys"][ids].permute(0, 2, 3, 1).double().contiguous()       # [rows, n_kv, hd, pages]
        q = s["q"][a:a + step].double().reshape(len(pos), n_kv, G, hd)
        out.append(_pick(case, pos, torch.matmul(q, key).amax(dim=2)))
    return torch.cat(out)


def _attend(s, dtype, limit):
    case = s["case"]
    m = MODELS[case["model"]]
    n_kv, G, hd, k = m["n_kv"], m["n_q"] // m["n_kv"], m["hd"], case["top_k"]
    head = torch.arange(n_kv, device="cuda")[None, :, None]
    step, out = max(1, limit // (n_kv * k * PAGE * hd)), []
    for a in range(0, len(s["pos"]), step):
        pos, sel = s["pos"][a:a + step], s["sel"][a:a + step]
        n = len(pos)
        row = s["table"][s["row_slot"][a:a + step].clamp(min=0).long()]
        page = torch.gather(row[:, None].expand(n, n_kv, -1), 2, sel.clamp(min=0).long()).clamp(min=0).long()
        key = s["k_pool"][page, head].to(dtype).reshape(n, n_kv, k * PAGE, hd)
        val = s["v_pool"][page, head].to(dtype).permute(0, 1, 2, 4, 3).reshape(n, n_kv, k * PAGE, hd)
        tok = sel[..., None] * PAGE + torch.arange(PAGE, device="cuda")
        live = ((sel[..., None] >= 0) & (tok <= pos[:, None, None, None])).reshape(n, n_kv, 1, k * PAGE)
        q = s["q"][a:a + step].to(dtype).reshape(n, n_kv, G, hd)
        x = torch.matmul(q, key.transpose(2, 3).contiguous()) / math.sqrt(hd)
        x = x.masked_fill(~live, -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = p.sum(dim=-1, keepdim=True)
        o = torch.matmul(p, val) / torch.where(total == 0, torch.ones_like(total), total)
        o = o.reshape(n, n_kv * G, hd)
        if s["gate"] is not None:
            o = o / (1 + torch.exp(-s["gate"][a:a + step].to(dtype)))
        out.append(o)
    return torch.cat(out)


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if op == "pages":
        if not s["case"]["admit"]:
            if s["left"] == 0:          # the batch has grown to its end: it starts over
                for k, v in zip(("flat", "seq", "free"), s["start"]):
                    s[k].copy_(v)
                s["left"] = GROW
            s["left"] -= 1
        if own:
            if s["case"]["admit"]:
                s["pt"].release(s["slots"])
            r = s["pt"].append(s["slots"], s["new"], s["rows"])
            out = dict(cu=r.cu, slot_map=r.slot_map, positions=r.positions, row_slot=r.row_slot, status=r.status)
        else:
            if s["case"]["admit"]:
                _plain_release(s)
            out = _plain_append(s)
        return dict(out, page_table=s["table"], seq_len=s["seq"], free_bits=s["free"])
    if op == "write":
        if own:
            s["kv"].write(s["slot_map"], s["k"], s["v"])
        else:
            _plain_write(s)
        return dict(k_pool=s["k_pool"], v_pool=s["v_pool"], block_keys=s["keys"])
    if op == "select":
        c = s["case"]
        if own:
            return s["kv"].select(s["q"], s["row_slot"], s["pos"], c["top_k"], c["sink"], c["local"])
        return _plain_select(s)
    if own:
        return s["kv"].attend(s["q"], s["row_slot"], s["pos"], s["sel"], gate=s["gate"])
    return _attend(s, torch.float32, 1 << 28).to(s["q"].dtype)


# ---------------------------------------------------------------- work

def work(case):
    m = MODELS[case["model"]]
    n_q, n_kv, hd = m["n_q"], m["n_kv"], m["hd"]
    eb = 4 if m["fmt"] == "f32" else 2
    lens, rows = _lengths(case)
    n, pad = len(lens), case["pad"]
    if case["op"] == "pages":
        new = lens if case["admit"] else [1] * n
        T = sum(new)
        old = [0 if case["admit"] else x for x in lens]
        fresh = sum((o + t + PAGE - 1) // PAGE - (o + PAGE - 1) // PAGE for o, t in zip(old, new))
        given = sum((x + PAGE - 1) // PAGE for x in lens) if case["admit"] else 0
        pages = sum((x + PAGE - 1) // PAGE for x in lens) + n * ((0 if case["admit"] else GROW) // PAGE + 1) + 200
        return {"bytes": 4 * (2 * (n + pad) + 2 * n + 3 * (T + pad) + fresh + 2 * given) + pages // 4,
                "flops": 8 * T + pages // 8}
    T = sum(rows)
    if case["op"] == "write":
        full = sum(x // PAGE - (x - t) // PAGE for x, t in zip(lens, rows))
        part = sum((x - t) % PAGE if x // PAGE > (x - t) // PAGE else 0 for x, t in zip(lens, rows))
        return {"bytes": (4 * T + part + full) * n_kv * hd * eb + 4 * (T + pad), "flops": full * PAGE * n_kv * hd}
    k, edge = case["top_k"], case["sink"] + case["local"]
    seen = scored = picked = read = 0
    for x, t in zip(lens, rows):
        nb = [p // PAGE + 1 for p in range(x - t, x)]
        mid = [b - edge if b > k else 0 for b in nb]
        scored += sum(mid)
        seen += max(mid)
        picked += sum(min(b, k) for b in nb)
        read += min(sum(min(b, k) for b in nb), nb[-1])
    if case["op"] == "select":
        return {"bytes": seen * n_kv * hd * eb + T * n_q * hd * eb + 4 * (T + pad) * (n_kv * k + 2) + 4 * seen,
                "flops": max(1, 2 * scored * n_q * hd)}
    cols = T * n_q * hd * eb * (3 if case["gate"] else 2)
    return {"bytes": read * n_kv * 2 * PAGE * hd * eb + cols + 4 * (T + pad) * (n_kv * k + 2) + 4 * read,
            "flops": 4 * picked * PAGE * n_q * hd}


# ---------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    """Block keys from the mean of each filled page, attention request by
    request; tables and selections are whole numbers and have none."""
    if case["op"] in ("pages", "select"):
        return None
    s = prepare(case, seed)
    m = MODELS[case["model"]]
    n_kv, hd, G = m["n_kv"], m["hd"], m["n_q"] // m["n_kv"]
    if case["op"] == "write":
        keys = s["keys"].double()
        slot_map = s["slot_map"].cpu().numpy()
        rows = np.flatnonzero(slot_map >= 0)
        at = torch.as_tensor(slot_map[rows], device="cuda").long()
        flat = s["k_pool"].double().transpose(1, 2).reshape(-1, n_kv, hd)       # one row a token
        flat[at] = s["k"][torch.as_tensor(rows, device="cuda")].double()
        done = torch.as_tensor(np.unique(slot_map[rows][slot_map[rows] % PAGE == PAGE - 1] // PAGE), device="cuda")
        if len(done):
            keys[done] = flat.view(-1, PAGE, n_kv, hd)[done].sum(dim=1) / PAGE
        return dict(k_pool=None, v_pool=None, block_keys=keys)
    out = torch.zeros((len(s["pos"]), m["n_q"], hd), dtype=torch.float64, device="cuda")
    pos, slot = s["pos"].tolist(), s["row_slot"].tolist()
    offs = torch.arange(PAGE, device="cuda")
    for r in range(len(pos)):
        if slot[r] < 0:
            continue
        row = s["table"][slot[r]].long()
        for h in range(n_kv):
            sel = s["sel"][r, h].long()
            tok = (sel[:, None] * PAGE + offs).reshape(-1)
            ok = ((sel >= 0)[:, None].expand(-1, PAGE).reshape(-1)) & (tok <= pos[r])
            page = row[sel.clamp(min=0)].clamp(min=0)
            key = s["k_pool"][page, h].double().reshape(-1, hd)
            val = s["v_pool"][page, h].double().transpose(1, 2).reshape(-1, hd)
            x = key @ s["q"][r, h * G:(h + 1) * G].double().T.contiguous() / hd ** 0.5
            x[~ok] = -math.inf
            w = torch.softmax(x, dim=0)
            out[r, h * G:(h + 1) * G] = (w[:, :, None] * val[:, None, :]).sum(dim=0)
    if s["gate"] is not None:
        out *= torch.sigmoid(s["gate"].double())
    return out
