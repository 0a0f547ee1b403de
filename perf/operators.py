"""The operators of the paged cache: their cases, inputs, plain forms and work.

A paged cache holds the K and V rows of S sequence slots in a pool of pages,
[n_pages][H][page][d] each.  table[s][j] is the page of rows [j * page, (j + 1) * page)
of slot s, length[s] its number of rows, ref[p] how many table entries name page p
(0: free).  Where `own` is true the operators are `paper_2606_03928_amd.pages`'s.

Kinds (`case["kind"]`):

  attn     attention of each slot's newest rows (a token of decoding, a chunk of a
           prompt) over the slot's pages, causal or not, with the rows' log-sum-exp
  write    the new K and V rows of a step into the last rows of their slots
  resize   slots truncated and grown: pages freed, taken, and copied where a slot
           grows within a page that it shares
  fork     slots that begin as another's rows, on the same pages
  compact  the survivors of an eviction round to the front of their slot's pages, the
           rest of the pages freed; shared pages are left to those who share them

A case's lengths follow from the case alone; values and page numbers from the seed.
Sizes are those of `synth.CONFIGS`: 8 KV heads of d = 128 (2 of 64 in the smallest), 2
to 8 query heads to each, caches of K + B rows for K = 128 to 8192.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SINKS, SINK_SCALE = 4, 10.0
OUTLIER_P, OUTLIER_LO, OUTLIER_HI = 0.005, 20.0, 100.0


def listed():
    return [
        # the smallest workload: two fp32 heads, a few tokens of three short sequences;
        # bound by launches
        dict(name="attn-tiny", kind="attn", dtype="f32", S=3, H=2, G=2, d=64, page=16, lo=100, hi=160,
             new=20, mix=2, causal=True, lse=True, pad=0),
        # a decode step of one layer of a 32B model at batch 64, full caches among part-filled ones
        dict(name="attn-decode-32b", kind="attn", dtype="bf16", S=64, H=8, G=8, d=128, page=64, lo=2000,
             hi=8320, new=1, mix=1, causal=True, lse=False, pad=0),
        # a mixed step of one layer of an 8B model: two prompt chunks among single tokens,
        # an idle slot, a batch padded at its end
        dict(name="attn-mixed-8b", kind="attn", dtype="bf16", S=16, H=8, G=4, d=128, page=32, lo=600,
             hi=4224, new=512, mix=8, causal=True, lse=True, pad=7),
        # a prompt chunk of 2048 tokens for each of four sequences, one layer of a 14B model
        dict(name="attn-prefill-14b", kind="attn", dtype="bf16", S=4, H=8, G=5, d=128, page=128, lo=4096,
             hi=8448, new=2048, mix=1, causal=True, lse=False, pad=0),
        # the rows of a decode step of one layer at batch 64
        dict(name="write-step", kind="write", dtype="bf16", S=64, H=8, d=128, page=64, lo=300, hi=4224,
             new=1, mix=1),
        # the rows of prompt chunks, fp32, chunks that begin and end inside pages
        dict(name="write-chunk-f32", kind="write", dtype="f32", S=9, H=8, d=128, page=16, lo=1300,
             hi=4224, new=1000, mix=1),
        # drafted tokens dropped, room for the next draft: 256 slots of one layer's cache
        dict(name="resize-draft", kind="resize", dtype="bf16", S=256, H=8, d=128, page=16, lo=500,
             hi=2176, more=5, samples=0),
        # eight samples of each of eight prompts, eight layers: forked, and each one's last
        # page copied as it grows
        dict(name="resize-samples", kind="resize", dtype="bf16", S=72, H=64, d=128, page=32, lo=700,
             hi=2176, more=40, samples=8),
        # beams of one request: half of the hypotheses leave, the others are forked
        dict(name="fork-beam", kind="fork", dtype="bf16", S=16, H=8, d=128, page=16, lo=400, hi=2176,
             samples=1),
        # a large batch in which three samples share each prompt
        dict(name="fork-batch", kind="fork", dtype="bf16", S=1024, H=1, d=64, page=16, lo=500, hi=8192,
             samples=3),
        # samples of one prompt, one layer, each evicted by its own map: every page is shared
        dict(name="compact-samples", kind="compact", dtype="bf16", S=5, H=8, d=128, page=64, K=2048,
             B=128, samples=4),
        # an eviction round of an 8B model at batch 8, every layer: the period's rows
        # written, then the survivors moved in place
        dict(name="compact-8b", kind="compact", dtype="bf16", S=8, H=288, d=128, page=64, K=4096, B=128,
             samples=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "write", "resize", "fork", "compact", "compact"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    e = 2 if dtype == "bf16" else 4
    d = rng.choice([64, 128, 128])
    H = rng.choice([1, 2, 4, 8, 8])
    page = rng.choice([16, 32, 64, 128, 48, 176])
    S = _log_int(rng, 1, 64)
    hi = _log_int(rng, 40, 8448)
    lo = rng.randint(1, hi)
    case = dict(kind=kind, dtype=dtype, S=S, H=H, d=d, page=page, lo=lo, hi=hi)
    if kind == "attn":
        G = rng.randint(1, 8)
        new = rng.choice([1, 1, 2, min(hi, _log_int(rng, 3, 2048)), min(hi, _log_int(rng, 3, 2048))])
        mix = rng.choice([1, 1, 2, 5])
        # below the largest listed cases: bytes of the cache, products (fp32 ones take the
        # fp32 units), and the plain form's padded score matrix
        S = min(S, int(1.2e9 / (2 * H * hi * d * e)))
        S = min(S, int((6e11 if e == 2 else 4e10) / (4.0 * new * G * H * hi * d)))
        S = min(S, int(8e9 / (4.0 * new * G * H * hi)))
        case.update(S=max(S, 1), G=G, new=new, mix=mix, causal=rng.random() < 0.8, lse=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 1, 13]))
    elif kind == "write":
        new = rng.choice([1, min(hi, _log_int(rng, 2, 1000))])
        case.update(new=new, mix=rng.choice([1, 2, 5]))
    elif kind == "resize":
        samples = rng.choice([0, 0, 2, 4])
        S = _log_int(rng, 1, 256)
        S = max(S, 1 + samples)
        S = max(1 + samples, min(S, int(1e9 / (H * hi * d * e))))
        case.update(S=S, more=_log_int(rng, 1, 300), samples=samples)
    elif kind == "fork":
        samples = rng.choice([1, 2, 7])
        S = max(_log_int(rng, 2, 1024), 1 + samples)
        case.update(S=S, H=1, d=64, samples=samples)
    else:
        K = _log_int(rng, 32, 8192)
        B = min(_log_int(rng, 1, 256), K)
        samples = rng.choice([0, 0, 3])
        S = max(1 + samples, min(rng.randint(1, 16), int(6e8 / (H * (K + B) * d * e))))
        H = H * rng.choice([1, 1, 4]) if S * H * 4 * (K + B) * d * e < 6e8 else H
        for name in ("lo", "hi"):
            del case[name]
        case.update(S=S, H=H, K=K, B=B, samples=samples)
    return case


# --- the lengths of a case, on the host -------------------------------------------------


def _spread(n, lo, hi, phase):
    """n whole numbers spread evenly over [lo, hi], in no order."""
    return [lo + int((phase + i * 0.6180339887) % 1.0 * (hi - lo + 1)) for i in range(n)]


def _parents(case):
    """The slot that each slot is forked from (-1: none): slots [0, r) are prompts."""
    S, samples = case["S"], case.get("samples", 0)
    if not samples:
        return [-1] * S
    r = max(1, S // (1 + samples))
    return [-1] * r + [(s - r) % r for s in range(r, S)]


def _lengths(case):
    """Rows that the slots hold before the pass."""
    S = case["S"]
    if case["kind"] == "compact":
        N = case["K"] + case["B"]
        return [0 if p >= 0 else (N if case["samples"] else case["K"]) for p in _parents(case)]
    got = _spread(S, case["lo"], case["hi"], 0.37)
    got[0] = case["hi"]
    return [0 if p >= 0 else n for p, n in zip(_parents(case), got)]


def _new(case):
    """New rows of each slot: `new` for every mix-th one and 1 for the others, none for every 11th."""
    if case["kind"] == "compact":
        return [0 if case["samples"] else case["B"]] * case["S"]
    got = [case["new"] if i % case["mix"] == 0 else 1 for i in range(case["S"])]
    if case["new"] > 1:
        got = [0 if i % 11 == 10 else n for i, n in enumerate(got)]
        got = [min(n, length) for n, length in zip(got, _lengths(case))]
    return got


def _target(case):
    """Rows that resize leaves to each slot."""
    length, parent = _lengths(case), _parents(case)
    if case["kind"] == "compact":
        return [-1 if case["samples"] else case["K"] + case["B"]] * case["S"]
    if case["samples"]:
        return [-1 if p < 0 else length[p] + case["more"] for p in parent]
    return [n + 1 + (i * 7) % case["more"] for i, n in enumerate(length)]


# --- inputs -----------------------------------------------------------------------------


def _inputs(case, seed):
    kind, S, H, d, page = (case[x] for x in ("kind", "S", "H", "d", "page"))
    dt = DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    host = random.Random(int(seed))

    def normal(shape, fix=None):
        out = torch.empty(shape, dtype=dt, device="cuda")
        step = max(1, (1 << 27) // max(1, math.prod(shape[1:])))
        for i in range(0, shape[0], step):
            t = torch.randn((min(step, shape[0] - i),) + tuple(shape[1:]), generator=gen, device="cuda")
            out[i:i + step] = fix(t) if fix else t
        return out

    def outliers(t):
        u = torch.rand(t.shape[:-1] + (1,), generator=gen, device="cuda")
        size = OUTLIER_LO * (OUTLIER_HI / OUTLIER_LO) ** (u / OUTLIER_P)
        return t * torch.where(u < OUTLIER_P, size, torch.ones_like(u))

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    length, parent = _lengths(case), _parents(case)
    most = max(length)
    if kind in ("resize", "compact"):
        most = max([most] + _target(case))
    M = -(-most // page) + 1
    used = [-(-n // page) for n in length]
    n_pages = sum(used) + 8
    if kind == "resize":
        n_pages += sum(max(0, -(-t // page) - u) + 1 for t, u in zip(_target(case), used))
    elif kind == "compact":
        grown = -(-(case["K"] + case["B"]) // page)
        n_pages += S * grown if case["samples"] else S * (grown - used[0])
    # a pool in use: a slot's pages lie anywhere in it
    order = list(range(n_pages))
    host.shuffle(order)
    table, ref = [[-1] * M for _ in range(S)], [0] * n_pages
    for s in range(S):
        for j in range(used[s]):
            table[s][j] = order.pop()
            ref[table[s][j]] = 1
    k, v = normal((n_pages, H, page, d)), normal((n_pages, H, page, d), outliers)
    first = ints([row[0] for row, n in zip(table, length) if n]).long()
    k[first, :, :SINKS] *= SINK_SCALE
    x = dict(k=k, v=v, ref=ints(ref), table=ints(table), length=ints(length))
    if kind in ("attn", "write", "compact"):
        new = _new(case)
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        x["cu"] = ints(cu)
        T = cu[-1] + case.get("pad", 0)
        # a step's queries and rows are parts of one projection's output
        G = case.get("G", 0)
        rows = normal((max(T, 1), H * (G + 2), d))
        if kind == "attn":
            x["q"] = rows[:, :H * G]
        else:
            x["k_new"], x["v_new"] = rows[:, H * G:H * (G + 1)], rows[:, H * (G + 1):]
    if kind in ("resize", "fork") or (kind == "compact" and case["samples"]):
        # drop the forks of the pass before; prompts keep their rows
        x["drop"] = ints([0 if p >= 0 else n if kind == "resize" and not case["samples"] else -1
                          for p, n in zip(parent, length)])
        x["parent"] = ints(parent)
    if kind in ("resize", "compact"):
        x["target"] = ints(_target(case))
    if kind == "compact":
        K, B, N = case["K"], case["B"], case["K"] + case["B"]
        live = [s for s in range(S) if not case["samples"] or parent[s] >= 0]
        x["map"] = ints([live.index(s) if s in live else -1 for s in range(S)])
        r = torch.rand((len(live), H, K), generator=gen, device="cuda")
        kept = torch.argsort(r, -1)[..., :K - B].sort(-1).values
        tail = torch.arange(K, N, device="cuda").expand(len(live), H, B)
        x["src"] = torch.cat([kept, tail], -1).int()
    return x


def prepare(case, seed):
    s = dict(case=case, x=_inputs(case, seed))
    x = s["x"]
    if case["kind"] == "attn":
        T, HG = x["q"].shape[0], case["H"] * case["G"]
        s["out"] = torch.zeros((T, HG, case["d"]), dtype=x["q"].dtype, device="cuda")
        s["lse"] = torch.zeros((T, HG), device="cuda") if case["lse"] else None
        s["max_len"], s["max_new"] = max(_lengths(case)), max(_new(case))
    return s


def run(s):
    if own:
        return _run_own(s)
    case, x, kind = s["case"], s["x"], s["case"]["kind"]
    if kind == "attn":
        _attn(s)
        return dict(out=s["out"], lse=s["lse"])
    if kind == "write":
        _write(x)
        return dict(k=x["k"], v=x["v"])
    if kind == "resize":
        _resize(x, x["drop"])
        if case["samples"]:
            _fork(x, x["parent"])
        _resize(x, x["target"])
        return _state(x)
    if kind == "fork":
        _resize(x, x["drop"])
        _fork(x, x["parent"])
        return dict(ref=x["ref"], table=x["table"], length=x["length"])
    if case["samples"]:
        _resize(x, x["drop"])
        _fork(x, x["parent"])
    else:
        _resize(x, x["target"])
        _write(x)
    _compact(x, case["K"])
    return _state(x)


def _run_own(s):
    from paper_2606_03928_amd import pages

    case, x, kind = s["case"], s["x"], s["case"]["kind"]
    c = s.get("cache")
    if c is None:
        c = s["cache"] = pages.PageCache(x["k"], x["v"], x["ref"], x["table"], x["length"])
    if kind == "attn":
        c.attn(x["q"], x["cu"], max_new=s["max_new"], max_len=s["max_len"], causal=case["causal"],
               out=s["out"], lse=s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if kind == "write":
        c.write(x["k_new"], x["v_new"], x["cu"])
        return dict(k=x["k"], v=x["v"])
    if kind == "resize":
        c.resize(x["drop"])
        if case["samples"]:
            c.fork(x["parent"])
        c.resize(x["target"])
        return _state(x)
    if kind == "fork":
        c.resize(x["drop"])
        c.fork(x["parent"])
        return dict(ref=x["ref"], table=x["table"], length=x["length"])
    if case["samples"]:
        c.resize(x["drop"])
        c.fork(x["parent"])
    else:
        c.resize(x["target"])
        c.write(x["k_new"], x["v_new"], x["cu"])
    c.compact(x["map"], x["src"])
    return _state(x)


def _state(x):
    return {n: x[n] for n in ("k", "v", "ref", "table", "length")}


# --- the plain forms ----------------------------------------------------------------------


def _token_slots(cu, T):
    """For each token its slot, its place in the slot's chunk, and whether it has one."""
    t = torch.arange(T, device="cuda")
    slot = torch.searchsorted(cu[1:].contiguous(), t.int(), right=True)
    ok = slot < cu.numel() - 1
    slot = torch.where(ok, slot, 0)
    return slot, t - cu.long()[slot], ok


def _attn(s):
    """softmax(q k^T / sqrt(d)) v over each slot's rows, the slots padded to one length."""
    case, x = s["case"], s["x"]
    S, H, G, d, page = (case[n] for n in ("S", "H", "G", "d", "page"))
    L, n_max = s["max_len"], s["max_new"]
    pages = x["table"][:, :-(-L // page)].long().clamp(min=0)

    def rows(pool):
        return pool[pages].permute(0, 2, 1, 3, 4).reshape(S, H, -1, d)[:, :, :L].float()

    cu, length, T = x["cu"].long(), x["length"].long(), x["q"].shape[0]
    n = cu[1:] - cu[:-1]
    i = torch.arange(n_max, device="cuda")
    q = x["q"][(cu[:-1, None] + i).clamp(max=T - 1)].float()
    q = q.view(S, n_max, H, G, d).permute(0, 2, 1, 3, 4).reshape(S * H, n_max * G, d)
    scores = torch.bmm(q, rows(x["k"]).reshape(S * H, L, d).transpose(1, 2).contiguous())
    scores = (scores / math.sqrt(d)).view(S, H, n_max, G, L)
    j = torch.arange(L, device="cuda")
    seen = (j < length[:, None]).view(S, 1, 1, 1, L)
    if case["causal"]:
        seen = seen & (j <= (length - n)[:, None, None] + i[:, None]).view(S, 1, n_max, 1, L)
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(S * H, n_max * G, L), rows(x["v"]).reshape(S * H, L, d))
    o = torch.where(total > 0, o.view(S, H, n_max, G, d) / total, 0.0)
    slot, at, ok = _token_slots(x["cu"], T)
    o = o.permute(0, 2, 1, 3, 4)[slot, at.clamp(0, n_max - 1)].reshape(T, H * G, d)
    s["out"].copy_(torch.where(ok[:, None, None], o.to(s["out"].dtype), s["out"]))
    if s["lse"] is not None:
        lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3)
        lse = lse[slot, at.clamp(0, n_max - 1)].reshape(T, H * G)
        s["lse"].copy_(torch.where(ok[:, None], lse, s["lse"]))


def _write(x):
    """Row i of a slot's n new ones is its row length - n + i."""
    T, page = x["k_new"].shape[0], x["k"].shape[2]
    slot, at, ok = _token_slots(x["cu"], T)
    cu, length = x["cu"].long(), x["length"].long()
    row = length[slot] - (cu[slot + 1] - cu[slot]) + at
    p = x["table"].long()[slot, row // page]
    x["k"][p, :, row % page] = x["k_new"]
    x["v"][p, :, row % page] = x["v_new"]


def _take_pages(x, need):
    """The lowest free pages, need[i] of them for entry i, in order: each entry's place in them."""
    free = (x["ref"] == 0).long()
    at = torch.cumsum(free, 0) - 1
    n = x["ref"].numel()
    every = torch.full((n + 1,), -1, dtype=torch.long, device="cuda")
    every.scatter_(0, torch.where(free > 0, at, n), torch.arange(n, device="cuda"))
    return every[:n], torch.cumsum(need, 0) - need


def _count(x, table, sign):
    """sign for each entry >= 0 of `table`, on the page's count."""
    n = x["ref"].numel()
    add = torch.zeros(2 * n, dtype=torch.int32, device="cuda")
    # the other entries fall behind the counts, spread so that they do not all meet in one
    other = n + torch.arange(table.numel(), device="cuda") % n
    at = torch.where(table.reshape(-1) >= 0, table.reshape(-1).long(), other)
    add.index_add_(0, at, torch.full_like(at, sign, dtype=torch.int32))
    return add[:n]


def _resize(x, target):
    page, M = x["k"].shape[2], x["table"].shape[1]
    length, table, ref = x["length"].long(), x["table"].long(), x["ref"]
    target = torch.where(target < 0, length, target.long())
    old, new = (length + page - 1) // page, (target + page - 1) // page
    last = table.gather(1, (old - 1).clamp(min=0)[:, None])[:, 0]
    grows = target > length
    copied = grows & (length % page > 0) & (ref[last.clamp(min=0)] > 1)
    begin = old - copied.long()
    need = torch.where(grows, new - begin, 0)
    free, at = _take_pages(x, need)
    j = torch.arange(M, device="cuda")[None]
    fresh = grows[:, None] & (j >= begin[:, None]) & (j < new[:, None])
    dropped = (j >= new[:, None]) & (j < old[:, None])
    took = torch.where(fresh, free[torch.where(fresh, at[:, None] + j - begin[:, None], 0)], -1)
    left = torch.where(copied, last, -1)
    x["ref"] += _count(x, took, 1) + _count(x, torch.where(dropped, table, -1), -1) + _count(x, left, -1)
    slots = copied.nonzero()[:, 0]
    if slots.numel():
        to = took[slots, begin[slots]]
        rows = (torch.arange(page, device="cuda") < (length[slots] % page)[:, None])[:, None, :, None]
        for pool in (x["k"], x["v"]):
            pool[to] = torch.where(rows, pool[last[slots]], pool[to])
    x["table"].copy_(torch.where(fresh, took, torch.where(dropped, -1, table)))
    x["length"].copy_(target)


def _fork(x, parent):
    page, M = x["k"].shape[2], x["table"].shape[1]
    forked, p = parent >= 0, parent.long().clamp(min=0)
    used = (x["length"][p] + page - 1) // page
    takes = forked[:, None] & (torch.arange(M, device="cuda")[None] < used[:, None])
    table = torch.where(takes, x["table"][p], x["table"])
    x["ref"] += _count(x, torch.where(takes, table, -1), 1)
    x["length"].copy_(torch.where(forked, x["length"][p], x["length"]))
    x["table"].copy_(table)


def _compact(x, K):
    page, M, H = x["k"].shape[2], x["table"].shape[1], x["k"].shape[1]
    table, ref = x["table"].long(), x["ref"]
    live = x["map"] >= 0
    old, new = (x["length"].long() + page - 1) // page, (K + page - 1) // page
    j = torch.arange(M, device="cuda")[None]
    fresh = live[:, None] & (j < new) & (ref[table.clamp(min=0)] > 1)
    free, at = _take_pages(x, fresh.long().reshape(-1))
    took = torch.where(fresh, free[torch.where(fresh, at.view(fresh.shape), 0)], -1)
    left = live[:, None] & (j >= new) & (j < old[:, None])
    x["ref"] += _count(x, took, 1) + _count(x, torch.where(left | fresh, table, -1), -1)
    to = torch.where(fresh, took, table)
    # row src[map[s]][h][i] of slot s to its row i, every row read before the first is written
    slots = live.nonzero()[:, 0]
    src = x["src"].long()[x["map"].long()[slots]]
    head = torch.arange(H, device="cuda")[None, :, None]
    page_of = table[slots].gather(1, (src // page).view(slots.numel(), -1)).view(src.shape)
    i = torch.arange(K, device="cuda")
    to_page = to[slots][:, i // page][:, None, :].expand(src.shape)
    for pool in (x["k"], x["v"]):
        pool[to_page, head, (i % page).expand(src.shape)] = pool[page_of, head, src % page]
    x["table"].copy_(torch.where(left, -1, to))
    x["length"].copy_(torch.where(live, K, x["length"]))


# --- work and exact values ------------------------------------------------------------------


def work(case):
    """Every input read once, every output written once, every product formed once."""
    kind, S, H, d, page = (case[x] for x in ("kind", "S", "H", "d", "page"))
    e = 2 if case["dtype"] == "bf16" else 4
    length, parent = _lengths(case), _parents(case)
    row, fl = H * d * e, 0.0

    def used(n):
        return -(-n // page)

    if kind == "attn":
        G, by = case["G"], 0.0
        for n, m in zip(length, _new(case)):
            if m:
                by += 2 * n * row + 2 * m * G * row + 4 * used(n)
                pairs = m * n - (m * (m - 1) / 2 if case["causal"] else 0)
                fl += 4.0 * pairs * H * G * d
            by += 4 * m * H * G * case["lse"]
    elif kind == "write":
        by = 4.0 * sum(_new(case)) * row
    else:
        # bookkeeping: lengths and the entries that change, with their counts
        target = [0] * S if kind == "fork" else _target(case)
        base = [length[p] if p >= 0 else n for p, n in zip(parent, length)]
        by = 12.0 * S
        for p, n in zip(parent, base):
            by += 2 * 12.0 * used(n) if p >= 0 else 0.0      # dropped, then forked
        if kind == "resize":
            for p, n, t in zip(parent, base, target):
                by += 2 * 12.0 * max(0, used(t) - used(n)) if t > n else 0.0
                if p >= 0 and n % page:
                    by += 4.0 * (n % page) * row
        if kind == "compact":
            for p in parent:
                if p >= 0 or not case["samples"]:
                    by += 4.0 * case["K"] * row + 4.0 * case["K"] * H
                    by += 0.0 if case["samples"] else 4.0 * case["B"] * row
    return {"bytes": float(by), "flops": float(fl)}


def exact(case, seed):
    """Attention in 64 bits, one slot at a time; the other kinds move rows and count."""
    if case["kind"] != "attn":
        return None
    x = _inputs(case, seed)
    H, G, d, page = (case[n] for n in ("H", "G", "d", "page"))
    T = x["q"].shape[0]
    out = torch.zeros((T, H, G, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((T, H, G), dtype=torch.float64, device="cuda")
    begin = 0
    for s, (n, m) in enumerate(zip(_lengths(case), _new(case))):
        if m == 0:
            continue
        ids = x["table"][s, :-(-n // page)].long()
        for h in range(H):
            k = x["k"][ids, h].reshape(-1, d)[:n].double()
            v = x["v"][ids, h].reshape(-1, d)[:n].double()
            for a in range(0, m, 512):
                b = min(m, a + 512)
                q = x["q"][begin + a:begin + b, h * G:(h + 1) * G].double().reshape(-1, d)
                z = torch.mm(q, k.t().contiguous()).view(b - a, G, n) / math.sqrt(d)
                if case["causal"]:
                    late = torch.arange(n, device="cuda")[None] > torch.arange(a, b, device="cuda")[:, None] + n - m
                    z.masked_fill_(late[:, None], -math.inf)
                w = torch.logsumexp(z, -1)
                lse[begin + a:begin + b, h] = w
                out[begin + a:begin + b, h] = torch.mm((z - w[..., None]).exp_().view(-1, n), v).view(b - a, G, d)
        begin += m
    return dict(out=out.view(T, H * G, d), lse=lse.view(T, H * G) if case["lse"] else None)
