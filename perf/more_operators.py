"""More operators of a cache in use, as a serving program has their work done: the cases that their speed is judged by.

Operators (paper_2605_01708_amd.cache_*)
  allot      from the requests' row counts: lengths, starts, pages out of a free list and back into it, block tables, and for every
             row its slot, its sequence and its position
  append     a step's projections: norms of the heads of Q and K, rotation by position, K and V into the cache, Q for attention
  write      new tokens' K and V into a cache of 4-bit words (E2M1, a power of two for each 32 elements), and back out of it, as
             a prompt in pieces has them: what comes back is what attention will see
  read       a sequence's tokens out of a cache of 4-bit words, as BF16
  attention  the rows of this step against a cache of 4-bit words

Fields of a case
  op                     which operator
  dtype                  the cache's words: "fp4"; append also "bf16" and "e4m3"
  seqs, longest, shortest, rows
                         sequences of the call; their lengths (spread evenly between the two, this call's rows included; allot: in front
                         of this call's rows); rows per sequence (0: every cached token; allot: the most of a sequence, fewer in others)
  kv_heads, group, dim   heads of the cache, query heads per head of the cache, elements of a head
  page                   tokens per page
  tree                   branches per node of the drafted tree, 0: a chain of tokens
  softcap, slopes, window
                         options of the scores: the cap, whether there is a bias by distance, how far back a row looks (0: all)
  rotary, interleaved, norm
                         append: elements of a head that rotate; whether pairs are neighbours or half of `rotary` apart; whether heads are normed
  given_back             allot: whether all pages are given back first, in a call of their own (requests leave, others come), or the
                         step keeps what is cached (the rejected drafts of the step before are dropped, this step's get their places)
"""
import math
import random

import torch

own = False   # the plain form, or the framework's kernels

MOST_TOKENS = 64 * 12000             # cached tokens x heads of the cache x elements / 1024, at most
MOST_SCORES = 16 * 64 * 8192 * 32    # rows x query heads x keys, padded to the longest sequence, at most
MOST_APPENDED = 16384 * 48 * 128     # rows x heads of Q, K and V x elements, at most
MOST_ALLOTTED = 262144               # rows of a call that allots
GROUP = 32                           # elements that share a power of two
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, op, dtype, seqs, longest, shortest, rows, kv_heads=8, group=4, dim=128, page=16, tree=0, softcap=0.0, slopes=False,
          window=0, rotary=0, interleaved=False, norm=False, given_back=False):
    c = {"op": op, "dtype": dtype, "seqs": seqs, "longest": longest, "shortest": shortest, "rows": rows, "kv_heads": kv_heads,
         "group": group, "dim": dim, "page": page, "tree": tree, "softcap": softcap, "slopes": slopes, "window": window,
         "rotary": rotary, "interleaved": interleaved, "norm": norm, "given_back": given_back}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a verifying step of 48 sequences: the last step's drafts are dropped, up to 5 new ones of each get their places
        _case("allot_step", "allot", "fp4", 48, 4001, 130, 5),
        # 1000 requests leave, and as many prompts of up to 500 tokens come in
        _case("allot_prompts", "allot", "fp4", 1000, 0, 0, 500, given_back=True),
        # a decoding step's projections, one token for each of 64 sequences
        _case("append_step", "append", "fp4", 64, 8192, 700, 1, rotary=128, norm=True),
        # a prompt's, of 16384 tokens, into an FP8 cache
        _case("append_prompt", "append", "e4m3", 1, 16384, 16384, 0, rotary=128, norm=True),
        # a decoding step's new tokens, one for each of 32 sequences
        _case("write4_step", "write", "fp4", 32, 4001, 130, 1),
        # a prompt of 32768 tokens
        _case("write4_prompt", "write", "fp4", 1, 32768, 32768, 0),
        # prompts of odd lengths, into the contiguous tensors that another engine takes
        _case("read4_ragged", "read", "fp4", 7, 1999, 37, 0),
        # a prompt of 65536 tokens
        _case("read4_prompt", "read", "fp4", 1, 65536, 65536, 0),
        # one sequence decodes one token: the smallest call
        _case("decode4_one", "attention", "fp4", 1, 901, 901, 1),
        # a full batch decodes
        _case("decode4_batch", "attention", "fp4", 64, 12000, 501, 1),
        # one long sequence, few heads of the cache
        _case("decode4_long", "attention", "fp4", 1, 131072, 131072, 1, kv_heads=4, group=8),
        # drafts of 64 tokens verified for 16 sequences
        _case("tree4_many", "attention", "fp4", 16, 8192, 3001, 64, tree=2),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("allot", "allot", "append", "append", "write", "read", "attention", "attention", "attention", "attention"))
    kv_heads, group, dim = rng.choice((1, 2, 4, 8, 8, 8)), rng.choice((1, 2, 4, 4, 5, 8)), rng.choice((64, 128, 128, 128, 256))
    page, tree = rng.choice((8, 16, 16, 32, 64, 128)), rng.choice((0, 0, 1, 2, 3, 4))
    if op == "allot":
        seqs = _spread(rng, 1, 4096)
        rows = _spread(rng, 1, min(8192, MOST_ALLOTTED // seqs))
        longest = _spread(rng, 1, 8192)
        back = rng.random() < 0.4
        return _case(None, op, "fp4", seqs, 0 if back else longest, 0 if back else rng.randrange(0, longest + 1), rows, page=page, given_back=back)
    seqs = _spread(rng, 1, 64)
    if op == "append":
        heads = kv_heads * (group + 2)
        rows = rng.choice((0, 1, rng.randrange(2, 65)))
        most = MOST_TOKENS * 128 // (kv_heads * dim) if rows else MOST_APPENDED // (heads * dim)
        longest = _spread(rng, max(rows, 20), max(rows, 20, min(131072, most // seqs)))
        return _case(None, op, rng.choice(("bf16", "e4m3", "fp4", "fp4")), seqs, longest, rng.randrange(max(1, rows), longest + 1), rows,
                     kv_heads, group, dim, page, rotary=rng.choice((dim, dim, dim // 2, 16 * rng.randrange(0, dim // 16 + 1))),
                     interleaved=rng.random() < 0.3, norm=rng.random() < 0.7)
    width = max(1, kv_heads * dim // 128)
    longest = _spread(rng, 20, min(131072, MOST_TOKENS * 8 // (width * seqs)))
    rows = 0 if op == "read" else rng.choice((0, 1)) if op == "write" else rng.choice((1, 1, rng.randrange(2, 17), rng.randrange(17, 65)))
    if op != "attention":
        longest = min(longest, 65536 * 8 // width // seqs // (2 if op == "write" else 1))
        return _case(None, op, "fp4", seqs, longest, rng.randrange(1, longest + 1), rows, kv_heads, 1, dim, page)
    rows = min(rows, longest, max(1, MOST_SCORES // (seqs * kv_heads * group * longest)))
    options = rng.choice((0, 0, 1, 2, 3))
    return _case(None, op, "fp4", seqs, longest, rng.randrange(rows, longest + 1), rows, kv_heads, group, dim, page, tree if rows > 1 else 0,
                 rng.choice((20.0, 30.0, 50.0)) if options & 1 else 0.0, options == 3, _spread(rng, 16, 8192) if options & 2 else 0)


def _lengths(case):
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    return [hi - (hi - lo) * (i * 5 % n) // max(1, n - 1) for i in range(n)]


def _rows(case):
    if case["op"] == "allot":   # some requests have none
        return [case["rows"] - i * 7 % (case["rows"] + 1) for i in range(case["seqs"])]
    return _lengths(case) if not case["rows"] else [case["rows"]] * case["seqs"]


def _room(case):
    """Rows that the outputs of an allotting call have room for: a padded batch."""
    return -(-(sum(_rows(case)) + 1) // 64) * 64


def _pages(n, case):
    return -(-n // case["page"])


def work(case):
    heads, dim, lens = case["kv_heads"], case["dim"], _lengths(case)
    rows = sum(_rows(case))
    if case["op"] == "allot":
        taken = sum(_pages(n + r, case) - _pages(n, case) for n, r in zip(lens, _rows(case)))
        moved = 16 * taken if case["given_back"] else 8 * taken if not any(lens) else 0
        return {"bytes": 16 * rows + 20 * case["seqs"] + moved, "flops": 0}
    token = heads * {"bf16": 2 * dim, "e4m3": dim + 1, "fp4": dim // 2 + dim // GROUP}[case["dtype"]]   # of K or of V
    if case["op"] == "write":
        return {"bytes": 2 * rows * (2 * token + 4 * heads * dim), "flops": 0}   # written, and read back
    if case["op"] == "read":
        return {"bytes": 2 * rows * (token + 2 * heads * dim), "flops": 0}
    if case["op"] == "append":
        back = 2 * (token + 2 * heads * dim) if case["dtype"] == "fp4" else 0    # read back
        return {"bytes": rows * (2 * heads * dim * (2 * case["group"] + 2) + 2 * token + back), "flops": 0}
    seen = sum(min(n, case["window"] + case["rows"] - 1) if case["window"] else n for n in lens)
    pairs = sum((min(n, case["window"]) if case["window"] else n) * case["rows"] for n in lens)
    q = rows * heads * case["group"]
    return {"bytes": 2 * token * seen + q * (4 * dim + 4), "flops": 4 * dim * heads * case["group"] * pairs}


# ---- what a program has in hand ----------------------------------------------------------------------


def _power(size, largest):
    """The least e for which size <= largest * 2^e, from -127 to 127."""
    _, e = torch.frexp(size / largest)                    # off by one at most
    e = torch.where(torch.ldexp(torch.full_like(size, largest), e - 1) >= size, e - 1, e)
    e = torch.where(torch.ldexp(torch.full_like(size, largest), e) < size, e + 1, e)
    return torch.where(size > 0, e, -127).clamp(-127, 127)


def _scaled(x, e):
    """x 2^-e, in two factors each of which is a normal number."""
    return torch.ldexp(torch.ldexp(x, -(e // 2)), -(e - e // 2))


def _fp4(x):
    """Words (two a byte, the even element in the low half) and scale bytes of x [..., dim] in 32 bits, all of it finite: for each
    32 elements the least power of two under which the largest magnitude fits, and one rounding, ties to even."""
    x = x.unflatten(-1, (-1, GROUP))
    e = _power(x.abs().amax(-1), 6.0)
    y = _scaled(x, e[..., None])
    a = y.abs()
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte()
            + (a > 5.0).byte() + torch.signbit(y).byte() * 8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _e4m3(x):
    """Words and scale bytes of x [..., dim] in 32 bits: the same for a whole row, to FP8."""
    e = _power(x.abs().amax(-1), 448.0)
    return _scaled(x, e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(gen, tokens, heads, dim, kind):
    """The cache's values: normal times a log-normal scale per channel, V at half the size."""
    channel = torch.exp(torch.randn(heads, dim, generator=gen, device="cuda")) * (0.5 if kind == "v" else 1.0)
    return (torch.randn(tokens, heads, dim, generator=gen, device="cuda") * channel).to(torch.bfloat16)


def _tree(rows, branches):
    """Bit j of entry i: row j is row i or one of its ancestors; and the rows' depths."""
    bits, depth = [1], [0]
    for i in range(1, rows):
        parent = (i - 1) // branches
        bits.append(bits[parent] | 1 << i)
        depth.append(depth[parent] + 1)
    return [b - (1 << 64) if b >> 63 else b for b in bits], depth


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _allot_inputs(case, seed):
    rng = random.Random(seed)
    lens, rows = _lengths(case), _rows(case)
    rng.shuffle(rows)
    used = [_pages(n, case) for n in lens]
    width = _pages(max(lens) + max(rows), case) + 1
    pages = sum(used) + sum(_pages(r, case) + 1 for r in rows) + 7
    order = list(range(pages))
    rng.shuffle(order)
    table = torch.zeros(case["seqs"], width, dtype=torch.int32)
    at = 0
    for k, n in enumerate(used):
        table[k, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    room = _room(case)
    return {"case": case, "table": table.cuda(), "lens": _i32(lens), "starts": _i32([0] * (case["seqs"] + 1)), "rows": _i32(rows),
            "keep": _i32(lens), "none": _i32([0] * case["seqs"]), "free": _i32(order[at:] + [0] * at), "state": _i32([pages - at] + [0] * 7),
            "slots": torch.zeros(room, dtype=torch.int64, device="cuda"), "row_seqs": _i32([0] * room), "positions": _i32([0] * room),
            "most": (max(rows), max(n + r for n, r in zip(lens, rows)))}


def _inputs(case, seed):
    if case["op"] == "allot":
        return _allot_inputs(case, seed)
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    heads, dim, page, dtype = case["kv_heads"], case["dim"], case["page"], case["dtype"]
    lens, rows = _lengths(case), _rows(case)
    used = [_pages(n, case) for n in lens]
    pages = sum(used) + 3
    order = list(range(pages))
    rng.shuffle(order)
    table, at = torch.zeros(len(lens), max(used), dtype=torch.int32), 0
    for k, n in enumerate(used):
        table[k, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    s = {"case": case, "table": table.cuda(), "starts": _i32(starts), "lens": _i32(lens)}
    words = {"bf16": (dim, torch.bfloat16), "e4m3": (dim, torch.float8_e4m3fn), "fp4": (dim // 2, torch.uint8)}[dtype]
    for kind in ("k", "v"):
        s[kind] = torch.zeros(pages, page, heads, words[0], device="cuda").to(words[1])
        s[kind + "_scales"] = None if dtype == "bf16" else torch.zeros(
            (pages, heads, page) if dtype == "e4m3" else (pages, heads, dim // GROUP, page), dtype=torch.uint8, device="cuda")
        if case["op"] in ("write", "append"):    # what was there before is overwritten or stays
            s["new_" + kind] = _values(gen, sum(rows), heads, dim, kind)
        else:
            w, b = _fp4(_values(gen, pages * page, heads, dim, kind).float())
            s[kind].copy_(w.view(pages, page, heads, -1))
            s[kind + "_scales"].copy_(b.view(pages, page, heads, -1).permute(0, 2, 3, 1))
        s["out_" + kind] = torch.empty(sum(rows), heads, dim, dtype=torch.bfloat16, device="cuda") if case["op"] != "attention" else None
    q_heads = heads * case["group"]
    if case["op"] in ("append", "attention"):
        s["q"] = torch.randn(sum(rows), q_heads, dim, generator=gen, device="cuda").to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
    if case["op"] == "append":
        half = case["rotary"] // 2
        s["freqs"] = (10000.0 ** (-torch.arange(half, device="cuda") / max(half, 1))).float() if half else None
        for kind in ("q", "k"):
            s[kind + "_weight"] = (1.0 + 0.3 * torch.randn(dim, generator=gen, device="cuda")).to(torch.bfloat16) if case["norm"] else None
        s["eps"] = 1e-6 if case["norm"] else None
    if case["op"] == "attention":
        s["lse"] = torch.empty(sum(rows), q_heads, device="cuda")
        s["scale"] = dim ** -0.5
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, q_heads + 1, device="cuda") / q_heads) if case["slopes"] else None
        s["tree"] = s["positions"] = None
        if case["tree"]:
            bits, depth = _tree(case["rows"], case["tree"])
            s["tree"] = torch.tensor(bits, device="cuda").repeat(len(lens))[:, None].contiguous()
            s["positions"] = ((s["lens"] - case["rows"])[:, None] + _i32(depth)).reshape(-1).contiguous()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:   # the descriptions of tensors that a program makes once, and the workspace
        import paper_2605_01708_amd as sz

        most = s["most"] if case["op"] == "allot" else (max(_rows(case)), case["longest"])
        s["seqs"] = sz.Sequences(s["table"], s["starts"], s["lens"], max_rows=most[0], max_len=most[1])
        if case["op"] == "allot":
            s["pool"] = sz.PagePool(s["free"], s["state"], case["page"])
            return s
        dtype = {"bf16": sz.BF16, "e4m3": sz.FP8_E4M3, "fp4": sz.FP4_E2M1}[case["dtype"]]
        s["cache"] = sz.KvCache(s["k"], s["v"], dtype, s["k_scales"], s["v_scales"])
        if case["op"] == "append":
            s["how"] = sz.Rotation(s["freqs"], interleaved=case["interleaved"], eps=s["eps"], q_weight=s["q_weight"], k_weight=s["k_weight"])
        if case["op"] == "attention":
            s["how"] = sz.Attention(s["scale"], softcap=case["softcap"], window=case["window"], slopes=s["slopes"], tree=s["tree"],
                                    positions=s["positions"])
            s["workspace"] = sz.attention_workspace(s["cache"], s["seqs"], s["q"].shape[0], s["q"].shape[1])
    return s


# ---- the framework's operators, and the plain form ---------------------------------------------------


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2605_01708_amd as sz

        if op == "allot":
            if case["given_back"]:
                sz.cache_allot(s["pool"], s["seqs"], s["none"], keep=s["keep"])
            sz.cache_allot(s["pool"], s["seqs"], s["rows"], keep=s["keep"], slots=s["slots"], row_seqs=s["row_seqs"], positions=s["positions"])
            return {name: s[name] for name in ("table", "lens", "starts", "free", "state", "slots", "row_seqs", "positions")}
        if op == "attention":
            sz.cache_attention(s["q"], s["cache"], s["seqs"], s["out"], s["workspace"], s["how"], lse=s["lse"])
            return {"out": s["out"], "lse": s["lse"]}
        if op == "append":
            sz.cache_append(s["q"], s["new_k"], s["new_v"], s["cache"], s["seqs"], s["how"], s["out"])
        elif op == "write":
            sz.cache_write(s["new_k"], s["new_v"], s["cache"], s["seqs"])
        if case["dtype"] == "fp4":
            sz.cache_read(s["cache"], s["seqs"], s["out_k"], s["out_v"])
            out = {"k": s["out_k"], "v": s["out_v"]}
        else:
            out = _words(s)
        return {"q": s["out"], **out} if op == "append" else out
    return {"allot": _allot, "append": _append, "write": _write, "read": _read, "attention": _attention}[op](s)


def _words(s):
    out = {"k": s["k"], "v": s["v"]}
    return out if s["k_scales"] is None else {**out, "k_scales": s["k_scales"], "v_scales": s["v_scales"]}


def _allot_call(s, rows, keep, n_rows):
    """Pages that sequences no longer need go onto the stack so that the first of them, in the sequences' order, is on top; then
    pages are taken off the top in that order.  (The cases' pools have enough.)"""
    page, top = s["case"]["page"], s["free"].shape[0]
    old = s["lens"].clamp(min=0)
    kept = torch.minimum(keep, old)
    new = kept + rows
    held, need = (old + page - 1) // page, (new + page - 1) // page
    column = torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)
    gives = (column >= need[:, None]) & (column < held[:, None])
    takes = (column >= held[:, None]) & (column < need[:, None])
    n_given, n_taken = gives.sum(), takes.sum()
    have = s["state"][0] + n_given
    place = have - 1 - (torch.cumsum(gives.flatten(), 0) - 1)
    stack = torch.cat([s["free"], s["free"].new_zeros(1)])
    stack[torch.where(gives.flatten(), place, top)] = s["table"].flatten()
    from_top = have - 1 - (torch.cumsum(takes.flatten(), 0) - 1)
    taken = stack[torch.where(takes.flatten(), from_top, top)].view_as(s["table"])
    s["table"].copy_(torch.where(takes, taken, s["table"]))
    s["free"].copy_(stack[:-1])
    s["lens"].copy_(new)
    s["starts"][1:] = torch.cumsum(rows, 0)
    zero = n_given * 0
    s["state"].copy_(torch.stack([have - n_taken, zero, zero, rows.sum(), rows.max(), new.max(), n_taken, n_given]))
    if n_rows:
        i = torch.arange(n_rows, device="cuda", dtype=torch.int32)
        of = torch.searchsorted(s["starts"][1:].contiguous(), i, right=True).clamp(max=rows.shape[0] - 1)
        there = i < s["starts"][-1]
        at = torch.where(there, kept[of] + i - s["starts"][of], 0)
        s["slots"].copy_(torch.where(there, s["table"][of, (at // page).long()].long() * page + at % page, -1))
        s["row_seqs"].copy_(torch.where(there, of, -1))
        s["positions"].copy_(torch.where(there, at, -1))


def _allot(s):
    if s["case"]["given_back"]:
        _allot_call(s, s["none"], s["keep"], 0)
    _allot_call(s, s["rows"], s["keep"], s["slots"].shape[0])
    return {name: s[name] for name in ("table", "lens", "starts", "free", "state", "slots", "row_seqs", "positions")}


def _slots(s):
    """Page and place in it of every row of the call, and its position."""
    starts, page = s["starts"], s["case"]["page"]
    counts = (starts[1:] - starts[:-1]).long()
    total = sum(_rows(s["case"]))
    of = torch.repeat_interleave(torch.arange(counts.numel(), device="cuda"), counts, output_size=total)
    at = s["lens"].long()[of] - counts[of] + torch.arange(total, device="cuda") - starts[of]
    return s["table"][of, at // page].long(), at % page, at


def _put(s, kind, page, place, x):
    dtype = s["case"]["dtype"]
    if dtype == "bf16":
        s[kind][page, place] = x.to(torch.bfloat16)
        return
    words, scales = _e4m3(x) if dtype == "e4m3" else _fp4(x)
    s[kind].view(torch.uint8)[page, place] = words.view(torch.uint8)
    s[kind + "_scales"].movedim(-1, 1)[page, place] = scales


def _gather(s, kind, page, place):
    """Cached rows of 4-bit words in 32 bits."""
    words = s[kind][page, place]
    code = torch.stack([words & 15, words >> 4], -1).flatten(-2)
    x = torch.tensor([*E2M1, *(-v for v in E2M1)], device="cuda")[code.int()].unflatten(-1, (-1, GROUP))
    e = s[kind + "_scales"].movedim(-1, 1)[page, place].int()[..., None] - 127
    return torch.ldexp(x, e).flatten(-2)


def _read(s):
    page, place, _ = _slots(s)
    return {kind: _gather(s, kind, page, place).to(torch.bfloat16) for kind in ("k", "v")}


def _write(s):
    page, place, _ = _slots(s)
    _put(s, "k", page, place, s["new_k"].float())
    _put(s, "v", page, place, s["new_v"].float())
    return _read(s)


def _normed_and_rotated(x, weight, s, angle):
    case = s["case"]
    x = x.float()
    if case["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight.float()
    if case["rotary"]:
        c, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        turned, rest = x[..., :case["rotary"]], x[..., case["rotary"]:]
        if case["interleaved"]:
            a, b = turned[..., 0::2], turned[..., 1::2]
            turned = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
        else:
            a, b = turned.chunk(2, -1)
            turned = torch.cat([a * c - b * sn, b * c + a * sn], -1)
        x = torch.cat([turned, rest], -1)
    return x


def _append(s):
    page, place, at = _slots(s)
    angle = at.double()[:, None] * s["freqs"].double() if s["case"]["rotary"] else None
    q = _normed_and_rotated(s["q"], s["q_weight"], s, angle).to(torch.bfloat16)
    _put(s, "k", page, place, _normed_and_rotated(s["new_k"], s["k_weight"], s, angle))
    _put(s, "v", page, place, s["new_v"].float())
    return {"q": q, **(_read(s) if s["case"]["dtype"] == "fp4" else _words(s))}


def _attention(s):
    c = s["case"]
    lens, T, n, heads, group = s["lens"].long(), c["rows"], c["seqs"], c["kv_heads"], c["group"]
    key = torch.arange(c["longest"], device="cuda")
    base = (lens - T)[:, None]
    page = s["table"][:, key // c["page"]].long()
    place = (key % c["page"]).expand(n, -1)
    valid = key < lens[:, None]                                                            # [n, keys]
    k = _gather(s, "k", page, place).permute(0, 2, 3, 1)                                   # [n, heads, dim, keys]
    v = torch.where(valid[:, :, None, None], _gather(s, "v", page, place), 0).transpose(1, 2)
    q = s["q"].float().view(n, T, heads, group, -1).permute(0, 2, 1, 3, 4).reshape(n, heads, T * group, -1)
    x = torch.matmul(q, k).view(n, heads, T, group, -1) * s["scale"]
    if c["softcap"]:
        x = torch.tanh(x / c["softcap"]) * c["softcap"]
    draft = key - base                                                                     # which row of the call a key is
    row = torch.arange(T, device="cuda")
    if s["tree"] is None:
        pos = base + row
        allowed = draft[:, None] <= row[:, None]
        key_pos = key.expand(n, -1)
    else:
        pos = s["positions"].long().view(n, T)
        bits = s["tree"].view(n, T, 1) >> draft.clamp(0, 63)[:, None] & 1
        allowed = (draft < 0)[:, None] | (bits != 0)
        key_pos = torch.where(draft < 0, key, torch.gather(pos, 1, draft.clamp(0, T - 1)))
    far = pos[:, :, None] - key_pos[:, None]                                               # [n, rows, keys]
    allowed = allowed & valid[:, None]
    if c["window"]:
        allowed = allowed & (far < c["window"])
    if s["slopes"] is not None:
        x = x - s["slopes"].view(heads, 1, group, 1) * far[:, None, :, None].float()
    x = torch.where(allowed[:, None, :, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, heads, T * group, -1), v).view(n, heads, T, group, -1)
    out = torch.where(total > 0, out / total, 0).permute(0, 2, 1, 3, 4).reshape(n * T, heads * group, -1)
    lse = (torch.log(total) + top).view(n, heads, T, group).permute(0, 2, 1, 3).reshape(n * T, -1)
    return {"out": out.to(torch.bfloat16), "lse": lse}


# ---- in 64 bits ---------------------------------------------------------------------------------------


def _to_grid(x, bits, least):
    """Values in 64 bits to the nearest of a floating format with so many mantissa bits and this least exponent, ties to even."""
    e = (torch.frexp(x)[1] - 1).clamp(min=least)
    unit = torch.exp2((e - bits).double())
    return torch.round(x / unit) * unit


def _on_grid(x, largest, bits, least, width):
    """x [..., dim] in 64 bits as quantised words (values without their power of two) and powers, for each `width` elements."""
    x = x.unflatten(-1, (-1, width))
    size = x.abs().amax(-1).clamp(min=2.0 ** -300)
    e = torch.ceil(torch.log2(size / largest)).clamp(-127, 127)
    e = e + (size > largest * torch.exp2(e)).double()              # the logarithm's own rounding
    e = e - ((size <= largest * torch.exp2(e - 1)) & (e > -127)).double()
    return _to_grid(x * torch.exp2(-e)[..., None], bits, least).flatten(-2), e


def _cached(s, kind, where):
    """Tokens of a cache of 4-bit words in 64 bits."""
    words = s[kind][where].long()
    nibble = torch.stack([words % 16, words // 16], -1).flatten(-2)
    size, exponent = nibble % 2, nibble // 2 % 4
    x = torch.where(exponent > 0, (1 + size / 2.0).double() * torch.exp2(exponent.double() - 1), size.double() / 2)
    x = torch.where(nibble > 7, -x, x).unflatten(-1, (-1, GROUP))
    return (x * torch.exp2(s[kind + "_scales"].movedim(-1, 1)[where].double() - 127)[..., None]).flatten(-2)


def _exact_turn(x, weight, s, case, at):
    x = x.double()
    if case["norm"]:
        x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]) * weight.double()
    half = case["rotary"] // 2
    if half:
        angle = at[:, None] * s["freqs"].double()
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        a = slice(0, 2 * half, 2) if case["interleaved"] else slice(0, half)
        b = slice(1, 2 * half, 2) if case["interleaved"] else slice(half, 2 * half)
        z = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * turn
        x[..., a], x[..., b] = z.real, z.imag
    return x


def _exact_allot(s, case):
    """One request after the other, on the host."""
    page, lens, rows, table = case["page"], s["lens"].tolist(), s["rows"].tolist(), s["table"].tolist()
    stack = s["free"].tolist()
    free = s["state"].tolist()[0]
    starts, slots, row_seqs, positions, taken = [0], [], [], [], 0
    for k, (n, r) in enumerate(zip(lens, rows)):
        for p in range(_pages(n, case), _pages(n + r, case)):
            free, taken = free - 1, taken + 1
            table[k][p] = stack[free]
        for t in range(n, n + r):
            slots.append(table[k][t // page] * page + t % page)
            row_seqs.append(k)
            positions.append(t)
        starts.append(starts[-1] + r)
    rest = [-1] * (_room(case) - len(slots))
    new = [n + r for n, r in zip(lens, rows)]
    return {"table": _i32(table), "lens": _i32(new), "starts": _i32(starts), "free": s["free"],
            "state": _i32([free, 0, 0, len(slots), max(rows), max(new), taken, 0]),
            "slots": torch.tensor(slots + rest, device="cuda"), "row_seqs": _i32(row_seqs + rest), "positions": _i32(positions + rest)}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "allot":
        return _exact_allot(s, case)
    lens, rows, page, dtype = _lengths(case), _rows(case), case["page"], case["dtype"]
    grid = {"bf16": None, "e4m3": (448.0, 3, -6, case["dim"]), "fp4": (6.0, 1, 0, GROUP)}[dtype]
    at, op, out, pool = 0, case["op"], {}, {}
    if op == "append" and dtype != "fp4":
        pool = {kind: s[kind].double() for kind in ("k", "v")}
        if dtype == "e4m3":
            pool |= {kind: s[kind].clone() for kind in ("k_scales", "v_scales")}
    for n, (length, count) in enumerate(zip(lens, rows)):
        token = torch.arange(length - count, length, device="cuda")
        where = (s["table"][n][token // page].long(), token % page)
        mine = slice(at, at + count)
        at += count
        if op == "attention":
            found = dict(zip(("out", "lse"), _exact_attention(s, case, n, mine, length)))
        elif op == "read":
            found = {kind: _cached(s, kind, where) for kind in ("k", "v")}
        else:
            found = {kind: s["new_" + kind][mine].double() for kind in ("k", "v")}
            if op == "append":
                found["k"] = _exact_turn(found["k"], s["k_weight"], s, case, token.double())
                found["q"] = _exact_turn(s["q"][mine], s["q_weight"], s, case, token.double())
            for kind in ("k", "v"):
                x, e = _on_grid(found[kind], *grid) if grid else (found[kind], None)
                if pool:
                    del found[kind]
                    pool[kind][where] = x
                    if grid:
                        pool[kind + "_scales"].movedim(-1, 1)[where] = (e[..., 0] + 127).to(torch.uint8)
                else:
                    found[kind] = (x.unflatten(-1, (-1, GROUP)) * torch.exp2(e)[..., None]).flatten(-2)
        for name, x in found.items():
            out.setdefault(name, []).append(x)
    return {**{name: torch.cat(x) for name, x in out.items()}, **pool}


def _exact_attention(s, case, n, mine, length):
    count, heads, group = case["rows"], case["kv_heads"], case["group"]
    position = torch.arange(length, device="cuda")
    where = (s["table"][n][position // case["page"]].long(), position % case["page"])
    k, v = _cached(s, "k", where), _cached(s, "v", where)                          # [keys, heads, dim]
    see = torch.ones(count, length, dtype=torch.bool, device="cuda")
    see[:, length - count:] = torch.ones(count, count, dtype=torch.bool, device="cuda").tril()
    if s["tree"] is not None:
        words = s["tree"][mine, 0].tolist()
        see[:, length - count:] = torch.tensor([[w >> j & 1 for j in range(count)] for w in words], device="cuda").bool()
        position[length - count:] = s["positions"][mine]
    far = position[length - count:, None] - position[None]
    if case["window"]:
        see &= far < case["window"]
    outs, sums = [], []
    for h in range(heads * group):
        x = s["q"][mine, h].double() @ k[:, h // group].T * s["scale"]
        if case["softcap"]:
            x = case["softcap"] * torch.tanh(x / case["softcap"])
        if s["slopes"] is not None:
            x = x - s["slopes"][h].double() * far
        x = x.masked_fill(~see, -math.inf)
        lse = torch.logsumexp(x, -1)
        outs.append(torch.exp(x - lse[:, None]) @ v[:, h // group])
        sums.append(lse)
    return torch.stack(outs, 1), torch.stack(sums, 1)
