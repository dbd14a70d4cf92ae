"""Sparse decode attention over the packed paged cache, and the management of its pages: what is measured, and the plain forms.

Five operators of a server that keeps long conversations in the 2/3/4-bit cache:

  bounds    after an append: per page and head, an upper and a lower bound of every channel of the packed keys, in 8 bits
  select    per sequence and key/value head, the pages whose bounds promise the largest scores for the step's queries
  sparse    one decode step's attention over the windows and the selected pages (selection included)
  fork      beams or a shared prefix: sequences that begin as copies of others, share their pages, and get a last page of their own
  compact   sequences end, their pages are given back, and the live pages move to the front of the pool

Definitions.  A page holds 64 tokens; a key is khat = fl32(x_min + Delta code).  Bounds of a page and head, over its tokens below the sequence's
length: e = the least integer >= -31 with max |khat| <= 127 2^e, upper[c] = ceil(max khat[c] / 2^e), lower[c] = floor(min khat[c] / 2^e).
Score of a page for query head j: q' = T_K^{-T} q, q_int = round(q' 32512 / max|q'|), dot = sum_c max(q_int, 0) upper + min(q_int, 0) lower,
s_j = fl32(fl32(dot) 2^e fl32(max|q'| / 32512 sm_scale)); the page's key is the largest fl32(s_j - (largest s_j of all pages)) of the heads that
share the key/value head.  The n_select pages with the largest keys are taken, of equal ones the lower; listed in ascending order, -1 behind them.
"""
import functools
import math

import numpy as np
import torch

own = False

D, PAGE = 128, 64
Q_MAX = 32512.0
RECORD = {2: 4608, 3: 6656, 4: 8704}       # bytes of one page and head


def _case(name, kind, batch, n_q, n_kv, bits, ctx_lo, ctx_hi, **more):
    return dict(dict(name=name, kind=kind, batch=batch, n_q=n_q, n_kv=n_kv, bits=bits, ctx_lo=ctx_lo, ctx_hi=ctx_hi, s_sink=4, s_keep=128, s_flush=1), **more)


def listed():
    return [
        # prompts of a batch have just been appended: the bounds of all their pages
        _case("bounds_prompts_8x8192_2bit", "bounds", 8, 28, 4, 2, 8192, 8192, new_lo=8192, new_hi=8192),
        # every decode step: one token more in the last page of each of many conversations
        _case("bounds_step_64_ragged_4bit", "bounds", 64, 32, 8, 4, 1024, 8192, new_lo=1, new_hi=1),
        # a full batch on long contexts: an eighth of the pages
        _case("select_16x32k", "select", 16, 32, 8, 2, 32768, 32768, budget=64),
        # one very long document, eight query heads per key/value head
        _case("select_1x128k", "select", 1, 64, 8, 2, 131072, 131072, budget=128),
        # the short end: one conversation on a small layer, latency and launches
        _case("sparse_1x2k_2bit", "sparse", 1, 8, 2, 2, 2048, 2048, s_keep=64, budget=8),
        # the headline serving step with an eighth of its pages
        _case("sparse_16x32k_2bit", "sparse", 16, 32, 8, 2, 32768, 32768, budget=64),
        # one very long document with a sixteenth of its pages
        _case("sparse_1x128k_2bit", "sparse", 1, 64, 8, 2, 131072, 131072, budget=128),
        # many users at different points of their conversations, some with fewer pages than the budget
        _case("sparse_64_ragged_4bit", "sparse", 64, 32, 8, 4, 1024, 8192, budget=32),
        # a beam of one short conversation splits in two
        _case("fork_1_of_300_2bit", "fork", 1, 8, 2, 2, 300, 300, beams=1, s_keep=64),
        # four long prompts, each continued by three more samples
        _case("fork_12_of_32k_2bit", "fork", 4, 32, 8, 2, 32001, 32761, beams=3),
        # a small pool in which two of five sequences end
        _case("compact_5_ragged_3bit", "compact", 5, 28, 4, 3, 501, 16001, ended=2),
        # half of a large batch ends
        _case("compact_64_ragged_4bit", "compact", 64, 32, 8, 4, 1024, 8192, ended=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["bounds", "select", "sparse", "sparse", "fork", "compact"])
    n_kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8])
    ctx = _log_int(rng, 100, 131072 if kind in ("select", "sparse") else 32768)
    most = max(1, min(64, 16 * 32768 * 8 // (ctx * n_kv)))
    if kind == "bounds":
        most = max(1, min(64, 8 * 8192 * 4 // (ctx * n_kv)))
    if kind in ("compact", "fork"):
        most = max(1, min(most, 32 * 32768 // ctx) // 2)
    case = _case("", kind, _log_int(rng, 1, most), n_kv * group, n_kv, rng.choice([2, 2, 3, 4]), max(90, ctx // rng.choice([1, 1, 3, 8])), ctx,
                 s_keep=rng.choice([64, 128]), s_flush=rng.choice([1, 1, 8, 16]))
    if kind == "bounds":
        new = _log_int(rng, 1, case["ctx_lo"])
        case.update(new_lo=max(1, new // rng.choice([1, 2, 16])), new_hi=new)
    elif kind in ("select", "sparse"):
        case.update(budget=_log_int(rng, 1, min(128, 64 * 16 * 8 // (case["batch"] * n_kv))))
    elif kind == "fork":
        case.update(beams=rng.choice([1, 1, 2, 3]))
    else:
        case["batch"] += 1
        case.update(ended=rng.randint(1, case["batch"] - 1))
    del case["name"]
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _spread(lo, hi, n, salt):
    """n lengths between lo and hi (they belong to the case, not to the seed)."""
    return [int(x) for x in np.random.default_rng(1000 + salt).integers(lo, hi + 1, size=n)]


def _slots(case):
    return case["batch"] * (1 + case.get("beams", 0))


def _pool_pages(case):
    longest = -(-case["ctx_hi"] // PAGE) + 1
    used = sum(-(-n // PAGE) for n in _spread(case["ctx_lo"], case["ctx_hi"], case["batch"], 1))
    return longest, used + _slots(case) + max(4, used // 8)          # a spare page per sequence, and an eighth more


def _queries_and_transform(case, seed):
    """q' in the scale of logits with standard deviation 2 on keys of unit variance; T_K^{-T}: a rotation with channel scales, fp32."""
    rng = np.random.default_rng([seed, 3])
    n_kv, group = case["n_kv"], case["n_q"] // case["n_kv"]
    rotation = np.linalg.qr(rng.standard_normal((n_kv, D, D)))[0]
    T_inv = torch.from_numpy((np.exp(0.25 * rng.standard_normal((n_kv, D, 1))) * rotation).astype(np.float32)).cuda()
    q = torch.from_numpy(2.0 * rng.standard_normal((case["batch"], case["n_q"], D)).astype(np.float32)).cuda()
    head = torch.from_numpy(np.exp(0.4 * rng.standard_normal((1, case["n_q"], 1))).astype(np.float32)).cuda()      # sharper and flatter heads
    return (q * head).to(torch.bfloat16), T_inv


def _vectors(gen, n, scale):
    """n pages of 64 vectors: what a page's tokens have in common, and what they do not."""
    common = torch.randn((n, 1, D), generator=gen, device="cuda")
    return (0.6 * common + 0.8 * torch.randn((n, PAGE, D), generator=gen, device="cuda")) * scale


def _quantized(x, bits, clip):
    """Codes (uint8) and the stored (step, offset) pair (fp16) of the clipped affine quantizer."""
    edge = clip * x.square().mean(-1, keepdim=True).sqrt()
    low = torch.maximum(x.amin(-1, keepdim=True), -edge)
    step = ((torch.minimum(x.amax(-1, keepdim=True), edge) - low) / ((1 << bits) - 1)).half()
    low = low.half()
    code = torch.round((x - low.float()) / step.float()).clamp_(0, (1 << bits) - 1).to(torch.uint8)
    return code, torch.cat([step, low], dim=-1)


def _content(case, seed, n_pages):
    """Key codes, key (step, offset), value codes, value (step, offset) of all pages and heads, 4096 of them at a time."""
    gen = torch.Generator(device="cuda").manual_seed(7919 * (seed + 1))
    n = n_pages * case["n_kv"]
    parts = [_quantized(_vectors(gen, min(4096, n - at), 1.0), case["bits"], 2.05) + _quantized(_vectors(gen, min(4096, n - at), 1.5), case["bits"], 1.75)
             for at in range(0, n, 4096)]
    return [torch.cat(part) for part in zip(*parts)]


@functools.lru_cache(maxsize=None)
def _places(bits):
    """Where the cache keeps the codes of a record: per plane (low bits; at 3 bits the high bit as well) and side (keys, values) the byte and
    the bit inside it of code (token, channel), as arrays of 64 x 128."""
    r, ch = np.meshgrid(np.arange(PAGE), np.arange(D), indexing="ij")
    block, rr = r >> 4, r & 15
    # keys: lanes of (token & 7, channel pair), words of (token half, channel half)
    s, hh, b, t = ch >> 5, (ch >> 4) & 1, 2 * ((ch >> 3) & 1) + (ch & 1), (ch >> 1) & 3
    lane, word = 4 * (rr & 7) + t, (rr >> 3) + 2 * hh
    # values: lanes of (channel & 7, token pair), half-words of (token & 1)
    ps, tv, hi, i, rsel = rr >> 3, (rr & 7) >> 1, rr & 1, ch >> 4, (ch & 15) >> 3
    lane_v = 4 * (ch & 7) + tv
    wide = 1024 if bits == 4 else 512
    side = 4 * (wide + (256 if bits == 3 else 0))
    if bits == 4:
        k = (block * 1024 + 512 * (s >> 1) + 16 * lane + 4 * word + b, 4 * (s & 1))
        v = (side + block * 1024 + 512 * ps + 16 * lane_v + 4 * (2 * rsel + (i >> 2)) + 2 * hi, 4 * (i & 3))
        return dict(low=(k, v), high=None, meta=2 * side)
    k = (block * 512 + 16 * lane + 4 * word + b, 2 * s)
    v = (side + block * 512 + 16 * lane_v + 4 * (2 * ps + rsel) + 2 * hi, 2 * i)
    high = None
    if bits == 3:
        target = np.where(i < 5, 2 * i + 2, 2 * (i - 5) + 2)
        shift = np.where(rsel == 0, np.where(i < 5, 0, 9), np.where(i < 5, -1, np.where(i < 7, 10, -6)))
        high = ((4 * 512 + block * 256 + 8 * lane + 4 * (rr >> 3) + b, 2 * s + hh), (side + 4 * 512 + block * 256 + 8 * lane_v + 4 * ps + 2 * hi, target + shift))
    return dict(low=(k, v), high=high, meta=2 * side)


@functools.lru_cache(maxsize=None)
def _flat(bits, plane, side):
    """Byte and bit of each code of a plane ("low", "high") and side as flat device tensors; a bit beyond 7 lies in the next byte."""
    byte, bit = _places(bits)[plane][side]
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a).reshape(-1)).cuda()  # noqa: E731
    return to(byte + (bit >> 3)), to((bit & 7).astype(np.uint8))


@functools.lru_cache(maxsize=None)
def _meta_bytes(bits, first, n):
    """Bytes first .. first + n - 1 of the eight that a token's steps and offsets (keys, values) take, of all 64 tokens."""
    r = np.arange(PAGE)
    at = _places(bits)["meta"] + 128 * (r >> 4) + 16 * (r & 7) + 8 * ((r >> 3) & 1)
    return torch.from_numpy((at[:, None] + first + np.arange(n)[None, :]).reshape(-1)).cuda()


def _write_plane(records, bits, plane, side, fields):
    """Puts one plane's fields ([records, 64 * 128] uint8) into its bytes, all fields of a byte together."""
    byte, bit = _flat(bits, plane, side)
    order = torch.argsort(byte, stable=True)
    first, n = int(byte.min()), int(byte.max()) - int(byte.min()) + 1
    per = byte.numel() // n
    records[:, first:first + n] = (fields[:, order] << bit[order]).view(-1, n, per).sum(-1, dtype=torch.uint8)


def _records(content, bits):
    """The packed records of all pages and heads."""
    kc, km, vc, vm = content
    records = torch.zeros((kc.shape[0], RECORD[bits]), dtype=torch.uint8, device="cuda")
    low = 15 if bits == 4 else 3
    _write_plane(records, bits, "low", 0, kc.view(-1, PAGE * D) & low)
    _write_plane(records, bits, "low", 1, vc.view(-1, PAGE * D) & low)
    if bits == 3:
        _write_plane(records, bits, "high", 0, kc.view(-1, PAGE * D) >> 2)
        _write_plane(records, bits, "high", 1, vc.view(-1, PAGE * D) >> 2)
    records[:, _meta_bytes(bits, 0, 8)] = torch.cat([km, vm], dim=-1).contiguous().view(torch.uint8).view(-1, PAGE * 8)
    return records


def prepare(case, seed):
    n_q, n_kv, bits, batch = case["n_q"], case["n_kv"], case["bits"], case["batch"]
    lens = _spread(case["ctx_lo"], case["ctx_hi"], batch, 1)
    longest, n_pages = _pool_pages(case)
    slots = _slots(case)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    # page table and reference counts of a pool that has been in use: the pages of the sequences lie anywhere
    order = np.random.default_rng([seed, 5]).permutation(n_pages)
    table, refs, at = np.full((slots, longest), -1, np.int32), np.zeros(n_pages, np.int32), 0
    for b, n in enumerate(lens):
        used = -(-n // PAGE)
        table[b, :used] = order[at:at + used]
        refs[order[at:at + used]] = 1
        at += used
    book = torch.from_numpy(np.concatenate([table.reshape(-1), refs])).cuda()
    gen = torch.Generator(device="cuda").manual_seed(104729 * (seed + 1))
    cap = case["s_keep"] + case["s_flush"] - 1
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    octets = lambda shape, kind: torch.randint(-128, 128, shape, generator=gen, device="cuda", dtype=torch.int16).to(torch.int8).view(kind)  # noqa: E731
    s = dict(case=case, batch=batch, lens=ints(lens), longest=max(lens), n_pages=n_pages, max_pages=longest, n_slots=slots, cap=cap,
             book=book, table=book[:slots * longest].view(slots, longest), refs=book[slots * longest:], status=torch.zeros(1, dtype=torch.int32, device="cuda"),
             slot=ints(list(range(batch))), ring=normal(slots, n_kv, 2, cap, D), sink=normal(slots, n_kv, 2, case["s_sink"], D))
    if case["kind"] in ("bounds", "sparse"):
        s["pages"] = _records(_content(case, seed, n_pages), bits).view(n_pages, n_kv, -1)
    elif case["kind"] in ("fork", "compact"):
        s["pages"] = octets((n_pages, n_kv, RECORD[bits]), torch.uint8)
    s["bounds"] = torch.zeros((n_pages, n_kv, 2, D), dtype=torch.int8, device="cuda")
    s["exponents"] = torch.zeros((n_pages, n_kv), dtype=torch.int8, device="cuda")
    if case["kind"] == "bounds":
        new = _spread(case["new_lo"], case["new_hi"], batch, 2)
        s.update(cu=ints([0] + list(np.cumsum(new))), max_new=max(new))
    if case["kind"] in ("select", "sparse"):
        s["Q"], s["T_inv"] = _queries_and_transform(case, seed)
        s["selected"] = torch.empty((batch, n_kv, case["budget"]), dtype=torch.int32, device="cuda")
        s["O"] = torch.empty((batch, n_q, D), dtype=torch.bfloat16, device="cuda")
        if case["kind"] == "sparse":
            for b, n in enumerate(lens):                      # kept up with every append of the sequence
                _plain_bounds(s, ints([b]), ints([n]), ints([n]))
        else:
            s.update(_drawn_bounds(n_pages, n_kv, seed))
    if case["kind"] == "fork":
        n = batch * case["beams"]
        s.update(n=n, src=ints([k // case["beams"] for k in range(n)]), dst=ints(list(range(batch, batch + n))), cu=ints(list(range(n + 1))), max_copies=n)
        s["src_len"] = s["lens"][s["src"].long()].contiguous()
    if case["kind"] == "compact":
        gone = np.random.default_rng([seed, 6]).permutation(batch)[:case["ended"]]
        s.update(n=len(gone), gone=ints(sorted(int(x) for x in gone)), start=book.clone(), max_copies=(n_pages + 1) // 2)
    if case["kind"] in ("fork", "compact"):
        s["bounds"], s["exponents"] = octets((n_pages, n_kv, 2, D), torch.int8), octets((n_pages, n_kv), torch.int8)
        s["copies"] = torch.full((2, s["max_copies"]), -1, dtype=torch.int32, device="cuda")
        s["count"], s["live"] = ints([0]), ints([0])
    return s


def _drawn_bounds(n_pages, n_kv, seed):
    """Bounds as pages of 64 unit-variance keys have them: about two and a half deviations of the tokens around the page's mean."""
    gen = torch.Generator(device="cuda").manual_seed(31 * (seed + 1))
    draw_one = lambda: torch.randn((n_pages, n_kv, D), generator=gen, device="cuda")  # noqa: E731
    mean = 0.6 * draw_one()
    upper, lower = mean + 1.9 + 0.3 * draw_one(), mean - 1.9 - 0.3 * draw_one()
    unit = 2.0 ** -4 * torch.ones((n_pages, n_kv), device="cuda")
    ints = torch.stack([torch.floor(lower / unit[..., None]), torch.ceil(upper / unit[..., None])], dim=2).clamp(-127, 127)
    return dict(bounds=ints.to(torch.int8), exponents=torch.full((n_pages, n_kv), -4, dtype=torch.int8, device="cuda"))


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _read_codes(records, bits, side):
    """Codes of the keys (side 0) or values (side 1) of records [..., bytes] as [..., 64, 128] uint8."""
    byte, bit = _flat(bits, "low", side)
    codes = (records[..., byte] >> bit) & (15 if bits == 4 else 3)
    if bits == 3:
        byte, bit = _flat(bits, "high", side)
        codes = codes + 4 * ((records[..., byte] >> bit) & 1)
    return codes.view(*records.shape[:-1], PAGE, D)


def _read_vectors(records, bits, side):
    """Dequantized keys or values, offset + step * code in 32 bits."""
    meta = records[..., _meta_bytes(bits, 4 * side, 4)].contiguous().view(torch.float16).view(*records.shape[:-1], PAGE, 2).float()
    return meta[..., 1:] + meta[..., :1] * _read_codes(records, bits, side).float()


def _power_of_two(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _plain_bounds(s, slot, lens, new):
    case = s["case"]
    first = (lens - new).long() // PAGE
    index = first[:, None] + torch.arange(int(new.max()) // PAGE + 2, device="cuda")[None, :]
    b, k = torch.nonzero((index * PAGE < lens[:, None]) & (new[:, None] > 0) & (index < s["max_pages"]), as_tuple=True)
    index = index[b, k]
    page = s["table"][slot[b].long(), index].long()
    keys = _read_vectors(s["pages"][page], case["bits"], 0)                                     # [pages, heads, 64, 128]
    there = (index[:, None] * PAGE + torch.arange(PAGE, device="cuda")[None, :] < lens[b][:, None])[:, None, :, None]
    upper, lower = keys.masked_fill(~there, -math.inf).amax(2), keys.masked_fill(~there, math.inf).amin(2)
    most = torch.maximum(upper.abs(), lower.abs()).amax(-1)
    part, e = torch.frexp(most)
    e = torch.where(most > 0, torch.where(part <= 127.0 / 128.0, e - 7, e - 6), -31).clamp(min=-31)
    scale = _power_of_two(-e)[..., None]
    s["bounds"][page] = torch.stack([torch.floor(lower * scale), torch.ceil(upper * scale)], dim=2).to(torch.int8)
    s["exponents"][page] = e.to(torch.int8)


def _ranges(s):
    """Per sequence: first and past-the-last packed position, first page, number of pages."""
    case, lens = s["case"], s["lens"].long()
    room = lens - case["s_keep"] - case["s_sink"]
    n = torch.where(room >= case["s_flush"], torch.div(room, case["s_flush"], rounding_mode="floor") * case["s_flush"], 0)
    lo = torch.full_like(n, case["s_sink"])
    first = lo // PAGE
    return lo, lo + n, first, torch.where(n > 0, (lo + n - 1) // PAGE - first + 1, 0)


def _compensated(s):
    """q' = T_K^{-T} q in 64 bits, [batch, heads, group, 128]."""
    case = s["case"]
    q = s["Q"].double().view(s["batch"], case["n_kv"], -1, D)
    return torch.einsum("hij,bhgj->bhgi", s["T_inv"].double(), q)


def _plain_select(s):
    case, budget = s["case"], s["case"]["budget"]
    _, _, first, n = _ranges(s)
    p_max = s["max_pages"]
    index = first[:, None] + torch.arange(p_max, device="cuda")[None, :]
    there = torch.arange(p_max, device="cuda")[None, :] < n[:, None]                              # [batch, pages]
    page = torch.gather(s["table"][s["slot"].long()].long(), 1, index.clamp(max=p_max - 1)).clamp(min=0)
    bounds, e = s["bounds"][page], s["exponents"][page].int()                                     # [batch, pages, heads, 2, 128]
    q = _compensated(s)
    most = q.abs().amax(-1, keepdim=True)
    q_int = torch.round(q * (Q_MAX / most))
    # whole numbers below 2^53: exact in any order
    dot = torch.einsum("bphc,bhgc->bhgp", bounds[..., 0, :].double(), q_int.clamp(max=0)) + torch.einsum("bphc,bhgc->bhgp", bounds[..., 1, :].double(), q_int.clamp(min=0))
    unit = (most / Q_MAX * float(np.float32(1.0 / math.sqrt(D)))).float()
    score = dot.float() * _power_of_two(e).permute(0, 2, 1)[:, :, None, :] * unit
    score = score.masked_fill(~there[:, None, None, :], -math.inf)
    best = score.amax(-1, keepdim=True)
    key = (score - torch.where(torch.isfinite(best), best, 0.0)).amax(2)                          # [batch, heads, pages]
    _, ranked = torch.sort(key, dim=-1, descending=True, stable=True)
    ranked = torch.nn.functional.pad(ranked, (0, max(0, budget - p_max)), value=p_max)[..., :budget]
    taken = torch.arange(budget, device="cuda")[None, None, :] < n[:, None, None]
    listed_ = torch.where(taken, ranked, p_max).sort(dim=-1).values
    s["selected"].copy_(torch.where(listed_ < p_max, listed_ + first[:, None, None], -1))


def _plain_attention(s):
    case, batch, n_kv = s["case"], s["batch"], s["case"]["n_kv"]
    lo, hi, _, _ = _ranges(s)
    slot, lens, selected = s["slot"].long(), s["lens"].long(), s["selected"].long()
    page = torch.gather(s["table"][slot].long()[:, None, :].expand(-1, n_kv, -1), 2, selected.clamp(min=0))
    records = s["pages"][page, torch.arange(n_kv, device="cuda")[None, :, None]]                  # [batch, heads, selected, bytes]
    keys, values = (_read_vectors(records, case["bits"], side).view(batch, n_kv, -1, D) for side in (0, 1))
    pos = selected[..., None] * PAGE + torch.arange(PAGE, device="cuda")
    there = ((selected[..., None] >= 0) & (pos >= lo[:, None, None, None]) & (pos < hi[:, None, None, None])).view(batch, n_kv, -1)
    # windows: the first s_sink positions, and all from the packed range's end on
    n_sink = lens.clamp(max=case["s_sink"])
    w = torch.arange(case["s_sink"] + s["cap"], device="cuda")[None, :]
    recent = torch.where(hi > lo, hi, lo)[:, None] + w - n_sink[:, None]
    in_sink = w < n_sink[:, None]
    ring = s["ring"][slot[:, None], :, :, recent.clamp(min=0) % s["cap"]]                         # [batch, window, heads, 2, 128]
    window = torch.where(in_sink[:, :, None, None, None], s["sink"][slot[:, None], :, :, w.clamp(max=case["s_sink"] - 1)], ring).float().permute(0, 2, 3, 1, 4)
    there = torch.cat([there, (in_sink | (recent < lens[:, None]))[:, None, :].expand(-1, n_kv, -1)], dim=2)
    keys, values = torch.cat([keys, window[:, :, 0]], dim=2), torch.cat([values, window[:, :, 1]], dim=2)
    z = torch.einsum("bhgc,bhkc->bhgk", _compensated(s).float(), keys) / math.sqrt(D)
    p = torch.softmax(z.masked_fill(~there[:, :, None, :], -math.inf), dim=-1)
    s["O"].copy_(torch.einsum("bhgk,bhkc->bhgc", p, values).reshape(batch, -1, D))


def _plain_fork(s):
    case, src, dst = s["case"], s["src"].long(), s["dst"].long()
    table, refs, n = s["table"], s["refs"], s["n"]
    one = torch.ones((), dtype=torch.int32, device="cuda")
    # what the destinations held before is given back
    held = table[dst]
    refs.index_put_((held[held >= 0].long(),), -one, accumulate=True)
    rows = torch.where(torch.arange(s["max_pages"], device="cuda")[None, :] * PAGE < s["src_len"][:, None], table[src], -1)
    refs.index_put_((rows[rows >= 0].long(),), one, accumulate=True)
    table[dst] = rows
    # the windows' rows in use
    row, lens = torch.arange(s["cap"], device="cuda")[None, :], s["src_len"][:, None]
    s["ring"][dst] = torch.where((row < lens)[:, None, None, :, None], s["ring"][src], s["ring"][dst])
    row = torch.arange(case["s_sink"], device="cuda")[None, :]
    s["sink"][dst] = torch.where((row < lens)[:, None, None, :, None], s["sink"][src], s["sink"][dst])
    # the page of each copy's next token: a page of its own, the lowest free ones in order
    index = s["src_len"].long() // PAGE
    tail = s["src_len"] % PAGE != 0
    old = rows[torch.arange(n, device="cuda"), index]
    new = torch.nonzero(refs == 0)[:n, 0].int()
    table[dst, index] = new
    refs.index_put_((new.long(),), one, accumulate=True)
    refs.index_put_((old[tail].long(),), -one, accumulate=True)
    k = int(tail.sum())
    s["copies"].fill_(-1)
    s["copies"][0, :k], s["copies"][1, :k] = old[tail], new[tail]
    s["count"].fill_(k)
    _plain_copy(s, old[tail].long(), new[tail].long())


def _plain_copy(s, src, dst):
    s["pages"][dst] = s["pages"][src]
    s["bounds"][dst] = s["bounds"][src]
    s["exponents"][dst] = s["exponents"][src]


def _plain_compact(s):
    s["book"].copy_(s["start"])
    table, refs, gone = s["table"], s["refs"], s["gone"].long()
    held = table[gone]
    refs.index_put_((held[held >= 0].long(),), torch.full((), -1, dtype=torch.int32, device="cuda"), accumulate=True)
    table[gone] = -1
    live = int((refs > 0).sum())
    src, dst = live + torch.nonzero(refs[live:] > 0)[:, 0], torch.nonzero(refs[:live] == 0)[:, 0]
    moved = torch.arange(s["n_pages"], dtype=torch.int32, device="cuda")
    moved[src] = dst.int()
    refs[dst] = refs[src]
    refs[src] = 0
    table.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()], table))
    s["copies"].fill_(-1)
    s["copies"][0, :src.numel()], s["copies"][1, :src.numel()] = src.int(), dst.int()
    s["count"].fill_(src.numel())
    s["live"].fill_(live)
    _plain_copy(s, src, dst)


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _handles(s):
    """What a program keeps between calls: the cache's and the pool's description, workspaces."""
    from paper_2609_38121_b200 import binding as B
    case, ptr = s["case"], lambda t: t.data_ptr()  # noqa: E731
    T = s.get("T_inv")
    if T is None:
        T = torch.zeros((case["n_kv"], D, D), dtype=torch.float32, device="cuda")
    pages = s.get("pages")
    if pages is None:
        pages = torch.zeros((s["n_pages"], case["n_kv"], RECORD[case["bits"]]), dtype=torch.uint8, device="cuda")
    desc = B.wushkv_cache(n_q=case["n_q"], n_kv=case["n_kv"], d=D, bits=case["bits"], page_tokens=PAGE, s_sink=case["s_sink"], s_keep=case["s_keep"],
                          s_flush=case["s_flush"], boundary_lag=0, n_slots=s["n_slots"], max_pages=s["max_pages"], ring_cap=s["cap"], kappa_k=0.96, kappa_v=0.92,
                          sm_scale=1.0 / math.sqrt(D), quantizer=0, n_pages=s["n_pages"], pages=ptr(pages), page_table=ptr(s["table"]), sink_kv=ptr(s["sink"]),
                          ring_kv=ptr(s["ring"]), T_K=ptr(T), T_K_invT=ptr(T), dev_status=ptr(s["status"]))
    s.update(B=B, desc=desc, keep=(T, pages))
    if case["kind"] == "sparse":
        s["ws_bytes"] = B.sparse_workspace_bytes(desc, s["batch"], s["longest"], case["budget"])
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
    if case["kind"] in ("fork", "compact"):
        s["pool"] = B.wushkv_page_pool(n_slots=s["n_slots"], max_pages=s["max_pages"], n_pages=s["n_pages"], page_table=ptr(s["table"]), refs=ptr(s["refs"]),
                                       dev_status=ptr(s["status"]))
        s["ws_bytes"] = B.pages_workspace_bytes(s["pool"], s["batch"])
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")


def _own_pass(s):
    if "B" not in s:
        _handles(s)
    B, desc, kind = s["B"], s["desc"], s["case"]["kind"]
    if kind == "bounds":
        B.update_page_bounds(desc, s["batch"], s["slot"], s["lens"], s["cu"], s["max_new"], s["bounds"], s["exponents"])
    elif kind == "select":
        B.select_pages(desc, s["batch"], s["slot"], s["lens"], s["longest"], s["Q"], s["bounds"], s["exponents"], s["case"]["budget"], s["selected"])
    elif kind == "sparse":
        B.decode_attn_sparse(desc, s["batch"], s["slot"], s["lens"], s["longest"], s["Q"], s["bounds"], s["exponents"], s["case"]["budget"], s["selected"], s["O"],
                             s["ws"], s["ws_bytes"])
    elif kind == "fork":
        B.pages_fork(s["pool"], s["n"], s["src"], s["dst"], s["src_len"])
        B.copy_windows(desc, s["n"], s["src"], s["dst"], s["src_len"])
        B.pages_reserve(s["pool"], s["n"], s["dst"], s["src_len"], s["cu"], s["copies"][0], s["copies"][1], s["count"], s["ws"], s["ws_bytes"])
        B.copy_pages(desc, s["max_copies"], s["copies"][0], s["copies"][1], s["count"], s["bounds"], s["exponents"])
    else:
        s["book"].copy_(s["start"])
        B.pages_release(s["pool"], s["n"], s["gone"])
        B.pages_compact(s["pool"], s["copies"][0], s["copies"][1], s["count"], s["live"], s["ws"], s["ws_bytes"])
        B.copy_pages(desc, s["max_copies"], s["copies"][0], s["copies"][1], s["count"], s["bounds"], s["exponents"])


def run(s):
    kind = s["case"]["kind"]
    if own:
        _own_pass(s)
    elif kind == "bounds":
        _plain_bounds(s, s["slot"], s["lens"], s["cu"][1:] - s["cu"][:-1])
    elif kind in ("select", "sparse"):
        _plain_select(s)
        if kind == "sparse":
            _plain_attention(s)
    elif kind == "fork":
        _plain_fork(s)
    else:
        _plain_compact(s)
    if kind == "bounds":
        return dict(bounds=s["bounds"], exponents=s["exponents"])
    if kind == "select":
        return dict(selected=s["selected"])
    if kind == "sparse":
        return dict(selected=s["selected"], O=s["O"])
    state = dict(table=s["table"], refs=s["refs"], copies=s["copies"], count=s["count"], pages=s["pages"], bounds=s["bounds"], exponents=s["exponents"], status=s["status"])
    return dict(state, ring=s["ring"], sink=s["sink"]) if kind == "fork" else dict(state, live=s["live"])


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    n_q, n_kv, batch = case["n_q"], case["n_kv"], case["batch"]
    lens = _spread(case["ctx_lo"], case["ctx_hi"], batch, 1)
    record = RECORD[case["bits"]]
    keys = PAGE * (D * case["bits"] // 8 + 4)                # codes, step and offset of a page's keys
    if case["kind"] == "bounds":
        new = _spread(case["new_lo"], case["new_hi"], batch, 2)
        pages = sum(-(-n // PAGE) - (n - m) // PAGE for n, m in zip(lens, new))
        return dict(bytes=pages * n_kv * (keys + 2 * D + 1), flops=4.0 * pages * n_kv * PAGE * D)
    if case["kind"] in ("select", "sparse"):
        budget, group = case["budget"], n_q // n_kv
        bytes_, flops = n_kv * D * D * 4 + batch * n_q * D * 2 + batch * n_kv * budget * 4, 2.0 * batch * n_q * D * D
        for n in lens:
            room = n - case["s_keep"] - case["s_sink"]
            packed = room // case["s_flush"] * case["s_flush"] if room >= case["s_flush"] else 0
            pages = -(-(case["s_sink"] + packed) // PAGE) if packed else 0
            bytes_ += pages * n_kv * (2 * D + 1)
            flops += 4.0 * pages * n_q * D
            if case["kind"] == "sparse":
                window = n - packed
                bytes_ += n_kv * (min(budget, pages) * record + window * 4 * D) + n_q * D * 2
                flops += 4.0 * D * n_q * (min(PAGE * budget, packed) + window)
        return dict(bytes=bytes_, flops=flops)
    if case["kind"] == "fork":
        total = 0
        for n in lens:
            rows = min(n, case["s_sink"]) + min(n, case["s_keep"] + case["s_flush"] - 1)
            tail = n_kv * (record + 2 * D + 1) if n % PAGE else 0
            total += case["beams"] * 2 * (n_kv * rows * 4 * D + tail + 4 * -(-n // PAGE))
        return dict(bytes=total, flops=0.0)
    # half of what lies behind the live pages' number moves, as pages lie anywhere
    _, n_pages = _pool_pages(case)
    used = sum(-(-n // PAGE) for n in lens)
    live = used * (1.0 - case["ended"] / batch)
    return dict(bytes=2.0 * live * (1.0 - live / n_pages) * n_kv * (record + 2 * D + 1) + 8.0 * (_slots(case) * _pool_pages(case)[0] + n_pages), flops=0.0)


# ---- the same in 64 bits --------------------------------------------------------------------------------------------

def exact(case, seed):
    """From the unpacked codes, sequence by sequence and head by head; the page operators table entry by table entry.  None: copies of records."""
    s = prepare(case, seed)
    if case["kind"] == "fork":
        return _exact_fork(case, s)
    if case["kind"] == "compact":
        return _exact_compact(case, s)
    if case["kind"] == "bounds":
        return _exact_bounds(case, s, seed)
    selected = torch.full((s["batch"], case["n_kv"], case["budget"]), -1, dtype=torch.int32)
    O = torch.zeros((s["batch"], case["n_q"], D), dtype=torch.float64, device="cuda")
    if case["kind"] == "sparse":
        kc, km, vc, vm = (x.view(s["n_pages"], case["n_kv"], PAGE, -1) for x in _content(case, seed, s["n_pages"]))
    group, scale = case["n_q"] // case["n_kv"], 1.0 / math.sqrt(D)
    for b, n in enumerate(s["lens"].tolist()):
        room = n - case["s_keep"] - case["s_sink"]
        packed = room // case["s_flush"] * case["s_flush"] if room >= case["s_flush"] else 0
        n_pages = -(-(case["s_sink"] + packed) // PAGE) if packed else 0
        row = s["table"][b, :n_pages].long()
        pos = torch.arange(n, device="cuda")
        for h in range(case["n_kv"]):
            q = [s["T_inv"][h].double() @ s["Q"][b, j].double() for j in range(h * group, (h + 1) * group)]
            if case["kind"] == "sparse":
                k, v = (m[row, h, :, 1:].double() + m[row, h, :, :1].double() * c[row, h].double() for c, m in ((kc, km), (vc, vm)))
                low, up, e = _exact_page_bounds(k, torch.arange(n_pages, device="cuda"), n)
            else:
                low, up, e = s["bounds"][row, h, 0].double(), s["bounds"][row, h, 1].double(), s["exponents"][row, h].double()
            # whole-number scores, each rounded to 32 bits as the definition says
            gain = []
            for x in q:
                most = float(x.abs().max())
                x_int = torch.round(x * (Q_MAX / most))
                dot = (torch.where(x_int > 0, up, low) * x_int).sum(1)
                z = dot.float() * torch.pow(2.0, e).float() * torch.tensor(most / Q_MAX * float(np.float32(scale)), device="cuda", dtype=torch.float64).float()
                gain.append(z - z.max() if n_pages else z)
            key = torch.stack(gain).amax(0).tolist()
            chosen = sorted(sorted(range(n_pages), key=lambda p: (-key[p], p))[:case["budget"]])
            selected[b, h, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
            if case["kind"] == "select":
                continue
            keep = torch.zeros(n_pages * PAGE, dtype=torch.bool, device="cuda")
            keep.view(n_pages, PAGE)[torch.tensor(chosen, dtype=torch.long, device="cuda")] = True
            where = torch.nonzero(keep)[:, 0]
            where = where[(where >= case["s_sink"]) & (where < case["s_sink"] + packed)]
            front, back = pos[pos < case["s_sink"]], pos[pos >= case["s_sink"] + packed]
            parts = [(x.reshape(-1, D)[where], s["sink"][b, h, i, front].double(), s["ring"][b, h, i, back % s["cap"]].double()) for i, x in enumerate((k, v))]
            keys, values = (torch.cat(p) for p in parts)
            for j, x in enumerate(q):
                O[b, h * group + j] = torch.softmax(keys @ x * scale, dim=0) @ values
    selected = selected.cuda()
    return dict(selected=selected, O=O) if case["kind"] == "sparse" else dict(selected=selected)


def _exact_page_bounds(k, index, n):
    """Lower and upper bounds as whole numbers and their exponents, from one head's keys [pages, 64, 128] in 64 bits, rounded to 32 as stored."""
    k = k.float().double()
    beyond = (index[:, None] * PAGE + torch.arange(PAGE, device="cuda")[None, :] >= n)[..., None]
    low, up = k.masked_fill(beyond, math.inf).amin(1), k.masked_fill(beyond, -math.inf).amax(1)
    most = torch.maximum(low.abs(), up.abs()).amax(1)
    e = torch.full_like(most, -31.0)
    for step in range(60):
        e = torch.where(most > 127.0 * torch.pow(2.0, e), e + 1, e)
    grid = torch.pow(2.0, e)[:, None]
    return torch.floor(low / grid), torch.ceil(up / grid), e


def _exact_bounds(case, s, seed):
    kc, km, _, _ = (x.view(s["n_pages"], case["n_kv"], PAGE, -1) for x in _content(case, seed, s["n_pages"]))
    cu = s["cu"].tolist()
    for b, n in enumerate(s["lens"].tolist()):
        index = torch.arange((n - (cu[b + 1] - cu[b])) // PAGE, -(-n // PAGE), device="cuda")
        row = s["table"][b, index].long()
        for h in range(case["n_kv"]):
            low, up, e = _exact_page_bounds(km[row, h, :, 1:].double() + km[row, h, :, :1].double() * kc[row, h].double(), index, n)
            s["bounds"][row, h] = torch.stack([low, up], dim=1).to(torch.int8)
            s["exponents"][row, h] = e.to(torch.int8)
    return dict(bounds=s["bounds"], exponents=s["exponents"])


def _exact_fork(case, s):
    table, refs, ring, sink = s["table"].cpu().numpy(), s["refs"].cpu().numpy(), s["ring"].double(), s["sink"].double()
    copies, src, dst, lens = [], s["src"].tolist(), s["dst"].tolist(), s["src_len"].tolist()
    for a, b, n in zip(src, dst, lens):
        for i in range(-(-n // PAGE)):
            table[b, i] = table[a, i]
            refs[table[a, i]] += 1
        rows, first = min(n, s["cap"]), min(n, case["s_sink"])
        ring[b, :, :, :rows], sink[b, :, :, :first] = ring[a, :, :, :rows], sink[a, :, :, :first]
    free = [p for p in range(len(refs)) if refs[p] == 0]
    for b, n in zip(dst, lens):
        page = free.pop(0)
        if n % PAGE:
            copies.append((int(table[b, n // PAGE]), page))
            refs[table[b, n // PAGE]] -= 1
        table[b, n // PAGE] = page
        refs[page] = 1
    return dict(table=torch.from_numpy(table), refs=torch.from_numpy(refs), copies=_padded(copies, s), count=torch.tensor([len(copies)], dtype=torch.int32),
                pages=None, bounds=None, exponents=None, status=torch.zeros(1, dtype=torch.int32), ring=ring, sink=sink)


def _exact_compact(case, s):
    table, refs = s["table"].cpu().numpy(), s["refs"].cpu().numpy()
    for b in s["gone"].tolist():
        for i, page in enumerate(table[b]):
            if page >= 0:
                refs[page] -= 1
            table[b, i] = -1
    live = int((refs > 0).sum())
    copies = list(zip([p for p in range(live, len(refs)) if refs[p] > 0], [p for p in range(live) if refs[p] == 0]))
    for a, b in copies:
        refs[b], refs[a] = refs[a], 0
        table[table == a] = b
    return dict(table=torch.from_numpy(table), refs=torch.from_numpy(refs), copies=_padded(copies, s), count=torch.tensor([len(copies)], dtype=torch.int32),
                pages=None, bounds=None, exponents=None, status=torch.zeros(1, dtype=torch.int32), live=torch.tensor([live], dtype=torch.int32))


def _padded(copies, s):
    pairs = torch.full((2, s["max_copies"]), -1, dtype=torch.int32)
    if copies:
        pairs[:, :len(copies)] = torch.tensor(copies, dtype=torch.int32).T
    return pairs
