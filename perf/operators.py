"""Rotary positions, a paged 8-bit key/value cache and the attention that reads it, as measurable calls.

Three operators of a program that serves a looped (or any other) Transformer next to the sparse loops:

  table    flashloop.rope_table: cosines and sines of every position, with the scalings for long contexts
  rope     flashloop.rope: queries or keys rotated by their positions
  append   flashloop.paged_append: new keys (rotated on the way) and values into pages of 8-bit codes, with one
           scale per page and head
  attn     flashloop.paged_attn: the last positions of a ragged batch attend over such a cache, causally, with or
           without a sliding window and leading positions that stay visible

`own` false: the same in elementary torch operations.  Pages lie in the cache in a random order, as they do once
sequences have come and gone; keys have a few loud channels, as real keys do.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False


def listed():
    return [
        # the rotary table of a 128K context stretched fourfold: what a program makes once
        dict(name="table_128k", kind="table", n_pos=131072, rot=128, scaling="yarn", factor=4.0, orig=32768),
        # and of a small one, without scaling
        dict(name="table_4k", kind="table", n_pos=4096, rot=64, scaling="none", factor=1.0, orig=4096),
        # the queries of a 32K prompt, read out of a fused projection; the eight tokens of a decoding batch
        dict(name="rope_32k", kind="rope", T=32768, H=16, d=128, rot=128, layout="half", dtype="bf16", fused=1, n_pos=32768),
        dict(name="rope_token", kind="rope", T=8, H=16, d=128, rot=64, layout="interleaved", dtype="f16", fused=0,
             n_pos=32768),
        # prompts of uneven length written into empty pages, one of them continued from the middle of a page
        dict(name="append_prompts", kind="append", new="16384,9001,4096,3200,87", past="0,0,0,1000,0", Hkv=8, d=128, rot=128,
             layout="half", dtype="bf16", page=64, fmt="int8"),
        # one token for each of 32 sequences
        dict(name="append_tokens", kind="append", new="1," * 31 + "1", past="4000,17,640,1,2999,63,64,65," * 3 +
             "8000,100,200,300,400,500,600,0", Hkv=8, d=128, rot=128, layout="half", dtype="bf16", page=64, fmt="e4m3"),
        # decoding: one short context of 16 heads (latency), a ragged batch with grouped heads, one very long context,
        # four positions at once over a window with leading positions kept
        dict(name="decode_short", kind="attn", new="1", past="299", Hq=16, Hkv=16, d=128, rot=128, layout="half", dtype="bf16",
             page=64, fmt="int8", window=0, sink=0),
        dict(name="decode_batch", kind="attn", new="1," * 31 + "1",
             past="8191,700,5000,33,4095,8000,2048,1," * 3 + "6100,7777,120,4500,3500,900,8100,64", Hq=32, Hkv=8, d=128,
             rot=128, layout="half", dtype="bf16", page=64, fmt="int8", window=0, sink=0),
        dict(name="decode_128k", kind="attn", new="1", past="131071", Hq=32, Hkv=8, d=128, rot=128, layout="half",
             dtype="bf16", page=64, fmt="e4m3", window=0, sink=0),
        dict(name="verify_window", kind="attn", new="4," * 15 + "4", past="30000,29000,12345,900," * 4, Hq=16, Hkv=4, d=64,
             rot=32, layout="interleaved", dtype="f16", page=16, fmt="int8", window=4096, sink=4),
        # prompts: the whole of a 16K prompt of 16 heads; chunks of a batch that arrive at different lengths, windowed
        dict(name="prompt_16k", kind="attn", new="16384", past="0", Hq=16, Hkv=16, d=128, rot=128, layout="half",
             dtype="bf16", page=64, fmt="int8", window=0, sink=0),
        dict(name="chunks_ragged", kind="attn", new="1009,512,2000,1", past="15000,0,6001,9000", Hq=32, Hkv=8, d=128,
             rot=64, layout="half", dtype="bf16", page=32, fmt="e4m3", window=8192, sink=64),
    ]


# ---- drawn cases: the ranges between and around the listed ones -------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed kinds: 1..48 sequences, 1..16384 new and up to 131072 cached positions (any, not only round
    ones), heads of 64 or 128 with groups of 1..8, pages of 16..128, both code types and both 16-bit types."""
    kind = rng.choice(("table", "rope", "append", "append", "decode", "decode", "decode", "prompt", "prompt"))
    d = rng.choice((64, 128))
    rot = rng.choice((d, d, d // 2, 16))
    layout, dtype = rng.choice(("half", "interleaved")), rng.choice(("bf16", "f16"))
    if kind == "table":
        scaling = rng.choice(("none", "linear", "ntk", "yarn"))
        return dict(kind=kind, n_pos=_log(rng, 256, 131072), rot=rng.choice((16, 32, 64, 96, 128)), scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.uniform(1.5, 16.0), orig=rng.choice((2048, 4096, 8192, 32768)))
    if kind == "rope":
        return dict(kind=kind, T=_log(rng, 1, 32768), H=rng.choice((1, 2, 5, 8, 12, 16)), d=d, rot=rot, layout=layout,
                    dtype=dtype, fused=rng.randint(0, 1), n_pos=32768)
    page, fmt = rng.choice((16, 32, 64, 128)), rng.choice(("int8", "e4m3"))
    Hkv = rng.choice((1, 2, 4, 5, 8))
    some = lambda n, lo, hi: ",".join(str(_log(rng, lo, hi)) for _ in range(n))  # noqa: E731
    if kind == "append":
        B = rng.randint(1, 32)
        new = rng.choice((",".join("1" * B), some(B, 1, max(2, 32768 // B))))
        return dict(kind=kind, new=new, past=some(B, 1, 8192), Hkv=Hkv, d=d, rot=rot, layout=layout, dtype=dtype,
                    page=page, fmt=fmt)
    window, sink = rng.choice(((0, 0), (0, 0), (_log(rng, 64, 8192), rng.choice((0, 4, 64)))))
    if kind == "decode":
        B = _log(rng, 1, 48)
        n = rng.choice((1, 1, 1, 2, 4))
        return dict(kind="attn", new=",".join([str(n)] * B), past=some(B, 1, 131072 // B), Hq=Hkv * rng.choice((1, 2, 4, 8)),
                    Hkv=Hkv, d=d, rot=rot, layout=layout, dtype=dtype, page=page, fmt=fmt, window=window, sink=sink)
    B = rng.randint(1, 6)
    return dict(kind="attn", new=some(B, 8, 8192 // B), past=some(B, 1, 8192), Hq=Hkv * rng.choice((1, 2, 3)),
                Hkv=Hkv, d=d, rot=rot, layout=layout, dtype=dtype, page=page, fmt=fmt, window=window, sink=sink)


# ---- what a case is ----------------------------------------------------------------------------------------
def _ints(text):
    return [int(x) for x in text.split(",") if x]


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _code_dtype(case):
    return torch.int8 if case["fmt"] == "int8" else torch.float8_e4m3fn


BASE = 10000.0                    # of the frequencies
YARN_LOW, YARN_HIGH = 1.0, 32.0   # turns within the original context between which a frequency is stretched in part


def _frequencies(rot, scaling, factor, orig, base):
    """fp64 frequencies of the pairs and the factor of the cosines and sines."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    base = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base
    f = torch.pow(torch.tensor(base, dtype=torch.float64, device="cuda"), -2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        turns = orig * f / (2.0 * math.pi)
        keep = ((turns - YARN_LOW) / (YARN_HIGH - YARN_LOW)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
    return f, 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def _plain_table(n_pos, rot, scaling="none", factor=1.0, orig=0, base=BASE):
    f, m = _frequencies(rot, scaling, factor, orig, base)
    angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return (torch.stack((angle.cos(), angle.sin()), dim=-1) * m).float()


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(g, *shape):
    """Keys with a few loud channels, the same ones at every position."""
    loud = torch.where(torch.rand(shape[-1], generator=g, device="cuda") < 0.06, 4.0, 1.0)
    return _normal(g, *shape) * loud


def _batch(case, g, spare=3):
    """Offsets of the new positions, lengths, and a block table over pages in random order (-1: no page)."""
    new, past = _ints(case["new"]), _ints(case["past"])
    lens = [a + b for a, b in zip(new, past)]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    pages = [-(-n // case["page"]) for n in lens]
    total = sum(pages) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(g.initial_seed()))).tolist()
    table = torch.full((len(new), max(pages) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    put = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    return SimpleNamespace(cu=put(cu), lens=put(lens), table=table.cuda(), pages=total, T=cu[-1], max_q=max(new),
                           max_len=max(lens))


def _stored(x, fmt):
    """Codes and scales of whole pages x [pages, heads, page, d]."""
    amax = x.abs().amax(dim=(2, 3))
    if fmt == "int8":
        s = amax / 127.0
        return torch.round(x / s[:, :, None, None]).clamp(-127, 127).to(torch.int8), s
    s = torch.exp2(torch.ceil(torch.log2(amax / 448.0)))
    return (x / s[:, :, None, None]).to(torch.float8_e4m3fn), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    if kind == "table":
        return SimpleNamespace(case=case, base=BASE * (1 + int(seed) % 50))      # a model's own base
    if kind == "rope":
        T, H, d = case["T"], case["H"], case["d"]
        x = _normal(g, T, (3 if case["fused"] else 1) * H * d).to(_dtype(case))[:, :H * d].view(T, H, d)
        pos = torch.randint(0, case["n_pos"], (T,), generator=g, device="cuda", dtype=torch.int32) if T < 1024 else \
            torch.arange(T, device="cuda", dtype=torch.int32)
        return SimpleNamespace(case=case, x=x, pos=pos, table=_plain_table(case["n_pos"], case["rot"]))
    b = _batch(case, g)
    Hkv, d, page = case["Hkv"], case["d"], case["page"]
    kc, ks = _stored(_keys(g, b.pages, Hkv, page, d), case["fmt"])
    vc, vs = _stored(_normal(g, b.pages, Hkv, page, d), case["fmt"])
    s = SimpleNamespace(case=case, b=b, kc=kc, vc=vc, ks=ks, vs=vs,
                        table=_plain_table(b.table.shape[1] * page, case["rot"]))
    if kind == "append":
        # the keys and values as a fused projection leaves them, one after the other in a row
        kv = torch.cat((_keys(g, b.T, Hkv, d) * 1.3, _normal(g, b.T, Hkv, d) * 1.3), dim=1).to(_dtype(case))
        s.k, s.v = kv[:, :Hkv], kv[:, Hkv:]
    else:
        s.q = _normal(g, b.T, case["Hq"], d).to(_dtype(case))
    return s


# ---- the calls ---------------------------------------------------------------------------------------------
def run(s):
    c = s.case
    if own:
        from paper_2609_29812_amd import flashloop as fl
        if c["kind"] == "table":
            return fl.rope_table(c["n_pos"], c["rot"], base=s.base, scaling=c["scaling"], factor=c["factor"],
                                 orig_len=c["orig"], low=YARN_LOW, high=YARN_HIGH)
        if c["kind"] == "rope":
            return fl.rope(s.x, s.table, s.pos, layout=c["layout"])
        if c["kind"] == "append":
            fl.paged_append(s.k, s.v, s.b.cu, s.b.lens, s.b.table, s.kc, s.vc, s.ks, s.vs, table=s.table,
                            layout=c["layout"])
            return s.kc, s.ks, s.vc, s.vs
        return fl.paged_attn(s.q, s.b.cu, s.b.lens, s.b.table, s.kc, s.vc, s.ks, s.vs, table=s.table, layout=c["layout"],
                             window=c["window"], n_sink=c["sink"], max_q=s.b.max_q, max_len=s.b.max_len)
    if c["kind"] == "table":
        return _plain_table(c["n_pos"], c["rot"], c["scaling"], c["factor"], c["orig"], s.base)
    if c["kind"] == "rope":
        return _plain_rotate(s.x.float(), s.table[s.pos.long()], c["layout"]).to(s.x.dtype)
    if c["kind"] == "append":
        return _plain_append(s)
    return _plain_attn(s)


def _plain_rotate(x, cs, layout):
    """x [T, H, d], cs [T, rot / 2, 2], in the type of x."""
    half = cs.shape[1]
    cos, sin = cs[:, None, :, 0].to(x.dtype), cs[:, None, :, 1].to(x.dtype)
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "half":
        a, b = r[..., :half], r[..., half:]
        return torch.cat((a * cos - b * sin, a * sin + b * cos, rest), dim=-1)
    a, b = r[..., 0::2], r[..., 1::2]
    return torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2), rest), dim=-1)


def _places(b):
    """Sequence and position of every new token."""
    t = torch.arange(b.T, device="cuda")
    seq = torch.searchsorted(b.cu[1:].long(), t, right=True)
    return seq, b.lens[seq].long() - (b.cu[seq + 1].long() - t)


def _coded(y, fmt):
    """Bytes of the codes of y, to the nearest (ties to even)."""
    if fmt == "int8":
        return torch.round(y).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return y.float().to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    c, b = s.case, s.b
    page = c["page"]
    seq, pos = _places(b)
    pid, slot = b.table[seq, pos // page].long(), pos % page
    past = (b.lens - (b.cu[1:] - b.cu[:-1])).long()            # lengths before
    last = b.table[torch.arange(past.numel(), device="cuda"), past // page].long()     # pages of the first new positions
    went_on = (past % page > 0)[:, None]                       # they hold earlier positions
    touched = torch.zeros(b.pages, 1, dtype=torch.bool, device="cuda").index_fill_(0, pid, True)
    # the rotation in 64 bits, rounded once: a code next to a border goes by it
    k = _plain_rotate(s.k.double(), s.table[pos], c["layout"]).float()
    for x, codes, scale in ((k, s.kc, s.ks), (s.v.float(), s.vc, s.vs)):
        most = torch.zeros_like(scale).index_reduce_(0, pid, x.abs().amax(dim=-1), "amax")
        if c["fmt"] == "int8":
            need = most / 127.0
        else:
            m, e = torch.frexp(most)                           # most = m 2^e, m in [0.5, 1): 448 = 0.875 * 2^9
            need = torch.ldexp(torch.ones_like(most), e - 9 + (m > 0.875).int())
        # pages that held positions before: the scale grows by the least power of two that covers the new ones
        m, e = torch.frexp(need[last].double() / scale[last].double())
        grow = torch.where(went_on, (e - (m == 0.5).int()).clamp(min=0), 0).float()
        kept = torch.where(went_on, scale[last] * torch.exp2(grow), need[last])
        held = codes[last].float() * torch.exp2(-grow)[:, :, None, None]
        codes.view(torch.uint8)[last] = _coded(held, c["fmt"])
        scale.copy_(torch.where(touched, need, scale))
        scale[last] = kept
        codes.view(torch.uint8)[pid, :, slot] = _coded(x.double() / scale[pid].double()[:, :, None], c["fmt"])
    return s.kc, s.ks, s.vc, s.vs


def _plain_attn(s):
    c, b = s.case, s.b
    page, Hq, Hkv, d = c["page"], c["Hq"], c["Hkv"], c["d"]
    G, B, n_pages = Hq // Hkv, b.lens.numel(), -(-b.max_len // page)
    seq, pos = _places(b)
    first = b.lens.long() - (b.cu[1:] - b.cu[:-1]).long()
    at = pos - first[seq]                                      # place among the sequence's new positions
    q = _plain_rotate(s.q.float(), s.table[pos], c["layout"])
    rows = torch.zeros(B, b.max_q, Hq, d, device="cuda").index_put_((seq, at), q)
    rows = rows.view(B, b.max_q, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, b.max_q * G, d)
    pid = b.table[:, :n_pages].long().clamp(min=0)

    def read(codes, scale):
        x = codes[pid].float() * scale[pid][:, :, :, None, None]
        return x.transpose(1, 2).reshape(B, Hkv, n_pages * page, d)

    k_t = read(s.kc, s.ks).transpose(2, 3).contiguous()
    x = torch.matmul(rows, k_t) / math.sqrt(d)
    i = (first[:, None] + torch.arange(b.max_q, device="cuda"))[:, None, :, None]      # positions of the rows
    j = torch.arange(n_pages * page, device="cuda")
    seen = j <= i
    if c["window"]:
        seen &= (j > i - c["window"]) | (j < c["sink"])
    x = x.view(B, Hkv, b.max_q, G, -1).masked_fill_(~seen[:, :, :, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, b.max_q * G, -1), read(s.vc, s.vs)).view(B, Hkv, b.max_q, G, d) / total
    return o[seq, :, at].reshape(b.T, Hq, d).to(s.q.dtype)


# ---- the least work ----------------------------------------------------------------------------------------
def _seen(n, past, window, sink):
    """Pairs of a new position and a position that it sees, and the positions that any of them sees."""
    if not window:
        return sum(range(past + 1, past + n + 1)), past + n
    pairs = 0
    for i in range(past, past + n):
        near = min(i + 1, window)
        pairs += near + min(sink, i + 1 - near)
    first = max(0, past - window + 1)
    return pairs, past + n - first + min(sink, first)


def work(case):
    kind = case["kind"]
    if kind == "table":
        return {"bytes": case["n_pos"] * case["rot"] * 4, "flops": 0}
    if kind == "rope":
        return {"bytes": 2 * 2 * case["T"] * case["H"] * case["d"] + min(case["T"], case["n_pos"]) * case["rot"] * 4,
                "flops": 3 * case["T"] * case["H"] * case["rot"]}
    new, past = _ints(case["new"]), _ints(case["past"])
    Hkv, d = case["Hkv"], case["d"]
    if kind == "append":
        pages = sum((n + p - 1) // case["page"] - p // case["page"] + 1 for n, p in zip(new, past))
        positions = min(sum(new), max(n + p for n, p in zip(new, past)))
        return {"bytes": sum(new) * Hkv * d * 2 * 3 + pages * Hkv * 8 + positions * case["rot"] * 4,
                "flops": 3 * sum(new) * Hkv * case["rot"]}
    seen = [_seen(n, p, case["window"], case["sink"]) for n, p in zip(new, past)]
    held = sum(u for _, u in seen)
    positions = min(sum(new), max(n + p for n, p in zip(new, past)))
    return {"bytes": held * Hkv * d * 2 + sum(-(-u // case["page"]) for _, u in seen) * Hkv * 8 +
            sum(new) * case["Hq"] * 4 * d + positions * case["rot"] * 4,
            "flops": 4 * d * case["Hq"] * sum(p for p, _ in seen)}


# ---- the definition in 64 bits -----------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"table": _exact_table, "rope": _exact_rope, "append": _exact_append, "attn": _exact_attn}[case["kind"]](s)


def _exact_table(s):
    c = s.case
    rot, factor = c["rot"], c["factor"]
    e = np.arange(0, rot, 2, dtype=np.float64) / rot
    f = (s.base * (factor ** (rot / (rot - 2.0)) if c["scaling"] == "ntk" else 1.0)) ** -e
    m = 1.0
    if c["scaling"] == "linear":
        f = f / factor
    elif c["scaling"] == "yarn":
        share = np.clip((c["orig"] * f / (2 * np.pi) - YARN_LOW) / (YARN_HIGH - YARN_LOW), 0, 1)
        f, m = f * (share + (1 - share) / factor), 1 + math.log(factor) / 10
    angle = np.multiply.outer(np.arange(c["n_pos"], dtype=np.float64), f)
    return np.stack((m * np.cos(angle), m * np.sin(angle)), axis=-1)


def _turned(x, cs, layout):
    """Rotation as complex products: x [T, H, d] and cs [T, rot / 2, 2] in 64 bits."""
    half = cs.shape[1]
    y = x.double().clone()
    turn = torch.view_as_complex(cs.double().contiguous())[:, None]
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rope(s):
    return _turned(s.x, s.table[s.pos.long()], s.case["layout"])


def _exact_append(s):
    c = s.case
    page, eight = c["page"], c["fmt"] == "int8"
    cu, lens, table = s.b.cu.tolist(), s.b.lens.tolist(), s.b.table.tolist()
    kc, vc = s.kc.double(), s.vc.double()

    def code(y):
        return torch.round(y) if eight else y.float().to(torch.float8_e4m3fn).double()   # (a power of two: y is exact)

    for b, n in enumerate(lens):
        at, end = n - (cu[b + 1] - cu[b]), n
        while at < end:
            stop = min(end, (at // page + 1) * page)
            rows = slice(cu[b] + at - (n - (cu[b + 1] - cu[b])), cu[b] + stop - (n - (cu[b + 1] - cu[b])))
            p, lo = table[b][at // page], at % page
            k = _turned(s.k[rows], s.table[at:stop], c["layout"]).float()
            for x, codes, scale in ((k, kc, s.ks), (s.v[rows].float(), vc, s.vs)):
                most = x.abs().amax(dim=(0, 2)).double()
                if eight:
                    need = (most / 127.0).float().double()
                else:
                    e = torch.ceil(torch.log2(most / 448.0))
                    need = torch.exp2(e - (most <= 448.0 * torch.exp2(e - 1)).double() + (most > 448.0 * torch.exp2(e)).double())
                if lo:
                    kept = scale[p].double()
                    for _ in range(40):
                        less = kept < need
                        codes[p] = torch.where(less[:, None, None], codes[p] * 0.5, codes[p])
                        kept = torch.where(less, kept * 2.0, kept)
                    codes[p] = code(codes[p])
                    need = kept
                scale[p] = need.float()
                codes[p][:, lo:lo + stop - at] = code(x.double() / scale[p].double()[:, None]).transpose(0, 1)
            at = stop
    whole = (lambda x: x.to(torch.int8)) if eight else (lambda x: x)
    return whole(kc), s.ks.double(), whole(vc), s.vs.double()


def _exact_attn(s):
    c = s.case
    Hq, Hkv, d, page = c["Hq"], c["Hkv"], c["d"], c["page"]
    G = Hq // Hkv
    o = torch.zeros(s.b.T, Hq, d, dtype=torch.float64, device="cuda")
    cu, lens = s.b.cu.tolist(), s.b.lens.tolist()
    for b, n in enumerate(lens):
        rows = slice(cu[b], cu[b + 1])
        i = torch.arange(n - (cu[b + 1] - cu[b]), n, device="cuda")
        j = torch.arange(n, device="cuda")
        hidden = j[None] > i[:, None]
        if c["window"]:
            hidden = hidden | ((j[None] <= i[:, None] - c["window"]) & (j[None] >= c["sink"]))
        q = _turned(s.q[rows], s.table[i], c["layout"])
        pid = s.b.table[b, :-(-n // page)].long()
        for h in range(Hkv):
            k, v = ((codes[pid, h].double() * scale[pid, h].double()[:, None, None]).reshape(-1, d)[:n]
                    for codes, scale in ((s.kc, s.ks), (s.vc, s.vs)))
            for e in range(h * G, h * G + G):
                x = (q[:, e] @ k.t().contiguous()) * d ** -0.5
                x[hidden] = -math.inf
                o[rows, e] = torch.softmax(x, dim=1) @ v
    return o
