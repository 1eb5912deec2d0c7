"""Attention over packed prompts, and a paged key/value cache in 4 bits, as measurable calls.

Four operators of a program that takes prompts in, keeps them in 4 bits and answers from there:

  packed  flashloop.packed_attn: causal attention of whole prompts of different lengths, packed one after the other, with
          grouped heads, with or without a sliding window and leading positions that stay visible
  append  flashloop.paged4_append: new keys (rotated on the way) and values into pages of 4-bit codes, in groups of 32
          channels; the rows that the codes stand for come back for the prompt's own attention
  read    flashloop.paged4_read: positions of a ragged batch back out of such a cache, as rows
  attn    flashloop.paged4_attn: the last positions of a ragged batch attend over such a cache

`own` false: the same in elementary torch operations.  Pages lie in the cache in a random order, as they do once
sequences have come and gone; keys have a few loud channels, as real keys do.
"""
import math
from types import SimpleNamespace

import torch

own = False

GROUP = 32                        # channels of a position and head that share a scale
MOST = 32768.0                    # magnitudes above count as this


def listed():
    return [
        # whole prompts: one short one (latency), one of 16K positions, six of very uneven length with grouped heads out of a
        # fused projection, half-width heads with a window and leading positions that stay visible
        dict(name="packed_short", kind="packed", new="300", Hq=16, Hkv=16, d=128, dtype="bf16", window=0, sink=0, fused=0),
        dict(name="packed_16k", kind="packed", new="16384", Hq=16, Hkv=16, d=128, dtype="bf16", window=0, sink=0, fused=0),
        dict(name="packed_ragged", kind="packed", new="5000,1,777,2048,333,4096", Hq=32, Hkv=8, d=128, dtype="bf16", window=0,
             sink=0, fused=1),
        dict(name="packed_window", kind="packed", new="9001,4096,1500", Hq=12, Hkv=4, d=64, dtype="f16", window=1024, sink=4,
             fused=1),
        # prompts of uneven length written into pages, one of them continued from the middle of a page; one token for each of
        # 32 sequences
        dict(name="append4_prompts", kind="append", new="16384,9001,4096,3200,87", past="0,0,0,1000,0", Hkv=8, d=128, rot=128,
             layout="half", dtype="bf16", page=64, fmt="int4"),
        dict(name="append4_tokens", kind="append", new="1," * 31 + "1", past="4000,17,640,1,2999,63,64,65," * 3 +
             "8000,100,200,300,400,500,600,0", Hkv=8, d=128, rot=64, layout="interleaved", dtype="f16", page=64, fmt="e2m1"),
        # a whole cache back as rows, for the loops that read states; the last positions of a few sequences
        dict(name="read4_32k", kind="read", new="20000,8000,4001,767", past="0,0,0,0", Hkv=8, d=128, dtype="bf16", page=64,
             fmt="int4"),
        dict(name="read4_tail", kind="read", new="64,64,64,64,64,64,64,33", past="500,4000,77,0,1,1200,31,900", Hkv=8, d=64,
             dtype="f16", page=16, fmt="e2m1"),
        # decoding: one short context of 16 heads (latency), a ragged batch with grouped heads, one very long context
        dict(name="decode4_short", kind="attn", new="1", past="299", Hq=16, Hkv=16, d=128, rot=128, layout="half", dtype="bf16",
             page=64, fmt="int4", window=0, sink=0),
        dict(name="decode4_batch", kind="attn", new="1," * 31 + "1",
             past="8191,700,5000,33,4095,8000,2048,1," * 3 + "6100,7777,120,4500,3500,900,8100,64", Hq=32, Hkv=8, d=128,
             rot=128, layout="half", dtype="bf16", page=64, fmt="int4", window=0, sink=0),
        dict(name="decode4_128k", kind="attn", new="1", past="131071", Hq=32, Hkv=8, d=128, rot=64, layout="interleaved",
             dtype="f16", page=64, fmt="e2m1", window=0, sink=0),
        # chunks of a batch that arrive at different lengths
        dict(name="chunks4_ragged", kind="attn", new="1009,512,2000,1", past="15000,0,6001,9000", Hq=32, Hkv=8, d=128,
             rot=128, layout="half", dtype="bf16", page=32, fmt="int4", window=8192, sink=64),
    ]


# ---- drawn cases: the ranges between and around the listed ones -------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed kinds: 1..48 sequences, 1..16384 new and up to 131072 cached positions (any, not only round
    ones), heads of 64 or 128 with groups of 1..8, pages of 16..128, both formats and both 16-bit types."""
    kind = rng.choice(("packed", "packed", "packed", "append", "append", "read", "decode", "decode", "decode", "chunk"))
    d, dtype = rng.choice((64, 128)), rng.choice(("bf16", "f16"))
    some = lambda n, lo, hi: ",".join(str(_log(rng, lo, hi)) for _ in range(n))  # noqa: E731
    window, sink = rng.choice(((0, 0), (0, 0), (_log(rng, 64, 8192), rng.choice((0, 4, 64)))))
    Hkv = rng.choice((1, 2, 4, 5, 8))
    if kind == "packed":
        B = _log(rng, 1, 16)
        return dict(kind=kind, new=some(B, 1, 11000 // B), Hq=Hkv * rng.choice((1, 2, 3, 4)), Hkv=Hkv, d=d, dtype=dtype,
                    window=window, sink=sink, fused=rng.randint(0, 1))
    rot, layout = rng.choice((d, d, d // 2, 16)), rng.choice(("half", "interleaved"))
    page, fmt = rng.choice((16, 32, 64, 128)), rng.choice(("int4", "e2m1"))
    if kind in ("append", "read"):
        B = rng.randint(1, 32)
        new = rng.choice((",".join("1" * B), some(B, 1, max(2, 32768 // B))))
        case = dict(kind=kind, new=new, past=some(B, 1, 8192), Hkv=Hkv, d=d, dtype=dtype, page=page, fmt=fmt)
        return dict(case, rot=rot, layout=layout) if kind == "append" else case
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


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(g, *shape):
    """Keys with a few loud channels, the same ones at every position."""
    loud = torch.where(torch.rand(shape[-1], generator=g, device="cuda") < 0.06, 4.0, 1.0)
    return _normal(g, *shape) * loud


def _turns(n_pos, rot):
    """Cosines and sines of every position."""
    f = torch.pow(torch.tensor(10000.0, dtype=torch.float64, device="cuda"),
                  -2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack((angle.cos(), angle.sin()), dim=-1).float()


def _put(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


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
    return SimpleNamespace(cu=_put(cu), lens=_put(lens), table=table.cuda(), pages=total, T=cu[-1], max_q=max(new),
                           max_len=max(lens))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, Hkv, d = case["kind"], case["Hkv"], case["d"]
    if kind == "packed":
        new, Hq = _ints(case["new"]), case["Hq"]
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        parts = [_normal(g, cu[-1], Hq, d), _keys(g, cu[-1], Hkv, d), _normal(g, cu[-1], Hkv, d)]
        if case["fused"]:         # queries, keys and values as a fused projection leaves them, one after the other in a row
            whole = torch.cat(parts, dim=1).to(_dtype(case))
            parts = [whole[:, :Hq], whole[:, Hq:Hq + Hkv], whole[:, Hq + Hkv:]]
        q, k, v = (x.to(_dtype(case)) for x in parts)
        return SimpleNamespace(case=case, q=q, k=k, v=v, cu=_put(cu), B=len(new), max_q=max(new))
    b = _batch(case, g)
    page = case["page"]
    kc, km = _stored(_keys(g, b.pages, Hkv, page, d), case["fmt"])
    vc, vm = _stored(_normal(g, b.pages, Hkv, page, d), case["fmt"])
    s = SimpleNamespace(case=case, b=b, kc=kc, vc=vc, km=km, vm=vm)
    if kind != "read":
        s.table = _turns(b.table.shape[1] * page, case["rot"])
    if kind == "append":
        # the keys and values as a fused projection leaves them, one after the other in a row
        kv = torch.cat((_keys(g, b.T, Hkv, d) * 1.3, _normal(g, b.T, Hkv, d) * 1.3), dim=1).to(_dtype(case))
        s.k, s.v = kv[:, :Hkv], kv[:, Hkv:]
    if kind == "attn":
        s.q = _normal(g, b.T, case["Hq"], d).to(_dtype(case))
    return s


# ---- the calls ---------------------------------------------------------------------------------------------
def run(s):
    c = s.case
    if own:
        from paper_2609_29812_amd import flashloop as fl
        if c["kind"] == "packed":
            return fl.packed_attn(s.q, s.k, s.v, s.cu, window=c["window"], n_sink=c["sink"], max_k=s.max_q)
        if c["kind"] == "append":
            k_rows, v_rows = torch.empty(s.k.shape, dtype=s.k.dtype, device="cuda"), torch.empty(s.v.shape, dtype=s.v.dtype, device="cuda")
            fl.paged4_append(s.k, s.v, s.b.cu, s.b.lens, s.b.table, s.kc, s.vc, s.km, s.vm, table=s.table, layout=c["layout"],
                             k_rows=k_rows, v_rows=v_rows)
            return (k_rows, v_rows, s.km, s.vm) if c["fmt"] == "int4" else (k_rows, v_rows)
        if c["kind"] == "read":
            return fl.paged4_read(s.b.cu, s.b.lens, s.b.table, s.kc, s.vc, s.km, s.vm, s.b.T, dtype=_dtype(c))
        return fl.paged4_attn(s.q, s.b.cu, s.b.lens, s.b.table, s.kc, s.vc, s.km, s.vm, table=s.table, layout=c["layout"],
                              window=c["window"], n_sink=c["sink"], max_q=s.b.max_q, max_len=s.b.max_len)
    if c["kind"] == "packed":
        return _plain_packed(s)
    if c["kind"] == "append":
        return _plain_append(s)
    if c["kind"] == "read":
        seq, pos = _places(s.b)
        pid, slot = s.b.table[seq, pos // c["page"]].long(), pos % c["page"]
        return tuple(_values(codes[pid, :, slot], meta[pid, :, slot]).to(_dtype(c)) for codes, meta in ((s.kc, s.km), (s.vc, s.vm)))
    return _plain_attn(s)


def _half_down(x):
    """Largest fp16 number that is at most x (64 bits, |x| <= 32768)."""
    h = x.to(torch.float16)
    bits = h.view(torch.int16).int()
    lower = torch.where(bits == 0, torch.full_like(bits, -32767), torch.where(bits > 0, bits - 1, bits + 1))
    down = torch.where(h == 0, torch.full_like(bits, -32767), lower).to(torch.int16).view(torch.float16)
    return torch.where(h.double() > x, down, h) + 0.0


def _stored(x, fmt):
    """Codes [..., d / 2] (channel 2 j in the low four bits of byte j) and the groups' numbers of values x [..., d]: int4 fp16
    (scale, zero), e2m1 exponents + 127 in 8 bits.  Borders are decided in 64 bits."""
    g = x.double().clamp(-MOST, MOST).unflatten(-1, (-1, GROUP))
    if fmt == "int4":
        lo, hi = g.amin(dim=-1), g.amax(dim=-1)
        zero = _half_down(lo)
        scale = -_half_down(-(hi - zero.double()) / 15.0) + 0.0
        by = torch.where(scale > 0, scale, 1.0).double()[..., None]
        c = torch.round((g - zero.double()[..., None]) / by).clamp(0, 15)
        c = torch.where(scale[..., None] > 0, c, 0.0).to(torch.uint8)
        meta = torch.stack((scale, zero), dim=-1)
    else:
        most = g.abs().amax(dim=-1)
        m, e = torch.frexp(most)                       # most = m 2^e, m in [0.5, 1): 6 = 0.75 * 2^3
        e = torch.where(most > 0, e - 3 + (m > 0.75).int(), -23).clamp(min=-23)
        y = torch.ldexp(g.abs(), -e[..., None])
        # 0, 0.5, 1, 1.5, 2, 3, 4, 6: to the nearest, ties to the even code
        c = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
        c = c + torch.signbit(g) * 8
        meta = (e + 127).to(torch.uint8)
    c = c.to(torch.uint8).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), meta


def _values(codes, meta):
    """fp32 values of codes [..., d / 2]."""
    c = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).unflatten(-1, (-1, GROUP))
    if meta.dtype == torch.float16:
        x = c.float() * meta[..., 0:1].float() + meta[..., 1:2].float()
    else:
        level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
        x = level[(c & 7).long()] * torch.where(c > 7, -1.0, 1.0) * torch.exp2(meta.float() - 127.0)[..., None]
    return x.flatten(-2)


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


def _plain_append(s):
    c, b = s.case, s.b
    seq, pos = _places(b)
    pid, slot = b.table[seq, pos // c["page"]].long(), pos % c["page"]
    # the rotation in 64 bits, rounded once: a code next to a border goes by it
    k = _plain_rotate(s.k.double(), s.table[pos], c["layout"]).float()
    rows = []
    for x, codes, meta in ((k, s.kc, s.km), (s.v.float(), s.vc, s.vm)):
        w, m = _stored(x, c["fmt"])
        codes[pid, :, slot] = w
        meta[pid, :, slot] = m
        rows.append(_values(w, m).to(_dtype(c)))
    return (*rows, s.km, s.vm) if c["fmt"] == "int4" else tuple(rows)


def _attend(rows, k, v, seen, d):
    """rows [B, Hkv, R G, d], k and v [B, Hkv, L, d] in fp32, seen [B or 1, 1, R, L] -> [B, Hkv, R, G, d]."""
    B, Hkv, RG, _ = rows.shape
    R = seen.shape[2]
    x = torch.matmul(rows, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    x = x.view(B, Hkv, R, RG // R, -1).masked_fill_(~seen[:, :, :, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p.view(B, Hkv, RG, -1), v).view(B, Hkv, R, RG // R, d) / total


def _plain_packed(s):
    c, cu = s.case, s.cu.long()
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    G, N = Hq // Hkv, s.max_q
    t = torch.arange(s.q.shape[0], device="cuda")
    seq = torch.searchsorted(cu[1:], t, right=True)
    at = t - cu[seq]
    lay = lambda x: torch.zeros(s.B, N, *x.shape[1:], device="cuda").index_put_((seq, at), x.float())  # noqa: E731
    rows = lay(s.q).view(s.B, N, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(s.B, Hkv, N * G, d)
    i, j = torch.arange(N, device="cuda")[:, None], torch.arange(N, device="cuda")
    seen = j <= i
    if c["window"]:
        seen &= (j > i - c["window"]) | (j < c["sink"])
    o = _attend(rows, lay(s.k).transpose(1, 2).contiguous(), lay(s.v).transpose(1, 2).contiguous(), seen[None, None], d)
    return o[seq, :, at].reshape(-1, Hq, d).to(s.q.dtype)


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
    k, v = (_values(codes[pid], meta[pid]).transpose(1, 2).reshape(B, Hkv, n_pages * page, d)
            for codes, meta in ((s.kc, s.km), (s.vc, s.vm)))
    i = (first[:, None] + torch.arange(b.max_q, device="cuda"))[:, None, :, None]      # positions of the rows
    j = torch.arange(n_pages * page, device="cuda")
    seen = j <= i
    if c["window"]:
        seen &= (j > i - c["window"]) | (j < c["sink"])
    return _attend(rows, k, v, seen, d)[seq, :, at].reshape(b.T, Hq, d).to(s.q.dtype)


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
    kind, new, Hkv, d = case["kind"], _ints(case["new"]), case["Hkv"], case["d"]
    T = sum(new)
    if kind == "packed":
        pairs = sum(_seen(n, 0, case["window"], case["sink"])[0] for n in new)
        return {"bytes": T * d * 2 * (2 * case["Hq"] + 2 * Hkv), "flops": 4 * d * case["Hq"] * pairs}
    past = _ints(case["past"])
    held = d // 2 + d // GROUP * (4 if case["fmt"] == "int4" else 1)          # bytes of a key or value of a head
    positions = min(T, max(n + p for n, p in zip(new, past)))
    if kind == "append":
        return {"bytes": 2 * T * Hkv * (2 * d + held + 2 * d) + positions * case["rot"] * 4, "flops": 3 * T * Hkv * case["rot"]}
    if kind == "read":
        return {"bytes": 2 * T * Hkv * (held + 2 * d), "flops": 0}
    seen = [_seen(n, p, case["window"], case["sink"]) for n, p in zip(new, past)]
    return {"bytes": 2 * sum(u for _, u in seen) * Hkv * held + T * case["Hq"] * 4 * d + positions * case["rot"] * 4,
            "flops": 4 * d * case["Hq"] * sum(p for p, _ in seen)}


# ---- the definition in 64 bits -----------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"packed": _exact_packed, "append": _exact_append, "read": _exact_read, "attn": _exact_attn}[case["kind"]](s)


def _softmax_of(q, k, v, i, window, sink):
    """Rows q [R, G, d] at positions i over k and v [L, d], all in 64 bits."""
    j = torch.arange(k.shape[0], device="cuda")
    hidden = j[None] > i[:, None]
    if window:
        hidden = hidden | ((j[None] <= i[:, None] - window) & (j[None] >= sink))
    out = torch.empty_like(q)
    for e in range(q.shape[1]):
        x = (q[:, e] @ k.t().contiguous()) * q.shape[2] ** -0.5
        x[hidden] = -math.inf
        out[:, e] = torch.softmax(x, dim=1) @ v
    return out


def _exact_packed(s):
    c = s.case
    G, at = c["Hq"] // c["Hkv"], s.cu.tolist()
    o = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    for a, b in zip(at, at[1:]):
        i = torch.arange(b - a, device="cuda")
        for h in range(c["Hkv"]):
            heads = slice(h * G, h * G + G)
            o[a:b, heads] = _softmax_of(s.q[a:b, heads].double(), s.k[a:b, h].double(), s.v[a:b, h].double(), i, c["window"], c["sink"])
    return o


def _turned(x, cs, layout):
    """Rotation as complex products: x [T, H, d] and cs [T, rot / 2, 2] in 64 bits."""
    half = cs.shape[1]
    y = x.double().clone()
    turn = torch.view_as_complex(cs.double().contiguous())[:, None]
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_held(codes, meta):
    """64-bit values of codes [..., d / 2], channel by channel of a byte."""
    out = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    pair = GROUP // 2
    for g in range(meta.shape[3]):
        w = codes[..., g * pair:(g + 1) * pair].int()
        for half, c in ((0, w % 16), (1, w // 16)):
            if meta.dtype == torch.float16:
                y = meta[..., g, 1].double()[..., None] + meta[..., g, 0].double()[..., None] * c.double()
            else:
                y = torch.zeros(c.shape, dtype=torch.float64, device=c.device)
                for n, level in enumerate(_E2M1):
                    y = torch.where(c == n, level, torch.where(c == n + 8, -level, y))
                y = y * 2.0 ** (meta[..., g].double()[..., None] - 127.0)
            out[..., g * GROUP + half:(g + 1) * GROUP:2] = y
    return out


def _exact_rounded(x, fmt):
    """The values that x [T, H, d] is held as, and with int4 the groups' (scale, zero): by search over all numbers that the
    format has."""
    out, meta = torch.empty_like(x), []
    halves = torch.arange(0, 0x7801, dtype=torch.int16, device=x.device).view(torch.float16).double()     # 0 .. 32768, ascending
    levels = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    for g in range(x.shape[2] // GROUP):
        y = x[..., g * GROUP:(g + 1) * GROUP].clamp(-MOST, MOST)
        if fmt == "int4":
            lo, hi = y.min(dim=-1).values, y.max(dim=-1).values
            below = halves[(torch.searchsorted(halves, lo.clamp(min=0), right=True) - 1).clamp(min=0)]
            z = torch.where(lo >= 0, below, -halves[torch.searchsorted(halves, (-lo).clamp(min=0))])
            s = halves[torch.searchsorted(halves, (hi - z) / 15.0)]
            n = ((y - z[..., None]) / torch.where(s > 0, s, 1.0)[..., None])
            n = torch.where((n - torch.floor(n) == 0.5) & (torch.floor(n) % 2 == 0), torch.floor(n), torch.floor(n + 0.5))
            out[..., g * GROUP:(g + 1) * GROUP] = z[..., None] + s[..., None] * torch.where(s[..., None] > 0, n, 0.0).clamp(max=15)
            meta.append(torch.stack((s, z), dim=-1))
        else:
            most, unit = y.abs().max(dim=-1).values, torch.full(y.shape[:-1], 2.0 ** -23, dtype=torch.float64, device=x.device)
            for _ in range(36):
                unit = torch.where(most > 6.0 * unit, unit * 2.0, unit)
            a = y.abs() / unit[..., None]
            up = torch.searchsorted(levels, a.contiguous()).clamp(max=7)
            dn = (up - 1).clamp(min=0)
            left, right = a - levels[dn], levels[up] - a
            n = torch.where((left < right) | ((left == right) & (dn % 2 == 0)), dn, up)
            out[..., g * GROUP:(g + 1) * GROUP] = levels[n] * unit[..., None] * torch.sign(y)
    return out, torch.stack(meta, dim=2) if meta else None


def _exact_append(s):
    c = s.case
    cu, lens, table, page = s.b.cu.tolist(), s.b.lens.tolist(), s.b.table.tolist(), c["page"]
    pos = torch.cat([torch.arange(n - (b - a), n, device="cuda") for a, b, n in zip(cu, cu[1:], lens)])
    k = _turned(s.k, s.table[pos], c["layout"]).float().double()
    rows, metas = [], []
    for x, meta in ((k, s.km), (s.v.double(), s.vm)):
        y, m = _exact_rounded(x, c["fmt"])
        rows.append(y)
        if m is not None:
            whole = meta.double()
            for a, b, n, pages in zip(cu, cu[1:], lens, table):
                at = n - (b - a)
                while at < n:
                    stop = min(n, (at // page + 1) * page)
                    whole[pages[at // page], :, at % page:at % page + stop - at] = m[b - (n - at):b - (n - stop)].transpose(0, 1)
                    at = stop
            metas.append(whole)
    return (*rows, *metas)


def _exact_read(s):
    c = s.case
    cu, lens = s.b.cu.tolist(), s.b.lens.tolist()
    out = []
    for codes, meta in ((s.kc, s.km), (s.vc, s.vm)):
        rows = []
        for b, n in enumerate(lens):
            pid = s.b.table[b, :-(-n // c["page"])].long()
            x = _exact_held(codes[pid], meta[pid]).transpose(1, 2).reshape(-1, c["Hkv"], c["d"])
            rows.append(x[n - (cu[b + 1] - cu[b]):n])
        out.append(torch.cat(rows))
    return tuple(out)


def _exact_attn(s):
    c = s.case
    Hq, Hkv, d, page = c["Hq"], c["Hkv"], c["d"], c["page"]
    G = Hq // Hkv
    o = torch.zeros(s.b.T, Hq, d, dtype=torch.float64, device="cuda")
    cu, lens = s.b.cu.tolist(), s.b.lens.tolist()
    for b, n in enumerate(lens):
        rows = slice(cu[b], cu[b + 1])
        i = torch.arange(n - (cu[b + 1] - cu[b]), n, device="cuda")
        q = _turned(s.q[rows], s.table[i], c["layout"])
        pid = s.b.table[b, :-(-n // page)].long()
        for h in range(Hkv):
            k, v = (_exact_held(codes[pid, h:h + 1], meta[pid, h:h + 1]).reshape(-1, d)[:n]
                    for codes, meta in ((s.kc, s.km), (s.vc, s.vm)))
            o[rows, h * G:h * G + G] = _softmax_of(q[:, h * G:h * G + G], k, v, i, c["window"], c["sink"])
    return o
