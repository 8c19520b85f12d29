"""The operators on either side of attention, as cases whose time is measured: each in its plain form, and as
the framework's entry points are called.

  rope    the norms of every query and key head with the position rotation, forward alone (`qk_rope_fwd`) or with
          the gradients from the fp32 dq, dk that the attention steps leave (`qk_rope_bwd`)
  append  new tokens' keys and values into a paged cache, rotated (and normed) on the way, their queries rotated
          beside them (`paged_append`)
  attn    attention of the new tokens of several sequences over that cache (`paged_attn`)

Inputs are drawn on the GPU from the seed.  Activations are N(0,1), what a norm leaves; norm weights lie around 1.
Sequence lengths belong to the case.  Pages are handed out in random order, as a cache that has been in use has them.
"""
import math
import random

import torch

own = False   # set by whoever measures: False: the plain form, True: the framework's kernels

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5


def rope(name, dtype, batch, len, hq, hkv, d, rot, norm=True, interleaved=False, packed=True, train=True, cp=1, rank=0):
    """`packed`: q and k are parts of one [batch, token, head, d] projection.  cp > 0: the tokens are the two zigzag
    chunks of `rank`; cp = 0: the positions are given, one per token."""
    case = dict(kind="rope", dtype=dtype, batch=batch, len=len, hq=hq, hkv=hkv, d=d, rot=rot, norm=norm, interleaved=interleaved,
                packed=packed, train=train, cp=cp, rank=rank)
    return dict(case, name=name) if name else case


def append(name, dtype, seqs, new, kv, page, hq, hkv, d, rot, norm, interleaved=False, ragged=False):
    case = dict(kind="append", dtype=dtype, seqs=seqs, new=new, kv=kv, page=page, hq=hq, hkv=hkv, d=d, rot=rot, norm=norm,
                interleaved=interleaved, ragged=ragged, mixed=False)
    return dict(case, name=name) if name else case


def attn(name, dtype, seqs, new, kv, page, hq, hkv, d, ragged=False, mixed=False):
    """`mixed`: one sequence has `new` new tokens, the others one."""
    case = dict(kind="attn", dtype=dtype, seqs=seqs, new=new, kv=kv, page=page, hq=hq, hkv=hkv, d=d, ragged=ragged, mixed=mixed)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the tiny fp32 shape of workloads.py: launches and host work count
        rope("rope_tiny_fp32_train", "fp32", batch=1, len=256, hq=2, hkv=2, d=64, rot=64, packed=False, cp=4, rank=0),
        # one rank's rows of the 1M-token GQA shard, from a packed projection: positions up to a million
        rope("rope_1m_shard_train", "bf16", batch=1, len=32768, hq=4, hkv=1, d=128, rot=128, cp=32, rank=5),
        # a prompt of 4096 tokens on a whole 7B model's heads, rotation alone
        rope("rope_prompt_forward", "bf16", batch=1, len=4096, hq=32, hkv=32, d=128, rot=128, norm=False, train=False),
        # head_dim 64 in half, a part of each head rotated in neighbouring pairs, odd lengths, positions given
        rope("rope_half_d64_train", "fp16", batch=2, len=3999, hq=8, hkv=2, d=64, rot=32, interleaved=True, packed=False, cp=0),
        # one new token for each of 64 sequences: what every layer of a decoding step does first
        append("append_one_token_each", "bf16", seqs=64, new=1, kv=8192, page=16, hq=32, hkv=8, d=128, rot=128, norm=True, ragged=True),
        # prompts of unequal length, half precision
        append("append_prompts_half", "fp16", seqs=5, new=3001, kv=4500, page=64, hq=12, hkv=4, d=64, rot=32, norm=False, interleaved=True,
               ragged=True),
        # one sequence, one token: the shortest call
        attn("attn_one_token_short", "bf16", seqs=1, new=1, kv=1000, page=16, hq=8, hkv=8, d=128),
        # a decoding step of many conversations
        attn("attn_decode_batch", "bf16", seqs=48, new=1, kv=8192, page=64, hq=32, hkv=8, d=128, ragged=True),
        # a decoding step of two long contexts on one shard's heads
        attn("attn_decode_long", "bf16", seqs=2, new=1, kv=262144, page=128, hq=4, hkv=1, d=128),
        # a few drafted tokens to be checked, half precision, three query heads to a key head
        attn("attn_drafted_half_d64", "fp16", seqs=16, new=5, kv=4000, page=24, hq=12, hkv=4, d=64, ragged=True),
        # a chunk of a long prompt: the largest
        attn("attn_chunk_32k", "bf16", seqs=1, new=2048, kv=32768, page=64, hq=32, hkv=8, d=128),
        # one prompt's chunk beside decoding sequences
        attn("attn_chunk_and_decodes", "bf16", seqs=9, new=1000, kv=6000, page=32, hq=8, hkv=2, d=128, ragged=True, mixed=True),
    ]


# ------------------------------------------------------------------------------------------------ draws
MOST_FLOPS = 1.08e12     # the chunk of a long prompt
MOST_BYTES = 7e8         # the decoding step of many conversations
MOST_SCORES = 2.15e9     # of the plain form, which holds them all


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    hkv = rng.choice([1, 2, 4, 8])
    return hkv * rng.choice([1, 2, 3, 4, 8]), hkv


def _draw_once(rng):
    kind = rng.choice(["rope", "rope", "append", "attn", "attn", "attn"])
    hq, hkv = _heads(rng)
    d = rng.choice([64, 128, 128])
    rot = rng.choice([d, d, d // 2])
    if kind == "rope":
        cp = rng.choice([0, 1, 4, 32])
        length = _log(rng, 2, 32768)
        return rope(None, rng.choice(["bf16", "bf16", "fp16", "fp32"]), batch=rng.choice([1, 1, 2, 3]), len=length if cp == 0 else 2 * (length // 2),
                    hq=hq, hkv=hkv, d=d, rot=rot, norm=rng.random() < 0.7, interleaved=rng.random() < 0.3, packed=rng.random() < 0.5,
                    train=rng.random() < 0.7, cp=cp, rank=rng.randrange(max(cp, 1)))
    page = rng.choice([16, 16, 24, 32, 64, 128, 256])
    kv = _log(rng, 20, 131072)
    seqs = _log(rng, 1, 96)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "append":
        return append(None, dtype, seqs=seqs, new=rng.choice([1, min(kv, _log(rng, 1, 4096))]), kv=kv, page=page, hq=hq, hkv=hkv, d=d, rot=rot,
                      norm=rng.random() < 0.6, interleaved=rng.random() < 0.3, ragged=rng.random() < 0.6)
    return attn(None, dtype, seqs=seqs, new=rng.choice([1, 1, min(kv, _log(rng, 2, 32)), min(kv, _log(rng, 33, 4096))]), kv=kv, page=page, hq=hq,
                hkv=hkv, d=d, ragged=rng.random() < 0.6, mixed=rng.random() < 0.2)


def _in_range(case):
    w = work(case)
    if w["flops"] > MOST_FLOPS or w["bytes"] > MOST_BYTES:
        return False
    if case["kind"] == "rope":
        return True
    new, kv = _lengths(case)
    pool = sum(-(-x // case["page"]) for x in kv) * case["page"] * 2 * case["hkv"] * case["d"] * 2
    return pool <= MOST_BYTES and (case["kind"] != "attn" or case["seqs"] * case["hq"] * max(new) * max(kv) <= MOST_SCORES)


def draw(rng):
    while True:
        case = _draw_once(rng)
        if _in_range(case):
            return case


# --------------------------------------------------------------------------------------------- the work
def _lengths(case):
    """New tokens and cached tokens (the new ones among them) of every sequence."""
    rng = random.Random(case["seqs"] * 1000003 + case["kv"] * 101 + case["new"])
    few = [1.0] + [math.exp(-rng.uniform(0, math.log(8))) if case["ragged"] else 1.0 for _ in range(case["seqs"] - 1)]
    kv = [max(1, round(case["kv"] * f)) for f in few]
    new = [1 if case["mixed"] and i else min(case["new"], kv[i]) for i in range(case["seqs"])]
    if case["ragged"] and not case["mixed"]:
        new = [max(1, round(n * f)) for n, f in zip(new, few)]
    return new, kv


def work(case):
    e, d, hq, hkv = SIZE[case["dtype"]], case["d"], case["hq"], case["hkv"]
    if case["kind"] == "rope":
        values = case["batch"] * case["len"] * (hq + hkv) * d
        # forward: in, out.  Backward: in and the fp32 gradient, out.
        return {"bytes": values * 2 * e + (values * (2 * e + 4) if case["train"] else 0), "flops": values * (8 + (14 if case["train"] else 0))}
    new, kv = _lengths(case)
    if case["kind"] == "append":
        return {"bytes": sum(new) * d * e * (2 * hq + 4 * hkv), "flops": 8 * sum(new) * d * (hq + hkv)}
    pairs = sum(n * c - n * (n - 1) // 2 for n, c in zip(new, kv))
    return {"bytes": sum(kv) * 2 * hkv * d * e + sum(new) * hq * (2 * d * e + 4), "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------------- data
def _normal(gen, shape, dtype):
    return torch.randn(shape, device=DEV, generator=gen).to(TORCH[dtype])


def _frequencies(rot):
    """Of the rotation, radians per position, fp32 as a model's configuration gives them."""
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).to(torch.float32).to(DEV)


def _zigzag_chunks(case):
    return case["len"] // 2, (case["rank"], 2 * case["cp"] - 1 - case["rank"])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"rope": _prepare_rope, "append": _prepare_append, "attn": _prepare_attn}[case["kind"]](case, gen)
    return dict(s, case=dict(case), kept={})   # kept: the program's descriptor and workspace, made at its first call


def run(state):
    if own:
        return {"rope": _own_rope, "append": _own_append, "attn": _own_attn}[state["case"]["kind"]](state)
    return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn}[state["case"]["kind"]](state)


def _weights(case, gen):
    if not case["norm"]:
        return None, None
    return tuple(1 + 0.2 * torch.randn(case["d"], device=DEV, generator=gen) for _ in range(2))


def _prepare_rope(case, gen):
    b, n, hq, hkv, d, dtype = (case[x] for x in ("batch", "len", "hq", "hkv", "d", "dtype"))

    def projection(make):
        """q and k as [batch, head, token, d] views of token-major memory."""
        if case["packed"]:   # the values' part is there too
            x = make((b, n, hq + 2 * hkv, d)).transpose(1, 2)
            return x[:, :hq], x[:, hq:hq + hkv]
        return make((b, n, hq, d)).transpose(1, 2), make((b, n, hkv, d)).transpose(1, 2)

    def heads(h, t=TORCH[dtype]):
        return torch.empty(b, h, n, d, dtype=t, device=DEV)

    s = {"inv_freq": _frequencies(case["rot"]), "positions": None}
    s["q"], s["k"] = projection(lambda shape: _normal(gen, shape, dtype))
    s["wq"], s["wk"] = _weights(case, gen)
    s["q_out"], s["k_out"] = heads(hq), heads(hkv)
    if case["cp"] == 0:
        s["positions"] = (torch.arange(n, device=DEV) + torch.randint(0, 1 << 20, (b, 1), device=DEV, generator=gen)).to(torch.int32)
    if case["train"]:
        s["dq_out"], s["dk_out"] = (torch.randn(b, h, n, d, device=DEV, generator=gen) for h in (hq, hkv))
        s["dq"], s["dk"] = projection(lambda shape: torch.zeros(shape, dtype=TORCH[dtype], device=DEV))
        s["dwq"], s["dwk"] = (torch.zeros(d, device=DEV) if case["norm"] else None for _ in range(2))
    return s


def _pages(kv, page, gen):
    """A page table of pages in random order, and how many there are."""
    need = [-(-x // page) for x in kv]
    width, total = max(need), sum(need)
    order = torch.randperm(total, device=DEV, generator=gen).to(torch.int32)
    table = torch.zeros(len(kv), width, dtype=torch.int32, device=DEV)
    first = torch.tensor([sum(need[:i]) for i in range(len(need))], device=DEV)
    at = first[:, None] + torch.arange(width, device=DEV)[None]
    return torch.where(torch.arange(width, device=DEV)[None] < torch.tensor(need, device=DEV)[:, None],
                       order[at.clamp(max=total - 1)], table), total


def _prepare_cache(case, gen):
    new, kv = _lengths(case)
    table, pages = _pages(kv, case["page"], gen)
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    s = {"table": table, "pages": pages, "tokens": starts[-1], "most_new": max(new), "most_kv": max(kv),
         "starts": torch.tensor(starts, dtype=torch.int32, device=DEV), "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV)}
    shape = (pages, case["hkv"], case["page"], case["d"])
    s["k_cache"], s["v_cache"] = _normal(gen, shape, case["dtype"]), _normal(gen, shape, case["dtype"])
    s["q"] = _normal(gen, (s["tokens"], case["hq"], case["d"]), case["dtype"])
    return s


def _prepare_append(case, gen):
    s = _prepare_cache(case, gen)
    shape = (s["tokens"], case["hkv"], case["d"])
    s["k"], s["v"] = _normal(gen, shape, case["dtype"]), _normal(gen, shape, case["dtype"])
    s["wq"], s["wk"] = _weights(case, gen)
    s["inv_freq"], s["q_out"] = _frequencies(case["rot"]), torch.empty_like(s["q"])
    return s


def _prepare_attn(case, gen):
    s = _prepare_cache(case, gen)
    s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(s["tokens"], case["hq"], device=DEV)
    return s


# ---------------------------------------------------------------------------------- the framework's calls
def _code(P, dtype):
    return {"bf16": P.BF16, "fp16": P.FP16, "fp32": P.FP32}[dtype]


def _flags(P, case):
    return (P.QK_NORM if case["norm"] else 0) | (P.ROPE_INTERLEAVED if case["interleaved"] else 0)


def _own_rope(s):
    import paper_2406_18485_amd as P
    c, kept = s["case"], s["kept"]
    if not kept:
        chunk_len, chunk = _zigzag_chunks(c) if c["cp"] else (0, (0, 0))
        kept["desc"] = P.make_rope_desc(batch=c["batch"], n_q_heads=c["hq"], n_kv_heads=c["hkv"], head_dim=c["d"], rot_dim=c["rot"],
                                        len=c["len"], chunk_len=chunk_len, chunk=chunk, dtype=_code(P, c["dtype"]), eps=EPS,
                                        flags=_flags(P, c), q_stride=s["q"].stride()[:3], k_stride=s["k"].stride()[:3])
        kept["workspace"] = torch.empty(max(P.qk_rope_workspace_bytes(kept["desc"]), 16), dtype=torch.uint8, device=DEV)
    P.qk_rope_fwd(kept["desc"], s["q"], s["k"], s["wq"], s["wk"], s["inv_freq"], s["positions"], s["q_out"], s["k_out"])
    if not c["train"]:
        return {"q": s["q_out"], "k": s["k_out"]}
    P.qk_rope_bwd(kept["desc"], s["q"], s["k"], s["wq"], s["wk"], s["inv_freq"], s["positions"], s["dq_out"], s["dk_out"],
                  s["dq"], s["dk"], s["dwq"], s["dwk"], kept["workspace"])
    return {"q": s["q_out"], "k": s["k_out"], "dq": s["dq"], "dk": s["dk"], "dwq": s["dwq"], "dwk": s["dwk"]}


def _paged_desc(P, s, **more):
    c = s["case"]
    return P.make_paged_desc(n_seqs=c["seqs"], n_tokens=s["tokens"], max_new=s["most_new"], n_q_heads=c["hq"], n_kv_heads=c["hkv"],
                             head_dim=c["d"], dtype=_code(P, c["dtype"]), n_pages=s["pages"], page_size=c["page"],
                             max_pages=s["table"].shape[1], **more)


def _own_append(s):
    import paper_2406_18485_amd as P
    c, kept = s["case"], s["kept"]
    if not kept:
        kept["desc"] = _paged_desc(P, s, rot_dim=c["rot"], eps=EPS, flags=_flags(P, c))
    P.paged_append(kept["desc"], s["q"], s["k"], s["v"], s["wq"], s["wk"], s["inv_freq"], None, s["starts"], s["kv_len"], s["table"],
                   s["q_out"], s["k_cache"], s["v_cache"])
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attn(s):
    import paper_2406_18485_amd as P
    kept = s["kept"]
    if not kept:
        kept["desc"] = _paged_desc(P, s, softmax_scale=1.0 / math.sqrt(s["case"]["d"]), causal=True, flags=P.WORKSPACE_CLEAN)
        kept["workspace"] = torch.zeros(max(P.paged_workspace_bytes(kept["desc"]), 16), dtype=torch.uint8, device=DEV)
    P.paged_attn(kept["desc"], s["q"], s["k_cache"], s["v_cache"], s["starts"], s["kv_len"], s["table"], None, s["o"], s["lse"],
                 kept["workspace"])
    return {"o": s["o"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------- plain forms
def _angles(positions, inv_freq):
    a = positions.double()[..., None] * inv_freq.double()
    return a.cos().float(), a.sin().float()


def _turned(x, cos, sin, rot, interleaved):
    """x [..., d] in fp32; cos, sin broadcast against [..., rot / 2]."""
    part, rest = x[..., :rot], x[..., rot:]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :rot // 2], part[..., rot // 2:])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((turned, rest), -1)


def _rms(x):
    return torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _normed(x, w):
    return x * _rms(x) * w


def _plain_positions(s):
    c = s["case"]
    if s["positions"] is not None:
        return s["positions"][:, None]          # [batch, 1, token]
    n, (low, high) = _zigzag_chunks(c)
    at = torch.arange(n, device=DEV)
    return torch.cat((low * n + at, high * n + at))[None, None]


def _plain_rope(s):
    c = s["case"]
    cos, sin = _angles(_plain_positions(s), s["inv_freq"])

    def forward(x, w, out):
        y = x.float()
        out.copy_(_turned(_normed(y, w) if c["norm"] else y, cos, sin, c["rot"], c["interleaved"]))

    def backward(x, w, g, dx, dw):
        g, x = _turned(g, cos, -sin, c["rot"], c["interleaved"]), x.float()
        if c["norm"]:
            r = _rms(x)
            dw.copy_((g * (x * r)).sum((0, 1, 2)))
            g = g * w
            g = r * g - x * (r * r * r) * ((g * x).mean(-1, keepdim=True))
        dx.copy_(g)

    forward(s["q"], s["wq"], s["q_out"])
    forward(s["k"], s["wk"], s["k_out"])
    if not c["train"]:
        return {"q": s["q_out"], "k": s["k_out"]}
    backward(s["q"], s["wq"], s["dq_out"], s["dq"], s["dwq"])
    backward(s["k"], s["wk"], s["dk_out"], s["dk"], s["dwk"])
    return {"q": s["q_out"], "k": s["k_out"], "dq": s["dq"], "dk": s["dk"], "dwq": s["dwq"], "dwk": s["dwk"]}


def _plain_places(s):
    """Of every new token: its sequence, its number among that sequence's, its position."""
    token = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(s["starts"], token.int(), right=True) - 1
    nth = token - s["starts"][seq]
    return seq, nth, s["kv_len"][seq] - (s["starts"][seq + 1] - s["starts"][seq]) + nth


def _plain_append(s):
    c = s["case"]
    seq, _, pos = _plain_places(s)
    cos, sin = _angles(pos[:, None], s["inv_freq"])

    def turned(x, w):
        x = x.float()
        return _turned(_normed(x, w) if c["norm"] else x, cos, sin, c["rot"], c["interleaved"]).to(TORCH[c["dtype"]])

    page, slot = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    s["q_out"].copy_(turned(s["q"], s["wq"]))
    s["k_cache"][page, :, slot] = turned(s["k"], s["wk"])
    s["v_cache"][page, :, slot] = s["v"]
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attn(s):
    c = s["case"]
    d, hkv, group = c["d"], c["hkv"], c["hq"] // c["hkv"]
    seq, nth, pos = _plain_places(s)

    def cached(cache):   # [sequence, kv head, key, d]
        return cache[s["table"].long()].transpose(1, 2).flatten(2, 3)[:, :, :s["most_kv"]].float()

    rows = torch.arange(s["most_new"], device=DEV)
    token = (s["starts"][:-1, None] + rows).clamp(max=s["tokens"] - 1)
    q = s["q"][token].float().unflatten(2, (hkv, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)   # [sequence, kv head, new x group, d]
    x = torch.matmul(q, cached(s["k_cache"]).transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    last = s["kv_len"][:, None] - (s["starts"][1:] - s["starts"][:-1])[:, None] + rows               # the last key that a row sees
    hidden = torch.arange(s["most_kv"], device=DEV) > last[:, :, None]
    hidden |= torch.arange(s["most_kv"], device=DEV) >= s["kv_len"][:, None, None]
    x = x.unflatten(2, (-1, group)).masked_fill_(hidden[:, None, :, None], -math.inf).flatten(2, 3)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, cached(s["v_cache"])) / total
    lse = (top + total.log()).squeeze(-1)
    o, lse = (y.unflatten(2, (-1, group)).transpose(1, 2).flatten(2, 3)[seq, nth] for y in (o, lse.unsqueeze(-1)))
    s["o"].copy_(o)
    s["lse"].copy_(lse.squeeze(-1))
    return {"o": s["o"], "lse": s["lse"]}


# ----------------------------------------------------------------------------------------- in 64 bits
def _rotation64(x, pos, c):
    """x [token, head, d], pos [token]: pairs as complex numbers, turned by exp(i pos f)."""
    rot = c["rot"]
    angle = pos.to(torch.float64)[:, None, None] * _frequencies(rot).to(torch.float64)
    by = torch.polar(torch.ones_like(angle), angle)
    part = x[..., :rot].reshape(*x.shape[:-1], *((rot // 2, 2) if c["interleaved"] else (2, rot // 2)))
    part = part if c["interleaved"] else part.transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * by)
    z = z if c["interleaved"] else z.transpose(-1, -2)
    return torch.cat((z.reshape(*x.shape[:-1], rot), x[..., rot:]), -1)


def _head64(x, w, pos, c):
    x = x.to(torch.float64)
    if w is not None:
        x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / c["d"] + EPS) * w.to(torch.float64)
    return _rotation64(x, pos, c)


def _exact_rope(s, c):
    if s["positions"] is None:
        n = c["len"] // 2
        i = torch.arange(c["len"], device=DEV)
        pos = torch.where(i < n, c["rank"] * n + i, (2 * c["cp"] - 1 - c["rank"]) * n + i - n).expand(c["batch"], -1)
    else:
        pos = s["positions"]
    got = {}
    for x, w in (("q", "wq"), ("k", "wk")):
        outs, grads, weight = [], [], 0
        for b in range(c["batch"]):
            rows = s[x][b].transpose(0, 1).to(torch.float64).requires_grad_()
            scale = None if s[w] is None else s[w].to(torch.float64).requires_grad_()
            y = _head64(rows, scale, pos[b], c)
            outs.append(y.detach().transpose(0, 1))
            if c["train"]:
                y.backward(s["d" + x + "_out"][b].transpose(0, 1).to(torch.float64))
                grads.append(rows.grad.transpose(0, 1))
                weight = weight + scale.grad if scale is not None else None
        got[x] = torch.stack(outs)
        if c["train"]:
            got["d" + x], got["d" + w] = torch.stack(grads), weight
    return got


def _exact_append(s, c):
    new, kv = _lengths(c)
    pos = torch.cat([torch.arange(k - n, k, device=DEV) for n, k in zip(new, kv)])
    got = {"q": _head64(s["q"], s["wq"], pos, c), "k_cache": s["k_cache"].to(torch.float64), "v_cache": s["v_cache"].to(torch.float64)}
    k, at = _head64(s["k"], s["wk"], pos, c), 0
    for b, n in enumerate(new):
        places = pos[at:at + n]
        page = s["table"][b].to(torch.int64)[torch.div(places, c["page"], rounding_mode="floor")]
        got["k_cache"][page, :, places % c["page"]] = k[at:at + n]
        got["v_cache"][page, :, places % c["page"]] = s["v"][at:at + n].to(torch.float64)
        at += n
    return got


def _exact_attn(s, c):
    new, kv = _lengths(c)
    group, at = c["hq"] // c["hkv"], 0
    o = torch.empty(s["tokens"], c["hq"], c["d"], dtype=torch.float64, device=DEV)
    lse = torch.empty(s["tokens"], c["hq"], dtype=torch.float64, device=DEV)
    for b, (n, m) in enumerate(zip(new, kv)):
        pages = s["table"][b, :-(-m // c["page"])].to(torch.int64)
        for h in range(c["hkv"]):
            keys, values = (s[x][pages, h].reshape(-1, c["d"])[:m].to(torch.float64) for x in ("k_cache", "v_cache"))
            for g in range(h * group, (h + 1) * group):
                scores = s["q"][at:at + n, g].to(torch.float64) @ keys.T / c["d"] ** 0.5
                if n > 1:
                    scores += torch.full((n, m), -math.inf, dtype=torch.float64, device=DEV).triu(m - n + 1)
                lse[at:at + n, g] = torch.logsumexp(scores, -1)
                o[at:at + n, g] = torch.exp(scores - lse[at:at + n, g, None]) @ values
        at += n
    return {"o": o, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "append": _exact_append, "attn": _exact_attn}[case["kind"]](s, case)
