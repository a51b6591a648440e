"""The operators that serve a model next to its LC-VQ layers, as cases to be timed.

Four operators, each through the package's public calls:

  kv_write   keys and values of new tokens, quantised as they are written into a paged
             cache (8-bit e4m3 codes with one power-of-two scale per token and head, or
             bf16 as they are), and read back
  kv_read    keys and values of any slots of such a cache, as the values they stand for
  attn       causal attention of each sequence's new tokens (one, or a chunk) over its
             pages of the cache, several query heads to a cached head
  int4       the layer output from 4-bit weights with a scale (and a zero point) per
             group of columns, for few tokens

With `own` false the same results come from elementary torch operations in 32 bits.

Shapes are those of the Llama-shaped models of the repository's workloads (4096 wide: 32
heads of 128; 8192 wide: 64 heads of 128 over 8 cached ones; 11008 and 28672 wide MLPs),
or generic.
"""
from __future__ import annotations

import math

import torch

own = False

_BF16 = torch.bfloat16
_E4M3 = torch.float8_e4m3fn
_E4M3_MAX = 448.0
_E_LO, _E_HI = -117, 119      # scale exponents of the 8-bit cache
_NONE = float("-inf")


def listed():
    return [
        # one token of one sequence into a 70B model's cache: the smallest call, latency
        dict(name="kv_write_1", kind="kv_write", T=1, Hkv=8, D=128, page=16, fp8=True),
        # a ragged batch of prompts, 7B model (32 cached heads), 8 bits
        dict(name="kv_write_4999", kind="kv_write", T=4999, Hkv=32, D=128, page=64, fp8=True),
        # the whole context of a few sequences read back, e.g. to move it or to attend
        # to it in another way
        dict(name="kv_read_100000", kind="kv_read", T=100000, Hkv=8, D=128, page=32, fp8=True),
        # one token of a short 7B conversation, cache in bf16: the smallest call, latency
        dict(name="decode_1x333", kind="attn", B=1, new=1, chunk=0, ctx=333, Hq=32, Hkv=32, D=128, page=16, fp8=False,
             window=0, ragged=False),
        # 64 conversations of very different lengths, 70B model, 8-bit cache
        dict(name="decode_64x8000", kind="attn", B=64, new=1, chunk=0, ctx=8000, Hq=64, Hkv=8, D=128, page=64, fp8=True,
             window=0, ragged=True),
        # one long document, 70B model: few rows, a long axis
        dict(name="decode_1x130001", kind="attn", B=1, new=1, chunk=0, ctx=130001, Hq=64, Hkv=8, D=128, page=64, fp8=True,
             window=0, ragged=False),
        # a chunk of a long prompt over what the cache holds already, 70B model
        dict(name="chunk_512_over_8192", kind="attn", B=1, new=512, chunk=0, ctx=8192, Hq=64, Hkv=8, D=128, page=64,
             fp8=True, window=0, ragged=False),
        # whole prompts, 7B model, bf16 cache, small pages
        dict(name="prefill_4x2048", kind="attn", B=4, new=2048, chunk=0, ctx=2048, Hq=32, Hkv=32, D=128, page=16, fp8=False,
             window=0, ragged=True),
        # a chunk beside decoding sequences in one call, heads of 64, a sliding window
        dict(name="mixed_32_chunk_1000", kind="attn", B=32, new=1, chunk=1000, ctx=6000, Hq=32, Hkv=8, D=64, page=32,
             fp8=True, window=2048, ragged=True),
        # one token through a 7B projection
        dict(name="int4_4096x4096_1", kind="int4", N=1, m=4096, n=4096, group=128, zeros=False, f32=False),
        # one token through a 70B up projection, asymmetric codes
        dict(name="int4_28672x8192_1", kind="int4", N=1, m=28672, n=8192, group=128, zeros=True, f32=False),
        # a batch of sequences through a 70B down projection, small groups
        dict(name="int4_8192x28672_16", kind="int4", N=16, m=8192, n=28672, group=64, zeros=False, f32=True),
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of step in [lo, hi], spread over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(v) // step * step)) // step * step


def draw(rng):
    most = max(_least(c) for c in listed())
    while True:                        # (few draws are larger than the largest listed case)
        case = _draw(rng)
        if _least(case) <= most:
            return case


def _least(case):
    """Seconds at 5 TB/s and 1300 TFLOP/s."""
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1.3e15)


def _draw(rng):
    kind = rng.choice(["kv_write", "kv_read", "attn", "attn", "attn", "attn", "int4", "int4"])
    if kind == "int4":
        group = rng.choice([32, 64, 128, 128])
        return dict(kind=kind, N=rng.choice([1, rng.randint(1, 4), rng.randint(1, 16), rng.randint(1, 16)]),
                    m=_log_int(rng, 256, 28672), n=_log_int(rng, 512, 28672, group), group=group,
                    zeros=rng.choice([False, True]), f32=rng.choice([False, True]))
    D, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 256])
    fp8, Hkv = rng.choice([True, True, False]), rng.choice([1, 2, 4, 8, 8, 32])
    if kind != "attn":
        most = min(100000, (1 << (20 if fp8 else 19)) // Hkv)
        return dict(kind=kind, T=_log_int(rng, 1, most), Hkv=Hkv, D=D, page=page, fp8=fp8)
    Hq = Hkv * (1 if Hkv == 32 else rng.choice([1, 4, 5, 8]))
    shape = rng.choice(["decode", "decode", "chunk", "mixed"])
    c = dict(kind=kind, Hq=Hq, Hkv=Hkv, D=D, page=page, fp8=fp8, window=rng.choice([0, 0, _log_int(rng, 16, 4096)]),
             ragged=rng.choice([False, True]))
    if shape == "decode":
        B = _log_int(rng, 1, 256)
        most = max(64, min(130000, (1 << (21 if fp8 else 20)) // (Hkv * B)))
        return dict(B=B, new=rng.choice([1, 1, rng.randint(1, 6)]), chunk=0, ctx=_log_int(rng, 16, most), **c)
    if shape == "chunk":
        B, new = rng.randint(1, 4), _log_int(rng, 16, 2048)
        most = max(new, min(16384, (1 << 28) // (Hq * B * new)))
        return dict(B=B, new=new, chunk=0, ctx=_log_int(rng, new, most), **c)
    B, chunk = _log_int(rng, 2, 64), _log_int(rng, 16, 1500)
    most = max(chunk, min(8192, (1 << 28) // (Hq * chunk), (1 << 20) // (Hkv * B)))
    return dict(B=B, new=1, chunk=chunk, ctx=_log_int(rng, chunk, most), **c)


# ---------------------------------------------------------------- preparation --

def _draws(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _sizes(case):
    """New tokens and cached tokens (the new ones among them) of each sequence.  Ragged
    lengths depend on the case alone, so that work() knows them."""
    B, new, ctx = case["B"], case["new"], case["ctx"]
    nq, lens = [], []
    for b in range(B):
        # from a seventh of the longest up to it, in an order without pattern
        f = 1.0 if b == 0 or not case["ragged"] else 1.0 / 7 + (b * 0.6180339887) % 1.0 * 6 / 7
        length = max(1, round(ctx * f))
        n = case["chunk"] if case["chunk"] and b == 0 else new
        if n == ctx:                     # a whole prompt
            n = length
        nq.append(min(n, length))
        lens.append(length)
    return nq, lens


def _normal(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _keys(g, T, H, D):
    """Keys or values as a model has them: some channels much larger than the rest."""
    gain = torch.exp(0.5 * _normal(g, H, D))
    return (_normal(g, T, H, D) * gain).to(_BF16)


def _e4m3(x):
    """x (fp32, (.., D)): e4m3 codes and the exponent of the scale, the smallest e with
    amax <= 448 * 2^e, in [-117, 119]."""
    frac, e = torch.frexp(x.abs().amax(-1))
    e = (e - 9 + (frac > 0.875).to(e.dtype)).clamp(_E_LO, _E_HI)
    q = torch.ldexp(x, -e.unsqueeze(-1)).clamp(-_E4M3_MAX, _E4M3_MAX).to(_E4M3)
    return q.view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What the cache's entries stand for, in fp32."""
    if codes.dtype == _BF16:
        return codes.float()
    return torch.ldexp(codes.view(_E4M3).float(), scales.to(torch.int32).unsqueeze(-1) - 127)


def _empty_cache(pages, H, page, D, fp8):
    data = torch.zeros((2, pages, H, page, D), dtype=torch.uint8 if fp8 else _BF16, device="cuda")
    return data, torch.full((2, pages, H, page), 127, dtype=torch.uint8, device="cuda") if fp8 else None


def _filled_cache(g, pages, H, page, D, fp8):
    data, scales = _empty_cache(pages, H, page, D, fp8)
    for i in range(2):
        x = _keys(g, pages * page, H, D).reshape(pages, page, H, D).transpose(1, 2).contiguous()
        if fp8:
            for p in range(0, pages, 256):   # some pages at a time: the 32-bit form is large
                data[i, p:p + 256], scales[i, p:p + 256] = _e4m3(x[p:p + 256].float())
        else:
            data[i] = x
    return data, scales


def prepare(case, seed):
    g, kind = _draws(seed), case["kind"]
    s = dict(case=case)
    if kind == "int4":
        m, n, group, N = case["m"], case["n"], case["group"], case["N"]
        w = _normal(g, m, n // group, group)
        if case["zeros"]:
            lo, hi = w.amin(-1), w.amax(-1)
            s["scales"] = ((hi - lo) / 15).to(_BF16)
            s["zeros"] = (-lo / s["scales"].float()).round().clamp(0, 15).to(_BF16)
        else:
            s["scales"] = (w.abs().amax(-1) / 7).to(_BF16)
            s["zeros"] = None
        z = s["zeros"].float() if case["zeros"] else torch.full_like(s["scales"], 8, dtype=torch.float32)
        c = (w / s["scales"].float().unsqueeze(-1)).round().add_(z.unsqueeze(-1)).clamp_(0, 15).to(torch.uint8)
        c = c.reshape(m, n)
        s["packed"] = c[:, 0::2] | (c[:, 1::2] << 4)          # two codes a byte, the even column low
        s["scales"].mul_(1.0 / math.sqrt(n))                 # outputs near 1
        s["X"] = _normal(g, N, n).to(_BF16)
        s["out"] = torch.empty((N, m), dtype=torch.float32 if case["f32"] else _BF16, device="cuda")
        if own:
            import paper_2606_10531_amd as lc
            s["ws"] = torch.empty(max(lc.int4_workspace_bytes(N, m, n), 16), dtype=torch.uint8, device="cuda")
        return s
    Hkv, D, page, fp8 = case["Hkv"], case["D"], case["page"], case["fp8"]
    if kind != "attn":
        T = case["T"]
        pages = -(-T // page) + 3
        slots = torch.randperm(pages, device="cuda", generator=g)[:-(-T // page)]
        s["slots"] = (slots.unsqueeze(1) * page + torch.arange(page, device="cuda")).reshape(-1)[:T].contiguous()
        if kind == "kv_read":
            s["data"], s["scales"] = _filled_cache(g, pages, Hkv, page, D, fp8)
        else:
            s["data"], s["scales"] = _empty_cache(pages, Hkv, page, D, fp8)
            # keys and values as the slices of one projection's output
            s["kv"] = torch.cat([_keys(g, T, Hkv, D), _keys(g, T, Hkv, D)], dim=1)
        return s
    nq, lens = _sizes(case)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((case["B"], max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    T = sum(nq)
    s["data"], s["scales"] = _filled_cache(g, pages, Hkv, page, D, fp8)
    s["table"], s["nq"], s["lens"] = table, nq, lens
    s["q"] = _normal(g, T, case["Hq"], D).to(_BF16)
    s["kv_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["q_starts"] = torch.tensor([sum(nq[:b]) for b in range(len(nq) + 1)], dtype=torch.int32, device="cuda")
    s["out"] = torch.empty((T, case["Hq"], D), dtype=_BF16, device="cuda")
    s["lse"] = torch.empty((T, case["Hq"]), dtype=torch.float32, device="cuda")
    if own:
        import paper_2606_10531_amd as lc
        need = lc.attn_workspace_bytes(T, case["B"], case["Hq"], Hkv, D, max(nq))
        s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ----------------------------------------------------------------------- passes --

def _plain_write(s):
    page = s["case"]["page"]
    H = s["case"]["Hkv"]
    at, off = s["slots"] // page, s["slots"] % page
    for i in range(2):
        x = s["kv"][:, i * H:(i + 1) * H]
        if s["scales"] is None:
            s["data"][i, at, :, off] = x
        else:
            s["data"][i, at, :, off], s["scales"][i, at, :, off] = _e4m3(x.float())


def _plain_read(s):
    page = s["case"]["page"]
    at, off = s["slots"] // page, s["slots"] % page
    return [_values(s["data"][i, at, :, off], None if s["scales"] is None else s["scales"][i, at, :, off]).to(_BF16)
            for i in range(2)]


def _plain_attn(s):
    c = s["case"]
    Hkv, D, G = c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    q0 = 0
    for b, (n, length) in enumerate(zip(s["nq"], s["lens"])):
        ids = s["table"][b, :-(-length // c["page"])].long()
        k, v = (_values(s["data"][i, ids], None if s["scales"] is None else s["scales"][i, ids])
                .transpose(0, 1).reshape(Hkv, -1, D)[:, :length].contiguous() for i in range(2))
        q = s["q"][q0:q0 + n].float().reshape(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * n, D)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(D)).reshape(Hkv, G, n, length)
        pos = torch.arange(length - n, length, device="cuda").unsqueeze(1)
        j = torch.arange(length, device="cuda").unsqueeze(0)
        hidden = j > pos
        if c["window"]:
            hidden = hidden | (j <= pos - c["window"])
        x.masked_fill_(hidden, _NONE)
        top = x.amax(-1, keepdim=True)
        x.sub_(top).exp_()
        total = x.sum(-1, keepdim=True)
        o = torch.matmul(x.reshape(Hkv, G * n, length), v).reshape(Hkv, G, n, D) / total
        s["out"][q0:q0 + n] = o.permute(2, 0, 1, 3).reshape(n, c["Hq"], D).to(_BF16)
        s["lse"][q0:q0 + n] = (top + total.log()).squeeze(-1).permute(2, 0, 1).reshape(n, c["Hq"])
        q0 += n
    return dict(out=s["out"], lse=s["lse"])


def _plain_int4(s):
    c = s["case"]
    w = torch.stack([s["packed"] & 15, s["packed"] >> 4], dim=-1).reshape(c["m"], -1, c["group"]).float()
    w.sub_(8.0 if s["zeros"] is None else s["zeros"].float().unsqueeze(-1)).mul_(s["scales"].float().unsqueeze(-1))
    return torch.matmul(s["X"].float(), w.reshape(c["m"], c["n"]).t()).to(s["out"].dtype)


def run(s):
    c, kind = s["case"], s["case"]["kind"]
    if not own:
        if kind == "kv_write":
            _plain_write(s)
            return _plain_read(s)
        return {"kv_read": _plain_read, "attn": _plain_attn, "int4": _plain_int4}[kind](s)
    import paper_2606_10531_amd as lc
    if kind == "int4":
        return lc.linear_fwd_int4(s["packed"], s["scales"], s["X"], c["group"], zeros=s["zeros"], workspace=s["ws"],
                                  out=s["out"])
    if kind == "kv_write":
        H = c["Hkv"]
        lc.kv_write(s["kv"][:, :H], s["kv"][:, H:], s["slots"], s["data"], s["scales"])
    if kind != "attn":
        return lc.kv_read(s["data"], s["slots"], s["scales"])
    out, lse = lc.attn_paged(s["q"], s["data"], s["table"], s["kv_lens"], s["q_starts"], s["scales"],
                             window=c["window"], max_q=max(s["nq"]), workspace=s["ws"], out=s["out"], lse=s["lse"])
    return dict(out=out, lse=lse)


# ------------------------------------------------------------------- least work --

def work(case):
    kind = case["kind"]
    if kind == "int4":
        m, n, N = case["m"], case["n"], case["N"]
        params = m * (n // case["group"]) * 2 * (2 if case["zeros"] else 1)
        return dict(bytes=m * n // 2 + params + N * n * 2 + N * m * (4 if case["f32"] else 2), flops=2 * N * m * n)
    Hkv, D = case["Hkv"], case["D"]
    entry = D + 1 if case["fp8"] else 2 * D     # bytes of one head's key or value in the cache
    if kind != "attn":
        T = case["T"]
        plain = T * Hkv * D * 2 * 2
        held = T * Hkv * entry * 2
        return dict(bytes=(2 if kind == "kv_write" else 1) * (plain + held) + T * 8, flops=0)
    nq, lens = _sizes(case)
    tokens = pairs = 0
    for n, length in zip(nq, lens):
        w = case["window"] or length
        tokens += min(length, w + n - 1)
        pairs += sum(min(p + 1, w) for p in range(length - n, length))
    T = sum(nq)
    return dict(bytes=tokens * Hkv * entry * 2 + T * case["Hq"] * (D * 4 + 4) + 4 * sum(-(-x // case["page"]) for x in lens),
                flops=4 * D * case["Hq"] * pairs)


# ------------------------------------------------------------- in 64 bits, apart --

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind = case["kind"]
    if kind == "int4":
        byte = s["packed"].cpu().to(torch.int64)
        code = torch.empty((case["m"], case["n"]), dtype=torch.float64)
        code[:, ::2], code[:, 1::2] = (byte % 16).double(), (byte // 16).double()
        y = torch.zeros((case["N"], case["m"]), dtype=torch.float64)
        X, scale = s["X"].cpu().double(), s["scales"].cpu().double()
        zero = None if s["zeros"] is None else s["zeros"].cpu().double()
        for k in range(case["n"] // case["group"]):
            cols = slice(k * case["group"], (k + 1) * case["group"])
            z = 8.0 if zero is None else zero[:, k:k + 1]
            y += (X[:, cols] @ (code[:, cols] - z).T) * scale[:, k]
        return y
    held = _decoded(s)
    if kind == "kv_read":
        at = s["slots"]
        return [h.transpose(1, 2).reshape(-1, case["Hkv"], case["D"])[at] for h in held]
    if kind == "kv_write":
        x = s["kv"].double()
        x = x if not case["fp8"] else _nearest_e4m3(x)
        return [x[:, :case["Hkv"]].contiguous(), x[:, case["Hkv"]:].contiguous()]
    nq, lens = _sizes(case)
    if sum(n * length for n, length in zip(nq, lens)) * case["Hq"] > 1 << 33:
        return None
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    group, first = case["Hq"] // case["Hkv"], 0
    for b, (n, length) in enumerate(zip(nq, lens)):
        t = torch.arange(length, device="cuda")
        page = s["table"][b].long()[t // case["page"]]
        i = torch.arange(n, device="cuda")[:, None] + (length - n)
        seen = (t[None, :] <= i) & ((i - t[None, :] < case["window"]) if case["window"] else True)
        for h in range(case["Hq"]):
            k, v = (x[page, h // group, t % case["page"]] for x in held)
            score = (s["q"][first:first + n, h].double() @ k.T) / math.sqrt(case["D"])
            score = torch.where(seen, score, torch.full_like(score, _NONE))
            lse[first:first + n, h] = torch.logsumexp(score, dim=1)
            out[first:first + n, h] = torch.exp(score - lse[first:first + n, h, None]) @ v
        first += n
    return dict(out=out, lse=lse)


def _decoded(s):
    """The cache's keys and values in 64 bits, from the bits of its codes."""
    if s["scales"] is None:
        return [s["data"][0].double(), s["data"][1].double()]
    byte = torch.arange(256, device="cuda")
    expo, mant = (byte >> 3 & 15).double(), (byte & 7).double()
    table = torch.where(expo > 0, torch.exp2(expo - 7) * (1 + mant / 8), torch.exp2(torch.full_like(mant, -6)) * mant / 8)
    table = torch.where(byte >= 128, -table, table)
    return [table[s["data"][i].long()] * torch.exp2(s["scales"][i].double() - 127).unsqueeze(-1) for i in range(2)]


def _nearest_e4m3(x):
    """Each value rounded to the 8-bit grid of its token and head."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 448)).clamp(-117, 119)
    e = torch.where(448 * torch.exp2(e - 1) >= top, e - 1, e).clamp(-117, 119)
    e = torch.where(448 * torch.exp2(e) < top, e + 1, e).clamp(-117, 119)
    unit = torch.exp2(e)
    y = x / unit
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step * unit
