"""Performance cases of the 4-bit KV cache: writing it, reading it back, and
decode attention over it.

A cache row holds one (sequence, position, KV head) of 128 dimensions: 64 bytes
of 4-bit codes, then for each group of ``quant_group`` (32, 64 or 128)
consecutive dimensions a bf16 scale, then for each group a bf16 lowest value;
a code c stands for low + scale * c.  The codes lie in sixteen little-endian
32-bit words: nibble n of word l holds dimension 32 (n mod 4) + 2 l + n // 4.
The caches are uint8 tensors [batch][L][n_kv][row] (token-major) or
[batch][n_kv][L][row] (head-major).  Row i of a call belongs to position
pos[b] + i and is written, or read, where 0 <= position < min(kv_len[b], L).

  write   new K/V rows quantised into the cache, then read back in fp32 (what
          4-bit rows are compared by); negative pos: left-padded prompts
  read    cached rows as bf16 or fp32 K/V rows, +0 outside the sequence, ready
          for prefill attention against a cached prefix
  attn    head-group masked decode attention, one query token a sequence

Quantisation, per group: low = the least value rounded down to bf16, scale =
(greatest - low) / 15 rounded to bf16 (0 below 2^-126), code = (x - low) /
scale rounded to nearest, ties to even.
"""
import math

import torch

own = False

HD = 128  # head dimension


# ---- the cases ---------------------------------------------------------------------

def listed():
    gqa = dict(n_q=32, n_kv=8, group=512)
    return [
        # one user generating: the K/V row of each new token of one layer
        dict(op="write", name="write_token_b1", n_seq=1, T=1, L=4096, n_kv=8, qg=32, dtype="bf16", head_major=False,
             ragged=False),
        # a serving batch generating together, every sequence at its own position
        dict(op="write", name="write_tokens_b32", n_seq=32, T=1, L=8192, n_kv=8, qg=64, dtype="bf16", head_major=True,
             ragged=True),
        # left-padded prompts of odd length kept in fp32 by a reference-numerics model
        dict(op="write", name="write_padded_f32_4x333", n_seq=4, T=333, L=1000, n_kv=8, qg=32, dtype="f32",
             head_major=False, ragged=True),
        # a long prompt
        dict(op="write", name="write_prompt_t8192", n_seq=1, T=8192, L=8192, n_kv=8, qg=32, dtype="bf16",
             head_major=True, ragged=False),
        # cached prefixes of a chunked prefill, left-padded to one length
        dict(op="read", name="read_prefix_4x1500", n_seq=4, T=1500, L=2048, n_kv=8, qg=32, dtype="bf16",
             head_major=False, ragged=True),
        # the caches of a whole batch of long sequences
        dict(op="read", name="read_8x32768", n_seq=8, T=32768, L=32768, n_kv=8, qg=128, dtype="bf16",
             head_major=True, ragged=False),
        # one user, a short chat: latency
        dict(gqa, op="attn", name="attn_b1_l500", B=1, L=500, qg=32, keep=1.0, ragged=False, head_major=True),
        # one user, a long document of odd length
        dict(gqa, op="attn", name="attn_b1_l50001", B=1, L=50001, qg=32, keep=1.0, ragged=False, head_major=True),
        # multi-head attention (no grouped queries), one scale a row, a small batch
        dict(op="attn", name="attn_mha_b8_l2000", n_q=32, n_kv=32, group=512, B=8, L=2000, qg=128, keep=0.5,
             ragged=True, head_major=False),
        # a serving batch, sequences of different ages, half of the head groups active
        dict(gqa, op="attn", name="attn_b32_ragged", B=32, L=8192, qg=32, keep=0.5, ragged=True, head_major=False),
        # a serving batch of equally long contexts, nothing masked
        dict(gqa, op="attn", name="attn_b32_l8192", B=32, L=8192, qg=32, keep=1.0, ragged=False, head_major=True),
        # the largest batch of long contexts
        dict(gqa, op="attn", name="attn_b64_l32768", B=64, L=32768, qg=64, keep=1.0, ragged=True, head_major=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["write", "write", "read", "attn", "attn", "attn"])
    qg = rng.choice([32, 32, 64, 128])
    head_major, ragged = rng.random() < 0.5, rng.random() < 0.6
    if op == "attn":
        n_q, n_kv, group = rng.choice([(32, 8, 512), (32, 8, 512), (32, 8, 128), (32, 32, 512), (16, 4, 256),
                                       (32, 4, 1024), (32, 2, 128), (8, 8, 128)])
        B = _log_int(rng, 1, 64)
        return dict(op=op, n_q=n_q, n_kv=n_kv, group=group, B=B, qg=qg, ragged=ragged, head_major=head_major,
                    L=_log_int(rng, 1, min(65536, 16777216 // (B * n_kv))), keep=rng.choice([1.0, 0.75, 0.5, 0.25]))
    n_kv = rng.choice([8, 8, 4, 2, 32])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    n_seq = _log_int(rng, 1, 32)
    if op == "write":
        T = _log_int(rng, 1, min(8192, 65536 * 4 // (n_seq * n_kv)))
        L = T + rng.randint(0, 2048)
    else:
        L = _log_int(rng, 1, min(32768, 2097152 // (n_seq * n_kv)))
        T = rng.randint(max(1, L // 2), L)
    return dict(op=op, n_seq=n_seq, T=T, L=L, n_kv=n_kv, qg=qg, dtype=dtype, head_major=head_major, ragged=ragged)


def _row_bytes(qg):
    return HD // 2 + 4 * (HD // qg)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def work(case):
    """Each input read once, each output written once (a ragged batch is half full on average)."""
    row = _row_bytes(case["qg"])
    if case["op"] == "attn":
        B, n_kv, qpk = case["B"], case["n_kv"], case["n_q"] // case["n_kv"]
        heads_per_group = case["group"] // HD
        read = 1.0 - (1.0 - case["keep"]) ** max(1, qpk // heads_per_group)  # share of KV heads read
        keys = B * n_kv * read * case["L"] * (0.5 if case["ragged"] else 1.0)
        heads = B * case["n_q"] * case["keep"] * case["L"] * (0.5 if case["ragged"] else 1.0)
        return {"bytes": 2 * keys * row + 2 * B * case["n_q"] * HD * 2, "flops": 4 * HD * heads}
    out = case["n_seq"] * case["T"] * case["n_kv"]
    elem = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "write":
        rows = out * (0.75 if case["ragged"] and case["T"] > 1 else 1.0)  # padding takes up to half of a prompt
        return {"bytes": 2 * (rows * (elem * HD + 2 * row) + out * 4 * HD), "flops": 2 * rows * HD * 8}
    rows = out * (0.75 if case["ragged"] else 1.0)
    return {"bytes": 2 * (rows * row + out * elem * HD), "flops": 2 * rows * HD * 2}


# ---- inputs ------------------------------------------------------------------------

def _cache_shape(case, batch):
    row = _row_bytes(case["qg"])
    return ((batch, case["n_kv"], case["L"], row) if case["head_major"] else
            (batch, case["L"], case["n_kv"], row))


def _fill_cache(g, case, batch):
    """A cache as quantised rows leave it: normal values with a bias per channel."""
    shape = _cache_shape(case, batch)
    cache = torch.empty(shape, dtype=torch.uint8, device="cuda")
    ng = HD // case["qg"]
    # one bias per (KV head, channel), as attention keys have
    bias = 0.7 * torch.randn((case["n_kv"], HD), generator=g, device="cuda")
    bias = bias[:, None] if case["head_major"] else bias
    for b in range(batch):
        x = torch.randn(shape[1:3] + (HD,), generator=g, device="cuda") + bias
        grp = x.view(shape[1:3] + (ng, case["qg"]))
        low = grp.amin(-1).bfloat16()
        scale = ((grp.amax(-1) - low.float()) / 15).bfloat16()
        code = ((grp - low.float()[..., None]) / scale.float()[..., None]).round_().clamp_(0, 15).to(torch.int32)
        # dimension 32 m + 2 l + e -> word l, nibble m + 4 e
        code = code.view(shape[1:3] + (4, 16, 2))
        shift = (4 * torch.arange(4, device="cuda")[:, None, None] + 16 * torch.arange(2, device="cuda")).int()
        words = (code << shift).sum((-3, -1), dtype=torch.int32)
        cache[b, ..., :64] = words.contiguous().view(torch.uint8)
        meta = torch.stack((scale, low), -2).contiguous()
        cache[b, ..., 64:] = meta.view(torch.uint8).flatten(-2)
    return cache


def _positions(g, case):
    """(pos, kv_len) int32 [n_seq] of a write or read, or None: whole rows from position 0."""
    n, T, L = case["n_seq"], case["T"], case["L"]
    if not case["ragged"]:
        return None, None
    u = torch.rand(n, generator=g, device="cuda")
    if case["op"] == "write" and T == 1:  # decode: sequences of different ages
        pos = (u * L).int().clamp_(max=L - 1)
    else:  # left padding of up to half of the rows
        pos = -(u * (T // 2 + 1)).int()
    return pos, pos + T


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] == "attn":
        B, n_q = case["B"], case["n_q"]
        ng = n_q * HD // case["group"]
        s["q"] = (1.5 * torch.randn((B, n_q * HD), generator=g, device="cuda")).bfloat16()
        s["mask"] = (torch.rand((B, ng), generator=g, device="cuda") < case["keep"]).to(torch.uint8)
        s["kv_len"] = None
        if case["ragged"]:  # ages evenly spread over the capacity, in random order
            step = (torch.randperm(B, generator=g, device="cuda") + 0.5) / B
            s["kv_len"] = (step * case["L"]).int().clamp_(min=1)
        s["k_cache"], s["v_cache"] = _fill_cache(g, case, B), _fill_cache(g, case, B)
        s["o"] = torch.empty_like(s["q"])
    else:
        n, rows, feat = case["n_seq"], case["n_seq"] * case["T"], case["n_kv"] * HD
        s["pos"], s["kv_len"] = _positions(g, case)
        if case["op"] == "write":
            bias = 0.7 * torch.randn((2, 1, feat), generator=g, device="cuda")
            kv = torch.randn((2, rows, feat), generator=g, device="cuda") + bias
            s["k"], s["v"] = (t.to(_dtype(case)).contiguous() for t in kv)
            s["k_cache"], s["v_cache"] = (torch.zeros(_cache_shape(case, n), dtype=torch.uint8, device="cuda")
                                          for _ in range(2))
        else:
            s["k_cache"], s["v_cache"] = _fill_cache(g, case, n), _fill_cache(g, case, n)
        dt = torch.float32 if case["op"] == "write" else _dtype(case)
        s["k_out"], s["v_out"] = (torch.empty((rows, feat), dtype=dt, device="cuda") for _ in range(2))
    if own:
        import paper_2607_28418_amd as W
        s["W"] = W
        if case["op"] == "attn":
            need = W.wide_attention_decode_kvq_workspace_size(case["B"], case["L"], case["n_q"], case["n_kv"], HD,
                                                              case["group"], case["qg"])
            s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ----------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    W = s["W"]
    if s["op"] == "attn":
        return W.wide_attention_decode_kvq(s["q"], s["k_cache"], s["v_cache"], s["mask"], s["n_q"], s["n_kv"], HD,
                                           s["group"], s["qg"], kv_len=s["kv_len"], head_major=s["head_major"],
                                           o=s["o"], ws=s["ws"])
    if s["op"] == "write":
        W.wide_kv_quantize(s["k"], s["v"], s["k_cache"], s["v_cache"], s["n_kv"], HD, s["qg"], pos=s["pos"],
                           kv_len=s["kv_len"], head_major=s["head_major"])
    return W.wide_kv_dequantize(s["k_cache"], s["v_cache"], s["T"], s["n_kv"], HD, s["qg"], pos=s["pos"],
                                kv_len=s["kv_len"], head_major=s["head_major"], k=s["k_out"], v=s["v_out"])


def _unpack(rows, qg):
    """Cache rows [...][row bytes] -> the values they stand for, fp32 [...][128]."""
    lead, ng = rows.shape[:-1], HD // qg
    words = rows[..., :64].contiguous().view(torch.int32)
    nib = torch.stack([(words >> (4 * n)) & 15 for n in range(8)], -1)      # [...][l][n = m + 4 e]
    code = nib.view(lead + (16, 2, 4)).movedim(-1, -3).reshape(lead + (ng, qg)).float()
    meta = rows[..., 64:].contiguous().view(torch.bfloat16).float().view(lead + (2, ng, 1))
    return (meta[..., 1, :, :] + meta[..., 0, :, :] * code).reshape(lead + (HD,))


def _div_even(a, b):
    """fp64 a / b (b > 0) to the nearest whole number, ties to even: the quotient's own rounding is undone."""
    k = torch.round(a / b)
    r, odd = a - b * k, torch.remainder(k, 2.0) == 1.0
    up = (r > b / 2) | ((r == b / 2) & odd)
    down = (r < -b / 2) | ((r == -b / 2) & odd)
    return k + up.double() - down.double()


def _values(x, qg):
    """The values that quantising fp64 rows [...][128] leaves, fp64 (in 64 bits: values next to a border)."""
    grp = x.view(x.shape[:-1] + (HD // qg, qg))
    least = grp.amin(-1, keepdim=True)
    # bf16, rounded down: the bits below its own are cut, and a negative number's size grows for them
    bits = least.float().view(torch.int32)
    cut = (bits >> 16) << 16
    low = (cut + ((bits < 0) & (cut != bits)).int() * 65536).view(torch.float32).double()
    span = grp.amax(-1, keepdim=True) - low
    # a bf16 step at span / 15: its binary exponent less 7, as a power of two put together from its bits
    unit = ((torch.frexp(span / 15.0)[1].long() - 8 + 1023) << 52).view(torch.float64)
    scale = unit * _div_even(span, 15.0 * unit)
    live = scale >= 2.0 ** -126
    one = torch.ones_like(scale)
    code = _div_even(grp - low, torch.where(live, scale, one)).clamp(0, 15)
    return torch.where(live, low + scale * code, low).reshape(x.shape)


def _run_plain(s):
    op, L, qg, n_kv = s["op"], s["L"], s["qg"], s["n_kv"]
    if op == "attn":
        B, n_q = s["B"], s["n_q"]
        q = s["q"].float().view(B, n_kv, n_q // n_kv, HD)
        o = torch.empty((B, n_kv, n_q // n_kv, HD), device="cuda")
        key = torch.arange(L, device="cuda")
        for b in range(B):
            k, v = (_unpack(s[c][b] if s["head_major"] else s[c][b].transpose(0, 1), qg)
                    for c in ("k_cache", "v_cache"))
            sc = torch.matmul(q[b], k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(HD))
            if s["kv_len"] is not None:
                sc = sc.masked_fill(key >= s["kv_len"][b], -math.inf)
            p = torch.exp(sc - sc.amax(-1, keepdim=True))
            o[b] = torch.matmul(p, v) / p.sum(-1, keepdim=True)
        on = s["mask"].bool().repeat_interleave(s["group"] // HD, dim=1).view(B, n_kv, -1, 1)
        return torch.where(on, o, torch.zeros_like(o)).view(B, n_q * HD).bfloat16()
    n, T = s["n_seq"], s["T"]
    pos = torch.arange(T, device="cuda").expand(n, T)
    pos = pos + s["pos"][:, None] if s["pos"] is not None else pos
    live = (pos >= 0) & (pos < L)
    if s["kv_len"] is not None:
        live = live & (pos < s["kv_len"][:, None])
    live = live.reshape(n * T, 1, 1)
    out = []
    for c in ("k", "v"):
        if op == "write":
            x = s[c].view(n * T, n_kv, HD)
            y = torch.cat([_values(part.double(), qg).float() for part in x.split(65536)])
        else:
            at = pos.clamp(0, L - 1).reshape(-1)
            seq = torch.arange(n, device="cuda").repeat_interleave(T)
            cache = s[c + "_cache"].transpose(1, 2) if s["head_major"] else s[c + "_cache"]
            y = _unpack(cache[seq, at], qg)
        y = torch.where(live, y, torch.zeros_like(y)).view(n * T, n_kv * HD)
        out.append(y if op == "write" else y.to(_dtype(s)))
    return tuple(out)


# ---- from the definition, in 64 bits ------------------------------------------------

def _exact_rows(rows, qg):
    """Cache rows -> values: every dimension's nibble picked by its byte and shift."""
    d = torch.arange(HD, device="cuda")
    m, l, e = d // 32, (d % 32) // 2, d % 2
    nib = m + 4 * e
    code = (rows[..., 4 * l + nib // 2] >> (4 * (nib % 2)).to(torch.uint8)) & 15
    grp = d // qg

    def bf16_at(first):
        lo, hi = rows[..., first + 2 * grp].long(), rows[..., first + 2 * grp + 1].long()
        bits = (lo | hi << 8) << 16
        return torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int().view(torch.float32).double()

    return bf16_at(64 + 2 * (HD // qg)) + bf16_at(64) * code.double()


def _exact_values(x, qg):
    """Rows as quantised: the bf16 roundings on the bits, the codes by counting borders."""
    shape = x.shape
    grp = x.double().reshape(-1, qg)
    lo, hi = grp.min(1).values, grp.max(1).values
    near = lo.float().bfloat16().double()                       # low: the nearest bf16 value, or the one before it
    down = torch.nextafter(near.bfloat16(), torch.full_like(near, -math.inf).bfloat16()).double()
    low = torch.where(near > lo, down, near)
    w = hi - low                                                # scale: the bf16 pattern at or below w / 15, or the next
    below = (((w / 15.0) * (1.0 - 2.0 ** -48)).view(torch.int64) >> 45) << 45
    above = below + (1 << 45)
    mid = 15.0 * (below + (1 << 44)).view(torch.float64)        # exact: 13 bits
    odd = (below >> 45) % 2 == 1
    scale = torch.where((w > mid) | ((w == mid) & odd), above, below).view(torch.float64)
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    d = grp - low[:, None]
    code = torch.zeros_like(d)
    for k in range(15):
        border = (scale * (k + 0.5))[:, None]
        code += (d >= border) if k % 2 else (d > border)        # ties to the even code
    return (low[:, None] + scale[:, None] * code).view(shape)


def exact(case, seed):
    s = prepare(case, seed)
    L, qg, n_kv = case["L"], case["qg"], case["n_kv"]
    if case["op"] == "attn":
        B, n_q = case["B"], case["n_q"]
        out = torch.zeros((B, n_q, HD), dtype=torch.float64, device="cuda")
        lens = [L] * B if s["kv_len"] is None else s["kv_len"].tolist()
        on = s["mask"].tolist()
        for b in range(B):
            for h in range(n_kv):
                pick = (b, h, slice(0, lens[b])) if case["head_major"] else (b, slice(0, lens[b]), h)
                heads = [i for i in range(h * (n_q // n_kv), (h + 1) * (n_q // n_kv))
                         if on[b][i * HD // case["group"]]]
                if not heads:
                    continue
                k, v = _exact_rows(s["k_cache"][pick], qg), _exact_rows(s["v_cache"][pick], qg)
                q = s["q"][b].view(n_q, HD)[heads].double()
                out[b, heads] = torch.softmax(q @ k.T / HD ** 0.5, dim=1) @ v
        return out.view(B, n_q * HD)
    res = []
    for c in ("k", "v"):
        y = torch.zeros((case["n_seq"], case["T"], n_kv, HD), dtype=torch.float64, device="cuda")
        for b in range(case["n_seq"]):
            first = 0 if s["pos"] is None else int(s["pos"][b])
            end = L if s["kv_len"] is None else min(L, int(s["kv_len"][b]))
            i0, i1 = max(0, -first), min(case["T"], end - first)
            if i1 <= i0:
                continue
            if case["op"] == "write":
                x = s[c].view(case["n_seq"], case["T"], n_kv, HD)[b, i0:i1].contiguous()
                y[b, i0:i1] = _exact_values(x, qg)
            else:
                rows = s[c + "_cache"][b].transpose(0, 1) if case["head_major"] else s[c + "_cache"][b]
                y[b, i0:i1] = _exact_rows(rows[first + i0:first + i1], qg)
        res.append(y.view(case["n_seq"] * case["T"], n_kv * HD))
    return tuple(res)
