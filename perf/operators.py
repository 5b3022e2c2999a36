"""Operators for decoding from compressed storage, and the calls they are measured by.

  w4      narrow product with 4-bit weights and group scales        nm_matmul_w4
  w4pack  weights to 4 bits and back                                nm_w4_quantize, nm_w4_dequantize
  write   latent-cache rows normalised, rotated, quantised, stored  nm_mla_cache_write_q8
  read    quantised cache rows back to bf16                         nm_mla_cache_read_q8
  attend  latent attention of a batch over the quantised cache,     nm_mla_attention_q8
          a prefix shared by all sequences and rows of their own

Weights in 4 bits: blocks of 16 columns n by 64 k, 512 bytes each, the blocks of one 16-column strip behind each other.  Byte
4 * (4 * (4 g + t) + j) + b of a block holds two codes; code p = 2 b + (high nibble) belongs to column g + 8 (p & 1) and
k = 32 (j >> 1) + 8 t + 4 (j & 1) + 2 ((p >> 1) & 1) + (p >> 2).  Scales: [group of k][16-column strip][8][2], the pair being columns
g and g + 8.  weight = (code - 8) * scale.

Quantised cache record of a row (kv_lora 512, rope 64): 512 e4m3 codes, 64 bf16, one fp32 scale (a power of two), 12 bytes unused;
row = scale * (codes | bf16 part).
"""
import math

import torch

own = False

KV, ROPE = 512, 64
REC = KV + 2 * ROPE + 16
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "bf16_f32out": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the smallest projection of the decode step (latent down-projection), one token
        {"name": "w4 one token 7168x576", "op": "w4", "M": 1, "N": 576, "K": 7168, "group": 128, "dtype": "bf16"},
        # the output projection, one token: the step's largest weight
        {"name": "w4 one token 16384x7168", "op": "w4", "M": 1, "N": 7168, "K": 16384, "group": 64, "dtype": "bf16"},
        # a full narrow batch over a wide matrix with a ragged edge and the smallest groups
        {"name": "w4 16 tokens 7168x18427", "op": "w4", "M": 16, "N": 18427, "K": 7168, "group": 32, "dtype": "f16"},
        # laying out weights once when a model is loaded
        {"name": "w4pack 7168x576 rows", "op": "w4pack", "N": 576, "K": 7168, "group": 128, "dtype": "bf16", "layout": 0},
        {"name": "w4pack 16384x7168 columns", "op": "w4pack", "N": 7168, "K": 16384, "group": 64, "dtype": "f16", "layout": 1},
        # the new rows of a decode batch; the rows of a prompt
        {"name": "write 16 rows", "op": "write", "T": 16, "rows": 1024, "full": True},
        {"name": "write 6001 rows", "op": "write", "T": 6001, "rows": 7000, "full": True},
        # rows handed to code that wants bf16: a short sequence, a long one
        {"name": "read 300 rows", "op": "read", "n": 300, "rows": 512},
        {"name": "read 50001 rows", "op": "read", "n": 50001, "rows": 65536},
        # one short sequence, few heads (a shard of the model): latency
        {"name": "attend 1x16 heads, 257 rows", "op": "attend", "T": 1, "H": 16, "prefix": 0, "mean": 257},
        # a ragged decode batch without a prefix, lengths from nothing to twice the mean
        {"name": "attend 16x128 heads, ragged 4096", "op": "attend", "T": 16, "H": 128, "prefix": 0, "mean": 4096},
        # a batch behind one long system prompt
        {"name": "attend 16x128 heads, prefix 32768", "op": "attend", "T": 16, "H": 128, "prefix": 32768, "mean": 500},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["w4", "w4", "w4pack", "write", "read", "attend", "attend"])
    if op == "w4":
        M, K = rng.randint(1, 16), _log(rng, 64, 18432)
        if rng.random() < 0.6:
            K = max(64, K // 64 * 64)
        N = _log(rng, 16, min(24576, 16384 * 7168 // K))
        return {"op": op, "M": M, "N": N, "K": K, "group": rng.choice([32, 64, 128]), "dtype": rng.choice(sorted(TYPES))}
    if op == "w4pack":
        K = _log(rng, 64, 18432)
        return {"op": op, "N": _log(rng, 16, min(24576, 16384 * 7168 // K)), "K": K, "group": rng.choice([32, 64, 128]), "dtype": rng.choice(["bf16", "f16"]),
                "layout": rng.randint(0, 1)}
    if op == "write":
        T = _log(rng, 1, 6000)
        return {"op": op, "T": T, "rows": min(7000, T + _log(rng, 1, 1000)), "full": rng.random() < 0.7}
    if op == "read":
        n = _log(rng, 1, 50000)
        return {"op": op, "n": n, "rows": _log(rng, 1, 65536)}
    T, H = _log(rng, 1, 32), rng.choice([8, 16, 24, 32, 64, 128, 128])
    prefix = 0 if rng.random() < 0.4 else _log(rng, 1, min(32768, 16 * 128 * 32768 // (T * H)))
    mean = _log(rng, 1, min(8192, 65536 // T))
    return {"op": op, "T": T, "H": H, "prefix": prefix, "mean": mean}


def lengths(case):
    """Own rows of each sequence: from none to twice the mean, in an order that is neither rising nor falling."""
    T, mean = case["T"], case["mean"]
    if T == 1:
        return [mean]
    return [2 * mean * ((7 * t + 3) % T) // (T - 1) if T % 7 else 2 * mean * t // (T - 1) for t in range(T)]


def padded(case):
    return -(-case["N"] // 16), -(-case["K"] // 64), -(-case["K"] // case["group"])


def work(case):
    op = case["op"]
    if op == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        out = 4 if case["dtype"] == "bf16_f32out" else 2
        return {"bytes": N * K / 2 + 2 * N * -(-K // case["group"]) + 2 * M * K + out * M * N, "flops": 2 * M * N * K}
    if op == "w4pack":  # there and back: weights in, codes and scales out, and the other way
        N, K = case["N"], case["K"]
        return {"bytes": 2 * (2 * N * K + N * K / 2 + 2 * N * -(-K // case["group"])), "flops": 6 * N * K}
    if op == "write":
        return {"bytes": case["T"] * (2 * (KV + ROPE) + 8 + (4 * ROPE if case["full"] else 0) + KV + 2 * ROPE + 4), "flops": case["T"] * 8 * (KV + ROPE)}
    if op == "read":
        return {"bytes": min(case["n"], case["rows"]) * (KV + 2 * ROPE + 4) + case["n"] * (8 + 2 * (KV + ROPE)), "flops": case["n"] * (KV + ROPE)}
    T, H, own_rows = case["T"], case["H"], sum(lengths(case))
    rows = case["prefix"] + own_rows
    return {"bytes": rows * (KV + 2 * ROPE + 4) + T * H * (2 * (KV + ROPE) + 2 * KV + 4), "flops": 2 * H * (KV + ROPE + KV) * (T * case["prefix"] + own_rows)}


def _records(n, g):
    """Cache records of n rows ~ N(0, 1), each row with a scale of its own, as they lie in memory."""
    x = torch.randn(n, KV + ROPE, generator=g, device="cuda") * torch.exp2(torch.randint(-2, 3, (n, 1), generator=g, device="cuda").float())
    s = torch.exp2(torch.ceil(torch.log2(x[:, :KV].abs().amax(1, keepdim=True) / 448)))
    rec = torch.zeros(n, REC, dtype=torch.uint8, device="cuda")
    rec[:, :KV] = (x[:, :KV] / s).to(torch.float8_e4m3fn).view(torch.uint8)
    rec[:, KV:KV + 2 * ROPE] = (x[:, KV:] / s).to(torch.bfloat16).view(torch.uint8)
    rec[:, KV + 2 * ROPE:KV + 2 * ROPE + 4] = s.view(torch.uint8)
    return rec


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    s, op = dict(case), case["op"]
    if op == "w4":
        t = TYPES[case["dtype"]]
        nb, kb, groups = padded(case)
        s["A"] = randn(case["M"], case["K"]).to(t)
        s["packed"] = torch.randint(0, 256, (nb * kb * 512,), generator=g, device="cuda", dtype=torch.uint8)
        s["scales"] = ((0.5 + torch.rand(groups * nb * 16, generator=g, device="cuda")) * (0.02 / 4)).to(t)
        s["C"] = torch.empty(case["M"], case["N"], dtype=torch.float32 if case["dtype"] == "bf16_f32out" else t, device="cuda")
    elif op == "w4pack":
        t = TYPES[case["dtype"]]
        nb, kb, groups = padded(case)
        shape = (case["N"], case["K"]) if case["layout"] else (case["K"], case["N"])
        s["B"] = (randn(*shape) * 0.02).to(t)
        s["packed"] = torch.empty(nb * kb * 512, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(groups * nb * 16, dtype=t, device="cuda")
        s["back"] = torch.empty_like(s["B"])
    elif op == "write":
        s["x"] = randn(case["T"], KV + ROPE).to(torch.bfloat16)
        s["index"] = torch.randperm(case["rows"], generator=g, device="cuda")[:case["T"]]
        if case["T"] > 2:
            s["index"][case["T"] // 2] = -1  # a padding token of the batch: written nowhere
        s["cache"] = torch.zeros(case["rows"], REC, dtype=torch.uint8, device="cuda")
        s["gamma"] = (1 + 0.02 * randn(KV)).to(torch.bfloat16) if case["full"] else None
        pos = torch.randint(0, 32768, (case["T"], 1), generator=g, device="cuda").double()
        angle = pos * 10000.0 ** (-torch.arange(0, ROPE, 2, device="cuda").double() / ROPE)
        s["cos_sin"] = torch.stack((angle.cos(), angle.sin()), -1).reshape(case["T"], ROPE).float() if case["full"] else None
    elif op == "read":
        s["cache"] = _records(case["rows"], g)
        s["index"] = torch.randint(0, case["rows"], (case["n"],), generator=g, device="cuda")
        if case["n"] > 2:
            s["index"][case["n"] // 2] = -1  # no such row: zeros
        s["rows_out"] = torch.empty(case["n"], KV + ROPE, dtype=torch.bfloat16, device="cuda")
    else:
        T, H, lens = case["T"], case["H"], lengths(case)
        s["lens"], s["most"] = lens, max(max(lens), 1)
        s["Q"] = randn(T, H, KV + ROPE).to(torch.bfloat16)
        s["shared"] = _records(case["prefix"], g) if case["prefix"] else None
        s["cache"] = _records(T * s["most"], g).view(T, s["most"], REC)
        s["o"] = torch.empty(T, H, KV, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(T, H, dtype=torch.float32, device="cuda")
        s["scale"] = 192 ** -0.5
        s["workspace"] = torch.empty(160 << 20, dtype=torch.uint8, device="cuda")
    return s


def _weights(s):
    """The 4-bit weights as fp32 [N][K]."""
    nb, kb, groups = padded(s)
    w = s["packed"].view(nb, kb, 8, 4, 2, 2, 4)  # strip, block, g, t, j >> 1, j & 1, byte
    w = torch.stack((w & 15, w >> 4), -1).view(nb, kb, 8, 4, 2, 2, 2, 2, 2)  # the byte's bits: p >> 2, (p >> 1) & 1; nibble: p & 1
    w = w.permute(0, 8, 2, 1, 4, 3, 5, 7, 6).reshape(nb * 16, kb * 64)
    sc = s["scales"].view(groups, nb, 8, 2).permute(1, 3, 2, 0).reshape(nb * 16, groups).float()
    sc = sc.repeat_interleave(s["group"], 1)[:s["N"], :s["K"]]
    return (w[:s["N"], :s["K"]].float() - 8) * sc


def _rows(rec):
    scale = rec[..., KV + 2 * ROPE:KV + 2 * ROPE + 4].contiguous().view(torch.float32)
    codes = rec[..., :KV].contiguous().view(torch.float8_e4m3fn).float()
    return torch.cat((codes, rec[..., KV:KV + 2 * ROPE].contiguous().view(torch.bfloat16).float()), -1) * scale


def _parts(cache):
    """A quantised cache as the values it stands for: codes, key part, scales."""
    return cache[:, :KV].view(torch.float8_e4m3fn), cache[:, KV:KV + 2 * ROPE].view(torch.bfloat16), cache[:, KV + 2 * ROPE:KV + 2 * ROPE + 4].view(torch.float32)


def _plain_w4(s):
    s["C"].copy_(s["A"].float() @ _weights(s).T)
    return s["C"]


def _plain_w4pack(s):
    nb, kb, groups = padded(s)
    N, K, grp = s["N"], s["K"], s["group"]
    w = s["B"].float() if s["layout"] else s["B"].float().T
    full = torch.zeros(nb * 16, groups * grp, device="cuda")
    full[:N, :K] = w
    full = full.view(nb * 16, groups, grp)
    scale = (full.abs().amax(2) / 7).to(s["scales"].dtype)
    sc = scale.float()[:, :, None]
    code = torch.where(sc > 0, torch.round(full / sc), 0).clamp(-8, 7) + 8
    s["scales"].copy_(scale.view(nb, 2, 8, groups).permute(3, 0, 2, 1).reshape(-1))
    back = ((code - 8) * sc).reshape(nb * 16, groups * grp)[:N, :K]
    cells = torch.full((nb * 16, kb * 64), 8, dtype=torch.uint8, device="cuda")
    keep = min(kb * 64, groups * grp)
    cells[:, :keep] = code.reshape(nb * 16, groups * grp)[:, :keep].to(torch.uint8)
    c = cells.view(nb, 2, 8, kb, 2, 4, 2, 2, 2).permute(0, 3, 2, 5, 4, 6, 8, 7, 1).reshape(-1, 2)
    s["packed"].copy_(c[:, 0] | (c[:, 1] << 4))
    s["back"].copy_(back if s["layout"] else back.T)
    return s["scales"], s["back"]


def _plain_write(s):
    x = s["x"].float()
    y, r = x[:, :KV], x[:, KV:]
    if s["gamma"] is not None:
        y = y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS) * s["gamma"].float()
    if s["cos_sin"] is not None:
        c, sn = s["cos_sin"][:, 0::2], s["cos_sin"][:, 1::2]
        r = torch.stack((r[:, 0::2] * c - r[:, 1::2] * sn, r[:, 0::2] * sn + r[:, 1::2] * c), -1).reshape(-1, ROPE)
    m, e = torch.frexp(y.abs().amax(1, keepdim=True))
    e = torch.where(m == 0, 0, torch.where(m <= 0.875, e - 9, e - 8).clamp(-32, 32))
    inv = torch.exp2(-e.float())
    keep = s["index"] >= 0
    at = s["index"][keep]
    s["cache"][at, :KV] = (y * inv).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)[keep]
    s["cache"][at, KV:KV + 2 * ROPE] = (r * inv).to(torch.bfloat16).view(torch.uint8)[keep]
    s["cache"][at, KV + 2 * ROPE:KV + 2 * ROPE + 4] = torch.exp2(e.float()).view(torch.uint8)[keep]
    return _parts(s["cache"])


def _plain_read(s):
    rows = _rows(s["cache"][s["index"].clamp(min=0)])
    s["rows_out"].copy_(torch.where(s["index"][:, None] >= 0, rows, 0))
    return s["rows_out"]


def _plain_attend(s):
    T, H = s["T"], s["H"]
    q = s["Q"].float() * s["scale"]
    mine = _rows(s["cache"])
    x = q @ mine.transpose(1, 2)
    out_of = torch.arange(s["most"], device="cuda")[None, :] >= torch.tensor(s["lens"], device="cuda")[:, None]
    x = x.masked_fill(out_of[:, None, :], -math.inf)
    if s["shared"] is not None:
        pre = _rows(s["shared"])
        x = torch.cat(((q.reshape(T * H, -1) @ pre.T).view(T, H, -1), x), -1)
    m = x.amax(-1, keepdim=True)
    p = torch.where(m > -math.inf, torch.exp(x - m), 0)
    total = p.sum(-1, keepdim=True)
    n = s["prefix"]
    o = p[..., n:] @ mine[..., :KV]
    if s["shared"] is not None:
        o = o + (p[..., :n].reshape(T * H, n) @ pre[:, :KV]).view(T, H, KV)
    s["o"].copy_(torch.where(total > 0, o / total, 0))
    s["lse"].copy_((m + torch.log(total))[..., 0])
    return s["o"], s["lse"]


def run(s):
    op = s["op"]
    if own:
        import paper_2609_16009_b200 as nm

        if op == "w4":
            nm.nm_matmul_w4(s["A"], s["packed"], s["scales"], s["C"], s["M"], s["N"], s["K"], s["group"], _dtype(nm, s["dtype"]))
            return s["C"]
        if op == "w4pack":
            d = _dtype(nm, s["dtype"])
            nm.nm_w4_quantize(s["B"], s["packed"], s["scales"], s["N"], s["K"], s["group"], d, s["layout"])
            nm.nm_w4_dequantize(s["packed"], s["scales"], s["back"], s["N"], s["K"], s["group"], d, s["layout"])
            return s["scales"], s["back"]
        if op == "write":
            nm.nm_mla_cache_write_q8(s["x"], s["gamma"], s["cos_sin"], s["index"], s["cache"], s["rows"], s["T"], KV, ROPE, EPS)
            return _parts(s["cache"])
        if op == "read":
            nm.nm_mla_cache_read_q8(s["cache"], s["rows"], s["index"], s["rows_out"], s["n"], KV, ROPE)
            return s["rows_out"]
        nm.nm_mla_attention_q8(s["Q"], s["shared"], s["prefix"], s["cache"], s["most"] * REC, s["lens"], s["o"], None, s["lse"], s["H"], KV, ROPE, s["scale"],
                               s["workspace"])
        return s["o"], s["lse"]
    return {"w4": _plain_w4, "w4pack": _plain_w4pack, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[op](s)


def _dtype(nm, name):
    return {"bf16": nm.BF16, "bf16_f32out": nm.BF16_F32OUT, "f16": nm.F16}[name]


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def _codes64(case, packed):
    """Codes [N16][K64] by the formula of each nibble's place."""
    nb, kb, _ = padded(case)
    n, k = torch.arange(nb * 16, device="cuda")[:, None], torch.arange(kb * 64, device="cuda")[None, :]
    r, kk = n % 16, k % 64
    j, t = 2 * (kk // 32) + (kk % 8) // 4, (kk % 32) // 8
    p = (r // 8) + 2 * ((kk % 4) // 2) + 4 * (kk % 2)
    byte = (n // 16 * kb + k // 64) * 512 + 4 * (4 * (4 * (r % 8) + t) + j) + p // 2
    return (packed[byte].int() >> (4 * (p % 2)).int()) & 15


def _scales64(case, scales):
    nb, kb, _ = padded(case)
    n, k = torch.arange(nb * 16, device="cuda")[:, None], torch.arange(case["K"], device="cuda")[None, :]
    return scales.double()[(k // case["group"] * nb + n // 16) * 16 + 2 * (n % 8) + (n % 16) // 8]


def _e4m3(x):
    """x in 64 bits to the nearest e4m3 value, ties to the even one; not beyond 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _rows64(rec):
    b = rec.reshape(-1, REC)
    code = b[:, :KV].long()
    exp, man = (code >> 3) & 15, code & 7
    v = torch.where(exp == 0, man.double() * 2.0 ** -9, (8 + man).double() * torch.exp2(exp.double() - 10)) * (1 - 2 * (code >> 7)).double()
    tail = b[:, KV:KV + 2 * ROPE].contiguous().view(torch.bfloat16).double()
    sc = b[:, KV + 2 * ROPE:KV + 2 * ROPE + 4].contiguous().view(torch.float32).double()
    return (torch.cat((v, tail), 1) * sc).view(*rec.shape[:-1], KV + ROPE)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    N, K = case.get("N"), case.get("K")
    if op == "w4":
        w = (_codes64(case, s["packed"])[:N, :K].double() - 8) * _scales64(case, s["scales"])[:N]
        return s["A"].double() @ w.T
    if op == "w4pack":
        nb, kb, groups = padded(case)
        w = s["B"].double() if case["layout"] else s["B"].double().T
        full = torch.zeros(nb * 16, groups * case["group"], device="cuda", dtype=torch.float64)
        full[:N, :K] = w
        amax = full.view(nb * 16, groups, -1).abs().amax(2)
        scale = (amax / 7).to(s["scales"].dtype).double()
        n, i = torch.arange(nb * 16, device="cuda")[:, None], torch.arange(groups, device="cuda")[None, :]
        flat = torch.zeros(groups * nb * 16, device="cuda", dtype=torch.float64)
        flat[((i * nb + n // 16) * 16 + 2 * (n % 8) + (n % 16) // 8).reshape(-1)] = scale.reshape(-1)
        return flat, None  # a code next to a border falls either way in 64 bits
    if op == "write":
        x = s["x"].double()
        y, r = x[:, :KV], x[:, KV:]
        if case["full"]:
            y = y / ((y ** 2).mean(1, keepdim=True) + EPS).sqrt() * s["gamma"].double()
            z = torch.view_as_complex(r.reshape(-1, ROPE // 2, 2).contiguous()) * torch.view_as_complex(s["cos_sin"].double().reshape(-1, ROPE // 2, 2).contiguous())
            r = torch.view_as_real(z).reshape(-1, ROPE)
        scale = torch.exp2(torch.ceil(torch.log2(y.abs().amax(1, keepdim=True) / 448)))
        codes, key, scales = (torch.zeros(case["rows"], n, device="cuda", dtype=torch.float64) for n in (KV, ROPE, 1))
        keep = s["index"] >= 0
        at = s["index"][keep]
        codes[at], key[at], scales[at] = _e4m3(y / scale)[keep], (r / scale)[keep], scale[keep]
        return codes, key, scales
    if op == "read":
        return _rows64(s["cache"])[s["index"].clamp(min=0)] * (s["index"] >= 0)[:, None]
    T, H = case["T"], case["H"]
    pre = _rows64(s["shared"]) if s["shared"] is not None else torch.zeros(0, KV + ROPE, device="cuda", dtype=torch.float64)
    out, lse = [], []
    for t in range(T):
        rows = torch.cat((pre, _rows64(s["cache"][t, :s["lens"][t]])))
        if not len(rows):
            out.append(torch.zeros(H, KV, device="cuda", dtype=torch.float64))
            lse.append(torch.full((H,), -math.inf, device="cuda", dtype=torch.float64))
            continue
        x = s["Q"][t].double() @ rows.T * s["scale"]
        lse.append(torch.logsumexp(x, 1))
        out.append(torch.softmax(x, 1) @ rows[:, :KV])
    return torch.stack(out), torch.stack(lse)
