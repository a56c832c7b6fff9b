"""The calls that a serving program makes of the 8-bit KV cache and of a shared prefix, as timed and checked cases.

Such a program keeps per layer an 8-bit cache (codes and absmax of keys and values), the lengths, and one
workspace. In each decode step it writes the new token and attends over the grown cache (``step``); a chunk
of a prompt is written and everything up to its end read back in bf16, which is what the chunk's own
attention uses (``chunk``); attention alone (``attend``) and reading back alone (``read``), as after a cache
was handed over; and a batch whose sequences begin with the same long prompt, which is kept once
(``prefix``, with bf16 or 8-bit caches). Head dimension 128, bf16 queries, keys and values throughout.

The 8-bit format: M = max |x| of a token's vector, n = rint(127 x / M) half to even, x ~ n M / 127.
"""
import math
import random

import torch

own = False

D = 128
BLOCK = 64
WORKSPACE = 256 << 20                # bytes of scratch that a program keeps for all of its layers
MAX_TOKENS = 4 << 20                 # largest drawn B * Hkv * Lcap
MAX_ROWS = 512 * 65536 * 8           # largest drawn B * G * Hkv * prefix tokens


def _attend(name, **kw):
    case = {"name": name, "kind": "attend", "B": 1, "Hkv": 8, "G": 4, "Lcap": 32768, "Lmin": 0}
    case.update(kw)
    case["Lmin"] = case["Lmin"] or case["Lcap"]
    return case


def listed():
    return [
        # One small layer at a short context: launches and latency are all there is.
        _attend("step_4k_b1", kind="step", Hkv=2, Lcap=4096, Lmin=3000),
        # One layer of a decode step of a busy server: 32 short sequences.
        _attend("step_8k_b32", kind="step", B=32, Lcap=8192, Lmin=500),
        # One sequence of an 8B-model layer (32 query heads, 8 KV heads) at a common context length.
        _attend("attend_32k_b1"),
        # Four long sequences.
        _attend("attend_128k_b4", B=4, Lcap=131072),
        # Mixed lengths from one token on, eight query heads per KV head.
        _attend("attend_ragged_g8", B=16, G=8, Lcap=65536, Lmin=1),
        # A few tokens of two short prompts, starting and ending inside a block.
        {"name": "chunk_37_b3", "kind": "chunk", "B": 3, "Hkv": 2, "Lcap": 1088, "start": 1000, "T": 37, "Tmin": 20},
        # A chunk of a chunked prefill, one of the sequences shorter than the chunk.
        {"name": "chunk_2k_b2", "kind": "chunk", "B": 2, "Hkv": 8, "Lcap": 32768, "start": 10007, "T": 2048, "Tmin": 1500},
        # A whole long cache read back.
        {"name": "read_128k_b1", "kind": "read", "B": 1, "Hkv": 8, "Lcap": 131072, "t0": 0, "t1": 131072},
        # Four conversations at their beginning on a short common prompt.
        {"name": "prefix_2k_b4", "kind": "prefix", "B": 4, "Hkv": 2, "G": 4, "Pcap": 2048, "Pmin": 2000, "Lcap": 128, "Lmin": 1, "bits": 16},
        # A serving batch on one long document.
        {"name": "prefix_32k_b32", "kind": "prefix", "B": 32, "Hkv": 8, "G": 4, "Pcap": 32768, "Pmin": 32768, "Lcap": 1024, "Lmin": 100, "bits": 16},
        # The same on a longer one, everything in 8 bits.
        {"name": "prefix8_128k_b16", "kind": "prefix", "B": 16, "Hkv": 8, "G": 4, "Pcap": 131072, "Pmin": 131072, "Lcap": 4096, "Lmin": 1, "bits": 8},
        # Many sequences with eight query heads per KV head, which share different parts of the document.
        {"name": "prefix_64k_g8_b64", "kind": "prefix", "B": 64, "Hkv": 8, "G": 8, "Pcap": 65536, "Pmin": 0, "Lcap": 512, "Lmin": 0, "bits": 16},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _blocks(n):
    return -(-n // BLOCK) * BLOCK


def draw(rng):
    """Another case: each kind about as often as a program calls it, sizes spread over their ranges."""
    kind = rng.choice(["attend", "attend", "step", "chunk", "read", "prefix", "prefix", "prefix"])
    Hkv, G = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 8])
    if kind == "prefix":
        Pcap = _blocks(_log_int(rng, 64, 131072))
        B = _log_int(rng, 1, min(256, max(1, MAX_ROWS // (G * Hkv * Pcap))))
        Lcap = _blocks(_log_int(rng, 64, max(64, min(4096, MAX_TOKENS // (4 * B * Hkv)))))
        return {"kind": kind, "B": B, "Hkv": Hkv, "G": G, "Pcap": Pcap, "Pmin": rng.choice([Pcap, rng.randrange(Pcap)]),
                "Lcap": Lcap, "Lmin": rng.choice([0, 1, Lcap // 2]), "bits": rng.choice([16, 16, 8])}
    Lcap = _blocks(_log_int(rng, 64, 16384 if kind in ("step", "chunk") else 262144))
    B = _log_int(rng, 1, min(64, max(1, MAX_TOKENS // (Hkv * Lcap * (4 if kind in ("read", "chunk") else 1)))))
    if kind == "chunk":
        T = _log_int(rng, 1, min(Lcap, 4096))
        return {"kind": kind, "B": B, "Hkv": Hkv, "Lcap": Lcap, "start": rng.randrange(Lcap - T + 1), "T": T, "Tmin": rng.randint(0, T)}
    if kind == "read":
        t0 = rng.choice([0, rng.randrange(Lcap // 2)])
        return {"kind": kind, "B": B, "Hkv": Hkv, "Lcap": Lcap, "t0": t0, "t1": rng.choice([Lcap, rng.randrange(t0 + 1, Lcap + 1)])}
    return {"kind": kind, "B": B, "Hkv": Hkv, "G": G, "Lcap": Lcap, "Lmin": rng.choice([Lcap, rng.randrange(1, Lcap)])}


def _spread(case, low, high):
    """Lengths that belong to the case: spread over [low, high], the same for every seed."""
    rng = random.Random(case["Lcap"] * 1000 + case["B"] + low)
    return [rng.randint(low, high) for _ in range(case["B"])]


def _lengths(case):
    """Each sequence's own tokens; a step's include the token that it writes."""
    return _spread(case, case["Lmin"], case["Lcap"])


def _prefix_lengths(case):
    """How much of the prefix each sequence uses: all of Pmin .. Pcap, both ends among them."""
    lens = _spread(case, case["Pmin"], case["Pcap"])
    lens[0], lens[-1] = case["Pmin"], case["Pcap"]
    return lens


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _as_8_bits(x):
    """(codes, absmax) of bf16 vectors [..., 128]."""
    M = x.abs().amax(-1)
    codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    flat, out, m = x.view(-1, D), codes.view(-1, D), M.view(-1, 1)
    for i in range(0, len(flat), 1 << 20):               # in pieces: the quotients are in 64 bits
        part = m[i:i + (1 << 20)].double()
        out[i:i + (1 << 20)] = torch.round(127 * flat[i:i + (1 << 20)].double() / torch.where(part > 0, part, 1)).to(torch.int8)
    return codes, M


def _inputs(case, seed):
    """What the program has in hand, on the GPU: N(0, 1) keys and values, queries that share half of their direction
    within a group. Cache rows behind a sequence hold what an earlier one left there."""
    gen = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, dtype=torch.bfloat16, device="cuda", generator=gen)

    B, Hkv, kind = case["B"], case["Hkv"], case["kind"]
    s = {"kind": kind}
    if kind != "prefix" or case["bits"] == 8:
        s["cache"] = [t for _ in range(2) for t in _as_8_bits(normal(B, Hkv, case["Lcap"], D))]
    else:
        s["cache"] = [normal(B, Hkv, case["Lcap"], D) for _ in range(2)]
    if kind in ("chunk", "step"):
        # keys and values are slices of one projection's output [B, T, (q,) k, v heads, 128]
        T = case.get("T", 1)
        qkv = normal(B, T, (case.get("G", 0) + 2) * Hkv, D)
        s["k_new"], s["v_new"] = qkv[:, :, -2 * Hkv:-Hkv], qkv[:, :, -Hkv:]
    if kind == "chunk":
        counts = _spread(case, case["Tmin"], case["T"])
        s.update(start=_int32([case["start"]] * B), counts=_int32(counts), t0=0, t1=case["start"] + max(counts),
                 lens=_int32([case["start"] + c for c in counts]))
        return s
    if kind == "read":
        return dict(s, t0=case["t0"], t1=case["t1"], lens=None)
    q = 0.5 * normal(B, Hkv, 1, D).float() + math.sqrt(0.75) * normal(B, Hkv, case["G"], D).float()
    s["q"] = q.view(B, Hkv * case["G"], D).bfloat16()
    s["lens"] = _int32(_lengths(case))
    if kind == "step":
        s["start"] = s["lens"] - 1
    if kind == "prefix":
        p = [normal(1, Hkv, case["Pcap"], D) for _ in range(2)]
        s["prefix"] = [t for x in p for t in _as_8_bits(x)] if case["bits"] == 8 else p
        s["prefix_lens"] = _int32(_prefix_lengths(case))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if "q" in s:
        s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms, in 32 bits ---------------------------------------------------------------------------------

def _plain_write(s):
    """The new tokens' codes and absmax at their positions in the cache."""
    k_codes, k_absmax, v_codes, v_absmax = s["cache"]
    B, T = s["k_new"].shape[:2]
    t = torch.arange(T, device="cuda").expand(B, T)
    at = s["start"].view(B, 1) + t
    valid = at < k_codes.shape[2]
    if "counts" in s:
        valid = valid & (t < s["counts"].view(B, 1))
    b, t = valid.nonzero(as_tuple=True)
    at = at[b, t]
    k, v = s["k_new"][b, t], s["v_new"][b, t]                            # [N, Hkv, 128]
    kM, vM = k.abs().amax(-1), v.abs().amax(-1)
    # in 64 bits: a quotient next to a half goes to the right side
    kd, vd = kM.double().unsqueeze(-1), vM.double().unsqueeze(-1)
    k_codes[b, :, at] = torch.round(127 * k.double() / torch.where(kd > 0, kd, 1)).to(torch.int8)
    v_codes[b, :, at] = torch.round(127 * v.double() / torch.where(vd > 0, vd, 1)).to(torch.int8)
    k_absmax[b, :, at], v_absmax[b, :, at] = kM, vM


def _plain_values(cache, t0=0, t1=None):
    """Keys and values in 32 bits: [B, Hkv, n, 128]."""
    if len(cache) == 2:
        return [x[:, :, t0:t1].float() for x in cache]
    kc, kM, vc, vM = [x[:, :, t0:t1].float() for x in cache]
    return kc * (kM / 127).unsqueeze(-1), vc * (vM / 127).unsqueeze(-1)


def _plain_read(s):
    k, v = _plain_values(s["cache"], s["t0"], s["t1"])
    if s["lens"] is not None:
        here = (torch.arange(s["t0"], s["t1"], device="cuda") < s["lens"].view(-1, 1)).view(len(k), 1, -1, 1)
        k, v = torch.where(here, k, 0), torch.where(here, v, 0)
    return k.bfloat16(), v.bfloat16()


def _plain_attention(s):
    """softmax over the prefix (if there is one) and the sequence's own tokens."""
    B, Hq, _ = s["q"].shape
    k, v = _plain_values(s["cache"])
    Hkv = k.shape[1]
    q = s["q"].float().view(B, Hkv, -1, D) / math.sqrt(D)
    n = torch.arange(k.shape[2], device="cuda")
    z = torch.where((n < s["lens"].view(B, 1)).view(B, 1, 1, -1), q @ k.transpose(-1, -2), -math.inf)
    m = z.amax(-1, keepdim=True)
    if "prefix" in s:
        pk, pv = _plain_values(s["prefix"])
        rows = q.transpose(0, 1).reshape(Hkv, -1, D)                     # [Hkv, B * G, 128]
        used = torch.arange(pk.shape[2], device="cuda") < s["prefix_lens"].view(B, 1)
        zp = (rows @ pk[0].transpose(-1, -2)).view(Hkv, B, Hq // Hkv, -1)
        zp = torch.where(used.view(1, B, 1, -1), zp, -math.inf)
        m = torch.maximum(m, zp.amax(-1, keepdim=True).transpose(0, 1))
    m0 = torch.where(m == -math.inf, 0, m)
    p = torch.exp(z - m0)
    total, out = p.sum(-1, keepdim=True), p @ v
    if "prefix" in s:
        p = torch.exp(zp - m0.transpose(0, 1))
        total = total + p.sum(-1, keepdim=True).transpose(0, 1)
        out = out + (p.view(Hkv, -1, p.shape[-1]) @ pv[0]).view(Hkv, B, -1, D).transpose(0, 1)
    out = torch.where(total > 0, out / total, 0).view(B, Hq, D).bfloat16()
    return out, (m0 + torch.log(total)).view(B, Hq)


def run(s):
    kind = s["kind"]
    if own:
        from paper_2609_00097_amd import ffd
        if kind in ("chunk", "step"):
            ffd.write_kv8(s["k_new"], s["v_new"], s["cache"], s["start"], counts=s.get("counts"))
        if kind in ("chunk", "read"):
            return ffd.read_kv8(s["cache"], s["t0"], s["t1"], seq_lens=s["lens"])
        if kind == "prefix":
            return ffd.shared_prefix_decode_attention(s["q"], s["prefix"], s["prefix_lens"], s["cache"], s["lens"],
                                                      workspace=s["workspace"])
        out = ffd.kv8_decode_attention(s["q"], s["cache"], s["lens"], workspace=s["workspace"])
        return out + (s["cache"][1], s["cache"][3]) if kind == "step" else out
    if kind in ("chunk", "step"):
        _plain_write(s)
    if kind in ("chunk", "read"):
        return _plain_read(s)
    # a step has written a row of the cache: the codes show in the attention, the absmax is returned
    return _plain_attention(s) + ((s["cache"][1], s["cache"][3]) if kind == "step" else ())


# ---- the same in 64 bits, one (sequence, KV head) after another ---------------------------------------------------

def _exact_8_bits(x):
    """The values that bf16 vectors x stand for in 8 bits."""
    x = x.double()
    M = x.abs().max(dim=-1, keepdim=True).values
    step = M / 127
    n = torch.round(x * 127 / M.clamp_min(1e-300))
    return n * step


def _exact_value(cache, which, b, h, n):
    """float64 [n, 128]: the first n keys (which = 0) or values (1) of sequence b, KV head h."""
    if len(cache) == 2:
        return cache[which][b, h, :n].double()
    return cache[2 * which][b, h, :n].double() * (cache[2 * which + 1][b, h, :n].double() / 127).unsqueeze(1)


def exact(case, seed):
    s = _inputs(case, seed)
    B, Hkv, kind = case["B"], case["Hkv"], case["kind"]
    if kind in ("chunk", "read"):
        n = s["t1"] - s["t0"]
        both = []
        for which in range(2):
            out = torch.zeros(B, Hkv, n, D, dtype=torch.float64, device="cuda")
            for b in range(B):
                for h in range(Hkv):
                    x = _exact_value(s["cache"], which, b, h, s["t1"])
                    if kind == "chunk":
                        c = int(s["counts"][b])
                        x[case["start"]:case["start"] + c] = _exact_8_bits((s["k_new"], s["v_new"])[which][b, :c, h])
                        x[case["start"] + c:] = 0
                    out[b, h] = x[s["t0"]:]
            both.append(out)
        return tuple(both)
    G, lens = case["G"], _lengths(case)
    out = torch.zeros(B, Hkv * G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hkv * G), -math.inf, dtype=torch.float64, device="cuda")
    for h in range(Hkv):
        if kind == "prefix":
            shared = [_exact_value(s["prefix"], w, 0, h, case["Pcap"]) for w in range(2)]
            shared_lens = _prefix_lengths(case)
        for b in range(B):
            k, v = [_exact_value(s["cache"], w, b, h, lens[b]) for w in range(2)]
            if kind == "step":
                k[-1], v[-1] = _exact_8_bits(s["k_new"][b, 0, h]), _exact_8_bits(s["v_new"][b, 0, h])
            q = s["q"][b, h * G:(h + 1) * G].double()
            z, values = [q @ k.T], [v]
            if kind == "prefix":
                z.append(q @ shared[0][:shared_lens[b]].T)
                values.append(shared[1][:shared_lens[b]])
            z = torch.cat(z, 1) * D ** -0.5
            if z.shape[1] == 0:
                continue
            rows = slice(h * G, (h + 1) * G)
            lse[b, rows] = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[b, rows, None])
            out[b, rows] = p[:, :lens[b]] @ values[0]
            if kind == "prefix":
                out[b, rows] += p[:, lens[b]:] @ values[1]
    return (out, lse, None, None) if kind == "step" else (out, lse)


def work(case):
    """Bytes and operations one pass cannot do without. A (token, KV head) of an 8-bit cache takes 2 (128 + 2)
    bytes, of a bf16 one 2 * 256; a shared prefix is read once, up to the longest use of it."""
    B, Hkv, kind = case["B"], case["Hkv"], case["kind"]
    row8, row16 = 2 * (D + 2), 4 * D
    if kind == "read":
        tokens = B * Hkv * (case["t1"] - case["t0"])
        return {"bytes": tokens * (row8 + row16), "flops": 2 * D * tokens}
    if kind == "chunk":
        counts = _spread(case, case["Tmin"], case["T"])
        new, end = Hkv * sum(counts), case["start"] + max(counts)
        old = Hkv * B * case["start"]
        # the new tokens are read, written to the cache and read back; every row of the result is written
        return {"bytes": new * (row16 + row8) + old * row8 + B * Hkv * end * row16, "flops": 2 * D * (old + 4 * new)}
    G, own_tokens = case["G"], Hkv * sum(_lengths(case))
    ends = 2 * B * Hkv * G * D * 2 + 4 * B * Hkv * G
    if kind == "step":
        ends += B * Hkv * (row16 + row8)
    row = row16 if case.get("bits") == 16 else row8
    bytes_, flops = own_tokens * row + ends, 4 * D * G * own_tokens
    if kind == "prefix":
        bytes_ += Hkv * max(_prefix_lengths(case)) * row
        flops += 4 * D * G * Hkv * sum(_prefix_lengths(case))
    return {"bytes": bytes_, "flops": flops}
