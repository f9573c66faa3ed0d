"""What the prefix-cache operators are timed on: caches held in 4 bits, the
attention that reads them, the attention weight that cached tokens gather, and
the eviction of tokens by it.

A case is a dict of plain values.  Its "kind" says which operator it takes:

  pack    the K and V caches of several robots' prefixes, all layers, to 4 bits
          and back to the model's type (kv_quantize, kv_expand)
  attend  one layer's attention of every request's action tokens over its own
          4-bit prefix cache and its action tokens (KvAttention.attention)
  score   the same with its log-sum-exp, and the attention weight that every
          cached token gathers (KvAttention.mass); caches in 4 bits or the
          model's type
  evict   per layer and KV head, the tokens worth most are kept and the caches
          compacted (kv_evict)

Horizons are comma-separated sets each request draws from; prefix lengths are
uniform in [prefix_lo, prefix_hi].  `cross`: the layer attends over the prefix
only (the even layers of the alternating layout).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
GROUP = 32       # elements along head_dim that share a scale
ALIGN = 256      # bytes between caches in one allocation
KEY_STD = 3.0    # prefix keys are larger than unit normal, so attention is peaked rather than uniform


class Shape:
    """The sizes a model configuration is made of."""

    def __init__(self, case):
        self.n_layers, self.d_model, self.d_mlp, self.action_dim, self.time_emb_dim = case["layers"], 1024, 4096, 32, 1024
        self.n_q_heads, self.n_kv_heads, self.head_dim = case["n_q"], case["n_kv"], case["head_dim"]
        self.rms_eps, self.attention_layout = 1e-6, 1 if case.get("cross") else 0


# ---------------------------------------------------------------- the cases

def _case(kind, robots, prefix, heads, layers, dtype, **more):
    return {"kind": kind, "robots": robots, "prefix_lo": prefix[0], "prefix_hi": prefix[1], "n_q": heads[0],
            "n_kv": heads[1], "head_dim": heads[2], "layers": layers, "dtype": dtype, **more}


def _named(name, c):
    return {"name": name, **c}


PI0 = (8, 1, 256)   # 8 query heads over one 256-wide KV head, 18 layers


def listed():
    return [
        # a new robot's prefix (three camera images and an instruction) goes into the 4-bit cache and comes back
        _named("pack_one", _case("pack", 1, (816, 816), PI0, 18, "bf16")),
        # the prefixes of 32 robots, after one call of the prefix producer
        _named("pack_32", _case("pack", 32, (512, 1280), PI0, 18, "bf16")),
        # one action token of one robot: the smallest call, launches count
        _named("attend_token", _case("attend", 1, (816, 816), PI0, 1, "bf16", horizons="1", cross=False)),
        # 32 robots of horizon 50
        _named("attend_32", _case("attend", 32, (600, 1024), PI0, 1, "bf16", horizons="50", cross=False)),
        # a fleet, short and long horizons mixed
        _named("attend_fleet", _case("attend", 256, (512, 1280), PI0, 1, "bf16", horizons="16,50", cross=False)),
        # the largest: a big fleet with long contexts
        _named("attend_512_long", _case("attend", 512, (1024, 2048), PI0, 1, "bf16", horizons="50", cross=False)),
        # a long observation history, single tokens over it
        _named("attend_history", _case("attend", 2, (60001, 131072), (8, 2, 128), 1, "bf16", horizons="1", cross=False)),
        # cross-attention of grouped 64-wide heads, odd and ragged lengths
        _named("attend_cross64", _case("attend", 37, (1, 700), (16, 4, 64), 1, "bf16", horizons="1,17,50", cross=True)),
        # which of a fleet's cached tokens the actions look at: caches in the model's type
        _named("score_fleet", _case("score", 256, (512, 1280), PI0, 1, "bf16", horizons="16,50", cross=False, bits=16)),
        # the same for one robot over its 4-bit cache
        _named("score_one", _case("score", 1, (816, 816), PI0, 1, "bf16", horizons="50", cross=False, bits=4)),
        # half of 32 robots' prefix tokens leave the caches; the last ones (the instruction) stay
        _named("evict_32", _case("evict", 32, (512, 1280), PI0, 18, "bf16", share=0.5, first=4, last=48)),
        # one robot, three quarters leave
        _named("evict_one", _case("evict", 1, (816, 816), PI0, 18, "bf16", share=0.25, first=4, last=48)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [PI0, PI0, (8, 2, 128), (16, 4, 64), (4, 4, 32), (3, 3, 128)]


def draw(rng):
    kind = rng.choice(["pack", "attend", "attend", "attend", "score", "score", "evict"])
    heads = rng.choice(HEADS)
    if heads == (3, 3, 128) and kind in ("attend", "score"):
        heads = (6, 3, 128)
    fp32 = rng.random() < 0.15
    lo = _log_int(rng, 1, 1024)
    prefix = (lo, lo + rng.randint(0, 256 if fp32 else 768))
    if kind in ("pack", "evict"):
        c = _case(kind, _log_int(rng, 1, 24), (min(lo, 900), min(lo, 900) + rng.randint(0, 380)), heads,
                  rng.randint(1, 9 if heads[1] > 2 else 18), "fp32" if fp32 else "bf16")
        if kind == "evict":
            c.update(share=round(rng.uniform(0.02, 1.0), 3), first=rng.choice([0, 1, 4, 17]), last=rng.choice([0, 1, 48]))
        return c
    if rng.random() < 0.15 and not fp32:
        prefix, robots, horizons = (_log_int(rng, 3000, 60000),) * 2, rng.randint(1, 4), rng.choice(["1", "1,4", "16"])
        prefix = (prefix[0], prefix[0] + rng.randint(0, 5000))
    else:
        robots = _log_int(rng, 1, 40 if fp32 else 300)
        horizons = rng.choice(["1", "16", "50", "16,50", "1,17,50", "3,33"])
    c = _case(kind, robots, prefix, heads, 1, "fp32" if fp32 else "bf16", horizons=horizons, cross=rng.random() < 0.3)
    if kind == "score":
        c["bits"] = rng.choice([4, 16])
    return c


def _lengths(case):
    """Prefix lengths and horizons of the requests: the case's own, the same for every seed."""
    r = np.random.default_rng([case["robots"], case["prefix_lo"], case["prefix_hi"]])
    P = r.integers(case["prefix_lo"], case["prefix_hi"], size=case["robots"], endpoint=True)
    H = r.choice([int(x) for x in case.get("horizons", "1").split(",")], size=case["robots"])
    return [int(p) for p in P], [int(h) for h in H]


def _keep(case, P):
    """Tokens kept of each prefix, the protected ones at its ends among them: (keep, first, last)."""
    out = []
    for p in P:
        first = min(case["first"], p)
        last = min(case["last"], p - first)
        out.append((max(first + last, min(p, max(1, round(case["share"] * p)))), first, last))
    return out


# ---------------------------------------------------------------- 4-bit caches, plainly

def _pack(x):
    """[.., n * 32] -> codes uint8 [.., n, 16] (element 2 i in the low four bits of byte i) and scale bytes [.., n]."""
    g = x.float().reshape(*x.shape[:-1], -1, GROUP)
    a = g.abs().amax(-1)
    m, e = torch.frexp(a)                      # a = m 2^e, m in [0.5, 1): the least s with a <= 7 * 2^s
    s = torch.where(a > 0, e - 3 + (m > 0.875), torch.full_like(e, -125)).clamp(-125, 125)
    y = torch.ldexp(g.abs(), -s[..., None])
    code = (y > 0.25).to(torch.uint8)
    # borders between neighbouring values; a value on one goes to the even code
    code += y >= 0.75
    code += y > 1.25
    code += y >= 1.75
    code += y > 2.5
    code += y >= 3.5
    code += y > 5.0
    code += torch.signbit(g).to(torch.uint8) * 8
    return code[..., 0::2] | (code[..., 1::2] << 4), (s + 127).to(torch.uint8)


def _unpack(codes, scales):
    """The values in fp32, [.., n * 32]."""
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    v = torch.stack([lut[(codes & 15).long()], lut[(codes >> 4).long()]], -1).flatten(-2)
    return torch.ldexp(v, scales.int()[..., None] - 127).flatten(-2)


def _cache_bytes(case, p):
    """Codes of all layers' rows, then their scales, and the room up to the next cache."""
    n = case["layers"] * p * case["n_kv"] * case["head_dim"]
    return n // 2, n // 2 + n // GROUP, -(-(n // 2 + n // GROUP) // ALIGN) * ALIGN


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    P, H = _lengths(case)
    n, L, nq, nkv, hd, dt = case["robots"], case["layers"], case["n_q"], case["n_kv"], case["head_dim"], _dtype(case)
    g = _gen(seed)
    rows = [L * p for p in P]                                  # cache rows of each request
    at = np.concatenate([[0], np.cumsum(rows)])
    k = (torch.randn((int(at[-1]), nkv, hd), device=DEV, generator=g) * KEY_STD).to(dt)
    v = torch.randn((int(at[-1]), nkv, hd), device=DEV, generator=g).to(dt)
    s = {"case": case, "shape": Shape(case), "P": P, "H": H, "k": k, "v": v, "at": [int(x) for x in at[:-1]],
         "Pt": torch.tensor(P, device=DEV), "Ht": torch.tensor(H, device=DEV), "att": torch.tensor(at[:-1], device=DEV)}
    if case["kind"] == "pack":
        s.update(k_back=torch.empty_like(k), v_back=torch.empty_like(v))
    if case["kind"] == "pack" or case.get("bits") == 4 or case["kind"] == "attend":
        sizes = [_cache_bytes(case, p) for p in P]
        off = np.concatenate([[0], np.cumsum([z[2] for z in sizes])])
        s["off"] = [int(x) for x in off[:-1]]
        s["codes_at"] = torch.tensor(off[:-1] // 16, device=DEV)
        s["scales_at"] = torch.tensor([o + z[0] for o, z in zip(off, sizes)], device=DEV)
        for name in ("k", "v"):
            q = torch.zeros(int(off[-1]), device=DEV, dtype=torch.uint8)
            if case["kind"] != "pack":
                codes, scales = _pack(s[name])
                for o, z, a, r in zip(s["off"], sizes, s["at"], rows):
                    q[o:o + z[0]] = codes[a:a + r].flatten()
                    q[o + z[0]:o + z[1]] = scales[a:a + r].flatten()
                del codes, scales
                s[name] = None                                 # the 4-bit cache is what is left of it
            s[name + "4"] = q
    if case["kind"] in ("attend", "score"):
        M = sum(H)
        first = np.concatenate([[0], np.cumsum(H)])[:-1]
        qkv = torch.randn((M, (nq + 2 * nkv) * hd), device=DEV, generator=g)
        qkv[:, nq * hd:(nq + nkv) * hd] *= KEY_STD
        s.update(qkv=(qkv * 0.64).to(dt), o=torch.empty((M, nq * hd), device=DEV, dtype=dt), first=torch.tensor(first, device=DEV))
        if case["kind"] == "score":
            s.update(lse=torch.empty((M, nq), device=DEV), mass=torch.empty(sum(P) * nkv, device=DEV))
    if case["kind"] == "evict":
        kp = _keep(case, P)
        # weights as attention leaves them: most tokens little, some much
        s["mass"] = torch.empty(sum(rows) * nkv, device=DEV).exponential_(generator=g) ** 3
        kept = [L * x[0] for x in kp]
        kat = np.concatenate([[0], np.cumsum(kept)])
        T = int(kat[-1])
        s.update(keep=kp, kat=[int(x) for x in kat[:-1]], kept=torch.empty(T * nkv, device=DEV, dtype=torch.int32),
                 kept_mass=torch.empty(T * nkv, device=DEV), k_out=torch.empty((T, nkv, hd), device=DEV, dtype=dt),
                 v_out=torch.empty((T, nkv, hd), device=DEV, dtype=dt), kept_t=torch.tensor(kp, device=DEV), katt=torch.tensor(kat[:-1], device=DEV))
    if own:
        _plan(s)
    return s


def _plan(s):
    """The calls' descriptions, and for attention the handle with its plan, as a program keeps them for a batch."""
    from paper_2607_01088_amd import rosa
    case, P, H = s["case"], s["P"], s["H"]
    e = 2 if case["dtype"] == "bf16" else 4
    row = case["n_kv"] * case["head_dim"] * e
    if case["kind"] == "pack":
        p4 = [(s["k4"].data_ptr() + o, s["v4"].data_ptr() + o) for o in s["off"]]
        src = [(s["k"].data_ptr() + a * row, s["v"].data_ptr() + a * row) for a in s["at"]]
        dst = [(s["k_back"].data_ptr() + a * row, s["v_back"].data_ptr() + a * row) for a in s["at"]]
        s["jobs"] = rosa.kv_jobs([(*x, *y, p) for x, y, p in zip(src, p4, P)])
        s["back"] = rosa.kv_jobs([(*y, *z, p) for y, z, p in zip(p4, dst, P)])
    elif case["kind"] == "evict":
        s["jobs"] = rosa.kv_evict_jobs([
            (s["k"].data_ptr() + a * row, s["v"].data_ptr() + a * row, s["k_out"].data_ptr() + b * row, s["v_out"].data_ptr() + b * row,
             s["mass"].data_ptr() + 4 * a * case["n_kv"], s["kept"].data_ptr() + 4 * b * case["n_kv"],
             s["kept_mass"].data_ptr() + 4 * b * case["n_kv"], p, *kp) for a, b, p, kp in zip(s["at"], s["kat"], P, s["keep"])])
    else:
        four = case["kind"] == "attend" or case["bits"] == 4
        if four:
            src = [(s["k4"].data_ptr() + o, s["v4"].data_ptr() + o) for o in s["off"]]
        else:
            src = [(s["k"].data_ptr() + a * row, s["v"].data_ptr() + a * row) for a in s["at"]]
        reqs = [rosa.request_struct(x, y, s["o"], s["o"], p, h, 1) for (x, y), p, h in zip(src, P, H)]
        mass = [s["mass"].data_ptr() + 4 * a * case["n_kv"] for a in s["at"]] if case["kind"] == "score" else None
        s["attention"] = rosa.KvAttention(s["shape"], case["dtype"], rosa.capacity(len(P), max(H), sum(H), 1, sum(P)))
        s["attention"].plan(reqs, rosa.ROSA_KV_FP4 if four else rosa.ROSA_KV_MODEL, mass=mass)


# ---------------------------------------------------------------- one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2607_01088_amd import rosa
        if kind == "pack":
            rosa.kv_quantize(s["shape"], s["case"]["dtype"], s["jobs"])
            rosa.kv_expand(s["shape"], s["case"]["dtype"], s["back"])
            return {"k": s["k_back"], "v": s["v_back"]}
        if kind == "evict":
            rosa.kv_evict(s["shape"], s["case"]["dtype"], rosa.ROSA_KV_MODEL, s["jobs"])
            return {"kept": s["kept"], "mass": s["kept_mass"], "k": s["k_out"], "v": s["v_out"]}
        if kind == "attend":
            s["attention"].attention(0, s["qkv"], s["o"])
            return s["o"]
        s["attention"].attention(0, s["qkv"], s["o"], lse=s["lse"])
        s["attention"].mass(0, s["qkv"], s["lse"], accumulate=False)
        return {"o": s["o"], "lse": s["lse"], "mass": s["mass"]}
    if kind == "pack":
        return {"k": _unpack(*_pack(s["k"])).to(s["k"].dtype).view(s["k"].shape), "v": _unpack(*_pack(s["v"])).to(s["v"].dtype).view(s["v"].shape)}
    if kind == "evict":
        return _plain_evict(s)
    o, lse, mass = _plain_attend(s, kind == "score")
    return o if kind == "attend" else {"o": o, "lse": lse, "mass": mass}


def _padded(s, name):
    """The prefix cache in fp32, [requests, longest prefix, n_kv, hd]; past a request's end its last row again."""
    case, Pm = s["case"], max(s["P"])
    t = torch.minimum(torch.arange(Pm, device=DEV)[None], s["Pt"][:, None] - 1)
    if name + "4" not in s:
        return s[name][s["att"][:, None] + t].float()
    c = case["n_kv"] * case["head_dim"] // GROUP              # groups of a row: 16 code bytes and a scale each
    at = t[..., None] * c + torch.arange(c, device=DEV)
    q = s[name + "4"]
    x = _unpack(q.view(-1, 16)[s["codes_at"][:, None, None] + at], q[s["scales_at"][:, None, None] + at])
    return x.view(len(s["P"]), Pm, case["n_kv"], case["head_dim"])


def _plain_attend(s, score):
    case = s["case"]
    n, nq, nkv, hd = case["robots"], case["n_q"], case["n_kv"], case["head_dim"]
    G, Pm, Hm = nq // nkv, max(s["P"]), max(s["H"])
    t = torch.arange(Hm, device=DEV)[None]
    real = t < s["Ht"][:, None]                               # [n, Hm]: action tokens that are there
    rows = s["first"][:, None] + torch.minimum(t, s["Ht"][:, None] - 1)
    x = s["qkv"][rows].float()
    q = x[..., :nq * hd].view(n, Hm, nkv, G, hd).permute(0, 2, 1, 3, 4).reshape(n, nkv, Hm * G, hd)
    k, v = _padded(s, "k"), _padded(s, "v")
    seen = torch.arange(Pm, device=DEV)[None] < s["Pt"][:, None]
    if not case["cross"]:
        k = torch.cat([k, x[..., nq * hd:(nq + nkv) * hd].reshape(n, Hm, nkv, hd)], 1)
        v = torch.cat([v, x[..., (nq + nkv) * hd:].reshape(n, Hm, nkv, hd)], 1)
        seen = torch.cat([seen, real], 1)
    w = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(hd)
    w = w.masked_fill(~seen[:, None, None, :], -math.inf)
    m = w.amax(-1, keepdim=True)
    e = torch.exp(w - m)
    l = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v.permute(0, 2, 1, 3).contiguous()) / l
    o = o.view(n, nkv, Hm, G, hd).permute(0, 2, 1, 3, 4).reshape(n, Hm, nq * hd)[real].to(s["o"].dtype)
    if not score:
        return o, None, None
    lse = (m + torch.log(l)).view(n, nkv, Hm, G).permute(0, 2, 1, 3).reshape(n, Hm, nq)[real]
    p = (e / l).view(n, nkv, Hm, G, -1) * real[:, None, :, None, None]
    mass = p.sum((2, 3))[..., :Pm]                            # [n, nkv, Pm]
    return o, lse, mass[seen[:, None, :Pm].expand(n, nkv, Pm)]


def _plain_evict(s):
    case = s["case"]
    n, L, nkv, Pm = case["robots"], case["layers"], case["n_kv"], max(s["P"])
    t = torch.arange(Pm, device=DEV)
    P, keep, first, last = s["Pt"][:, None], s["kept_t"][:, 0:1], s["kept_t"][:, 1:2], s["kept_t"][:, 2:3]
    tc = torch.minimum(t[None], P - 1)
    lay, head = torch.arange(L, device=DEV)[None, :, None, None], torch.arange(nkv, device=DEV)[None, None, :, None]
    per = s["Pt"][:, None, None, None]
    at = s["att"][:, None, None, None] * nkv + (lay * nkv + head) * per + tc[:, None, None, :]
    mass = s["mass"][at]                                      # [n, L, nkv, Pm]
    rank = torch.where((t[None] < first) | (t[None] >= P - last), math.inf, 0.0)[:, None, None, :] + mass
    rank = torch.where((t[None] < P)[:, None, None, :], rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(order)
    place.scatter_(-1, order, t.expand_as(order).contiguous())
    b, l, h, i = (place < keep[:, None, None, :]).nonzero(as_tuple=True)   # in the order (request, layer, head, token)
    kb = s["kept_t"][:, 0][b]
    slot = torch.arange(b.numel(), device=DEV) - s["katt"][b] * nkv - (l * nkv + h) * kb   # place among the kept of its row
    to = (s["katt"][b] + l * kb + slot) * nkv + h
    src = (s["att"][b] + l * s["Pt"][b] + i) * nkv + h
    out = {"kept": i.int(), "mass": mass[b, l, h, i]}
    for name in ("k", "v"):
        y = torch.empty((s["kept"].numel(), case["head_dim"]), device=DEV, dtype=s[name].dtype)
        y[to] = s[name].view(-1, case["head_dim"])[src]
        out[name] = y.view(s[name + "_out"].shape)
    return out


# ---------------------------------------------------------------- work

def work(case):
    P, H = _lengths(case)
    L, nq, nkv, hd = case["layers"], case["n_q"], case["n_kv"], case["head_dim"]
    e = 2 if case["dtype"] == "bf16" else 4
    four = 0.5 + 1 / GROUP
    n = 2 * sum(P) * L * nkv * hd                              # cached values, K and V
    if case["kind"] == "pack":
        return {"bytes": 2 * n * (e + four), "flops": 4 * n}
    if case["kind"] == "evict":
        kept = sum(x[0] for x in _keep(case, P)) * L * nkv
        return {"bytes": 4 * sum(P) * L * nkv + 8 * kept + 2 * 2 * kept * hd * e, "flops": sum(P) * L * nkv}
    bits4 = case["kind"] == "attend" or case["bits"] == 4
    keys = [p + (0 if case["cross"] else h) for p, h in zip(P, H)]
    bytes_ = n * (four if bits4 else e) + sum(H) * (2 * nq + 2 * nkv) * hd * e
    if case["kind"] == "score":
        bytes_ += 4 * sum(P) * nkv + 4 * sum(H) * nq
    return {"bytes": bytes_, "flops": sum(4 * nq * hd * h * x for h, x in zip(H, keys))}


# ---------------------------------------------------------------- 64-bit values

def _exact_unpack(codes, scales):
    """codes [rows, 16 n] uint8, scales [rows, n] -> [rows, 32 n]: sign, two exponent bits and one mantissa bit each."""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2).long()
    sign, ex, man = 1 - 2 * (c // 8), (c // 2) % 4, c % 2
    mag = torch.where(ex == 0, man * 0.5, (1 + man * 0.5) * torch.pow(2.0, (ex - 1).double()))
    return sign * mag * torch.pow(2.0, scales.double() - 127).repeat_interleave(GROUP, -1)


def _exact_round(x):
    """The 4-bit value of every element: the nearest of the group's 8 magnitudes, of two equally near the even one."""
    g = x.double().reshape(-1, GROUP)
    a = g.abs().amax(-1, keepdim=True)
    s = torch.full_like(a, -125.0)
    s = torch.where(a > 0, torch.ceil(torch.log2(a / 7)), s)
    s = torch.where(a > 7 * torch.pow(2.0, s), s + 1, s)       # log2 next to a power of two
    s = torch.where((a > 0) & (a <= 7 * torch.pow(2.0, s - 1)), s - 1, s).clamp(-125, 125)
    y = g.abs() / torch.pow(2.0, s)
    best, off = torch.zeros_like(y), y.clone()
    for i, m in enumerate([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], 1):
        d = (y - m).abs()
        nearer = (d < off) | ((d == off) & (i % 2 == 0))
        best, off = torch.where(nearer, torch.full_like(y, m), best), torch.where(nearer, d, off)
    return (torch.sign(g) * best * torch.pow(2.0, s)).view(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    P, H, L, nq, nkv, hd = s["P"], s["H"], case["layers"], case["n_q"], case["n_kv"], case["head_dim"]
    if case["kind"] == "pack":
        out = {}
        for name in ("k", "v"):
            y = torch.empty(s[name].shape, device=DEV, dtype=torch.float64)
            for a, p in zip(s["at"], P):
                y[a:a + L * p] = _exact_round(s[name][a:a + L * p])
            out[name] = y
        return out
    if case["kind"] == "evict":
        mass = s["mass"].cpu().numpy().astype(np.float64)
        rows, ms = [], []
        for a, p, (keep, first, last) in zip(s["at"], P, s["keep"]):
            per = np.empty((L, keep, nkv), np.int64)
            for l in range(L):
                for h in range(nkv):
                    m = mass[a * nkv + (l * nkv + h) * p:][:p]
                    rest = sorted(range(first, p - last), key=lambda i: (-m[i], i))[:keep - first - last]
                    ids = np.array(sorted([*range(first), *rest, *range(p - last, p)]))
                    per[l, :, h] = (a + l * p + ids) * nkv + h
                    ms.append(m[ids])
            rows.append(per.reshape(-1))
        rows = torch.tensor(np.concatenate(rows), device=DEV)
        out = {"kept": None, "mass": torch.tensor(np.concatenate(ms))}
        for name in ("k", "v"):
            out[name] = s[name].view(-1, hd)[rows].double().view(-1, nkv, hd)
        return out
    four = case["kind"] == "attend" or case["bits"] == 4
    o, lse, mass, r0 = [], [], [], 0
    for i, (p, h) in enumerate(zip(P, H)):
        kv = []
        for name in ("k", "v"):
            if four:
                nb, ns, _ = _cache_bytes(case, p)
                b = s[name + "4"][s["off"][i]:s["off"][i] + ns]
                kv.append(_exact_unpack(b[:nb].view(p, -1), b[nb:].view(p, -1)).view(p, nkv, hd))
            else:
                kv.append(s[name][s["at"][i]:s["at"][i] + p].double())
        x = s["qkv"][r0:r0 + h].double()
        r0 += h
        q, k, v = x[:, :nq * hd].view(h, nkv, -1, hd), kv[0], kv[1]
        if not case["cross"]:
            k = torch.cat([k, x[:, nq * hd:(nq + nkv) * hd].reshape(h, nkv, hd)])
            v = torch.cat([v, x[:, (nq + nkv) * hd:].reshape(h, nkv, hd)])
        oo, ll = torch.empty(q.shape, device=DEV, dtype=torch.float64), torch.empty(q.shape[:3], device=DEV, dtype=torch.float64)
        for j in range(nkv):
            w = q[:, j].reshape(-1, hd) @ k[:, j].t().contiguous() / math.sqrt(hd)
            z = torch.logsumexp(w, -1, keepdim=True)
            w = torch.exp(w - z)
            oo[:, j], ll[:, j] = (w @ v[:, j].contiguous()).view(h, -1, hd), z.view(h, -1)
            mass.append(w.sum(0)[:p])
        o.append(oo.reshape(h, nq * hd))
        lse.append(ll.reshape(h, nq))
    o = torch.cat(o)
    return o if case["kind"] == "attend" else {"o": o, "lse": torch.cat(lse), "mass": torch.cat(mass)}
