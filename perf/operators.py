"""Timed cases of the operators around a key/value cache held in 4 bits: head norms with the position rotation in one pass,
writing into the cache and reading it back, attention over it, the sum of the attention weights of each key, and eviction by
that sum.

`run` computes them in elementary torch operations, or, where `own` is true, through `binding.qk_norm_rope` and
`binding.KvCache4`.  The cache holds, for each key and head, dh codes c of 4 bits and two bf16 numbers: value = c s + m with
m the row's minimum and s a fifteenth of its range.  Sizes: the head layouts of `workloads` (32 heads of 128, 4 of 64), blocks of
16 to 64 rows, grouped heads, caches of up to 2048 keys as its decodes have them, and longer ones.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------------------

def _rope(name, dtype, rows, hq, hk, dh, theta, start):
    return {"name": name, "op": "rope", "dtype": dtype, "rows": rows, "hq": hq, "hk": hk, "dh": dh, "theta": theta, "start": start}


def _store(name, batch, rows, heads, dh, start, out, ragged=False):
    return {"name": name, "op": "store", "batch": batch, "rows": rows, "hk": heads, "dh": dh, "start": start, "out": out,
            "ragged": ragged}


def _attn(name, op, batch, rows, hq, hk, dh, keys, ragged=False, empty=False):
    return {"name": name, "op": op, "batch": batch, "rows": rows, "hq": hq, "hk": hk, "dh": dh, "keys": keys, "ragged": ragged,
            "empty": empty}


def _evict(name, batch, heads, dh, keys, keep, ragged=False):
    return {"name": name, "op": "evict", "batch": batch, "hk": heads, "dh": dh, "keys": keys, "keep": keep, "ragged": ragged}


def listed():
    return [
        # the tiny fp32 model's whole sequence, 96 rows of 4 heads of 64: latency
        _rope("norm+rope fp32 96x(4+4)x64", "fp32", 96, 4, 4, 64, 10000.0, 0),
        # a server's batch of 16 x 1024 rows before a whole-sequence step, 32 query and 8 key heads, positions far out
        _rope("norm+rope bf16 16384x(32+8)x128", "bf16", 16384, 32, 8, 128, 500000.0, 100000),
        # one block of 32 rows written into the cache at its place: a cached step's write, latency
        _store("store 1x32 rows 32x128", 1, 32, 32, 128, 256, "fp32"),
        # a block's first step: the rows of eight sequences of 2048 positions
        _store("store 8x2048 rows 32x128", 8, 2048, 32, 128, 0, "bf16"),
        # one new token of one request, 32 query heads on 8 key heads, 4000 keys
        _attn("attention 1x1 token 32/8x128 4000 keys", "attend", 1, 1, 32, 8, 128, 4000),
        # a dual-cache step of a small model with heads of 64: three ragged sequences
        _attn("attention 3x27 rows 8/8x64 1500 keys", "attend", 3, 27, 8, 8, 64, 1500, ragged=True),
        # the dual-cache step of the 8B shape: eight blocks of 32 rows on 2048 keys
        _attn("attention 8x32 rows 32/32x128 2048 keys", "attend", 8, 32, 32, 32, 128, 2048),
        # blocks of 32 rows with grouped heads far into long documents
        _attn("attention 4x32 rows 32/8x128 65000 keys", "attend", 4, 32, 32, 8, 128, 65000, ragged=True),
        # the weights of those 8B blocks, summed per key before an eviction
        _attn("weights 8x32 rows 32/32x128 2048 keys", "weigh", 8, 32, 32, 32, 128, 2048),
        # the weights that sixteen single tokens give to long caches
        _attn("weights 16x1 token 32/8x128 30000 keys", "weigh", 16, 1, 32, 8, 128, 30000, ragged=True),
        # the 8B cache halved after the prompt
        _evict("evict 8x32 heads 2048 -> 1024", 8, 32, 128, 2048, 1024),
        # long documents cut to an eighth
        _evict("evict 4x8 heads 65000 -> 8000", 4, 8, 128, 65000, 8000, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_KEYS = 4 * 8 * 65000          # keys x heads of the largest listed cache


def draw(rng):
    op = rng.choice(["rope", "store", "attend", "attend", "attend", "weigh", "evict"])
    if op == "rope":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        dh = rng.choice([64, 128]) if dtype == "bf16" else rng.choice([32, 48, 64, 128, 256])
        hk = rng.choice([1, 2, 4, 8, 16, 32])
        hq = hk * rng.choice([1, 1, 2, 4, 7, 8])
        cost = {"bf16": 2, "fp32": 4}[dtype] * (hq + hk) * dh
        rows = _log_int(rng, 1, min(32768, 16384 * 40 * 128 * 2 // cost))
        case = _rope("", dtype, rows, hq, hk, dh, rng.choice([10000.0, 500000.0, 1000000.0]), rng.choice([0, 0, 1000, 1000000]))
    elif op == "store":
        hk, dh = rng.choice([1, 2, 4, 8, 12, 32]), rng.choice([64, 128])
        batch = _log_int(rng, 1, 16)
        rows = _log_int(rng, 1, max(2, min(4096, 8 * 2048 * 32 * 128 // (batch * hk * dh))))
        case = _store("", batch, rows, hk, dh, rng.choice([0, 1, 63, 64, 1000]), rng.choice(["bf16", "fp32"]), rng.random() < 0.5)
        if case["out"] == "fp32":
            case["rows"] = max(1, rows // 2)
    elif op in ("attend", "weigh"):
        dh, hk, group = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8, 8, 32]), rng.choice([1, 1, 2, 4, 5, 8])
        rows = rng.choice([1, 1, 1, 2, 5, 16, 32, 32, 33, 64])
        while rows * group > 128:
            rows //= 2
        batch = _log_int(rng, 1, 32)
        top = MAX_KEYS // (batch * hk)
        if op == "weigh":
            top = min(top, 16 * 8 * 30000 * 4 // (batch * hk * max(4, rows * group)))
        keys = _log_int(rng, 1, max(2, min(131072, top)))
        case = _attn("", op, batch, rows, hk * group, hk, dh, keys, rng.random() < 0.5, rng.random() < 0.2)
    else:
        dh, hk, batch = rng.choice([64, 128]), rng.choice([1, 2, 8, 32]), _log_int(rng, 1, 16)
        keys = _log_int(rng, 64, min(131072, MAX_KEYS // (batch * hk)))
        keep = max(1, min(int(keys * rng.choice([0.1, 0.25, 0.5, 0.9])), 4 * 8 * 8000 // (batch * hk)))
        case = _evict("", batch, hk, dh, keys, keep, rng.random() < 0.5)
    case.pop("name")
    return case


def _key_counts(case):
    """Keys of each sequence: all the same, or spread over the upper half of the length; `empty`: the last has none."""
    n, b = case["keys"], case["batch"]
    lens = [n - (n * (5 * i % 8)) // 16 for i in range(b)] if case["ragged"] else [n] * b
    if case.get("empty") and b > 1:
        lens[-1] = 0
    return lens


def _row_counts(case):
    r, b = case["rows"], case["batch"]
    return [r - (r * (3 * i % 4)) // 8 for i in range(b)] if case["ragged"] else [r] * b


def work(case):
    op = case["op"]
    if op == "rope":
        e = 2 if case["dtype"] == "bf16" else 4
        values = case["rows"] * (case["hq"] + case["hk"]) * case["dh"]
        return {"bytes": 2 * e * values + 4 * case["rows"] + 8 * case["dh"], "flops": 7 * values}
    record = case["dh"] + 8                                       # K and V of a key and head: 2 x (dh / 2 + 4) bytes
    if op == "store":
        rows = sum(_row_counts(case)) * case["hk"]
        out = 2 if case["out"] == "bf16" else 4
        # bf16 rows in, records written and read once, their values out
        return {"bytes": rows * (4 * case["dh"] + 2 * record + 2 * out * case["dh"]), "flops": 12 * rows * case["dh"]}
    keys = _key_counts(case)
    if op == "attend":
        rows = _row_counts(case)
        pairs = sum(r * n for r, n in zip(rows, keys)) * case["hq"]
        return {"bytes": sum(keys) * case["hk"] * record + sum(rows) * case["hq"] * (4 * case["dh"] + 4), "flops": 4 * pairs * case["dh"]}
    if op == "weigh":
        rows = _row_counts(case)
        pairs = sum(r * n for r, n in zip(rows, keys)) * case["hq"]
        return {"bytes": sum(keys) * case["hk"] * (record // 2 + 8) + sum(rows) * case["hq"] * (2 * case["dh"] + 4),
                "flops": 2 * pairs * case["dh"]}
    kept = sum(min(n, case["keep"]) for n in keys) * case["hk"]
    # all weights read; of the kept keys the record, weight and position moved, the record read back and its values (bf16) out
    return {"bytes": 4 * sum(keys) * case["hk"] + kept * (3 * record + 16 + 4 * case["dh"]), "flops": 2 * kept * case["dh"]}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _inputs(case, seed):
    """Tensors made from the seed alone.  Keys have the few large channels that trained models show, values do not."""
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    rnd = lambda *shape, dtype=torch.bfloat16: torch.randn(*shape, generator=g, device=DEVICE, dtype=dtype)
    op, dh = case["op"], case["dh"]
    if op == "rope":
        dt = DTYPES[case["dtype"]]
        t = case["rows"]
        return {"q": rnd(t, case["hq"], dh, dtype=dt), "k": rnd(t, case["hk"], dh, dtype=dt) * 3,
                "q_gain": 1 + 0.2 * rnd(dh, dtype=torch.float32), "k_gain": 1 + 0.2 * rnd(dh, dtype=torch.float32),
                "positions": torch.arange(case["start"], case["start"] + t, dtype=torch.int32, device=DEVICE)}
    channels = torch.exp(0.7 * rnd(case["hk"], dh, dtype=torch.float32)).to(torch.bfloat16)
    if op == "store":
        n = sum(_row_counts(case))
        return {"k": rnd(n, case["hk"], dh) * channels, "v": rnd(n, case["hk"], dh)}
    b, n = case["batch"], case["keys"]
    d = {"k": rnd(b, n, case["hk"], dh) * channels, "v": rnd(b, n, case["hk"], dh) + 0.25}
    if op == "evict":
        w = torch.rand(b, case["hk"], n, generator=g, device=DEVICE) ** 8 * 16
        d["weights"] = torch.round(w * 4096) / 4096                # sums of few rows: many small ones, and ties
    else:
        d["q"] = rnd(sum(_row_counts(case)), case["hq"], dh) * 2
        if op == "weigh":
            d["weights"] = torch.rand(b, case["hk"], n, generator=g, device=DEVICE)
    return d


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _quantise(x):
    """bf16 [..., dh] -> codes (uint8), s, m (fp32, exact in bf16).  Decided in 64 bits: a code hangs on which side of a
    border a value lies."""
    xf = x.float()
    m = xf.amin(-1, keepdim=True).to(torch.bfloat16).float()
    s = ((xf.amax(-1, keepdim=True) - m) / 15.0).to(torch.bfloat16).float()
    t = (xf.double() - m.double()) / s.double()
    codes = torch.where(s > 0, torch.round(t).clamp(0, 15), torch.zeros_like(t)).to(torch.uint8)
    return codes, s, m


def _pack(x):
    """As the cache keeps it: two codes to a byte."""
    codes, s, m = _quantise(x)
    return codes[..., 0::2] | codes[..., 1::2] << 4, s.to(torch.bfloat16), m.to(torch.bfloat16)


def _unpack(packed):
    codes, s, m = packed
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    return c * s.float() + m.float()


def _rope_plain(st):
    def one(x, gain):
        xf = x.float()
        y = xf * gain / torch.sqrt((xf * xf).mean(-1, keepdim=True) + st["eps"])
        h = x.shape[-1] // 2
        freq = st["theta"] ** (-torch.arange(h, dtype=torch.float64, device=x.device) / h)
        angle = st["positions"].double()[:, None] * freq           # far positions: 64 bits
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        a, b = y[..., :h], y[..., h:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)
    return one(st["q"], st["q_gain"]), one(st["k"], st["k_gain"])


def _attend_plain(st):
    out, lse = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:2], device=DEVICE)
    kf, vf = _unpack(st["k4"]), _unpack(st["v4"])                  # [B, keys, heads, dh]
    for b, n in enumerate(st["key_counts"]):
        lo, hi = st["row_starts"][b], st["row_starts"][b + 1]
        if n == 0:
            out[lo:hi], lse[lo:hi] = 0, -math.inf
            continue
        q = _by_head(st["q"][lo:hi].float(), kf.shape[2])
        s = q @ kf[b, :n].permute(1, 2, 0) * st["scale"]
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o = p @ vf[b, :n].permute(1, 0, 2) / total
        out[lo:hi] = _by_row(o, hi - lo).to(out.dtype)
        lse[lo:hi] = _by_row(top + torch.log(total), hi - lo)[..., 0]
    return out, lse


def _by_head(q, heads):
    """[rows, Hq, x] -> [heads, rows * group, x]: the query heads h * group ... of a group share the key head h."""
    r, hq, x = q.shape
    return q.reshape(r, heads, hq // heads, x).permute(1, 0, 2, 3).reshape(heads, r * (hq // heads), x)


def _by_row(o, rows):
    h, n, x = o.shape
    return o.reshape(h, rows, n // rows, x).permute(1, 0, 2, 3).reshape(rows, h * (n // rows), x)


def _weigh_plain(st):
    out = st["weights"].clone()
    kf = _unpack(st["k4"])
    for b, n in enumerate(st["key_counts"]):
        lo, hi = st["row_starts"][b], st["row_starts"][b + 1]
        if n == 0:
            continue
        q = _by_head(st["q"][lo:hi].float(), kf.shape[2])
        lse = _by_head(st["lse"][lo:hi, :, None], kf.shape[2])
        s = q @ kf[b, :n].permute(1, 2, 0) * st["scale"]
        out[b, :, :n] += torch.exp(s - lse).sum(1)
    return out


def _evict_plain(st):
    b, h, _ = st["weights"].shape
    keep = st["keep"]
    dh = st["k4"][0].shape[-1] * 2
    kept = torch.full((b, h, keep), -1, dtype=torch.int32, device=DEVICE)
    w_out, p_out = torch.zeros(b, h, keep, device=DEVICE), torch.zeros(b, h, keep, dtype=torch.int32, device=DEVICE)
    k_out = torch.zeros(b, keep, h, dh, dtype=torch.bfloat16, device=DEVICE)
    v_out = torch.zeros_like(k_out)
    heads = torch.arange(h, device=DEVICE)[:, None]
    for i, n in enumerate(st["key_counts"]):
        m = min(n, keep)
        w, pos = st["weights"][i, :, :n], st["positions"][i, :, :n]
        rank = torch.where((pos < st["first"]) | (pos >= st["protect_from_host"][i]), math.inf, w)
        chosen = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:, :m]
        stays = torch.zeros(h, n, dtype=torch.bool, device=DEVICE)
        stays.scatter_(1, chosen, True)
        # kept keys below m stay; the others take the free places in order
        front, back = stays[:, :m], stays[:, m:]
        source = torch.arange(m, device=DEVICE).expand(h, m).clone()
        if n > m:
            order = torch.argsort((~back).to(torch.uint8), dim=1, stable=True) + m       # kept ones first, ascending
            turn = (~front).long().cumsum(1) - 1
            source = torch.where(front, source, torch.gather(order, 1, turn.clamp(0, n - m - 1)))
        kept[i, :, :m] = source.int()
        w_out[i, :, :m], p_out[i, :, :m] = torch.gather(w, 1, source), torch.gather(pos, 1, source)
        for packed, out in ((st["k4"], k_out), (st["v4"], v_out)):
            out[i, :m] = _unpack(tuple(t[i][source, heads] for t in packed)).permute(1, 0, 2).to(torch.bfloat16)
    return kept, _clipped(st), w_out, p_out, k_out, v_out


def _clipped(st):
    return torch.clamp(st["lens"], max=st["keep"])


# ---- what a program has in hand, and one pass --------------------------------------------------------------------------

def prepare(case, seed):
    d = _inputs(case, seed)
    op = case["op"]
    if op == "rope":
        d.update(op=op, theta=case["theta"], eps=1e-5)
        return d
    if own:
        from paper_2509_25188_b200 import binding
    b, dh, hk = case["batch"], case["dh"], case["hk"]
    if op == "store":
        counts = _row_counts(case)
        d.update(op=op, out=DTYPES[case["out"]], max_rows=case["rows"], row_start=_int32(_starts(counts)),
                 key_start=_int32([case["start"]] * b), counts=counts)
        if own:
            d["cache"] = binding.KvCache4(b, hk, dh, case["start"] + case["rows"])
        return d
    counts = _key_counts(case)
    st = {"op": op, "key_counts": counts, "lens": _int32(counts), "max_len": case["keys"]}
    k, v = d.pop("k"), d.pop("v")
    if own:
        st["cache"] = binding.KvCache4(b, hk, dh, case["keys"])
        st["cache"].store(k, v)
    else:
        st["k4"], st["v4"] = _pack(k), _pack(v)
    if op == "evict":
        st.update(keep=case["keep"], first=4, protect_from_host=[max(n - 32, 0) for n in counts])
        st["protect_from"] = _int32(st["protect_from_host"])
        st["positions"] = torch.arange(case["keys"], dtype=torch.int32, device=DEVICE).expand(b, hk, -1).contiguous()
        st["weights"] = d["weights"]
        if own:
            st["into"] = binding.KvCache4(b, hk, dh, case["keep"])
            st["weights_into"] = torch.zeros(b, hk, case["keep"], device=DEVICE)
            st["positions_into"] = torch.zeros(b, hk, case["keep"], dtype=torch.int32, device=DEVICE)
        return st
    rows = _row_counts(case)
    st.update(q=d["q"], scale=1.0 / math.sqrt(dh), row_starts=_starts(rows), row_start=_int32(_starts(rows)), max_rows=case["rows"])
    if op == "weigh":
        st["weights"] = d["weights"]
        if own:
            st["out"] = torch.empty_like(d["weights"])
            st["out"].copy_(d["weights"])
            st["lse"] = st["cache"].attention(st["q"], st["lens"], st["max_len"], row_start=st["row_start"],
                                              max_rows=st["max_rows"], scale=st["scale"])[1]
        else:
            st["lse"] = _attend_plain(st)[1]
    return st


def run(state):
    op = state["op"]
    if not own:
        if op == "rope":
            return _rope_plain(state)
        if op == "store":
            out = tuple(_unpack(_pack(state[n])).to(state["out"]) for n in ("k", "v"))
            return out
        return {"attend": _attend_plain, "weigh": _weigh_plain, "evict": _evict_plain}[op](state)
    from paper_2509_25188_b200 import binding
    st = state
    if op == "rope":
        return binding.qk_norm_rope(st["q"], st["k"], st["q_gain"], st["k_gain"], st["positions"], theta=st["theta"], eps=st["eps"])
    if op == "store":
        # written, then read back as a reader of the cache sees them
        st["cache"].store(st["k"], st["v"], key_start=st["key_start"], row_start=st["row_start"], max_rows=st["max_rows"])
        return st["cache"].load(st["max_rows"], key_start=st["key_start"], row_start=st["row_start"], total_rows=st["k"].shape[0],
                                dtype=st["out"])
    if op == "attend":
        return st["cache"].attention(st["q"], st["lens"], st["max_len"], row_start=st["row_start"], max_rows=st["max_rows"],
                                     scale=st["scale"])
    if op == "weigh":
        return st["cache"].attention_weights(st["q"], st["lse"], st["lens"], st["max_len"], st["weights"], out=st["out"],
                                             row_start=st["row_start"], max_rows=st["max_rows"], scale=st["scale"])
    kept, lens = st["cache"].evict(st["weights"], st["lens"], st["max_len"], st["keep"], positions=st["positions"], first=st["first"],
                                   protect_from=st["protect_from"], into=st["into"], weights_into=st["weights_into"],
                                   positions_into=st["positions_into"])
    k, v = st["into"].load(st["keep"], dtype=torch.bfloat16)
    return kept, lens, st["weights_into"], st["positions_into"], k, v


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _values64(x):
    """What the cache keeps of x, in 64 bits.  s and m are defined with their roundings (fp32 range and quotient, then bf16);
    the code is the number of borders m + (k + 1/2) s below x, a value on a border going to the even side."""
    x = x.double()
    m = x.min(-1, keepdim=True).values
    s = ((x.max(-1, keepdim=True).values - m).float().double() / 15).float().to(torch.bfloat16).double()
    t = (x - m) / s
    low = torch.floor(t)
    up = (t - low > 0.5) | ((t - low == 0.5) & (low % 2 == 1))
    code = torch.minimum(low + up, torch.full_like(t, 15.0))
    return torch.where(s > 0, code * s + m, m.expand_as(x))


def _scores64(q, k, scale):
    """q [rows, Hq, dh], k [keys, Hk, dh] -> [rows, Hq, keys]"""
    group = q.shape[1] // k.shape[1]
    return torch.stack([q[:, h] @ k[:, h // group].T for h in range(q.shape[1])], 1) * scale


def exact(case, seed):
    d, op = _inputs(case, seed), case["op"]
    if op == "rope":
        h = case["dh"] // 2
        angle = d["positions"].double().unsqueeze(1) * torch.exp(-math.log(case["theta"]) / h * torch.arange(h, device=DEVICE).double())
        turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
        out = []
        for x, gain in ((d["q"], d["q_gain"]), (d["k"], d["k_gain"])):
            x = x.double()
            x = x * torch.rsqrt(x.square().sum(-1, keepdim=True) / case["dh"] + 1e-5) * gain.double()
            z = torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous()) * turn
            out.append(torch.cat((z.real, z.imag), -1))
        return tuple(out)
    if op == "store":
        return _values64(d["k"]), _values64(d["v"])
    lens = _key_counts(case)
    if op == "evict":
        return _evict64(case, d, lens)
    starts, scale = _starts(_row_counts(case)), 1.0 / math.sqrt(case["dh"])
    group = case["hq"] // case["hk"]
    q = d["q"].double()
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    out = torch.zeros_like(q)
    weights = d["weights"].double() if op == "weigh" else None
    for i, n in enumerate(lens):
        rows = slice(starts[i], starts[i + 1])
        if n == 0:
            continue
        s = _scores64(q[rows], _values64(d["k"][i, :n]), scale)
        lse[rows] = torch.logsumexp(s, -1)
        p = torch.softmax(s, -1)
        if weights is not None:
            weights[i, :, :n] += p.sum(0).reshape(case["hk"], group, n).sum(1)
        else:
            v = _values64(d["v"][i, :n])
            out[rows] = torch.stack([p[:, h] @ v[:, h // group] for h in range(case["hq"])], 1)
    return weights if weights is not None else (out, lse)


def _evict64(case, d, lens):
    b, h, keep, dh = case["batch"], case["hk"], case["keep"], case["dh"]
    kept = torch.full((b, h, keep), -1, dtype=torch.int64)
    for i, n in enumerate(lens):
        m = min(n, keep)
        for j in range(h):
            w = d["weights"][i, j, :n].tolist()
            order = sorted(range(n), key=lambda x: (not (x < 4 or x >= max(n - 32, 0)), -w[x], x))
            chosen = set(order[:m])
            late = iter(sorted(x for x in chosen if x >= m))
            kept[i, j, :m] = torch.tensor([x if x in chosen else next(late) for x in range(m)])
    kept = kept.to(DEVICE)
    there = kept >= 0
    src = kept.clamp(min=0)
    rows = src.transpose(1, 2).unsqueeze(-1).expand(-1, -1, -1, dh)
    values = [torch.gather(_values64(d[x]), 1, rows) * there.transpose(1, 2).unsqueeze(-1) for x in ("k", "v")]
    weights = torch.gather(d["weights"].double(), 2, src) * there
    return (kept.int(), _int32([min(n, keep) for n in lens]), weights, src * there, values[0], values[1])
