"""The operators over a cache held in 4 bits, as measurable cases.

A context made for 4 bits keeps keys and values as e2m1 codes with one power-of-two scale for 32 dimensions of a head: 17/32 of a
byte a value in the pool and in the tier.  The operators are the ones a serving program calls for every layer:

  op "append"  a turn's keys and values, quantised, to their pages and to the tier (heads of the keys normalised first where the
               model does so), and read back as the values that the cache holds from then on
  op "attend"  attention of the new tokens over the context in the pool: decode steps, turns, first turns; the heads of the queries
               are normalised where the model does so, and rotated to their positions, in the same pass
  op "turn"    all of a turn: load of the kept history from the tier, append and save, attention

Each pass begins with the plan of its batch (positions, work lists), as a step of a serving program does.

Format.  A row is the head_dim values of one token and kv head.  Of every 32 of them, with the largest magnitude M, p is the smallest
integer from -127 on with M <= 6 * 2^p, the scale byte is p + 127, and a value x becomes the e2m1 number nearest to x / 2^p (0, 0.5, 1,
1.5, 2, 3, 4, 6 with a sign; of two at the same distance the one with the even code).  Two codes a byte, the first in the low half.
A page of a head is 16 rows of codes, then 16 rows of scale bytes; a row of the tier is a token's codes of all heads, then their
scale bytes, up to a multiple of 16 bytes.

Shapes and length mixes are those of this repository's configurations and of its benchmark's decode leg; values are ~N(0, 1).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
BLOCK = 32
EPS = 1e-6

_BASE = dict(op="attend", layers=1, batch=1, q_heads=32, kv_heads=32, head_dim=128, rope_style=0, norm=False, window=8192, tier="hbm",
             overflow=False, hist_lo=0, hist_hi=0, new_lo=1, new_hi=1, lengths=0)


def _case(name: str, **kw) -> dict:
    return dict(_BASE, name=name, **kw)


def listed() -> list:
    return [
        # one decoding user's new token into the cache and the tier: all latency
        _case("append_b1", op="append", kv_heads=8, q_heads=64, hist_lo=2777, hist_hi=2777),
        # the new turns of a full grouped-query batch; the model normalises the heads of its keys
        _case("append_gqa_b64_norm", op="append", q_heads=64, kv_heads=8, norm=True, batch=64, hist_lo=1024, hist_hi=4096, new_lo=64, new_hi=512),
        # first turns of very different length with 64-wide heads
        _case("append_first_b16_d64", op="append", kv_heads=4, head_dim=64, rope_style=1, batch=16, new_lo=128, new_hi=2048),
        # one user waiting for tokens on the 70B-shaped layer: few bytes
        _case("attend_decode_gqa_b1", q_heads=64, kv_heads=8, hist_lo=2777, hist_hi=2777),
        # a full batch of decoding users on the same layer, of a model that normalises its heads
        _case("attend_decode_gqa_b64_norm", q_heads=64, kv_heads=8, norm=True, batch=64, hist_lo=1024, hist_hi=4096),
        # decoding on the 7B-shaped multi-head layer
        _case("attend_decode_mha_b16", batch=16, window=4096, hist_lo=1000, hist_hi=1600),
        # an ordinary batch of turns, multi-head: every key is used for a few dozen rows
        _case("attend_turn_mha_b16", batch=16, window=4096, hist_lo=512, hist_hi=2048, new_lo=32, new_hi=256),
        # the largest batch of turns, grouped-query, heads normalised: bound by the matrix cores
        _case("attend_turn_gqa_b64_norm", q_heads=64, kv_heads=8, norm=True, batch=64, hist_lo=1024, hist_hi=4096, new_lo=64, new_hi=512),
        # one conversation with a long document behind it
        _case("attend_turn_gqa_b1_long", q_heads=64, kv_heads=8, window=65536, hist_lo=31003, hist_hi=31003, new_lo=301, new_hi=301),
        # first turns: nothing saved yet; 64-wide heads, interleaved rotary pairs
        _case("attend_first_b16_d64", kv_heads=4, head_dim=64, rope_style=1, batch=16, new_lo=128, new_hi=2048),
        # conversations that overflow their window and keep the most recent half, the whole turn over four layers
        _case("turn_overflow_b8", op="turn", layers=4, batch=8, window=4096, hist_lo=4700, hist_hi=5500, new_lo=64, new_hi=512, overflow=True),
        # the whole turn with the tier where the method keeps it, pinned host memory: bound by the host link
        _case("turn_gqa_b16_pinned", op="turn", layers=2, batch=16, q_heads=64, kv_heads=8, hist_lo=1024, hist_hi=4096, new_lo=16, new_hi=64,
              tier="pinned"),
    ]


_MODELS = ((32, 32, 128), (40, 40, 128), (64, 8, 128), (32, 4, 64), (8, 2, 128), (4, 4, 64), (12, 4, 64), (5, 5, 128))
_MOST_SECONDS = 2.2e-3          # of a drawn case, at rates that the card sustains (the largest listed one takes 2.5e-3)


def _log_int(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> dict:
    q_heads, kv_heads, head_dim = rng.choice(_MODELS)
    c = dict(_BASE, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, rope_style=rng.randrange(2), norm=rng.random() < 0.4,
             batch=_log_int(rng, 1, 64), lengths=rng.randrange(1 << 20))
    kind = rng.choice(("append", "decode", "decode", "turn", "turn", "first", "long", "whole", "whole"))
    hist, new = _log_int(rng, 1, 4000), _log_int(rng, 1, 400)
    c.update(hist_lo=hist, hist_hi=_log_int(rng, hist, 4100), new_lo=new, new_hi=_log_int(rng, new, 520))
    if kind == "append":
        c["op"] = "append"
    elif kind == "decode":
        c.update(new_lo=1, new_hi=rng.choice((1, 1, 4)))
    elif kind == "first":
        c.update(hist_lo=0, hist_hi=0, new_hi=_log_int(rng, new, 2048))
    elif kind == "long":
        c.update(batch=rng.choice((1, 2)), window=65536, hist_lo=_log_int(rng, 4000, 31000), hist_hi=31003)
    elif kind == "whole":
        c.update(op="turn", layers=rng.choice((1, 2, 3)), tier="pinned" if rng.random() < 0.4 else "hbm")
        if rng.random() < 0.4:
            c.update(window=4096, hist_lo=4000, hist_hi=_log_int(rng, 4000, 5500), overflow=True)
    while _seconds(c) > _MOST_SECONDS and c["layers"] > 1:
        c["layers"] -= 1
    while _seconds(c) > _MOST_SECONDS and c["batch"] > 1:
        c["batch"] = (c["batch"] + 1) // 2
    while _seconds(c) > _MOST_SECONDS:
        c["new_lo"], c["new_hi"] = (c["new_lo"] + 1) // 2, (c["new_hi"] + 1) // 2
    return c


def _seconds(case: dict) -> float:
    w = work(case)
    host = case["layers"] * 2.0 * float(_lengths(case)[2].sum()) * _row_bytes(case) if case["tier"] == "pinned" else 0.0
    return max(w["bytes"] / 4e12, w["flops"] / 0.7e15, host / 5e10)


def _lengths(case: dict):
    """saved, new and kept tokens of every conversation"""
    rng = np.random.default_rng([case["lengths"], 77])
    hist = rng.integers(case["hist_lo"], case["hist_hi"] + 1, case["batch"]).astype(np.int32)
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, case["batch"]).astype(np.int32)
    kept = np.where(case["overflow"] & (hist + new > case["window"]), np.maximum(0, case["window"] // 2 - new), hist).astype(np.int32)
    return hist, new, kept


def _row_bytes(case: dict) -> int:
    return (case["kv_heads"] * 17 * case["head_dim"] // 32 + 15) // 16 * 16


def work(case: dict) -> dict:
    _, new, kept = _lengths(case)
    n, k = float(new.sum()), float(kept.sum())
    newf, keptf = new.astype(np.float64), kept.astype(np.float64)
    values = case["kv_heads"] * case["head_dim"]
    four = 2.0 * values * 17 / 32                   # bytes of a token's keys and values in 4 bits
    rows = 2.0 * values * 2                         # ... in bf16
    attend_b = four * (n + k) + 2.0 * case["q_heads"] * case["head_dim"] * 2 * n
    attend_f = 4.0 * case["head_dim"] * case["q_heads"] * float(np.sum(newf * keptf + newf * (newf + 1) / 2))
    append_b = rows * n + 2 * four * n + rows * n   # in; pages and tier; the values read back
    append_f = 2.0 * values * 8 * n
    if case["op"] == "append":
        b, f = append_b, append_f
    elif case["op"] == "attend":
        b, f = attend_b, attend_f
    else:
        b, f = 2 * four * k + append_b + attend_b, append_f + attend_f
    return {"bytes": case["layers"] * b, "flops": case["layers"] * f}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------


def _pack(x: torch.Tensor):
    """codes (two a byte) and scale bytes of bf16 rows, by comparisons in 32 bits (every step is exact)"""
    x = x.float().unflatten(-1, (-1, BLOCK))
    most = x.abs().amax(-1, keepdim=True)
    bits = most.view(torch.int32)
    byte = torch.clamp((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000).int(), min=0)
    y = torch.ldexp(x.abs(), 127 - byte)
    code = (y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
    code = torch.where(x < 0, code | 8, code).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, byte.squeeze(-1).to(torch.uint8)


def _tables(dev):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=dev)
    return torch.cat([grid, -grid]), torch.cat([2.0 ** torch.arange(-127.0, 127.0, device=dev, dtype=torch.float64), torch.full((2,), math.nan, device=dev)]).float()


def _angles(case: dict, dev):
    half = case["head_dim"] // 2
    freq = 10000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) * 2 / case["head_dim"])
    return torch.arange(int(case["window"]), device=dev, dtype=torch.float64)[:, None] * freq


def _to_rows(codes, scales, row_bytes: int) -> torch.Tensor:
    """[tokens, heads, ...] -> rows of the tier"""
    row = torch.cat([codes.flatten(-2), scales.flatten(-2)], -1)
    return torch.nn.functional.pad(row, (0, row_bytes - row.shape[-1]))


def _inputs(case: dict, seed: int) -> dict:
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    L, B, D, Hq, Hkv = case["layers"], case["batch"], case["head_dim"], case["q_heads"], case["kv_heads"]
    hist, new, kept = _lengths(case)
    context, total_q = kept + new, int(new.sum())

    def normal(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen)

    pages = (context + PAGE - 1) // PAGE
    num_pages = int(pages.sum()) + 5
    perm = np.random.default_rng([case["lengths"], 78]).permutation(num_pages).astype(np.int32)
    table = np.full((B, int(pages.max())), -1, np.int32)
    first = np.concatenate([[0], np.cumsum(pages)])
    for c in range(B):
        table[c, :pages[c]] = perm[first[c]:first[c + 1]]
    s = dict(case=case, hist=hist, new=new, kept=kept, table=table, num_pages=num_pages, scale=1.0 / math.sqrt(D),
             cu_q=np.concatenate([[0], np.cumsum(new)]), rows=np.concatenate([[0], np.cumsum(hist.astype(np.int64) + new)]),
             pages=[torch.from_numpy(table[c, :pages[c]]).long().to(dev) for c in range(B)])
    s["q_weight"], s["k_weight"] = ((1 + 0.2 * normal(L, D)).contiguous() for _ in range(2)) if case["norm"] else (None, None)
    # attending finds the whole context in the pool
    if case["op"] == "attend":
        s["k_pool"], s["v_pool"] = (torch.cat([t.flatten(-2) for t in _pack(normal(L, num_pages, Hkv, PAGE, D))], -1) for _ in range(2))
    else:
        s["k_pool"], s["v_pool"] = (torch.zeros(L, num_pages, Hkv, PAGE * 17 * D // 32, dtype=torch.uint8, device=dev) for _ in range(2))
        s["new_k"], s["new_v"] = normal(L, total_q, Hkv, D), normal(L, total_q, Hkv, D)
        for name in ("tier_k", "tier_v"):
            t = _to_rows(*_pack(normal(L, int(s["rows"][-1]), Hkv, D)), _row_bytes(case))
            s[name] = torch.empty(t.shape, dtype=torch.uint8, pin_memory=True).copy_(t) if case["tier"] == "pinned" else t
    if case["op"] != "append":
        s["q"] = normal(L, total_q, Hq, D)
    return s


def prepare(case: dict, seed: int) -> dict:
    s = _inputs(case, seed)
    dev = s["k_pool"].device
    s["grid"], s["powers"] = _tables(dev)
    angles = _angles(case, dev)
    s["cos"], s["sin"] = torch.cos(angles).float(), torch.sin(angles).float()
    if own:
        import paper_2403_19708_amd as ca

        L, D, context = case["layers"], case["head_dim"], s["kept"] + s["new"]
        total_q = int(s["new"].sum())
        ctx = ca.Context(ca.Config(n_layers=L, n_q_heads=case["q_heads"], n_kv_heads=case["kv_heads"], head_dim=D, max_positions=case["window"],
                                   rope_style=case["rope_style"], max_seqs=case["batch"], max_batch_kv_tokens=int(context.sum()) + 64,
                                   max_batch_q_tokens=total_q + 16, require_load=1 if case["op"] == "turn" else 0), kv_bits=4)
        s["ctx"], s["keep_start"], s["end"] = ctx, (s["hist"] - s["kept"]).astype(np.int32), context.astype(np.int32)
        if case["norm"]:
            for l in range(L):
                ctx.head_norm_set(l, s["q_weight"][l], s["k_weight"][l], EPS)
        if case["op"] != "append":
            s["out"] = torch.zeros_like(s["q"])
        if case["op"] != "attend":
            s["read_k"], s["read_v"] = torch.zeros_like(s["new_k"]), torch.zeros_like(s["new_v"])
            for name in ("tier_k", "tier_v"):
                s["at_" + name] = [ca.pointer_array([s[name][l].data_ptr() + int(r) * _row_bytes(case) for r in s["rows"][:-1]]) for l in range(L)]
        torch.cuda.synchronize()
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------------


def run(state: dict):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s: dict):
    ctx, case, stream = s["ctx"], s["case"], torch.cuda.current_stream()
    layers = range(case["layers"])
    # the plan of the batch: every step has another one, whatever of the step is measured
    ctx.rope_rebase(s["hist"], s["keep_start"], s["new"], s["table"], s["num_pages"], stream)
    if case["op"] == "attend":
        for l in layers:
            ctx.cached_prefill_attn(l, s["q"][l], s["k_pool"][l], s["v_pool"][l], s["out"][l], s["scale"], stream)
        return {"out": s["out"]}
    if case["op"] == "turn":
        for l in layers:
            ctx.kv_load_layer(l, s["at_tier_k"][l], s["at_tier_v"][l], s["k_pool"][l], s["v_pool"][l])
    for l in layers:
        ctx.kv_append_save_layer(l, s["new_k"][l], s["new_v"][l], s["k_pool"][l], s["v_pool"][l], s["at_tier_k"][l], s["at_tier_v"][l], stream)
        if case["op"] == "turn":
            ctx.cached_prefill_attn(l, s["q"][l], s["k_pool"][l], s["v_pool"][l], s["out"][l], s["scale"], stream)
        ctx.kv_read_layer(l, s["k_pool"][l], s["v_pool"][l], s["read_k"][l], s["read_v"][l], s["kept"], s["end"], stream)
    ctx.join(stream)
    return {"k": s["read_k"], "v": s["read_v"]} if case["op"] == "append" else {"out": s["out"], "k": s["read_k"], "v": s["read_v"]}


def _values(s: dict, codes, scales):
    """what codes [..., dims / 2] and scale bytes [..., dims / 32] stand for"""
    x = s["grid"][torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, BLOCK)) * s["powers"][scales.int()][..., None]).flatten(-2)


def _from_pages(s: dict, pool, c: int):
    """[tokens, heads, dims] of conversation c"""
    D = s["case"]["head_dim"]
    p = pool[s["pages"][c]]
    codes, scales = p[..., :PAGE * D // 2].unflatten(-1, (PAGE, -1)), p[..., PAGE * D // 2:].unflatten(-1, (PAGE, -1))
    return _values(s, codes, scales).transpose(1, 2).flatten(0, 1)[:int(s["kept"][c] + s["new"][c])]


def _from_rows(s: dict, rows):
    case = s["case"]
    H, D = case["kv_heads"], case["head_dim"]
    rows = rows.to(s["grid"].device, non_blocking=True)
    return _values(s, rows[:, :H * D // 2].unflatten(-1, (H, -1)), rows[:, H * D // 2:H * D * 17 // 32].unflatten(-1, (H, -1)))


def _rotate(s: dict, x, first: int):
    """rows [tokens, heads, dims] at positions first, first + 1, .."""
    cos, sin = s["cos"][first:first + x.shape[0], None], s["sin"][first:first + x.shape[0], None]
    if s["case"]["rope_style"] == 0:
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _held(s: dict, l: int):
    """values of the new keys and values in the cache; normalised in 64 bits, since a key next to a border falls on either side of it"""
    k = s["new_k"][l]
    if s["k_weight"] is not None:
        k = k.double()
        k = (k / torch.sqrt(k.square().mean(-1, keepdim=True) + EPS) * s["k_weight"][l].double()).to(torch.bfloat16)
    return _values(s, *_pack(k)), _values(s, *_pack(s["new_v"][l]))


def _attend(s: dict, q, k, v, kept: int):
    """softmax over the visible keys for new tokens q [new, heads, dims]; k, v [context, kv heads, dims]"""
    new, heads, D = q.shape
    k = _rotate(s, k, 0).permute(1, 2, 0)
    q = _rotate(s, q, kept).transpose(0, 1).reshape(k.shape[0], -1, D)
    score = torch.matmul(q, k).mul_(s["scale"]).view(heads, new, -1)
    at = torch.arange(kept + new, device=q.device)
    score.masked_fill_(at > at[kept:, None], -math.inf)
    p = score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(k.shape[0], -1, kept + new), v.transpose(0, 1)).view(heads, new, D) / total
    return out.transpose(0, 1)


def _run_plain(s: dict):
    case = s["case"]
    kinds = {"out": [], "k": [], "v": []}
    for l in range(case["layers"]):
        if case["op"] != "attend":
            new_k, new_v = _held(s, l)
            kinds["k"].append(new_k.to(torch.bfloat16))
            kinds["v"].append(new_v.to(torch.bfloat16))
        if case["op"] == "append":
            continue
        q = s["q"][l].float()
        if s["q_weight"] is not None:
            q = q / torch.sqrt(q.square().mean(-1, keepdim=True) + EPS) * s["q_weight"][l].float()
        out = []
        for c in range(case["batch"]):              # conversations of different length
            mine = slice(int(s["cu_q"][c]), int(s["cu_q"][c + 1]))
            if case["op"] == "attend":
                k, v = _from_pages(s, s["k_pool"][l], c), _from_pages(s, s["v_pool"][l], c)
            else:
                rows = slice(int(s["rows"][c] + s["hist"][c] - s["kept"][c]), int(s["rows"][c] + s["hist"][c]))
                k = torch.cat([_from_rows(s, s["tier_k"][l][rows]), new_k[mine]])
                v = torch.cat([_from_rows(s, s["tier_v"][l][rows]), new_v[mine]])
            out.append(_attend(s, q[mine], k, v, int(s["kept"][c])))
        kinds["out"].append(torch.cat(out).to(torch.bfloat16))
    return {name: torch.stack(x) for name, x in kinds.items() if x}


# ---- the definition, in 64 bits -------------------------------------------------------------------------------------------------


def exact(case: dict, seed: int):
    s = _inputs(case, seed)
    dev, D, H, G = s["k_pool"].device, case["head_dim"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    f64 = torch.float64
    magnitude = torch.tensor([(m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)) for e in range(4) for m in range(2)], dtype=f64, device=dev)

    def decode(codes, scales):
        both = torch.empty(*codes.shape[:-1], D, dtype=torch.int64, device=dev)
        both[..., 0::2], both[..., 1::2] = codes % 16, codes // 16
        sign = 1.0 - 2.0 * (both // 8)
        return sign * magnitude[both % 8] * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1)

    def held(x):
        x = x.double().reshape(-1, BLOCK)
        fraction, exponent = torch.frexp(x.abs().amax(-1))                # 6 * 2^p is 0.75 * 2^(p + 3)
        p = torch.clamp(exponent - 3 + (fraction > 0.75), min=-127)
        p = torch.where(fraction == 0, torch.full_like(p, -127), p)
        step = torch.exp2(p.double())[:, None]
        best, value = torch.full_like(x, math.inf), torch.zeros_like(x)
        for code in (0, 2, 4, 6, 1, 3, 5, 7):                             # of two at the same distance the first, an even one
            off = (x.abs() - magnitude[code] * step).abs()
            value = torch.where(off < best, magnitude[code] * step, value)
            best = torch.minimum(off, best)
        return torch.copysign(value, x)

    def normed(x, weight):
        x = x.double()
        return x if weight is None else x * torch.rsqrt((x * x).sum(-1, keepdim=True) / D + EPS) * weight.double()

    turn = _angles(case, dev)

    def spun(x, first):
        z = torch.complex(x[..., :D // 2], x[..., D // 2:]) if case["rope_style"] == 0 else torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous())
        z = z * torch.polar(torch.ones_like(turn[first:first + x.shape[0]]), turn[first:first + x.shape[0]])
        return torch.cat([z.real, z.imag], -1)

    kinds = {"out": [], "k": [], "v": []}
    for l in range(case["layers"]):
        if case["op"] != "attend":
            key = s["new_k"][l] if s["k_weight"] is None else normed(s["new_k"][l], s["k_weight"][l]).to(torch.bfloat16)
            kinds["k"].append(held(key).reshape(key.shape))
            kinds["v"].append(held(s["new_v"][l]).reshape(key.shape))
        if case["op"] == "append":
            continue
        q = normed(s["q"][l], None if s["q_weight"] is None else s["q_weight"][l])
        out = torch.empty(q.shape, dtype=f64, device=dev)
        for c in range(case["batch"]):
            kept, a, b = int(s["kept"][c]), int(s["cu_q"][c]), int(s["cu_q"][c + 1])
            t = torch.arange(kept + b - a, device=dev)
            hidden = t[None] > t[kept:, None]
            for g in range(H):
                both = []
                for name in ("k", "v"):
                    if case["op"] == "attend":
                        where, slot = s["pages"][c][t // PAGE], t % PAGE
                        pool = s[name + "_pool"][l][:, g]
                        codes, scales = pool[:, :PAGE * D // 2].reshape(-1, PAGE, D // 2), pool[:, PAGE * D // 2:].reshape(-1, PAGE, D // BLOCK)
                        both.append(decode(codes[where, slot], scales[where, slot]))
                    else:
                        end = int(s["rows"][c] + s["hist"][c])
                        rows = s["tier_" + name][l][end - kept:end].to(dev)
                        saved = decode(rows[:, g * D // 2:(g + 1) * D // 2], rows[:, H * D // 2 + g * D // BLOCK:H * D // 2 + (g + 1) * D // BLOCK])
                        both.append(torch.cat([saved, kinds[name][l][a:b, g]]))
                k = spun(both[0], 0)
                for h in range(g * G, (g + 1) * G):
                    score = spun(q[a:b, h], kept) @ k.T * s["scale"]
                    out[a:b, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ both[1]
        kinds["out"].append(out)
    return {name: torch.stack(x) for name, x in kinds.items() if x}
