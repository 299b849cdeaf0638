"""Attention over the 4-bit cache on the GPU, held closer than a worst case allows: the mean square of its error against 64 bits on every path,
every key counted exactly once, keys and queries of very different sizes side by side."""
import numpy as np
import pytest
import torch

import kv4_oracle as o4
from synth import bf16_bits_to_f64, draw_values_bf16
from test_gpu_kv4 import Turn, to_bits, to_torch, turn  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

# path: the switches that choose it, most rows a unit may have there, roundings of the operands of the score product (in units of the root mean
# square of one, for the root of their sum), and of the probabilities and the output
ROWS, TILES128, TILES256, EXPANDED, SCALAR = "few rows", "tiles of 128", "tiles of 256", "expanded", "scalar"
SWITCHES = {ROWS: dict(), TILES128: dict(attn_prerotate=1, attn_tile_rows=128), TILES256: dict(attn_prerotate=1, attn_tile_rows=256), EXPANDED: dict(attn_prerotate=2),
            SCALAR: dict(attn_variant=1)}
# Relative root mean square of a rounding to s significant bits: the error is uniform up to half a step, 2^-s of the power of two below the
# value, and mantissas m are spread like their logarithm: 2^-s / sqrt(3) * sqrt(mean of 1 / m^2) = 2^-s * 0.425.
U8, U11 = 2.0 ** -8 * 0.425, 2.0 ** -11 * 0.425
# Of a rotation in fp16 the angle, a product and the sum are rounded, and the part of the pair that is left out of a component is no larger than
# the pair: 3 roundings, of up to sqrt(2) of the component.  Queries are rounded before they are rotated (few rows), or behind (tiles), keys not.
# The expanded path rounds either once, rotated in fp32, and leaves to the tiles what is too large or small for that.
OPERANDS = {ROWS: 2 ** 0.5 * 7 ** 0.5 * U11, TILES128: 2 ** 0.5 * 4 ** 0.5 * U11, TILES256: 2 ** 0.5 * 4 ** 0.5 * U11, EXPANDED: 2 ** 0.5 * 4 ** 0.5 * U11, SCALAR: 0.0}
PROBABILITIES = {ROWS: U8, TILES128: U8, TILES256: U8, EXPANDED: U8, SCALAR: 0.0}


def exact(t, c, g):
    """outputs of the heads of kv head g of conversation c, and the root mean square of the size that score errors scale with"""
    G, mine = t.Hq // t.H, slice(t.cu[c], t.cu[c + 1])
    q = bf16_bits_to_f64(t.q[mine, g * G:(g + 1) * G])
    if t.qw is not None:
        q = o4.head_norm(q, t.qw, t.eps)
    k, v = t.context(0, c)[:, g], t.context(1, c)[:, g]
    n = int(t.n[c])
    qr, kr = o4.rotate(q, n + np.arange(len(q)), t.style), o4.rotate(k[:, None], np.arange(len(k)), t.style)[:, 0]
    s = np.einsum("jhd,td->jht", qr, kr) * t.scale
    size = np.einsum("jhd,td->jht", qr * qr, kr * kr) * t.scale ** 2
    hidden = np.arange(len(k))[None] > (n + np.arange(len(q)))[:, None]
    s = np.where(hidden[:, None], -np.inf, s)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, float((p * size).sum(-1).mean())


def check_rms(t, path, slack=1.25):
    """Root mean square of the error over that of the outputs.  Output and probabilities are rounded to 8 bits; a score off by d moves the output by
    its probability times d (v - out), no more than the output's own size times d where values have no common part.  The slack is for
    how far a mean over few rows may be off (a hundred roundings: 7 %), and for values with one."""
    got = bf16_bits_to_f64(to_bits(t.out))
    G = t.Hq // t.H
    err = size = 0.0
    score = []
    for c in range(t.B):
        for g in range(t.H):
            want, s = exact(t, c, g)
            score.append(s * len(want))
            err += ((got[t.cu[c]:t.cu[c + 1], g * G:(g + 1) * G] - want) ** 2).sum()
            size += (want ** 2).sum()
    s2 = sum(score) / (t.H * t.cu[-1])
    limit = slack * np.sqrt(U8 ** 2 + PROBABILITIES[path] ** 2 + OPERANDS[path] ** 2 * s2)
    assert np.sqrt(err / size) <= limit, (np.sqrt(err / size), limit, np.sqrt(s2))


def run(t):
    t.rebase()
    t.load()
    t.append()
    t.attend()
    t.finish()


# ---- every path's error ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("q_scale", [1.0, 4.0])
@pytest.mark.parametrize("style,norm", [(0, True), (1, False)])
@pytest.mark.parametrize("path,hist,new,Hq,H,D", [
    (ROWS, [700, 40, 301], [1, 4, 2], 16, 4, 128), (ROWS, [500, 3, 129], [5, 16, 1], 4, 4, 64),
    (TILES128, [300, 0], [90, 140], 4, 2, 128), (TILES128, [300, 0], [90, 140], 3, 3, 64),
    (TILES256, [200, 60], [150, 33], 4, 2, 128), (TILES256, [200, 60], [150, 33], 4, 4, 64),
    (EXPANDED, [200, 60], [150, 33], 4, 2, 128), (EXPANDED, [300, 0], [90, 140], 3, 3, 64),
    (SCALAR, [100, 0], [20, 31], 4, 2, 128), (SCALAR, [100, 0], [20, 31], 2, 2, 64)])
def test_mean_square_of_the_error(turn, path, hist, new, Hq, H, D, style, norm, q_scale):
    t = turn(hist, new, Hq, H, D, style=style, norm=norm, q_scale=q_scale, seed=3, **SWITCHES[path])
    run(t)
    check_rms(t, path)


# ---- every key counts once --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("marks", ["step", "place"])
@pytest.mark.parametrize("path,hist,new,Hq,H,D", [
    (ROWS, [1990, 700, 33], [1, 3, 2], 8, 2, 128), (ROWS, [1200, 64, 1], [2, 1, 16], 2, 2, 64), (ROWS, [1999], [1], 1, 1, 128),
    (TILES128, [1000, 31], [130, 70], 4, 1, 128), (TILES128, [1300, 31], [130, 70], 2, 2, 64), (TILES256, [1500, 100], [300, 1], 2, 2, 128),
    (TILES256, [900, 100], [70, 300], 4, 1, 64), (EXPANDED, [1500, 100], [300, 70], 2, 1, 128), (EXPANDED, [900, 3], [300, 20], 4, 2, 64)])
def test_every_key_counts_once(turn, path, hist, new, Hq, H, D, marks):
    """Queries of zeros give every visible key the same weight, exactly.  The values of a step of 32 keys are ones in a dimension of the step's
    own (or those of the same place in a step in the place's own), so that the output is how many of them were counted: one key more or less is a
    32nd (or one in at most 72) of that, the output's rounding a 256th."""
    T = sum(new)
    def ones(tokens, first):
        at = np.arange(first, first + tokens)
        v = np.zeros((tokens, H, D), np.uint16)
        v[np.arange(tokens), :, at // 32 % D if marks == "step" else at % 32] = 0x3F80
        return v
    cu = np.concatenate([[0], np.cumsum(new)])
    v_new = np.concatenate([ones(m, h) for h, m in zip(hist, new)])
    t = turn(hist, new, Hq, H, D, v_new=v_new, seed=5, **SWITCHES[path])
    t.q = np.zeros_like(t.q)
    t.dq.zero_()
    for c, h in enumerate(hist):
        t.saved[c][1] = o4.quantise(ones(h, 0))
        t.tier[1][c][:h] = torch.from_numpy(o4.rows(*t.saved[c][1])).to(t.tier[1][c].device)
    torch.cuda.synchronize()
    run(t)
    got = bf16_bits_to_f64(to_bits(t.out))
    for c, h in enumerate(hist):
        v = o4.values(*o4.quantise(ones(h + new[c], 0)))[:, 0]
        counts = np.cumsum(v, 0)[h:] / (h + 1 + np.arange(new[c]))[:, None]
        err = np.abs(got[cu[c]:cu[c + 1]] - counts[:, None])
        assert (err <= counts[:, None] * (2.0 ** -8 + 1e-6)).all(), (c, np.unravel_index(err.argmax(), err.shape))


# ---- batches as they come ----------------------------------------------------------------------------------------------------------------
HEADS = ((8, 8, 128), (5, 5, 128), (16, 2, 128), (8, 2, 128), (4, 4, 64), (12, 4, 64), (16, 2, 64), (33, 11, 64))


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(turn, seed):
    """whole turns of decode steps, short and long turns and first turns in any mixture, truncated, by the plan the library chooses"""
    rng = np.random.default_rng([seed, 41])
    Hq, H, D = HEADS[seed % len(HEADS)]
    B = int(rng.integers(1, 7))
    hist = np.where(rng.random(B) < 0.2, 0, np.exp(rng.uniform(0, np.log(1500), B)).astype(int))
    new = np.where(rng.random(B) < 0.4, 1, np.exp(rng.uniform(0, np.log(250), B)).astype(int))
    if seed % 3 == 0:
        new = np.minimum(new, 4)                                     # a batch of decode steps
    keep = (hist * rng.random(B) * (rng.random(B) < 0.4)).astype(int)
    t = turn(hist, new, Hq, H, D, keep=keep, style=int(rng.integers(2)), norm=bool(rng.integers(2)), seed=seed, tier=("device", "pinned")[int(rng.integers(2))],
             load_mode=int(rng.integers(3)), save_mode=int(rng.integers(3)))
    t.rebase()
    t.load()
    t.append_save()
    t.attend()
    t.finish()
    t.check_pools()
    t.check_tiers()
    check_rms(t, ROWS)                                               # the loosest of the limits
    t.out.fill_(float("nan"))
    before = t.out.clone()
    t.attend(out=before)
    t.attend()
    t.finish()
    assert torch.equal(before, t.out)


@pytest.mark.parametrize("path", [ROWS, TILES128, TILES256, EXPANDED, SCALAR])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_behind_the_last_sequence_stay_on_every_path(turn, path, D):
    t = turn([40, 10], [3, 4 if path == ROWS else 70], 4, 2, D, **SWITCHES[path])
    T = int(t.cu[-1])
    out = torch.full((T + 4, 4, D), 3.0, dtype=torch.bfloat16, device=t.out.device)
    t.rebase()
    t.load()
    t.append()
    t.attend(out=out[2:T + 2])
    t.finish()
    assert (out[:2] == 3.0).all() and (out[T + 2:] == 3.0).all()
    t.out.copy_(out[2:T + 2])
    check_rms(t, path)


@pytest.mark.parametrize("path,hist,new", [(ROWS, [700, 40, 301], [1, 4, 2]), (TILES128, [300, 0, 9], [90, 140, 1]), (TILES256, [200, 60, 3], [150, 33, 1]),
                                           (EXPANDED, [200, 60, 0], [150, 33, 1]), (SCALAR, [100, 0, 5], [20, 31, 1])])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tier", ["device", "pinned"])
@pytest.mark.parametrize("offset", [2, 5])
def test_memory_of_any_alignment(turn, path, hist, new, D, tier, offset):
    """queries, outputs, new keys and values aligned to their elements, pools and tiers to bytes"""
    t = turn(hist, new, 8, 2, D, seed=6, tier=tier, norm=True, **SWITCHES[path])

    def elsewhere(x, by, pin=False):
        flat = x.contiguous().reshape(-1).view(torch.uint8)
        room = torch.zeros(flat.numel() + 64, dtype=torch.uint8, device=x.device)
        room = room.pin_memory() if pin else room
        room[by:by + flat.numel()] = flat
        return room
    rooms = [elsewhere(x, 2) for x in (t.dq, t.dk, t.dv, t.out)]
    q, k, v, out = (r.data_ptr() + 2 for r in rooms)
    pool_rooms = [elsewhere(x, offset) for x in t.pools]
    pools = [r.data_ptr() + offset for r in pool_rooms]
    tier_rooms = [[elsewhere(x, offset, tier == "pinned") for x in mine] for mine in t.tier]
    tiers = [[r.data_ptr() + offset for r in mine] for mine in tier_rooms]
    got = [torch.zeros(int(t.cu[-1]) * 2 * D + 8, dtype=torch.bfloat16, device=t.dq.device) for _ in range(2)]
    torch.cuda.synchronize()
    t.rebase()
    t.ctx.kv_load_layer(0, *tiers, *pools)
    t.ctx.kv_append_save_layer(0, k, v, *pools, *tiers)
    t.ctx.cached_prefill_attn(0, q, *pools, out, t.scale)
    t.ctx.kv_read_layer(0, *pools, *(x.data_ptr() + 2 for x in got))
    t.finish()
    for room, x in [(rooms[3], t.out)] + list(zip(pool_rooms, t.pools)) + [y for a, b in zip(tier_rooms, t.tier) for y in zip(a, b)]:
        by = 2 if x is t.out else offset
        x.reshape(-1).view(torch.uint8).copy_(room[by:by + x.numel() * x.element_size()])
        assert not room[:by].any() and not room[by + x.numel() * x.element_size():].any()
    torch.cuda.synchronize()
    t.check_pools()
    t.check_tiers()
    check_rms(t, path)
    for i in range(2):
        assert np.array_equal(bf16_bits_to_f64(to_bits(got[i][1:1 + int(t.cu[-1]) * 2 * D])).reshape(-1, 2, D), o4.values(*t.appended[i]))


# ---- keys of very different sizes side by side -------------------------------------------------------------------------------------------
LOW = 8          # rotary pairs of the lowest frequencies, which a few hundred positions hardly turn


@pytest.mark.parametrize("where", ["hidden", "outweighed"])
@pytest.mark.parametrize("exponent", [18, 20, 24, 40, 100])
@pytest.mark.parametrize("path,T,Hq,H,D", [(ROWS, 8, 4, 2, 128), (ROWS, 16, 2, 2, 64), (TILES128, 90, 4, 2, 128), (TILES128, 90, 2, 2, 64), (TILES256, 150, 4, 2, 128),
                                          (TILES256, 150, 2, 2, 64), (EXPANDED, 90, 4, 2, 128), (SCALAR, 20, 2, 2, 64)])
def test_a_large_key_takes_no_bits_from_the_others(turn, path, T, Hq, H, D, exponent, where):
    """hidden: the last token's key, which only its own row sees; outweighed: one in the middle whose scores are far below the others'"""
    f = lambda x: (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    k = bf16_bits_to_f64(draw_values_bf16((T, H, D), 8, 2))
    q = bf16_bits_to_f64(draw_values_bf16((T, Hq, D), 8, 1))
    low = np.concatenate([np.arange(D // 2 - LOW, D // 2), np.arange(D - LOW, D)])
    q[..., low] = 3.0
    at = T - 1 if where == "hidden" else T // 2
    k[at] = 0.0
    k[at, :, low] = -2.0 ** exponent
    t = turn([0], [T], Hq, H, D, k_new=f(k), seed=8, window=512, **SWITCHES[path])
    t.q = f(q)
    t.dq.copy_(to_torch(t.q))
    run(t)
    t.check_pools()
    check_rms(t, path)


# ---- norms of queries and keys whose squares are past the range of 32 bits ------------------------------------------------------------------
@pytest.mark.parametrize("eps", [1e-6, 0.0])
@pytest.mark.parametrize("exponent", [120, 70, -60, -70, -125, "mixed"])
@pytest.mark.parametrize("path,T,Hq,H,D", [(ROWS, 8, 4, 2, 128), (ROWS, 16, 2, 2, 64), (TILES128, 90, 4, 2, 128), (TILES256, 150, 2, 2, 64), (EXPANDED, 90, 4, 2, 128),
                                          (EXPANDED, 90, 2, 2, 64), (SCALAR, 20, 4, 2, 128)])
def test_norms_of_heads_of_any_size(turn, path, T, Hq, H, D, exponent, eps):
    f = lambda x: (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    sizes = 2.0 ** (np.array([0, 100, -70, 64, -10, -124])[np.arange(T) % 6] if exponent == "mixed" else np.full(T, float(exponent)))
    k = f(bf16_bits_to_f64(draw_values_bf16((T, H, D), 8, 2)) * sizes[:, None, None])
    t = turn([0], [T], Hq, H, D, k_new=k, seed=8, norm=True, style=T % 4 // 2, window=512, **SWITCHES[path])
    t.eps = eps
    t.ctx.head_norm_set(0, *t.weights, eps)
    t.appended[0] = o4.quantise(o4.f64_to_bf16_bits(o4.head_norm(bf16_bits_to_f64(k), t.kw, eps)))
    t.q = f(bf16_bits_to_f64(draw_values_bf16((T, Hq, D), 8, 1)) * sizes[:, None, None])
    t.dq.copy_(to_torch(t.q))
    run(t)
    t.check_pools()
    check_rms(t, path)


@pytest.mark.parametrize("D,Hq", [(128, 4), (64, 4)])
@pytest.mark.parametrize("bad", [False, True])
def test_shares_over_the_expanded_cache_from_both_kernels(turn, D, Hq, bad):
    """one share of a row tile loads a key outside the middle of fp16's range, the others do not; then a value that is NaN as well"""
    H, hist, new = 1, 3000, 130
    t = turn([hist], [new], Hq, H, D, seed=12, **SWITCHES[EXPANDED])
    k = bf16_bits_to_f64(draw_values_bf16((hist, H, D), 12, 10))
    v = bf16_bits_to_f64(draw_values_bf16((hist, H, D), 12, 11))
    low = np.concatenate([np.arange(D // 2 - LOW, D // 2), np.arange(D - LOW, D)])
    k[100], k[1700] = 0.0, k[1700] * 2.0 ** -30
    k[100, :, low] = 2.0 ** 30
    if bad:
        v[2001, :, 40] = np.nan
    f = lambda x: (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    q = bf16_bits_to_f64(t.q)
    q[..., low] = 0.0                                                # its scores are none: among 3000 keys it is one more
    t.q = f(q)
    t.dq.copy_(to_torch(t.q))
    t.saved[0] = [o4.quantise(f(x)) for x in (k, v)]
    for i in range(2):
        t.tier[i][0][:hist] = torch.from_numpy(o4.rows(*t.saved[0][i])).to(t.tier[i][0].device)
    torch.cuda.synchronize()
    t.rebase()
    items = t.ctx.rebase_read(6).reshape(-1, 8)
    assert (items[items[:, 0] >= 0][:, 6] >= 0).any()
    t.load()
    t.append()
    t.attend()
    t.finish()
    got = bf16_bits_to_f64(to_bits(t.out))
    if bad:
        assert np.isnan(got[:, :, 32:64]).all() and np.isfinite(got[:, :, :32]).all() and np.isfinite(got[:, :, 64:]).all()
        t.saved[0][1] = o4.quantise(f(np.nan_to_num(v)))             # the other dimensions are those without it
        clean = t.out.clone()
        clean[:, :, 32:64] = to_torch(f(np.concatenate([exact(t, 0, 0)[0][:, :, 32:64]]))).reshape(clean[:, :, 32:64].shape)
        t.out.copy_(clean)
    check_rms(t, EXPANDED)
