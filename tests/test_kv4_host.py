"""The 4-bit cache without a GPU: the oracle's codes against a search over all of them, the format's edges, and what the host refuses."""
import ctypes

import numpy as np
import pytest

import kv4_oracle as o4
import paper_2403_19708_amd as ca
from hip_model import Turn, in_model
from paper_2403_19708_amd import binding
from synth import bf16_bits_to_f64, draw_values_bf16


@pytest.mark.parametrize("D", [64, 128])
def test_codes_are_the_nearest_ones(D):
    bits = draw_values_bf16((50, 3, D), 5, 1)
    x = bf16_bits_to_f64(bits)
    codes, scales = o4.quantise(bits)
    v = o4.values(codes, scales)
    step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    every = np.concatenate([o4.GRID, -o4.GRID])
    assert np.array_equal(np.abs(v - x), np.abs(x[..., None] - every * step[..., None]).min(-1))
    most = np.abs(x).reshape(50, 3, -1, 32).max(-1)
    s = 2.0 ** (scales.astype(float) - 127)
    assert (most <= 6 * s).all() and (most > 3 * s).all()            # the smallest scale that cuts nothing off


def test_edges_of_the_format():
    def one(values):
        x = np.zeros(64, np.float32)
        x[:len(values)] = values
        bits = (x.view(np.uint32) >> 16).astype(np.uint16)
        return o4.quantise(bits)

    codes, scales = one([6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.0, -6.0])
    assert scales.tolist() == [127, 0]                                # 6 = 6 * 2^0; a block of zeros has the smallest scale
    assert [int(c) & 15 for c in codes[:5]] == [7, 6, 4, 2, 8] and [int(c) >> 4 for c in codes[:5]] == [6, 4, 2, 0, 15]
    assert one([6.03125])[1][0] == 128 and one([3.0])[1][0] == 126 and one([3.015625])[1][0] == 127
    codes, scales = one([3.3895313892515355e38, 6 * 2.0 ** 125, 2.0 ** 125])        # the largest finite bf16
    assert scales[0] == 252 and codes[0] == 0x77 and codes[1] == 2    # 6 * 2^125 is the largest that is kept
    assert one([2.0 ** -133])[1][0] == 0
    for bad in (np.inf, -np.inf, np.nan):
        codes, scales = one([1.0, bad])
        assert scales.tolist() == [255, 0] and not codes.any() and np.isnan(o4.values(codes, scales)[:32]).all()


def test_rows_are_multiples_of_16_bytes():
    assert [o4.row_bytes(h, d) for h, d in ((8, 128), (5, 128), (1, 128), (4, 64), (1, 64), (3, 64))] == [544, 352, 80, 144, 48, 112]


@pytest.mark.parametrize("kw,status", [
    (dict(attn_variant=4), "CA_ERR_UNSUPPORTED"),
    (dict(attn_schedule=1), "CA_ERR_UNSUPPORTED"),
    (dict(head_dim=96), "CA_ERR_UNSUPPORTED"),
])
def test_configurations_that_are_refused(kw, status):
    with pytest.raises(ca.CaError) as e:
        ca.config_validate(ca.Config(**kw), kv_bits=4)
    assert e.value.status_name == status


def test_other_switches_are_served():
    for kw in (dict(), dict(attn_variant=1), dict(attn_variant=2), dict(attn_tile_rows=256), dict(attn_prerotate=1), dict(attn_prerotate=1, attn_variant=2, attn_tile_rows=256), dict(attn_prerotate=2), dict(attn_split=1),
               dict(load_mode=1, save_mode=1), dict(head_dim=64, rope_style=1)):
        ca.config_validate(ca.Config(**kw), kv_bits=4)
    with pytest.raises(ValueError):
        ca.config_validate(ca.Config(), kv_bits=8)


def test_calls_without_a_context():
    lib = ca.load_library()
    n = ctypes.c_int64(0)
    c = ca.Config().to_c()
    assert lib.ca_create_kv4(ctypes.byref(c), None) == 1
    assert lib.ca_kv_sizes(None, ctypes.byref(n), ctypes.byref(n)) == 1
    assert lib.ca_kv_read_layer(None, 0, None, None, None, None, None, None, None) == 1
    assert lib.ca_head_norm_set(None, 0, None, None, 1e-6, None) == 1
    assert {"ca_create_kv4", "ca_kv_sizes", "ca_kv_read_layer", "ca_head_norm_set"} <= set(binding.SYMBOLS)


# ---- on the model of the HIP runtime ------------------------------------------------------------------------------------------------
class Turn4(Turn):
    """hip_model's batch over a 4-bit cache"""

    def __init__(self, m, hist, new, tier=0, heads=(4, 2, 128), layers=1, **cfg):
        hq, hkv, d = heads
        self.m, self.hist, self.new = m, np.array(hist, np.int32), np.array(new, np.int32)
        m.device(0)
        pages = (self.hist + self.new + 15) // 16
        self.num_pages = int(pages.sum()) + 1
        self.table = np.full((len(hist), int(pages.max())), -1, np.int32)
        first = np.concatenate([[0], np.cumsum(pages)])
        for c in range(len(hist)):
            self.table[c, :pages[c]] = range(first[c], first[c + 1])
        total, context = int(self.new.sum()), int((self.hist + self.new).sum())
        self.ctx = ca.Context(ca.Config(n_layers=layers, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_positions=int((self.hist + self.new).max()), max_seqs=len(hist),
                                        max_batch_kv_tokens=context + 64, max_batch_q_tokens=total + 16, **cfg), kv_bits=4)
        self.row = self.ctx.kv_row_bytes
        self.kp, self.vp = (m.alloc(self.num_pages * self.ctx.kv_page_bytes) for _ in range(2))
        self.tk, self.tv = ([m.alloc(int(r) * self.row, tier) for r in self.hist + self.new] for _ in range(2))
        self.q, self.out = (m.alloc(total * hq * d * 2) for _ in range(2))
        self.nk, self.nv = (m.alloc(total * hkv * d * 2) for _ in range(2))
        self.scale = d ** -0.5


# Four heads to a thread where one would give every compute unit more than 16 workgroups: here 1200 of them
@pytest.mark.parametrize("cus,heads_to_a_thread", [(256, 1), (80, 1), (64, 4)])
@in_model
def test_an_append_is_spread_over_the_compute_units_there_are(m, cus, heads_to_a_thread):
    m.lib.model_cus(cus)
    t = Turn4(m, [0], [1200], heads=(8, 8, 128))
    t.rebase()
    op, = m.queued(t.append)
    assert f"kv4_append_kernelILi128ELb0ELi{heads_to_a_thread}E" in m.what(op)
    assert m.lib.model_workgroups(op) == 75 * 8 // heads_to_a_thread


# Shares of 33 MiB, which the static call takes only where nothing but the last round of workgroups is cut
@pytest.mark.parametrize("heads,hist,new", [((64, 4, 64), [3327, 5094, 3895, 2850], [223, 355, 348, 368]),
                                            ((64, 4, 64), [15489, 6862, 10754, 7958, 14590, 5666], [315, 248, 210, 149, 292, 215]),
                                            ((32, 4, 64), [6625, 10010, 3869], [1450, 1023, 1182])])
@in_model
def test_what_the_static_call_takes_does_not_depend_on_plans_that_were_not_taken(m, heads, hist, new):
    t = Turn4(m, hist, new, heads=heads, require_load=0, attn_tile_rows=128)
    t.rebase()
    taken = t.ctx.rebase_read(6)
    answers = []
    for prerotate in (0, 1, 2):                    # both ways, then each for itself
        one = t if prerotate == 0 else Turn4(m, hist, new, heads=heads, require_load=0, attn_tile_rows=128, attn_prerotate=prerotate)
        one.rebase()
        same = np.array_equal(one.ctx.rebase_read(6), taken)
        try:
            one.attn(static=True)
            answers.append((same, "taken"))
        except ca.CaError as e:
            answers.append((same, e.status_name))
    alone = [a for a in answers[1:] if a[0]]
    assert alone and all(a == (True, "CA_ERR_OUT_OF_RANGE") for a in [answers[0]] + alone), answers


@pytest.mark.parametrize("load_mode", [0, 1])
@pytest.mark.parametrize("tier", [0, 1], ids=["device", "pinned"])
@in_model
def test_a_whole_turn_waits_for_what_it_reads(m, tier, load_mode):
    t = Turn4(m, [4000, 30], [200, 1], tier=tier, load_mode=load_mode)
    s, other = m.stream(), m.stream()
    ops = m.queued(lambda: (t.rebase(s), t.load(), t.append(s), t.attn(s), t.save(s)))
    load, save = m.named(ops, "kv4_move_kernel")
    append, = m.named(ops, "kv4_append_kernel")
    assert all(m.behind(load, op) for op in m.named(ops, "copy")) and len(m.named(ops, "copy")) == 4 * load_mode
    attn = m.named(ops, "attn_kv4") + m.named(ops, "attn_prerot") + m.named(ops, "kv4_expand") + m.named(ops, "kv4_mark")
    assert attn and all(m.behind(op, load) and m.behind(op, append) for op in attn) and m.behind(save, append) and m.behind(save, load)
    t.ctx.join(other)
    assert m.stream_behind(other, load) and m.stream_behind(other, save)
    t.ctx.sync()
    assert m.done(load) and m.done(save)


@pytest.mark.parametrize("new", [[5, 40], [2, 9000]], ids=["short", "long"])
@pytest.mark.parametrize("tier", [0, 1], ids=["device", "pinned"])
@in_model
def test_a_staged_write_back_copies_what_was_packed(m, tier, new):
    """new_k and new_v are not what the tier holds: the codes are packed from the pools first"""
    t = Turn4(m, [33, 0], new, tier=tier, save_mode=1, pipeline_depth=2)
    s, other = m.stream(), m.stream()
    t.rebase(s)
    for _ in range(3):                                    # (the third takes the first one's slot)
        ops = m.queued(lambda: t.append_save(s))
        append, = m.named(ops, "kv4_append_kernel")
        pack, = m.named(ops, "kv4_move_kernel")
        copies = m.named(ops, "copy")
        assert len(copies) == 4 and m.behind(pack, append) and all(m.behind(op, pack) for op in copies)
    t.ctx.join(other)
    assert all(m.stream_behind(other, op) for op in copies)
    t.ctx.sync()
    assert all(m.done(op) for op in copies)


@pytest.mark.parametrize("tier,mode", [(0, 0), (1, 2), (1, 0)], ids=["device", "pinned-mode2", "pinned"])
@pytest.mark.parametrize("new", [2, 20000], ids=["short", "long"])
@in_model
def test_sync_and_join_cover_append_save(m, new, tier, mode):
    t = Turn4(m, [0], [new], tier=tier, save_mode=mode)
    s, s2, other = m.stream(), m.stream(), m.stream()
    t.rebase(s)
    saves = [m.queued(lambda: t.append_save(x))[-1] for x in (s, s, s2)]        # (the third while the others are under way)
    t.ctx.join(other)
    assert all(m.stream_behind(other, op) for op in saves)
    t.ctx.sync()
    assert all(m.done(op) for op in saves)


@pytest.mark.parametrize("new", [1, 40])
@in_model
def test_a_step_can_be_captured(m, new):
    t = Turn4(m, [100], [new], require_load=0)
    s, s2 = m.stream(), m.stream()
    got = [m.alloc(new * t.ctx.cfg.n_kv_heads * t.ctx.cfg.head_dim * 2) for _ in range(2)]
    t.rebase(s)
    t.append_save(s2)
    m.lib.model_capture(s, 1)
    m.queued(lambda: (t.append_save(s), t.attn(s), t.ctx.kv_read_layer(0, t.kp, t.vp, *got, stream=s)))
    assert m.lib.model_capture(s, 0)
    t.ctx.join(s2)
    t.ctx.sync()
    t.rebase(s)


@in_model
def test_scratch_copies_are_for_plans_that_may_expand(m):
    """two bf16 copies of a batch's context and their marks; a context that never expands has none"""
    def bytes_of(**cfg):
        before = m.lib.model_device_bytes()
        t = Turn4(m, [4000], [200], heads=(8, 8, 128), **cfg)
        made = m.lib.model_device_bytes() - before
        t.ctx.close()
        return made
    bytes_of()                                      # (the first context finds the library's static memory)
    copies = bytes_of() - bytes_of(attn_prerotate=1)
    context = (4200 + 64) * 8 * 128 * 2
    assert 2 * context <= copies <= 2.1 * context
