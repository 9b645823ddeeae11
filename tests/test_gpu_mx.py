"""hsadmm_compact_mx and hsadmm_expand_mx against a plain numpy quantisation of the plain packing.  Everything about them is
exact: scales are powers of two, codes are nearest values, sums of fp32 are formed in a stated order; so codes, scale bytes
and expanded bits have to be equal."""
import numpy as np
import pytest
import torch

import paper_2512_14628_amd as pkg
import workloads as wk
from tests.ref_e4m3 import E2M1, E4M3, nearest_code

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
N, F, C, B = wk.MODE_NONE, wk.MODE_FILTER, wk.MODE_CHANNEL, wk.MODE_BOTH
FORMATS = [pkg.MX_FP8, pkg.MX_FP4]
TOP = {pkg.MX_FP8: 448.0, pkg.MX_FP4: 6.0}
# rows of one element, of odd and even lengths, shorter and longer than a block and than an item; 1x1 and 3x3 layers
SHAPES = [(1, 1, 1, F, 1), (7, 3, 9, F, 3), (16, 16, 9, F, 8), (33, 31, 1, F, 20), (5, 1030, 1, F, 2), (3, 2500, 1, F, 2),
          (10, 64, 1, N, 10), (9, 5, 9, N, 9), (40, 24, 1, C, 7), (12, 10, 9, C, 4), (65, 33, 1, C, 11), (2, 3000, 1, C, 900),
          (24, 20, 9, B, 9, 8), (31, 17, 1, B, 30, 5), (3, 2100, 1, B, 2, 1001)]


def random_mask(wl, rng, keep=None):
    """keep: None: the plan's counts at random places; else the probability of every group's byte (any nonzero value)."""
    parts = []
    for l in wl.layers:
        for groups, k in ([(l.c_out, l.k), (l.c_in, l.k_in)] if l.mode == B else [(l.groups, l.k)]):
            m = np.zeros(groups, np.uint8)
            if keep is None:
                m[rng.permutation(groups)[:k]] = 1
            else:
                m = np.where(rng.random(groups) < keep, rng.integers(1, 256, groups), 0).astype(np.uint8)
            parts.append(m)
    return np.concatenate(parts)


def packing(wl, mask, align):
    """Per layer: the arena elements in packed order; layer_off; kept_idx."""
    places, off, kept = [], [0], []
    for l in wl.layers:
        g = l.group_base
        rows, cols = np.arange(l.c_out), np.arange(l.c_in)
        if l.mode in (F, B):
            rows = np.flatnonzero(mask[g:g + l.c_out])
        if l.mode == C:
            cols = np.flatnonzero(mask[g:g + l.c_in])
        if l.mode == B:
            cols = np.flatnonzero(mask[g + l.c_out:g + l.c_out + l.c_in])
        kept += [rows] if l.mode in (N, F) else [cols] if l.mode == C else [rows, cols]
        at = (rows[:, None, None] * l.c_in + cols[None, :, None]) * l.khw + np.arange(l.khw)
        places.append(at.reshape(-1) + l.elem_off)
        off.append(off[-1] + -(-at.size // align) * align)
    return places, np.array(off), np.concatenate(kept)


def quantise(c, fmt):
    """Codes (one a value) and scale bytes of fp32 values, a whole number of blocks."""
    b = c.astype(np.float64).reshape(-1, 32)
    bad = ~np.isfinite(b).all(1)
    b = np.where(bad[:, None], 0, b)
    top = np.abs(b).max(1)
    e = np.full(top.shape, -127)
    while (over := top > TOP[fmt] * np.ldexp(1.0, e)).any():
        e = np.where(over, e + 1, e)
    # (a code that stands for 2^128 has no value in fp32: the code below)
    limit = np.where(e == (120 if fmt == pkg.MX_FP8 else 126), 240.0 if fmt == pkg.MX_FP8 else 3.0, np.inf)[:, None]
    codes = nearest_code(np.clip(b / np.ldexp(1.0, e)[:, None], -limit, limit), fmt)
    codes[bad] = 0
    return codes.reshape(-1), np.where(bad, 255, e + 127).astype(np.uint8)


def stored(codes, fmt):
    return codes if fmt == pkg.MX_FP8 else (codes[0::2] | (codes[1::2] << 4)).astype(np.uint8)


def values(codes, scales, fmt):
    """What codes (one a value) stand for, fp32."""
    v = (E4M3 if fmt == pkg.MX_FP8 else E2M1)[codes].reshape(-1, 32)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v * s[:, None]).astype(np.float32).reshape(-1)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


class Case:
    def __init__(self, shapes=SHAPES, seed=0, align=32):
        self.wl = wk.custom_workload(shapes, R=1, seed=seed)
        self.plan = pkg.Plan(self.wl.table(), pack_align_elems=align)
        self.align = align
        self.ws = torch.zeros(self.plan.workspace_bytes, dtype=torch.uint8, device=DEV)
        self.rng = np.random.default_rng(seed)
        cap = self.plan.packed_capacity_elems
        self.codes = torch.full((cap + 64,), 0xAB, dtype=torch.uint8, device=DEV)
        self.scales = torch.full((cap // 32 + 8,), 0xCD, dtype=torch.uint8, device=DEV)
        self.off = torch.full((self.plan.n_layers + 1,), -1, dtype=torch.int64, device=DEV)
        self.kept = torch.full((self.plan.groups_total,), -1, dtype=torch.int32, device=DEV)

    def arena(self, spread=4.0):
        n = self.wl.n_arena
        x = self.rng.standard_normal(n) * 10.0 ** self.rng.uniform(-spread, spread, n)
        x = x.astype(np.float32)
        on = np.zeros(n, bool)
        for l in self.wl.layers:
            on[l.elem_off:l.elem_off + l.n] = True
        x[~on] = np.nan
        return x

    def write(self, src0, src1, mask, fmt):
        pkg.hsadmm_compact_mx(self.plan, dev(src0), None if src1 is None else dev(src1), mask, fmt, self.codes, self.scales,
                              self.off, self.kept, self.ws)

    def check_written(self, c, mask, fmt):
        """Codes, scales, offsets and kept lists against the plain form; nothing beyond the blocks is touched."""
        places, off, kept = packing(self.wl, mask, self.align)
        want_codes = np.full(self.codes.numel(), 0xAB, np.uint8)
        want_scales = np.full(self.scales.numel(), 0xCD, np.uint8)
        half = 1 if fmt == pkg.MX_FP8 else 2
        for p, o in zip(places, off):
            x = np.concatenate([c[p], np.zeros(-p.size % 32, np.float32)])
            code, scale = quantise(x, fmt) if x.size else (np.zeros(0, np.uint8),) * 2
            assert o % 32 == 0
            want_codes[o // half:(o + x.size) // half] = stored(code, fmt)
            want_scales[o // 32:(o + x.size) // 32] = scale
        got = self.scales.cpu().numpy()
        assert np.array_equal(got, want_scales), np.flatnonzero(got != want_scales)[:8]
        got = self.codes.cpu().numpy()
        assert np.array_equal(got, want_codes), np.flatnonzero(got != want_codes)[:8]
        assert np.array_equal(self.off.cpu().numpy(), off)
        got = self.kept.cpu().numpy()
        assert np.array_equal(got[:kept.size], kept) and (got[kept.size:] == -1).all()

    def close(self):
        self.plan.close()


@pytest.mark.parametrize("keep", [None, 0.0, 0.05, 0.9, 1.0])
@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
def test_written_codes_are_the_nearest_values(fmt, two, keep):
    case = Case(seed=3)
    z, v = case.arena(), case.arena() if two else None
    mask = random_mask(case.wl, case.rng, keep)
    case.write(z, v, dev(mask), fmt)
    with np.errstate(invalid="ignore"):
        case.check_written(z + v if two else z, mask, fmt)
    # again under the mappings that call has left in the workspace
    case.codes.fill_(0xAB)
    case.scales.fill_(0xCD)
    case.write(z, v, None, fmt)
    case.check_written(z + v if two else z, mask, fmt)
    case.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_wider_alignment_leaves_its_padding_alone(fmt):
    case = Case(align=96, seed=5)
    z = case.arena()
    mask = random_mask(case.wl, case.rng)
    case.write(z, None, dev(mask), fmt)
    case.check_written(z, mask, fmt)
    case.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_special_values(fmt):
    """Zeros of both signs, denormals, the largest numbers, ties, and values that are not finite, in kept and pruned places."""
    case = Case([(40, 32, 1, F, 20)], seed=1)
    z = case.arena(0.0)
    rows = z.reshape(40, 32)
    tiny = np.float32(2.0 ** -149)
    rows[0] = 0.0
    rows[1] = -0.0
    rows[2] = tiny
    rows[3] = tiny * np.arange(32, dtype=np.float32)
    rows[4] = np.float32(3.4028235e38)
    rows[5] = np.linspace(-3.4e38, 3.4e38, 32, dtype=np.float32)
    rows[6] = np.float32(2.0 ** -126) * np.arange(32, dtype=np.float32)
    rows[7] = np.concatenate([[448.0], np.arange(31) + 0.5])                     # ties
    rows[8] = np.concatenate([[6.0], np.arange(31) * 0.25])
    rows[9] = np.concatenate([[np.nextafter(np.float32(448), np.float32(500))], np.arange(31)])    # one more power of two
    rows[10] = np.concatenate([[np.nextafter(np.float32(6), np.float32(7))], np.arange(31) * 0.1])
    rows[11, 5] = np.inf
    rows[12, 31] = np.nan
    rows[13, 0] = -np.inf
    rows[14] = np.float32(1.1754944e-38)
    rows[15] = 2.0 ** np.arange(-16, 16)
    rows[20:] = np.nan                                                           # pruned: not looked at
    mask = (np.arange(40) < 20).astype(np.uint8)
    case.write(z, None, dev(mask), fmt)
    case.check_written(z, mask, fmt)
    dst = torch.full((case.wl.n_arena,), 5.0, device=DEV)
    pkg.hsadmm_expand_mx(case.plan, [case.codes], [case.scales], fmt, dev(mask), dst, None, None, case.ws)
    got = dst.cpu().numpy().reshape(40, 32)
    assert np.isnan(got[11:14]).all() and np.isfinite(np.delete(got, [11, 12, 13], 0)).all()
    assert not got[20:].view(np.uint32).any()
    case.close()


def buffers(case, mask, fmt, M):
    """M nodes' buffers (random values under one mask), as stored and as they read."""
    places, off, _ = packing(case.wl, mask, case.align)
    half, out = (1 if fmt == pkg.MX_FP8 else 2), []
    for _ in range(M):
        c = case.arena(2.0)
        # (what no one writes is never read: codes of NaN and scales of NaN between the blocks)
        codes = np.full(max(int(off[-1]), 32) // half, 0x7F, np.uint8)
        scales = np.full(max(int(off[-1]), 32) // 32, 255, np.uint8)
        read = []
        for p, o in zip(places, off):
            x = np.concatenate([c[p], np.zeros(-p.size % 32, np.float32)])
            if x.size == 0:
                read.append(x)
                continue
            code, scale = quantise(x, fmt)
            codes[o // half:(o + x.size) // half], scales[o // 32:(o + x.size) // 32] = stored(code, fmt), scale
            read.append(values(code, scale, fmt)[:p.size])
        out.append((codes, scales, read))
    return places, out


@pytest.mark.parametrize("keep", [None, 0.0, 0.5, 1.0])
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("M", [1, 2, 5, 64])
@pytest.mark.parametrize("fmt", FORMATS)
def test_reading_is_the_mean_of_the_values_on_kept_elements(fmt, M, dual, keep):
    case = Case(seed=M)
    mask = random_mask(case.wl, case.rng, keep)
    places, nodes = buffers(case, mask, fmt, M)
    n = case.wl.n_arena
    want = np.full(n, 7.0, np.float32)
    for li, (l, p) in enumerate(zip(case.wl.layers, places)):
        want[l.elem_off:l.elem_off + l.n] = 0.0
        acc = nodes[0][2][li]
        for node in nodes[1:]:
            acc = acc + node[2][li]
        want[p] = acc * np.float32(1.0 / M)
    zi, vd = case.arena(1.0), case.arena(1.0)
    dst, dvd = torch.full((n,), 7.0, device=DEV), dev(vd)
    args = (dev(zi), dvd) if dual else (None, None)
    codes, scales = [dev(c) for c, _, _ in nodes], [dev(s) for _, s, _ in nodes]
    pkg.hsadmm_expand_mx(case.plan, codes, scales, fmt, dev(mask), dst, *args, case.ws)
    got = dst.cpu().numpy()
    assert np.array_equal(got.view(np.uint32), want.view(np.uint32)), np.flatnonzero(got.view(np.uint32) != want.view(np.uint32))[:8]
    if dual:
        on = ~np.isnan(vd)
        new = (vd + (zi - want))[on]
        assert np.array_equal(dvd.cpu().numpy()[on].view(np.uint32), new.view(np.uint32))
        assert np.isnan(dvd.cpu().numpy()[~on]).all()
    # the same under the mappings in the workspace
    dst.fill_(7.0)
    pkg.hsadmm_expand_mx(case.plan, codes, scales, fmt, None, dst, None, None, case.ws)
    assert np.array_equal(dst.cpu().numpy().view(np.uint32), want.view(np.uint32))
    case.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_code_and_every_scale_byte_reads_as_the_formats_say(fmt):
    """A layer of 256 blocks, block s with scale byte s, all codes in it in turn."""
    case = Case([(256, 32, 1, N, 256)])
    codes = np.tile(np.arange(256, dtype=np.uint8), 32) if fmt == pkg.MX_FP8 else np.tile(np.arange(16, dtype=np.uint8), 512)
    codes = np.concatenate([np.roll(codes[32 * s:32 * s + 32], s) for s in range(256)])
    scales = np.arange(256, dtype=np.uint8)
    dst = torch.zeros(case.wl.n_arena, device=DEV)
    mask = dev(np.zeros(256, np.uint8))                        # (an unconstrained layer is kept whatever the bytes say)
    pkg.hsadmm_expand_mx(case.plan, [dev(stored(codes, fmt))], [dev(scales)], fmt, mask, dst, None, None, case.ws)
    got = dst.cpu().numpy()
    with np.errstate(over="ignore"):
        want = values(codes, scales, fmt)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.array_equal(got[ok].view(np.uint32), want[ok].view(np.uint32))
    case.close()


@pytest.mark.parametrize("fmt,step", [(pkg.MX_FP8, 2.0 ** -4), (pkg.MX_FP4, 2.0 ** -2)])
def test_what_comes_back_is_within_half_a_step(fmt, step):
    """A round trip of values next to the fp32 pack and expand of the same: relative to the value half a step at most
    (2^-4, 2^-2), or half the smallest code's step in units of the block's scale."""
    case = Case(seed=11)
    mask = random_mask(case.wl, case.rng)
    z, v = case.arena(1.0), case.arena(1.0)
    case.write(z, v, dev(mask), fmt)
    n = case.wl.n_arena
    a, b = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    pkg.hsadmm_expand_mx(case.plan, [case.codes], [case.scales], fmt, None, a, None, None, case.ws)
    packed = torch.zeros(case.plan.packed_capacity_elems, device=DEV)
    pkg.hsadmm_compact_sum(case.plan, dev(z), dev(v), dev(mask), packed, case.off, case.kept, case.ws)
    pkg.hsadmm_expand(case.plan, packed, None, b, case.ws)
    a, b = a.cpu().numpy().astype(np.float64), b.cpu().numpy().astype(np.float64)
    places, off, _ = packing(case.wl, mask, 32)
    scales = case.scales.cpu().numpy()
    smallest = np.zeros(n)
    for p, o in zip(places, off):
        smallest[p] = np.ldexp(2.0 ** -9 if fmt == pkg.MX_FP8 else 0.5, scales[o // 32 + np.arange(p.size) // 32].astype(int) - 127)
    assert (np.abs(a - b) <= np.maximum(np.abs(b) * step, smallest / 2)).all()
    case.close()


def test_refusals():
    case = Case(SHAPES[:4])
    p, ws, n = case.plan, case.ws, case.wl.n_arena
    z, v, dst = (torch.zeros(n + 8, device=DEV) for _ in range(3))
    mask = torch.ones(p.groups_total, dtype=torch.uint8, device=DEV)

    def write(plan=p, src0=z, src1=None, mask=mask, fmt=0, codes=case.codes, scales=case.scales, off=case.off, kept=case.kept,
              ws=ws, **k):
        return pkg.hsadmm_compact_mx(plan, src0, src1, mask, fmt, codes, scales, off, kept, ws, check=False, **k)

    def read(plan=p, codes=[case.codes], scales=[case.scales], fmt=0, mask=mask, dst=dst, Zi=None, Vd=None, ws=ws, **k):
        return pkg.hsadmm_expand_mx(plan, codes, scales, fmt, mask, dst, Zi, Vd, ws, check=False, **k)

    assert write() == 0 and read() == 0
    tight = pkg.Plan(case.wl.table(), pack_align_elems=16)
    for call in (write, read):
        assert call(plan=tight) == -4                          # blocks would hold two layers
        assert call(fmt=2) == -4 and call(fmt=-1) == -4
        assert call(ws=ws, workspace_bytes=p.workspace_bytes - 1) == -2
        assert call(ws=None, workspace_bytes=p.workspace_bytes) == -1
    tight.close()
    for bad in (dict(src0=None), dict(src0=z[1:]), dict(src1=v[2:]), dict(codes=None), dict(codes=case.codes[8:]),
                dict(scales=None), dict(off=None), dict(kept=None)):
        assert write(**bad) == -1, bad
    for bad in (dict(codes=[], scales=[]), dict(codes=[None]), dict(codes=[case.codes[4:]]), dict(scales=[None]), dict(dst=None),
                dict(dst=dst[1:]), dict(Zi=z), dict(Vd=v), dict(Zi=z, Vd=z), dict(Zi=dst, Vd=v), dict(Zi=z, Vd=dst),
                dict(Zi=z[1:], Vd=v)):
        assert read(**bad) == -1, bad
    assert read(codes=[case.codes] * 65, scales=[case.scales] * 65) == -4
    with pytest.raises(ValueError):
        pkg.hsadmm_expand_mx(p, [case.codes], [], 0, mask, dst, None, None, ws)
    torch.cuda.synchronize()
    case.close()
