"""GPU parity of positions, cache pages, masks and differences where the other file's shapes do not reach: far positions of every pair, calls large
enough for the kernels of large calls, buffers of eight-byte alignment, and what the calls refuse."""
import math
from decimal import Decimal

import numpy as np
import pytest

from oracle.ckks_oracle import AttnDesc
from paper_2609_12378_b200 import binding
from tests.harness import params
from tests.test_frequencies_host import PI, angles
from tests.test_gpu_positions import EXP, RSQRT, SCALE, _dev_cts, _dev_keys, _keys, _refused, _residues, _ring

pytestmark = pytest.mark.gpu


# ---- the table -------------------------------------------------------------------------------------------------------
def _unit(position, w):
    """cos, sin of position * w as Decimals good to 2^-100: a double's functions at the angle's nearest double, and the rest's first order."""
    a = position * w % (2 * PI)
    if a > PI:
        a -= 2 * PI
    r = float(a)
    rest = a - Decimal(r)                     # below 2^-52: its square is left out, the functions at r are exact to 2^-53
    c, s = Decimal(math.cos(r)), Decimal(math.sin(r))
    return c - rest * s, s + rest * c


@pytest.mark.parametrize("rot,theta", [(128, 500000.0), (96, 10000.0), (256, 1.5)])
@pytest.mark.parametrize("kind,factor", [("none", 1.0), ("linear", 3.0), ("base", 8.0), ("bands", 8.0), ("ramp", 32.0)])
def test_every_pair_of_a_far_position_is_as_exact_as_of_a_near_one(rot, theta, kind, factor):
    """A unit is off by less than 3 * 2^-52 (the rounding of its argument, at most pi 2^-53, and two units in the last place of each value), a value by two
    units, the magnitude's product and its own, 7 * 2^-52, and by the frequency's 2^-103 relative times the position, 2^-52 at most: 2^-49
    in all, times the magnitude; the comparison's own functions add 2^-53."""
    _, ctx = _ring(10)
    few, many = (1.0, 4.0) if kind == "bands" else (1.0, 32.0)
    w = angles(rot, theta, kind, factor, 8192.0, few, many)
    pairs = sorted({0, 1, 2, 5, rot // 8, rot // 4, rot // 2 - 1})
    for first in (0, (1 << 20) + 3, (1 << 36) - 7, (1 << 50) - 9):
        cos, sin = (t.cpu().numpy() for t in ctx.rotary_table(rot, first, 9, theta=theta, scaling=kind, factor=factor, original_length=8192.0, magnitude=1.25))
        for i in (0, 3, 8):
            for j in pairs:
                c, s = _unit(Decimal(first + i), w[j])
                for got, want in ((cos[i, j], c), (sin[i, j], s)):
                    assert abs(Decimal(float(got)) - Decimal(1.25) * want) <= Decimal(1.25) * (Decimal(2) ** -49 + Decimal(2) ** -53), (first + i, j, got)


def test_a_long_table_of_an_odd_shape():
    """Enough rows for the large tiles, the last one cut, and columns that fill no tile: sampled rows, the last ones among them, against the same
    positions' rows of short tables and the definition."""
    _, ctx = _ring(10)
    rot, first, count = 70, 1000003, 131072 * 2 + 77                     # 35 pairs: two column tiles; 1025 row tiles of 256
    cos, sin = (t.cpu().numpy() for t in ctx.rotary_table(rot, first, count, theta=10000.0))
    w = angles(rot, 10000.0, "none", 1.0, 0.0, 1.0, 4.0)
    assert cos.shape == (count, rot // 2)
    for i in (0, 1, 15, 16, 255, 256, 4095, 77777, count - 78, count - 77, count - 2, count - 1):
        for j in (0, 1, 31, 32, 33, 34):
            c, s = _unit(Decimal(first + i), w[j])
            assert abs(Decimal(float(cos[i, j])) - c) <= Decimal(2) ** -49 + Decimal(2) ** -53, (i, j)
            assert abs(Decimal(float(sin[i, j])) - s) <= Decimal(2) ** -49 + Decimal(2) ** -53, (i, j)
    near = ctx.rotary_table(rot, first + count - 5, 5, theta=10000.0)
    for got, want in zip((cos[-5:], sin[-5:]), near):
        assert np.abs(got - want.cpu().numpy()).max() <= 2.0 ** -48


# ---- scales of two maps ------------------------------------------------------------------------------------------------------
def test_maps_whose_scales_part_in_the_softmax_are_refused():
    """A round takes a relative difference of the scales to about twenty times itself (u^2 and the polynomial of degree 2 in its square, times u, squared):
    scores just within 2^-30 of each other leave probabilities that may not be subtracted."""
    import torch
    from tests.gpu_util import context, key_dev
    P, ctx = params(10, 13, 4, 4), context(10, 13, 4, 4)
    o, desc = P.oracle, AttnDesc(8, 2, 4)
    tok, lad = o.attention_rotations(desc)
    keys, rlk = _dev_keys(_keys(P, 5, tok + lad)), key_dev(_keys(P, 6, [0]).popitem()[1], 0)
    q, k = _dev_cts(_residues(P, 1, 13, 2)), _dev_cts(_residues(P, 2, 13, 2))
    w = torch.ones(2, dtype=torch.float64, device="cuda")

    def diff(off, rounds, **kw):
        q2 = _dev_cts(_residues(P, 3, 13, 2), SCALE * (1 + off))
        return ctx.attention_differential(q, k, q2, k, k, w, 0.5, rounds, EXP, [RSQRT] * rounds, rlk, keys, 8, 2, 4, **kw)
    launches = binding.kernel_launches()
    for kw in (dict(), dict(masked=True, causal=True)):
        _refused(binding.ERR_SCALE, diff, 0.9 * 2.0 ** -30, 1, **kw)
        _refused(binding.ERR_SCALE, diff, -0.2 * 2.0 ** -30, 1, **kw)
    assert binding.kernel_launches() == launches
    assert len(diff(2.0 ** -36, 1)) == 2


# ---- buffers on one another ----------------------------------------------------------------------------------------------------
def test_a_table_s_halves_may_not_overlap():
    import torch
    _, ctx = _ring(10)
    buf = torch.zeros(33 * 8, dtype=torch.float64, device="cuda")
    at = lambda x: buf[8 * x: 8 * x + 128].view(16, 8)  # noqa: E731
    launches = binding.kernel_launches()
    for a, b in ((0, 0), (0, 15), (15, 0), (3, 4)):
        _refused(binding.ERR_ARG, ctx.rotary_table, 16, 0, 16, out=(at(a), at(b)))
    assert binding.kernel_launches() == launches
    ctx.rotary_table(16, 0, 16, out=(at(16), at(0)))          # neighbours


def _as_table(t, rows, half):
    import torch
    return t.view(-1)[:rows * half].view(torch.float64).view(rows, half)


def test_calls_on_tables_keys_weights_or_workspaces_in_their_results_place_are_refused():
    import torch
    P, ctx = _ring(10)
    a, level = (16, 4, 8), 4
    C = lambda t, s=SCALE: binding.Ciphertext(t, s)  # noqa: E731
    x, v = _dev_cts(_residues(P, 1, level, 1)), _dev_cts(_residues(P, 2, level, 1))
    pk, pv = _dev_cts(_residues(P, 3, level - 1, 1)), _dev_cts(_residues(P, 4, level - 1, 1))
    keys = _dev_keys(_keys(P, 2, P.oracle.rotary_rotations(*a, 16, False)))
    cos, sin = ctx.rotary_table(16, 0, 8)
    out = [C(torch.empty((2, level - 1, P.N), dtype=torch.uint64, device="cuda"))]
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    on_ws = lambda shape: ws[4096: 4096 + 8 * int(np.prod(shape))].view(torch.uint64).view(shape)  # noqa: E731
    launches = binding.kernel_launches()

    def rotary(**kw):
        kw = dict(cts=x, cos=cos, sin=sin, keys=keys, outs=out, ws=ws) | kw
        return ctx.rotary(kw["cts"], [0], kw["cos"], kw["sin"], kw["keys"], *a, outs=kw["outs"], ws=kw["ws"])

    def append(**kw):
        kw = dict(k=x, v=v, pk=pk, pv=pv, cos=cos, sin=sin, keys=keys, ws=ws, out_k=None) | kw
        return ctx.cache_append(kw["k"], kw["v"], [0], [(1, 3, 0)], kw["pk"], kw["pv"], kw["cos"], kw["sin"], kw["keys"], *a, out_k=kw["out_k"], ws=kw["ws"])
    key_ws = [binding.SwitchKey(on_ws(tuple(k.data.shape)), k.galois) for k in keys]
    on_key = lambda l: [C(keys[0].data.view(-1)[:2 * l * P.N].view(2, l, P.N))]  # noqa: E731
    for name in ("cos", "sin"):
        _refused(binding.ERR_ARG, rotary, **{name: _as_table(out[0].data, 8, 8)})
        _refused(binding.ERR_ARG, rotary, **{name: _as_table(on_ws((64,)), 8, 8)})
        _refused(binding.ERR_ARG, append, **{name: _as_table(pk[0].data, 8, 8)})
        _refused(binding.ERR_ARG, append, **{name: _as_table(pv[0].data, 8, 8)})
        _refused(binding.ERR_ARG, append, **{name: _as_table(on_ws((64,)), 8, 8)})
    _refused(binding.ERR_ARG, rotary, outs=on_key(level - 1))
    _refused(binding.ERR_ARG, rotary, keys=key_ws)
    _refused(binding.ERR_ARG, rotary, cts=[C(on_ws((2, level, P.N)))])
    _refused(binding.ERR_ARG, rotary, outs=[C(on_ws((2, level - 1, P.N)))])
    _refused(binding.ERR_ARG, append, out_k=on_key(level - 1))
    _refused(binding.ERR_ARG, append, pv=on_key(level - 1))
    _refused(binding.ERR_ARG, append, keys=key_ws)
    _refused(binding.ERR_ARG, append, k=[C(on_ws((2, level, P.N)))])
    _refused(binding.ERR_ARG, append, v=[C(on_ws((2, level, P.N)))])
    _refused(binding.ERR_ARG, append, pk=[C(on_ws((2, level - 1, P.N)))])
    # score maps
    y, z = _dev_cts(_residues(P, 5, level, 2)), _dev_cts(_residues(P, 6, level, 2))
    outs = [C(torch.empty((2, level - 1, P.N), dtype=torch.uint64, device="cuda")) for _ in y]
    w = torch.ones(2, dtype=torch.float64, device="cuda")
    mask = lambda **kw: ctx.attention_mask(kw.get("x", y), 8, 2, 4, outs=kw.get("outs", outs), ws=ws)  # noqa: E731
    diff = lambda **kw: ctx.attention_difference(kw.get("x", y), kw.get("y", z), kw.get("w", w), 8, 2, 4, outs=kw.get("outs", outs), ws=ws)  # noqa: E731
    for f in (mask, diff):
        _refused(binding.ERR_ARG, f, x=[y[0], C(on_ws((2, level, P.N)))])
        _refused(binding.ERR_ARG, f, outs=[outs[0], C(on_ws((2, level - 1, P.N)))])
    _refused(binding.ERR_ARG, diff, y=[C(on_ws((2, level, P.N))), z[1]])
    _refused(binding.ERR_ARG, diff, w=_as_table(outs[1].data, 1, 2).view(-1))
    _refused(binding.ERR_ARG, diff, w=_as_table(on_ws((64,)), 1, 2).view(-1))
    assert binding.kernel_launches() == launches
    rotary(), append(), mask(), diff()                       # and none of it with buffers of their own


def test_keys_of_another_level_and_workspaces_on_the_host_are_refused():
    import torch
    P, ctx = _ring(10)
    a = (16, 4, 8)
    x = _dev_cts(_residues(P, 1, 4, 1))
    keys = _dev_keys(_keys(P, 2, P.oracle.rotary_rotations(*a, 16, False)))
    cos, sin = ctx.rotary_table(16, 0, 8)
    short = [binding.SwitchKey(k.data[:, :, :-1].contiguous(), k.galois) for k in keys]
    launches = binding.kernel_launches()
    with pytest.raises(ValueError):
        ctx.rotary(x, [0], cos, sin, short, *a)
    with pytest.raises(ValueError):
        ctx.cache_append(x, None, [0], [(0, 1, 0)], _dev_cts(_residues(P, 3, 3, 1)), None, cos, sin, short, *a)
    with pytest.raises(ValueError):
        ctx.rotary(x, [0], cos, sin, keys, *a, ws=torch.empty(64 << 20, dtype=torch.uint8))
    assert binding.kernel_launches() == launches


# ---- large calls and eight-byte alignment ------------------------------------------------------------------------------------------
def _odd(arr):
    """A ciphertext or key on the device eight bytes behind a sixteen-byte boundary."""
    import torch
    t = torch.empty(arr.size + 1, dtype=torch.int64, device="cuda")[1:].view(arr.shape)
    t.copy_(torch.from_numpy(arr.view(np.int64)))
    assert t.data_ptr() % 16 == 8
    return t.view(torch.uint64)


def _cts(x, odd):
    return [binding.Ciphertext(_odd(c), SCALE) for c in x] if odd else _dev_cts(x)


@pytest.mark.parametrize("odd", ["", "x", "y", "out", "x y out"])
def test_masks_and_differences_of_many_limbs(odd):
    """Sixteen groups at N = 2^13, level 7: more rows than are taken by a warp each."""
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(13)
    o, level, shape = P.oracle, 7, (128, 4, 8)
    desc = AttnDesc(*shape)
    assert (P.N >> 10) * 2 * desc.groups() * (level - 1) > 6 * 148
    x, y = _residues(P, 51, level, 16), _residues(P, 52, level, 16)
    dx, dy = _cts(x, "x" in odd), _cts(y, "y" in odd)
    fresh = lambda: _cts(np.zeros((16, 2, level - 1, P.N), dtype=np.uint64), "out" in odd)  # noqa: E731
    kw = dict(causal=True, key_begin=2, key_end=120, window=70)
    got, want = ctx.attention_mask(dx, *shape, outs=fresh(), **kw), o.attention_mask(desc, x, **kw)
    for g in range(16):
        assert np.array_equal(host(got[g].data), want[g]), g
    w = np.array([0.5, -1.25, 0.0, 0.7])
    got, want = ctx.attention_difference(dx, dy, torch.from_numpy(w).cuda(), *shape, outs=fresh()), o.attention_difference(desc, x, y, w)
    for g in range(16):
        assert np.array_equal(host(got[g].data), want[g]), g


@pytest.mark.parametrize("log_n,level,shape,n", [(12, 6, (32, 4, 16), 3), (13, 7, (64, 8, 8), 16)])
@pytest.mark.parametrize("odd", ["", "in", "page", "out", "key", "in page out key"])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_unaligned_buffers(log_n, level, shape, n, odd, in_place):
    """Whole pages and parts of pages, rotated keys, values and keys without positions; the larger case has more rows than are taken by a warp each."""
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(log_n)
    o, inner, half = P.oracle, shape[2], shape[0] // 2
    keys = _keys(P, 61, o.rotary_rotations(*shape, shape[0], False))
    dk = [binding.SwitchKey(_odd(k), g) for g, k in keys.items()] if "key" in odd else _dev_keys(keys)
    xk, xv = _residues(P, 62, level, n), _residues(P, 63, level, n)
    pk, pv = _residues(P, 64, level - 1, n), _residues(P, 65, level - 1, n)
    spans = [(0, inner, 0)] + [(i % 5, inner - i % 3 - 1, i) for i in range(1, n)]
    a = np.random.default_rng(66).uniform(-4, 4, (n + inner, half))
    cos, sin = np.cos(a), np.sin(a)
    dc, ds = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    pages = list(range(n))
    for table, parts in (((dc, ds), spans), ((dc, ds), [(1, inner, 0)] + spans[1:]), ((None, None), spans)):
        dxk, dxv = _cts(xk, "in" in odd), _cts(xv, "in" in odd)
        dpk, dpv = _cts(pk, "page" in odd), _cts(pv, "page" in odd)
        fresh = lambda: _cts(np.zeros_like(pk), "out" in odd)  # noqa: E731
        ok, ov = ctx.cache_append(dxk, dxv, pages, parts, dpk, dpv, *table, dk, *shape, out_k=None if in_place else fresh(), out_v=None if in_place else fresh())
        for i, (b, e, r) in enumerate(parts):
            want = o.append_keys(pk[i], xk[i], cos, sin, keys, *shape, shape[0], False, b, e, r) if table[0] is not None else o.append_values(pk[i], xk[i], inner, b, e)
            assert np.array_equal(host(ok[i].data), want), i
            assert np.array_equal(host(ov[i].data), o.append_values(pv[i], xv[i], inner, b, e)), i


# ---- options on the ring that they change ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layout,rot", [("half", 128), ("interleaved", 40)])
def test_rotation_with_options_that_change_its_kernels(layout, rot):
    """N = 2^16: conversions on the tensor cores, a share of the plain transforms on the integer pipe, and both, which leave the fused row kernel."""
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(16)
    o, a, il = P.oracle, (128, 32, 8), layout == "interleaved"
    keys = _keys(P, 71, o.rotary_rotations(*a, rot, il))
    x, dk = _residues(P, 72, 3, 2), _dev_keys(keys)
    ang = np.random.default_rng(73).uniform(-4, 4, (16, rot // 2))
    cos, sin = np.cos(ang), np.sin(ang)
    dc, ds = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    want, d = o.rotary(x, [0, 5], cos, sin, keys, *a, rot, il), _dev_cts(x)
    both = {binding.OPT_CONV_KERNEL: binding.CONV_TENSOR, binding.OPT_NTT_FP_SHARE: 3}
    for options in (both, {binding.OPT_CONV_KERNEL: binding.CONV_TENSOR}, {binding.OPT_NTT_FP_SHARE: 3}, {binding.OPT_CONV_KERNEL: binding.CONV_TENSOR, binding.OPT_NTT_FP_SHARE: 0}):
        old = {k: ctx.get_option(k) for k in options}
        try:
            for k, v in options.items():
                ctx.set_option(k, v)
            out = ctx.rotary(d, [0, 5], dc, ds, dk, *a, rot_dim=rot, layout=layout)
        finally:
            for k, v in old.items():
                ctx.set_option(k, v)
        assert all(np.array_equal(host(out[i].data), want[i]) for i in range(2)), options


# ---- five to eight digits: the row kernel and the launches apart ----------------------------------------------------------------------
@pytest.mark.parametrize("ring,level,shape,n", [((12, 6, 1, 6), 6, (16, 4, 32), 13), ((12, 6, 1, 6), 6, (16, 4, 32), 18), ((13, 8, 1, 8), 8, (16, 4, 32), 5),
                                                ((13, 8, 1, 8), 7, (16, 4, 32), 16), ((14, 6, 1, 6), 6, (32, 8, 16), 1), ((14, 6, 1, 6), 5, (32, 8, 16), 16),
                                                ((15, 10, 2, 5), 10, (64, 16, 16), 1), ((15, 10, 2, 5), 9, (64, 16, 16), 3)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_of_many_digits_on_both_sides_of_its_rule(ring, level, shape, n, layout):
    import torch
    from tests.gpu_util import context, host
    P, ctx = params(*ring), context(*ring)
    o, il, rows = P.oracle, layout == "interleaved", [i % 3 for i in range(n)]
    keys = _keys(P, 81, o.rotary_rotations(*shape, shape[0], il))
    x, dk = _residues(P, 82, level, n), _dev_keys(keys)
    a = np.random.default_rng(83).uniform(-4, 4, (2 + shape[2], shape[0] // 2))
    cos, sin = np.cos(a), np.sin(a)
    out = ctx.rotary(_dev_cts(x), rows, torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), dk, *shape, layout=layout)
    want = o.rotary(x, rows, cos, sin, keys, *shape, shape[0], il)
    for i in range(n):
        assert np.array_equal(host(out[i].data), want[i]), i
