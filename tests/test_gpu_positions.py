"""GPU parity: position tables, the rotation of shard ciphertexts by them, the append to pages of a cache, masks and differences of score
maps, and masked and differential attention.  Every limb bit-exact against the CPU checker's definitions; the chain a decoder runs on
decrypted results."""
import ctypes as C
import math
import threading

import numpy as np
import pytest

from oracle.ckks_oracle import AttnDesc
from paper_2609_12378_b200 import binding, inputs
from tests.harness import Client, params
from tests.test_oracle_positions import TOL, rotate_clear

pytestmark = pytest.mark.gpu

SCALE = 2.0 ** 50
RINGS = {10: (10, 6, 3, 2), 11: (11, 6, 1, 6), 12: (12, 6, 2, 3), 13: (13, 7, 7, 1), 15: (15, 4, 2, 2), 16: (16, 3, 1, 3), 100: (10, 9, 1, 9), 101: (10, 20, 10, 2)}       # parameters by log_n, or another number for a second set


def _ring(log_n):
    from tests.gpu_util import context
    return params(*RINGS[log_n]), context(*RINGS[log_n])


def _residues(P, seed, level, count=1):
    return inputs.uniform_residues(inputs.rng(seed, level), P.q[:level], P.N, 2 * count).reshape(count, 2, level, P.N)


def _keys(P, seed, rots):
    g, allp = inputs.rng(seed, 99), list(P.q) + list(P.p)
    return {P.oracle.galois_element(r): inputs.uniform_residues(g, allp, P.N, 2 * P.dnum).reshape(P.dnum, 2, P.L + P.K, P.N) for r in rots}


def _dev_cts(x, scale=SCALE):
    from tests.gpu_util import ct_dev
    return [ct_dev(c, scale) for c in x]


def _dev_keys(keys):
    from tests.gpu_util import key_dev
    return [key_dev(k, g) for g, k in keys.items()]


def _table(seed, rows, half):
    import torch
    a = inputs.rng(seed, 5).uniform(-4, 4, (rows, half))
    c, s = np.cos(a), np.sin(a)
    return c, s, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


# ---- the table -------------------------------------------------------------------------------------------------------
def _angles(rot, theta, kind, factor, length, few, many):
    """Turns per position, from the definition, in extended precision."""
    ld = np.longdouble
    j, pi = np.arange(rot // 2).astype(ld), ld("3.14159265358979323846264338327950288")
    t = ld(theta) * ld(factor) ** (ld(rot) / (rot - 2)) if kind == "base" else ld(theta)
    w = t ** (-2 * j / rot)
    if kind == "linear":
        return w / factor
    if kind == "bands":
        keep = np.clip((length * w / (2 * pi) - few) / (many - few), 0, 1)
        return keep * w + (1 - keep) * w / factor
    if kind == "ramp":
        lo, hi = (rot * np.log(length / (b * 2 * pi)) / (2 * np.log(t)) for b in (many, few))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
        keep = 1 - np.clip((j - lo) / max(hi - lo, 0.001), 0, 1)
        return keep * w + (1 - keep) * w / factor
    return w


@pytest.mark.parametrize("rot,first,count", [(128, 0, 128), (2, 5, 1), (256, 7, 33), (96, 131000, 300), (64, (1 << 20) - 5, 10)])
@pytest.mark.parametrize("kind,factor", [("none", 1.0), ("linear", 4.0), ("base", 8.0), ("bands", 8.0), ("ramp", 32.0)])
def test_table_of_angles(rot, first, count, kind, factor):
    """A frequency is a double, formed with a power, at most four products and a sum, each off by 2^-53 relative (the power by 2^-52): the angle of
    position p is off by at most p w (2^-52 + 5 * 2^-53) < p 2^-50, and the values by two roundings and the function's own two units."""
    if kind == "base" and rot < 4:
        rot = 4
    _, ctx = _ring(10)
    args = dict(theta=500000.0, scaling=kind, factor=factor, original_length=8192.0)
    few, many = (1.0, 4.0) if kind == "bands" else (1.0, 32.0)
    cos, sin = ctx.rotary_table(rot, first, count, magnitude=1.25, **args)
    w = _angles(rot, 500000.0, kind, factor, 8192.0, few, many)
    pos = (first + np.arange(count)).astype(np.longdouble)
    a = np.remainder(pos[:, None] * w, 2 * np.longdouble("3.14159265358979323846264338327950288"))
    tol = 1.25 * ((first + count) * 2.0 ** -50 + 4 * 2.0 ** -52)
    assert cos.shape == (count, rot // 2)
    assert np.abs(cos.cpu().numpy() - 1.25 * np.cos(a)).max() <= tol
    assert np.abs(sin.cpu().numpy() - 1.25 * np.sin(a)).max() <= tol


def test_far_positions_are_as_exact_as_near_ones():
    """Pair 0 turns by exactly one radian per position: the angle is the position, and no rounding of a frequency is in the way."""
    _, ctx = _ring(10)
    pi = "3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211707"
    from decimal import Decimal, getcontext
    getcontext().prec = 90
    for first in (0, 1 << 30, (1 << 50) - 4):
        cos, sin = ctx.rotary_table(8, first, 4)
        for i in range(4):
            r = float(Decimal(first + i) % (2 * Decimal(pi)))
            assert abs(float(cos[i, 0]) - math.cos(r)) < 2.0 ** -50 and abs(float(sin[i, 0]) - math.sin(r)) < 2.0 ** -50, (first, i)


def test_table_refusals():
    import torch
    _, ctx = _ring(10)
    for kw, code in [(dict(rot_dim=0), binding.ERR_ARG), (dict(rot_dim=7), binding.ERR_UNSUPPORTED), (dict(rot_dim=258), binding.ERR_UNSUPPORTED),
                     (dict(count=0), binding.ERR_ARG), (dict(theta=1.0), binding.ERR_ARG), (dict(theta=math.nan), binding.ERR_ARG),
                     (dict(scaling="linear", factor=0.5), binding.ERR_ARG), (dict(scaling="bands", factor=2.0), binding.ERR_ARG),
                     (dict(scaling="ramp", factor=2.0, original_length=100.0, turns_few=4.0, turns_many=2.0), binding.ERR_ARG),
                     (dict(scaling="base", factor=2.0, rot_dim=2), binding.ERR_UNSUPPORTED), (dict(magnitude=-1.0), binding.ERR_ARG),
                     (dict(magnitude=math.inf), binding.ERR_ARG), (dict(first=1 << 50, count=1), binding.ERR_UNSUPPORTED)]:
        a = dict(rot_dim=8, first=0, count=4) | kw
        rot, n = a["rot_dim"], max(a["count"], 1)
        out = (torch.zeros(a["count"], rot // 2, dtype=torch.float64, device="cuda"), torch.zeros(a["count"], rot // 2, dtype=torch.float64, device="cuda"))
        with pytest.raises(binding.CkksError) as e:
            if not out[0].numel():      # a null buffer for nothing to write
                f = binding.CRotaryScaling(0, rot, 1e4, 1.0, 0.0, 0.0, 0.0, 1.0)
                buf = torch.zeros(8, dtype=torch.float64, device="cuda")
                ctx._check(binding.load().ckks_rotary_table(ctx._h, C.byref(f), 0, a["count"], buf.data_ptr(), buf.data_ptr(), None))
            ctx.rotary_table(**a, out=out)
        assert e.value.code == code, kw


# ---- the rotation --------------------------------------------------------------------------------------------------------
CASES = [
    # log_n, level, dim, heads, inner, rot, layout, ciphertexts, rows, same position
    (10, 6, 16, 4, 8, 16, "half", 1, [0], False),                       # one rotation serves both channels of a pair
    (10, 5, 16, 2, 4, 16, "half", 3, [4, 0, 4], False),                 # copies; two ciphertexts share positions; a partial last digit
    (10, 2, 16, 4, 8, 16, "interleaved", 2, [1, 9], False),             # the smallest level
    (10, 4, 16, 2, 8, 10, "half", 2, [3, 3], True),                     # part of the head, one token in all slots
    (11, 6, 32, 8, 4, 32, "half", 2, [0, 4], False),                    # six digits
    (11, 5, 32, 8, 4, 22, "interleaved", 3, [0, 4, 8], False),          # five, two rotations
    (11, 6, 32, 8, 4, 22, "interleaved", 9, [0, 4, 8, 0, 4, 8, 1, 2, 3], False),     # six, two rotations of many ciphertexts
    (100, 7, 16, 4, 8, 12, "half", 2, [0, 1], True),                    # seven
    (100, 8, 16, 4, 8, 16, "half", 17, list(range(17)), False),         # eight
    (101, 20, 16, 4, 8, 16, "half", 2, [0, 8], False),                  # digits of ten limbs, ten special primes
    (101, 11, 16, 4, 8, 14, "half", 3, [2, 0, 2], False),
    (100, 9, 16, 4, 8, 16, "interleaved", 2, [0, 8], False),            # nine: the kernel for any number of them
    (11, 3, 2, 4, 128, 2, "interleaved", 1, [2], False),                # a head of one pair, three digits
    (12, 6, 32, 4, 16, 24, "interleaved", 4, [0, 16, 32, 48], False),
    (12, 3, 64, 32, 1, 64, "half", 19, list(range(19)), False),         # more ciphertexts than run side by side, one token each
    (12, 4, 32, 4, 16, 32, "half", 20, [16 * (i % 17) for i in range(20)], False),   # more sets of positions than are encoded at a time
    (13, 7, 64, 8, 8, 2, "half", 1, [0], False),                        # one digit; one pair rotated
    (15, 4, 64, 16, 16, 64, "half", 2, [0, 16], False),                 # side by side: the plaintexts' encoding next to the digits
    (15, 3, 64, 16, 8, 40, "interleaved", 9, [i % 4 for i in range(9)], True),       # one more than run side by side
    (16, 3, 128, 32, 8, 128, "half", 1, [3], True),
]


@pytest.mark.parametrize("log_n,level,dim,heads,inner,rot,layout,n,rows,same", CASES)
def test_rotation_bit_exact(log_n, level, dim, heads, inner, rot, layout, n, rows, same):
    from tests.gpu_util import host
    P, ctx = _ring(log_n)
    o, il = P.oracle, layout == "interleaved"
    rots = o.rotary_rotations(dim, heads, inner, rot, il)
    assert ctx.rotary_rotations(dim, heads, inner, rot, layout) == rots
    x, keys = _residues(P, 100 + log_n + dim, level, n), _keys(P, 7 + log_n, rots)
    cos, sin, dc, ds = _table(log_n + rot, max(rows) + (1 if same else inner), rot // 2)
    d = _dev_cts(x)
    out = ctx.rotary(d, rows, dc, ds, _dev_keys(keys), dim, heads, inner, rot_dim=rot, layout=layout, same_position=same)
    want = o.rotary(x, rows, cos, sin, keys, dim, heads, inner, rot, il, 0 if same else 1)
    for i in range(n):
        assert out[i].scale == SCALE and out[i].level == level - 1
        assert np.array_equal(host(out[i].data), want[i]), i
        assert np.array_equal(host(d[i].data), x[i])
    assert ctx.encode_range_flag() == binding.OK


@pytest.mark.parametrize("log_n", [10, 12])
def test_rotation_of_unaligned_buffers(log_n):
    """Ciphertexts and keys need only 8-byte alignment."""
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(log_n)
    o, level, a = P.oracle, 4, (16, 4, 8)
    rots = o.rotary_rotations(*a, 16, True)
    x, keys = _residues(P, 3, level, 2), _keys(P, 4, rots)
    cos, sin, dc, ds = _table(9, 16, 8)

    def odd(arr):
        buf = torch.empty(arr.size + 1, dtype=torch.uint64, device="cuda")
        t = buf[1:].view(arr.shape)
        t.view(torch.int64).copy_(torch.from_numpy(arr.view(np.int64)))
        assert t.data_ptr() % 16 == 8
        return t
    cts = [binding.Ciphertext(odd(c), SCALE) for c in x]
    ks = [binding.SwitchKey(odd(k), g) for g, k in keys.items()]
    outs = [binding.Ciphertext(odd(np.zeros((2, level - 1, P.N), dtype=np.uint64)), 0.0) for _ in x]
    want = o.rotary(x, [0, 8], cos, sin, keys, *a, 16, True)
    even = [binding.Ciphertext(torch.empty((2, level - 1, P.N), dtype=torch.uint64, device="cuda"), 0.0) for _ in x]
    for c, k, to in ((cts, ks, outs), (_dev_cts(x), ks, even), (cts, _dev_keys(keys), even), (_dev_cts(x), _dev_keys(keys), outs)):
        ctx.rotary(c, [0, 8], dc, ds, k, *a, layout="interleaved", outs=to)
        for i in range(2):
            assert np.array_equal(host(to[i].data), want[i])


def test_rotation_with_other_options_and_on_another_stream():
    """Options change no result; a call on a side stream is ordered by that stream alone."""
    import torch
    from tests.gpu_util import context, host
    P, ctx = _ring(12)
    o, a, rows = P.oracle, (32, 4, 16), [0, 16, 32]
    rots = o.rotary_rotations(*a, 32, False)
    x, keys = _residues(P, 13, 6, 3), _keys(P, 14, rots)
    cos, sin, dc, ds = _table(15, 48, 16)
    want = o.rotary(x, rows, cos, sin, keys, *a, 32, False)
    d, dk = _dev_cts(x), _dev_keys(keys)
    for option, value in ((binding.OPT_CONV_KERNEL, binding.CONV_TENSOR), (binding.OPT_NTT_FP_SHARE, 3)):
        old = ctx.get_option(option)
        ctx.set_option(option, value)
        try:
            out = ctx.rotary(d, rows, dc, ds, dk, *a)
        finally:
            ctx.set_option(option, old)
        assert all(np.array_equal(host(out[i].data), want[i]) for i in range(3))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(int(binding.load().ckks_rotary_workspace_bytes(ctx._h, C.byref(ctx._rotary_desc(*a, None, "half")), 6, 3)), dtype=torch.uint8, device="cuda")
    out = ctx.rotary(d, rows, dc, ds, dk, *a, ws=ws, stream=side)
    side.synchronize()
    assert all(np.array_equal(host(out[i].data), want[i]) for i in range(3))


@pytest.mark.parametrize("log_n,top", [(12, 5), (15, 4)])
def test_rotation_and_append_replay_from_a_graph(log_n, top):
    """Captured once, replayed on new inputs, tables and pages in the same buffers, an eager call between the replays."""
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(log_n)
    o, a = P.oracle, (32, 4, 16)
    rots = o.rotary_rotations(*a, 32, False)
    keys = _keys(P, 24, rots)
    dk = _dev_keys(keys)
    x, v, pk = (_residues(P, s, l, 1) for s, l in ((1, top), (2, top), (3, top - 1)))
    d, dv, dp = _dev_cts(x), _dev_cts(v), _dev_cts(pk)
    cos, sin, dc, ds = _table(3, 16, 16)
    outs = [[binding.Ciphertext(torch.empty_like(dp[0].data), 0.0)] for _ in range(3)]

    def step():
        ctx.rotary(d, [0], dc, ds, dk, *a, outs=outs[0], ws=ws)
        ctx.cache_append(d, dv, [0], [(3, 9, 0)], dp, dp, dc, ds, dk, *a, out_k=outs[1], out_v=outs[2], ws=ws)
    L, desc = binding.load(), ctx._rotary_desc(*a, None, "half")
    ws = torch.empty(max(L.ckks_rotary_workspace_bytes(ctx._h, C.byref(desc), top, 1), L.ckks_cache_append_workspace_bytes(ctx._h, C.byref(desc), top - 1, 1)),
                     dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (31, 32):
        x, v, pk = (_residues(P, seed + s, l, 1) for s, l in ((1, top), (2, top), (3, top - 1)))
        c2, s2, _, _ = _table(seed, 16, 16)
        for t, arr in ((d[0].data, x[0]), (dv[0].data, v[0]), (dp[0].data, pk[0])):
            t.view(torch.int64).copy_(torch.from_numpy(arr.view(np.int64)))
        dc.copy_(torch.from_numpy(c2)); ds.copy_(torch.from_numpy(s2))
        graph.replay()
        eager = ctx.rotary(d, [0], dc, ds, dk, *a)[0]
        want = o.rotary(x, [0], c2, s2, keys, *a, 32, False)[0]
        assert np.array_equal(host(outs[0][0].data), want) and np.array_equal(host(eager.data), want)
        assert np.array_equal(host(outs[1][0].data), o.append_keys(pk[0], x[0], c2, s2, keys, *a, 32, False, 3, 9, 0))
        assert np.array_equal(host(outs[2][0].data), o.append_values(pk[0], v[0], 16, 3, 9))


def test_calls_on_two_streams_of_one_context():
    """Each with a workspace of its own, nothing ordering one after the other, from one host thread and from two; with one lane and with several."""
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(15)
    o, a = P.oracle, (64, 16, 16)
    keys = _keys(P, 33, o.rotary_rotations(*a, 64, False))
    x, v, pk = _residues(P, 34, 4, 2), _residues(P, 35, 4, 2), _residues(P, 36, 3, 2)
    cos, sin, dc, ds = _table(37, 16, 32)
    d, dv, dp, dk = _dev_cts(x), _dev_cts(v), _dev_cts(pk), _dev_keys(keys)
    want_k = [o.append_keys(pk[i], x[i], cos, sin, keys, *a, 64, False, 2, 7, 1) for i in range(2)]
    want_v = [o.append_values(pk[i], v[i], 16, 2, 7) for i in range(2)]
    need = int(binding.load().ckks_cache_append_workspace_bytes(ctx._h, C.byref(ctx._rotary_desc(*a, None, "half")), 3, 1))
    for lanes in (1, 2, 4):
        old = ctx.get_option(binding.OPT_LANES)
        ctx.set_option(binding.OPT_LANES, lanes)
        try:
            streams = [torch.cuda.Stream() for _ in range(2)]
            wss = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
            outs = [[_dev_cts(np.zeros_like(pk[:1])) for _ in range(2)] for _ in range(2)]
            torch.cuda.synchronize()

            def call(i):
                ctx.cache_append([d[i]], [dv[i]], [0], [(2, 7, 1)], [dp[i]], [dp[i]], dc, ds, dk, *a, out_k=outs[i][0], out_v=outs[i][1], ws=wss[i], stream=streams[i])
            for _ in range(3):
                call(0), call(1)
            # and from two host threads
            threads = [threading.Thread(target=lambda i=i: [call(i) for _ in range(20)]) for i in range(2)]
            [t.start() for t in threads], [t.join() for t in threads]
            torch.cuda.synchronize()
        finally:
            ctx.set_option(binding.OPT_LANES, old)
        for i in range(2):
            assert np.array_equal(host(outs[i][0][0].data), want_k[i]) and np.array_equal(host(outs[i][1][0].data), want_v[i]), (lanes, i)


def _refused(code, f, *args, **kw):
    with pytest.raises(binding.CkksError) as e:
        f(*args, **kw)
    assert e.value.code == code, (e.value.code, kw)


def test_rotation_refusals():
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(10)
    a = (16, 4, 8)
    x = _dev_cts(_residues(P, 1, 4, 2))
    keys = _dev_keys(_keys(P, 2, P.oracle.rotary_rotations(*a, 16, True)))
    _, _, dc, ds = _table(2, 20, 8)
    run = lambda cts=x, rows=(0, 12), k=keys, c=dc, s=ds, shape=a, **kw: ctx.rotary(cts, list(rows), c, s, k, *shape, **({"layout": "interleaved"} | kw))  # noqa: E731
    launches = binding.kernel_launches()
    _refused(binding.ERR_ARG, run, rows=(0, 13))                                     # past the table
    _refused(binding.ERR_ARG, run, rows=(0, 0xffffffff))
    _refused(binding.ERR_NO_KEY, run, k=keys[:1])
    _refused(binding.ERR_NO_KEY, run, k=[])
    _refused(binding.ERR_UNSUPPORTED, run, shape=(16, 3, 8))                         # does not divide the slots
    _refused(binding.ERR_UNSUPPORTED, run, shape=(16, 64, 8))
    _refused(binding.ERR_UNSUPPORTED, ctx.rotary_rotations, 16, 4, 8, 7)
    _refused(binding.ERR_UNSUPPORTED, ctx.rotary_rotations, 16, 4, 8, 18)
    _refused(binding.ERR_ARG, ctx.rotary_rotations, 0, 4, 8, 2)
    _refused(binding.ERR_ARG, ctx.rotary_rotations, 16, 4, 8, 0)
    low = _dev_cts(_residues(P, 1, 1, 1))
    one = [binding.Ciphertext(torch.empty((2, 1, P.N), dtype=torch.uint64, device="cuda"), 0.0)]
    _refused(binding.ERR_LEVEL, run, cts=low, rows=(0,), outs=one)
    _refused(binding.ERR_LEVEL, run, cts=[x[0], _dev_cts(_residues(P, 1, 3, 1))[0]])
    big = torch.empty((2, 5, P.N), dtype=torch.uint64, device="cuda")
    inside = binding.Ciphertext(big.view(-1)[P.N: P.N + 6 * P.N].view(2, 3, P.N), 0.0)
    other = binding.Ciphertext(torch.empty((2, 3, P.N), dtype=torch.uint64, device="cuda"), 0.0)
    _refused(binding.ERR_ARG, run, outs=[inside, binding.Ciphertext(big.view(-1)[:6 * P.N].view(2, 3, P.N), 0.0)])       # results on each other
    _refused(binding.ERR_ARG, run, outs=[other, binding.Ciphertext(x[0].data.view(-1)[:6 * P.N].view(2, 3, P.N), 0.0)])  # a result on an input
    need = int(binding.load().ckks_rotary_workspace_bytes(ctx._h, C.byref(ctx._rotary_desc(*a, None, "interleaved")), 4, 2))
    _refused(binding.ERR_WORKSPACE, run, ws=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        run(c=dc.float())
    with pytest.raises(TypeError):
        run(s=ds[:, :4].contiguous())
    with pytest.raises(ValueError):
        run(rows=(0,))
    with pytest.raises(ValueError):
        run(outs=[other])
    assert binding.kernel_launches() == launches
    assert np.array_equal(host(x[0].data), _residues(P, 1, 4, 2)[0])


# ---- the cache -----------------------------------------------------------------------------------------------------------
APPENDS = [
    # log_n, page level, input level, dim, heads, inner, rot, layout, pages in the pool, page numbers, spans
    (10, 3, 4, 16, 4, 8, 16, "half", 1, [0], [(3, 4, 11)]),                                              # one token
    (10, 3, 6, 16, 2, 8, 12, "half", 5, [4, 1, 2], [(0, 8, 0), (0, 8, 8), (0, 3, 16)]),                  # a prompt; inputs of a higher level
    (101, 19, 20, 16, 4, 8, 16, "half", 2, [1], [(2, 6, 0)]),
    (10, 1, 2, 16, 4, 8, 16, "interleaved", 3, [2, 0], [(7, 8, 0), (1, 7, 5)]),                          # the lowest page level; copies of rows
    (11, 5, 6, 32, 8, 4, 32, "half", 2, [1], [(0, 1, 3)]),                                               # six digits
    (15, 3, 4, 64, 16, 16, 64, "half", 3, [1, 2], [(0, 1, 0), (3, 16, 5)]),                                 # keys and values side by side
    (15, 2, 4, 64, 16, 16, 30, "interleaved", 2, [1, 0], [(0, 16, 0), (2, 9, 0)]),                       # a whole page among them
    (12, 5, 6, 32, 4, 16, 20, "interleaved", 20, [19 - i for i in range(18)], [(i % 5, 16 - i % 3, i) for i in range(18)]),
]


@pytest.mark.parametrize("log_n,lp,lx,dim,heads,inner,rot,layout,npages,pages,spans", APPENDS)
@pytest.mark.parametrize("in_place", [False, True])
def test_append_bit_exact(log_n, lp, lx, dim, heads, inner, rot, layout, npages, pages, spans, in_place):
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(log_n)
    o, il, n = P.oracle, layout == "interleaved", len(pages)
    rots = o.rotary_rotations(dim, heads, inner, rot, il)
    keys = _keys(P, 70 + log_n, rots)
    xk, xv = _residues(P, 71, lx, n), _residues(P, 72, lx, n)
    pk, pv = _residues(P, 73, lp, npages), _residues(P, 74, lp, npages)
    rows = max(r + e - b for b, e, r in spans)
    cos, sin, dc, ds = _table(75, rows, rot // 2)
    dpk, dpv = _dev_cts(pk), _dev_cts(pv)
    ok, ov = (dpk, dpv) if in_place else tuple([binding.Ciphertext(torch.full_like(c.data.view(torch.int64), 5).view(torch.uint64), 0.0) for c in s] for s in (dpk, dpv))
    got_k, got_v = ctx.cache_append(_dev_cts(xk), _dev_cts(xv), pages, spans, dpk, dpv, dc, ds, _dev_keys(keys), dim, heads, inner, rot_dim=rot, layout=layout,
                                    out_k=None if in_place else ok, out_v=None if in_place else ov)
    assert got_k is ok and got_v is ov
    wk, wv = (pk.copy(), pv.copy()) if in_place else (np.full_like(pk, 5), np.full_like(pv, 5))       # pages that are not named stay as they are
    for i, (p, (b, e, r)) in enumerate(zip(pages, spans)):
        wk[p] = o.append_keys(pk[p], xk[i], cos, sin, keys, dim, heads, inner, rot, il, b, e, r)
        wv[p] = o.append_values(pv[p], xv[i], inner, b, e)
    for p in range(npages):
        assert np.array_equal(host(ok[p].data), wk[p]), p
        assert np.array_equal(host(ov[p].data), wv[p]), p
        if p in pages:
            assert ok[p].scale == SCALE and ov[p].scale == SCALE
        if not in_place:
            assert np.array_equal(host(dpk[p].data), pk[p])


def test_append_of_one_side_and_of_keys_without_positions():
    from tests.gpu_util import host
    P, ctx = _ring(10)
    o, a = P.oracle, (16, 2, 8)
    xk, pk = _residues(P, 81, 5, 2), _residues(P, 82, 4, 3)
    spans, pages = [(0, 8, 0), (2, 5, 0)], [2, 0]
    want = [o.append_values(pk[p], xk[i], 8, b, e) for i, (p, (b, e, _)) in enumerate(zip(pages, spans))]
    for side in ("k", "v"):
        d, pool = _dev_cts(xk), _dev_cts(pk)
        args = (d, None) if side == "k" else (None, d)
        pools = (pool, None) if side == "k" else (None, pool)
        ctx.cache_append(*args, pages, spans, *pools, None, None, [], *a)
        for i, p in enumerate(pages):
            assert np.array_equal(host(pool[p].data), want[i]), side
        assert np.array_equal(host(pool[1].data), pk[1])


def test_append_refusals():
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(10)
    a = (16, 4, 8)
    x, v = _dev_cts(_residues(P, 1, 4, 2)), _dev_cts(_residues(P, 2, 4, 2))
    pk, pv = _dev_cts(_residues(P, 3, 3, 3)), _dev_cts(_residues(P, 4, 3, 3))
    keys = _dev_keys(_keys(P, 2, P.oracle.rotary_rotations(*a, 16, False)))
    _, _, dc, ds = _table(2, 16, 8)

    def run(k=x, vv=v, pages=(0, 2), spans=((0, 8, 0), (0, 3, 8)), page_k=pk, page_v=pv, kk=keys, shape=a, c=dc, s=ds, **kw):
        return ctx.cache_append(k, vv, list(pages), list(spans), page_k, page_v, c, s, kk, *shape, **kw)
    launches = binding.kernel_launches()
    _refused(binding.ERR_ARG, run, pages=(0, 3))                                     # no such page
    _refused(binding.ERR_ARG, run, pages=(1, 1))                                     # one page twice
    _refused(binding.ERR_ARG, run, pages=(0, 0xffffffff))
    _refused(binding.ERR_ARG, run, spans=((0, 8, 0), (3, 3, 8)))                     # an empty span
    _refused(binding.ERR_ARG, run, spans=((0, 8, 0), (3, 9, 0)))                     # past the page
    _refused(binding.ERR_ARG, run, spans=((0, 8, 9), (0, 3, 8)))                     # past the table
    _refused(binding.ERR_ARG, run, k=None, vv=None)
    _refused(binding.ERR_NO_KEY, run, kk=[])
    _refused(binding.ERR_UNSUPPORTED, run, shape=(16, 4, 5), spans=((0, 5, 0), (0, 3, 8)))
    _refused(binding.ERR_LEVEL, run, k=_dev_cts(_residues(P, 1, 3, 2)))              # no limb to spare
    _refused(binding.ERR_LEVEL, run, page_v=_dev_cts(_residues(P, 4, 2, 3)))         # keys and values at other levels
    _refused(binding.ERR_SCALE, run, vv=_dev_cts(_residues(P, 2, 4, 2), SCALE * 1.001))
    _refused(binding.ERR_ARG, run, page_v=pk)                                        # keys' and values' pages in one place
    _refused(binding.ERR_ARG, run, page_k=[binding.Ciphertext(x[0].data.view(-1)[:6 * P.N].view(2, 3, P.N), SCALE)] + pk[1:])
    _refused(binding.ERR_ARG, run, out_k=[pk[2], pk[1], pk[0]])                      # pages in each other's place
    need = int(binding.load().ckks_cache_append_workspace_bytes(ctx._h, C.byref(ctx._rotary_desc(*a, None, "half")), 3, 2))
    _refused(binding.ERR_WORKSPACE, run, ws=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert binding.kernel_launches() == launches
    assert np.array_equal(host(pk[0].data), _residues(P, 3, 3, 3)[0])


# ---- masks and differences -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("log_n,level,tokens,heads,E,Ti", [(10, 6, 8, 2, 4, 2), (10, 2, 16, 1, 4, 1), (10, 3, 32, 4, 1, 1), (11, 4, 16, 4, 16, 8), (12, 5, 64, 4, 2, 2)])
def test_masks_and_differences_bit_exact(log_n, level, tokens, heads, E, Ti):
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(log_n)
    o, desc = P.oracle, AttnDesc(tokens, heads, E, 1, Ti)
    G = desc.groups()
    x, y = _residues(P, 90 + tokens, level, G), _residues(P, 91 + tokens, level, G)
    for kw in (dict(causal=True, key_begin=0, key_end=tokens), dict(causal=False, key_begin=1, key_end=tokens - 3), dict(causal=True, key_begin=0, key_end=0),
               dict(causal=True, key_begin=0, key_end=tokens, window=3, query_offset=2), dict(causal=False, key_begin=0, key_end=tokens, window=2, query_offset=-3),
               dict(causal=True, key_begin=0, key_end=tokens, query_offset=-tokens)):
        d = _dev_cts(x)
        out = ctx.attention_mask(d, tokens, heads, E, token_inner=Ti, **kw)
        want = o.attention_mask(desc, x, **kw)
        for g in range(G):
            assert out[g].scale == SCALE and np.array_equal(host(out[g].data), want[g]), (kw, g)
    w = inputs.rng(92, heads).uniform(-2, 2, heads)
    d, e = _dev_cts(x), _dev_cts(y)
    out = ctx.attention_difference(d, e, torch.from_numpy(w).cuda(), tokens, heads, E, token_inner=Ti)
    want = o.attention_difference(desc, x, y, w)
    for g in range(G):
        assert out[g].scale == SCALE and np.array_equal(host(out[g].data), want[g]), g
        assert np.array_equal(host(d[g].data), x[g]) and np.array_equal(host(e[g].data), y[g])


def test_shapes_whose_products_leave_64_bits_are_refused():
    _, ctx = _ring(10)
    for tokens, heads, block in ((1 << 31, 4, 1 << 31), (1 << 31, 1 << 31, 4), (4, 1 << 31, 4), (1 << 30, 1, 1 << 30)):
        _refused(binding.ERR_UNSUPPORTED, ctx.attention_rotations, tokens, heads, block)
    for shape in ((1 << 31, 1 << 31, 4, 2), (4, 1 << 31, 1 << 31, 2), (1 << 16, 1 << 16, 1, 2), (512, 512, 512, 512)):
        _refused(binding.ERR_UNSUPPORTED, ctx.rotary_rotations, *shape)


def test_many_groups_and_a_ciphertext_in_several_places():
    """512 groups of one score diagonal; one ciphertext as several inputs, and as both maps."""
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(10)
    o, desc = P.oracle, AttnDesc(512, 1, 1)
    x = _residues(P, 17, 2, 2)
    d = _dev_cts(x)
    out = ctx.attention_mask([d[g % 2] for g in range(512)], 512, 1, 1, causal=True, key_end=500)
    for g in (0, 1, 15, 16, 255, 511):
        want = o.rescale(o.mul_plain_acc(x[g % 2], o.encode(o.mask_slots(desc, g, True, 0, 500), float(P.q[1]), 2)))
        assert np.array_equal(host(out[g].data), want), g
    w = torch.tensor([1.0], dtype=torch.float64, device="cuda")
    out = ctx.attention_difference([d[0]] * 2, [d[0]] * 2, w, 2, 1, 1)
    want = o.attention_difference(AttnDesc(2, 1, 1), x[[0, 0]], x[[0, 0]], [1.0])
    assert np.array_equal(host(out[0].data), want[0]) and np.array_equal(host(out[1].data), want[1])


def test_weights_that_no_plaintext_holds_set_the_range_flag():
    import torch
    P, ctx = _ring(10)
    x = _dev_cts(_residues(P, 1, 3, 2))
    assert ctx.encode_range_flag() == binding.OK
    for bad in (math.nan, math.inf, 1e6):
        ctx.attention_difference(x, x, torch.tensor([0.5, bad], dtype=torch.float64, device="cuda"), 8, 2, 4)
        assert ctx.encode_range_flag() == binding.ERR_RANGE
        assert ctx.encode_range_flag() == binding.OK


def test_masks_and_differences_of_unaligned_buffers():
    import torch
    from tests.gpu_util import host
    P, ctx = _ring(10)
    o, desc, level = P.oracle, AttnDesc(8, 2, 4, 1, 2), 4
    x, y = _residues(P, 1, level, 2), _residues(P, 2, level, 2)

    def odd(shape, arr=None):
        t = torch.zeros(int(np.prod(shape)) + 1, dtype=torch.int64, device="cuda")[1:].view(shape)
        if arr is not None:
            t.copy_(torch.from_numpy(arr.view(np.int64)))
        return binding.Ciphertext(t.view(torch.uint64), SCALE)
    w = torch.tensor([0.5, -0.75], dtype=torch.float64, device="cuda")
    want = o.attention_difference(desc, x, y, w.cpu().numpy())
    for a, b, outs in (([odd(c.shape, c) for c in x], _dev_cts(y), None), (_dev_cts(x), [odd(c.shape, c) for c in y], None),
                       (_dev_cts(x), _dev_cts(y), [odd((2, level - 1, P.N)) for _ in x])):
        out = ctx.attention_difference(a, b, w, 8, 2, 4, token_inner=2, outs=outs)
        assert all(np.array_equal(host(out[g].data), want[g]) for g in range(2))


def test_mask_and_difference_refusals():
    import torch
    P, ctx = _ring(10)
    a = (8, 2, 4)
    x, y = _dev_cts(_residues(P, 1, 4, 2)), _dev_cts(_residues(P, 2, 4, 2))
    w = torch.ones(2, dtype=torch.float64, device="cuda")
    launches = binding.kernel_launches()
    mask = lambda cts=x, shape=a, **kw: ctx.attention_mask(cts, *shape, **kw)  # noqa: E731
    diff = lambda p=x, q=y, ww=w, shape=a, **kw: ctx.attention_difference(p, q, ww, *shape, **kw)  # noqa: E731
    _refused(binding.ERR_ARG, mask, key_begin=5, key_end=4)
    _refused(binding.ERR_ARG, mask, key_end=9)
    _refused(binding.ERR_ARG, mask, query_offset=1 << 32)
    _refused(binding.ERR_UNSUPPORTED, mask, token_inner=3)
    _refused(binding.ERR_UNSUPPORTED, mask, shape=(8, 3, 4))
    _refused(binding.ERR_LEVEL, mask, cts=_dev_cts(_residues(P, 1, 1, 2)), outs=[binding.Ciphertext(torch.empty((2, 1, P.N), dtype=torch.uint64, device="cuda"), 0.0) for _ in x])
    _refused(binding.ERR_LEVEL, diff, q=_dev_cts(_residues(P, 2, 3, 2)))
    _refused(binding.ERR_SCALE, diff, q=_dev_cts(_residues(P, 2, 4, 2), SCALE * 1.5))
    on = [binding.Ciphertext(c.data.view(-1)[:6 * P.N].view(2, 3, P.N), 0.0) for c in y]
    _refused(binding.ERR_ARG, diff, outs=on)
    _refused(binding.ERR_ARG, mask, cts=y, outs=on)
    _refused(binding.ERR_WORKSPACE, mask, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    _refused(binding.ERR_WORKSPACE, diff, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    for bad in (w.float(), w[:1], w.cpu()):
        with pytest.raises(TypeError):
            diff(ww=bad)
    with pytest.raises(ValueError):
        mask(cts=x[:1])
    assert binding.kernel_launches() == launches
    assert len(mask(key_begin=3, key_end=3)) == 2          # every key masked is a mask like any other


# ---- attention with masks, and of two maps ---------------------------------------------------------------------------------
EXP, RSQRT = [0.92, 0.38, 0.07], [1.9, -1.1, 0.25]


def _operands(P, seed, level, dim, sets, cl=None):
    return [_residues(P, seed + 10 * s, level, dim) for s in range(sets)]


@pytest.mark.parametrize("tokens,heads,E,Ti,Gb,rounds", [(8, 2, 4, 2, 1, 1), (8, 2, 8, 1, 1, 1), (16, 1, 4, 4, 2, 0)])
def test_masked_and_differential_attention_bit_exact(tokens, heads, E, Ti, Gb, rounds):
    import torch
    from tests.gpu_util import context, host, key_dev
    P, ctx = params(10, 13, 4, 4), context(10, 13, 4, 4)
    o, desc, level, dim, dim_v = P.oracle, AttnDesc(tokens, heads, E, Gb, Ti), 13, 2, 2
    tok, lad = o.attention_rotations(desc)
    keys = _keys(P, 5, tok + lad + o.attention_query_rotations(desc))
    rlk = _keys(P, 6, [0]).popitem()[1]
    q1, k1, q2, k2 = _operands(P, 200 + tokens, level, dim, 4)
    v = _residues(P, 7, level, dim_v)
    mask = dict(causal=True, key_begin=0, key_end=tokens - 1)
    poly = (0.5, rounds, EXP, [RSQRT] * rounds)
    dq1, dk1, dq2, dk2, dv = (_dev_cts(x) for x in (q1, k1, q2, k2, v))
    drlk, dkeys, shape = key_dev(rlk, 0), _dev_keys(keys), dict(tokens=tokens, heads=heads, diag_block=E, token_inner=Ti)
    opoly = (0.5, rounds, EXP, np.array([RSQRT] * rounds).reshape(rounds, 3))
    # Softmax alone
    S = _residues(P, 8, level - 1, desc.groups())
    want, sp = o.softmax_rows(desc, S, SCALE, *opoly, rlk, keys, mask)
    got = ctx.softmax_rows_masked(_dev_cts(S), *poly, drlk, dkeys, **shape, **mask)
    for g in range(desc.groups()):
        assert got[g].scale == sp and np.array_equal(host(got[g].data), want[g]), g
    # one map, masked
    want, so = o.attention_masked(desc, q1, k1, v, SCALE, SCALE, *opoly, rlk, keys, mask)
    got = ctx.attention_masked(dq1, dk1, dv, *poly, drlk, dkeys, **shape, group_baby=Gb, **mask)
    for d in range(dim_v):
        assert got[d].scale == so and np.array_equal(host(got[d].data), want[d]), d
    # two maps
    w = inputs.rng(9, heads).uniform(0.1, 0.9, heads)
    for masked in (False, True):
        want, so = o.attention_masked(desc, (q1, q2), (k1, k2), v, SCALE, SCALE, *opoly, rlk, keys, mask if masked else None, w)
        got = ctx.attention_differential(dq1, dk1, dq2, dk2, dv, torch.from_numpy(w).cuda(), *poly, drlk, dkeys, **shape, group_baby=Gb, masked=masked,
                                         **(mask if masked else {}))
        for d in range(dim_v):
            assert abs(got[d].scale - so) <= 2.0 ** -40 * so and np.array_equal(host(got[d].data), want[d]), (masked, d)
    for arr, t in ((q1, dq1), (k2, dk2), (v, dv)):
        assert all(np.array_equal(host(t[x].data), arr[x]) for x in range(2))


def test_masked_and_differential_attention_refusals():
    import torch
    from tests.gpu_util import context, key_dev
    P, ctx = params(10, 13, 4, 4), context(10, 13, 4, 4)
    o, desc, dim = P.oracle, AttnDesc(8, 2, 4), 2
    tok, lad = o.attention_rotations(desc)
    keys = _dev_keys(_keys(P, 5, tok + lad))
    rlk = key_dev(_keys(P, 6, [0]).popitem()[1], 0)
    q, k = _dev_cts(_residues(P, 1, 13, dim)), _dev_cts(_residues(P, 2, 13, dim))
    w = torch.ones(2, dtype=torch.float64, device="cuda")
    launches = binding.kernel_launches()

    def masked(qq=q, kk=k, vv=k, ks=keys, r=rlk, exp=EXP, rounds=1, **kw):
        return ctx.attention_masked(qq, kk, vv, 0.5, rounds, exp, [RSQRT] * rounds, r, ks, 8, 2, 4, **kw)

    def diff(q1=q, k1=k, q2=q, k2=k, vv=k, ks=keys, r=rlk, rounds=1, **kw):
        return ctx.attention_differential(q1, k1, q2, k2, vv, w, 0.5, rounds, EXP, [RSQRT] * rounds, r, ks, 8, 2, 4, **kw)
    S = _dev_cts(_residues(P, 4, 12, desc.groups()))
    for rounds in (3, 1 << 30, 0xffffffff):              # their levels leave 32 bits
        poly = binding.Context._softmax_desc(0.5, 1, EXP, [RSQRT])
        poly.rounds = rounds
        d = binding.CAttnDesc(8, 2, 4, 1, 1)
        ca = (binding.CCt * len(S))(*[ctx._ct2(x) for x in S])
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        for name, extra in (("ckks_softmax_rows", ()), ("ckks_softmax_rows_masked", (C.byref(binding.CAttnMask(1, 0, 8, 0, 0)),))):
            rc = getattr(binding.load(), name)(ctx._h, C.byref(d), C.byref(poly), *extra, ca, C.byref(binding.CEvk(rlk.data.data_ptr(), 0)), ctx._evks(keys), len(keys), ca,
                                               ws.data_ptr(), ws.numel(), None)
            assert rc == binding.ERR_LEVEL, (name, rounds, rc)
    for f in (masked, diff):
        _refused(binding.ERR_NO_KEY, f, ks=keys[:-1])
        _refused(binding.ERR_LEVEL, f, rounds=3)
        _refused(binding.ERR_LEVEL, f, vv=_dev_cts(_residues(P, 3, 2, dim)))
        _refused(binding.ERR_WORKSPACE, f, ws=torch.empty(4096, dtype=torch.uint8, device="cuda"))
    _refused(binding.ERR_LEVEL, diff, q2=_dev_cts(_residues(P, 3, 12, dim)))
    _refused(binding.ERR_SCALE, diff, q2=_dev_cts(_residues(P, 3, 13, dim), SCALE * 2))
    _refused(binding.ERR_ARG, masked, key_begin=3, key_end=2)
    _refused(binding.ERR_ARG, diff, masked=True, key_end=9)
    _refused(binding.ERR_RANGE, masked, exp=[0.1, 1e300, 0.1])
    assert binding.kernel_launches() == launches


# ---- together: what a decoder's layer does between its projections ----------------------------------------------------------------
def test_decoder_attention_from_cached_pages():
    """Two steps of a cache: a prompt of five tokens, then two more, appended to pages of four; keys and queries rotated to their positions;
    pages packed to operands; causal attention over the tokens there are.  Decrypted against the same pipeline in the clear."""
    from tests.gpu_util import context, ct_dev, host, key_dev
    P, ctx = params(10, 16, 4, 4), context(10, 16, 4, 4)
    o, cl = P.oracle, Client(P, 77)
    tokens, heads, dim, inner, E = 8, 8, 4, 4, 8
    pages, half = tokens // inner, dim // 2
    desc, n = AttnDesc(tokens, heads, E, 1, inner), P.n
    assert E * tokens * heads == n
    g = inputs.rng(78, 0)
    Q, K, V = (g.uniform(-0.7, 0.7, (tokens, heads, dim)) for _ in range(3))
    live = 7
    first = 1000                                          # the sequence's positions start far from 0
    cos, sin = ctx.rotary_table(dim, first, tokens)
    angle = (first + np.arange(tokens))[:, None] * 10000.0 ** (-2.0 * np.arange(half) / dim)
    Qr, Kr = rotate_clear(Q, angle, False, dim), rotate_clear(K, angle, False, dim)

    def shards(x, level):        # [pages][slots], copies behind one another
        flat = x.reshape(pages, inner, heads, dim).transpose(0, 3, 2, 1).reshape(pages, -1)
        return [ct_dev(cl.encrypt_slots(np.tile(z, n // z.size), SCALE, level), SCALE) for z in flat]
    a = (dim, heads, inner)
    assert dim * heads * inner * 4 == n
    rots = set(ctx.rotary_rotations(*a)) | set(ctx.attention_rotations(tokens, heads, E))
    for kind in (binding.ATTN_QUERY, binding.ATTN_KEY_VALUE):
        rots |= set(ctx.attention_pack_rotations(kind, dim, tokens, heads, E, inner))
    keys = [key_dev(cl.rotation_key(o.galois_element(r)), o.galois_element(r)) for r in sorted(rots)]
    rlk = key_dev(cl.relin_key(), 0)
    level = 16
    q, k, v = shards(Q, level), shards(K, level), shards(V, level)
    rq = ctx.rotary(q, [0, inner], cos, sin, keys, *a)
    pool_k, pool_v = ([ct_dev(np.zeros((2, level - 1, P.N), dtype=np.uint64), SCALE) for _ in range(3)] for _ in range(2))
    table = [2, 0]                                        # the sequence's pages in the pool
    ctx.cache_append(k, v, table, [(0, 4, 0), (0, 1, 4)], pool_k, pool_v, cos, sin, keys, *a)
    ctx.cache_append(k[1:], v[1:], table[1:], [(1, 3, 5)], pool_k, pool_v, cos, sin, keys, *a)
    for x, want, pool in ((0, Kr, pool_k), (1, V, pool_v)):
        for p in range(pages):
            z = want.reshape(pages, inner, heads, dim)[p].copy()
            z[max(0, live - p * inner):] = 0.0
            z = z.transpose(2, 1, 0).reshape(-1)
            assert np.abs(cl.decrypt_slots(host(pool[table[p]].data), SCALE) - np.tile(z, n // z.size)).max() < TOL
        assert not host(pool[1].data).any()
    shape = (tokens, heads, E, inner)
    oq = ctx.attention_pack(binding.ATTN_QUERY, rq, dim, keys, *shape)
    ok = ctx.attention_pack(binding.ATTN_KEY_VALUE, [pool_k[p] for p in table], dim, keys, *shape)
    ov = ctx.attention_pack(binding.ATTN_KEY_VALUE, [pool_v[p] for p in table], dim, keys, *shape)
    lk = ok[0].level
    oq = [binding.Ciphertext(x.data[:, :lk].contiguous(), x.scale) for x in oq]
    Kc = Kr.copy()
    Kc[live:] = 0.0                                       # empty slots of the cache
    S = np.einsum("ihd,jhd->hij", Qr, Kc)
    spread = 2 * np.abs(S).max()
    shift = spread / 2
    fit = lambda f, lo, hi, deg: np.polynomial.polynomial.polyfit(np.linspace(lo, hi, 200), f(np.linspace(lo, hi, 200)), deg)  # noqa: E731
    pv = np.polynomial.polynomial.polyval
    ce = fit(np.exp, -spread / 2, 0.0, 4) / 2.0 ** np.arange(5)
    seen = (np.arange(tokens)[None, :] <= np.arange(tokens)[:, None]) & (np.arange(tokens)[None, :] < live)
    u = pv(S - shift, ce) * seen
    s = (u * u).sum(2)
    cr = fit(lambda t: 1 / np.sqrt(t), s.min() / 1.3, s.max() * 1.3, 4)
    u = (pv(s, cr)[:, :, None] * u) ** 2
    want = np.einsum("hij,jhd->ihd", u, V)
    out = ctx.attention_masked(oq, ok, ov, shift, 1, ce, [cr], rlk, keys, tokens, heads, E, token_inner=inner, causal=True, key_end=live)
    _, i, h = inputs.attention_slot_index(tokens, heads, E, n, inner)
    for d in range(dim):
        got = cl.decrypt_slots(host(out[d].data), out[d].scale).real
        # a chain of about twelve products at scale 2^50, each adding slot errors below 2^-30, through polynomials of slope at most
        # about 30 on values below 4: 2^-30 * 12 * 30 * 4 < 2^-19
        assert np.abs(got - want[i, h, d]).max() < 2.0 ** -19, d
    assert ctx.encode_range_flag() == binding.OK and ctx.device_status() == binding.OK
