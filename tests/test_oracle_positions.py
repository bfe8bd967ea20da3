"""Pins for the checker's position rotation, cache pages, masks and differences of score maps: slot by slot against the same
formulas in the clear, on decrypted results."""
import numpy as np
import pytest

from oracle.ckks_oracle import AttnDesc
from paper_2609_12378_b200 import inputs
from tests.harness import Client, params
from tests.test_oracle_attention import _key_of

SCALE = 2.0 ** 50
# Slot errors of values of magnitude 1 at scale 2^50, N = 2^10: encryption and key switching leave coefficients of standard deviation
# below 2^8, rescaling and encoding below 2^4; a slot sums N of them with unit weights, so its deviation is below 2^8 sqrt(N) 2^-50 =
# 2^-37.  2^-30 is more than a hundred deviations.
TOL = 2.0 ** -30


def rotate_clear(x, angle, interleaved, rot):
    """x [tokens][heads][dim], angle [tokens][rot / 2]: the rotated channels, from the definition."""
    y = x.copy()
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c, s = np.cos(angle[:, j])[:, None], np.sin(angle[:, j])[:, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


def shard_slots(x, n):
    """x [token_inner][heads][dim] -> slots, copies behind one another."""
    v = np.ascontiguousarray(x.transpose(2, 1, 0)).reshape(-1)
    return np.tile(v, n // v.size)


@pytest.mark.parametrize("dim,heads,inner,rot,interleaved", [(16, 4, 8, 16, False), (16, 2, 4, 16, False), (16, 4, 8, 16, True), (16, 2, 8, 10, False),
                                                             (8, 4, 16, 6, True), (2, 4, 16, 2, True), (2, 4, 64, 2, False), (16, 4, 1, 12, False)])
def test_rotation_of_positions_decrypts_to_the_definition(dim, heads, inner, rot, interleaved):
    P = params(10, 5, 2, 3)
    o, cl = P.oracle, Client(P, 40 + dim + heads + rot)
    g = inputs.rng(41, dim * inner + rot)
    x = g.uniform(-1, 1, (inner, heads, dim))
    table = g.uniform(0, 6, (inner + 3, rot // 2))
    ct = cl.encrypt_slots(shard_slots(x, P.n), SCALE, 4)
    rots = o.rotary_rotations(dim, heads, inner, rot, interleaved)
    assert len(rots) == (1 if (2 if interleaved else rot) == dim else 2)
    keys = {o.galois_element(r): cl.rotation_key(o.galois_element(r)) for r in rots}
    for step in (0, 1):
        out = o.rotary(ct[None], [2], np.cos(table), np.sin(table), keys, dim, heads, inner, rot, interleaved, step)[0]
        want = rotate_clear(x, table[2 + step * np.arange(inner)], interleaved, rot)
        assert out.shape == (2, 3, P.N)
        assert np.abs(cl.decrypt_slots(out, SCALE) - shard_slots(want, P.n)).max() < TOL


@pytest.mark.parametrize("begin,end", [(0, 8), (3, 4), (5, 8), (0, 1)])
def test_appended_tokens_join_a_page_and_leave_its_other_slots(begin, end):
    P = params(10, 5, 2, 3)
    dim, heads, inner, rot = 16, 2, 8, 12
    o, cl = P.oracle, Client(P, 50 + begin + end)
    g = inputs.rng(51, begin * 8 + end)
    x, old = g.uniform(-1, 1, (inner, heads, dim)), g.uniform(-1, 1, (inner, heads, dim))
    old[begin:end] = 0.0
    angle = g.uniform(0, 6, (20, rot // 2))
    page, ct = cl.encrypt_slots(shard_slots(old, P.n), SCALE, 3), cl.encrypt_slots(shard_slots(x, P.n), SCALE, 5)
    keys = {o.galois_element(r): cl.rotation_key(o.galois_element(r)) for r in o.rotary_rotations(dim, heads, inner, rot, False)}
    k = o.append_keys(page, ct, np.cos(angle), np.sin(angle), keys, dim, heads, inner, rot, False, begin, end, 7)
    v = o.append_values(page, ct, inner, begin, end)
    pos = np.zeros((inner, rot // 2))
    pos[begin:end] = angle[7:7 + end - begin]
    want_k, want_v = old.copy(), old.copy()
    want_k[begin:end], want_v[begin:end] = rotate_clear(x, pos, False, rot)[begin:end], x[begin:end]
    assert np.abs(cl.decrypt_slots(k, SCALE) - shard_slots(want_k, P.n)).max() < TOL
    assert np.abs(cl.decrypt_slots(v, SCALE) - shard_slots(want_v, P.n)).max() < TOL


@pytest.mark.parametrize("tokens,heads,E,Ti", [(8, 2, 4, 2), (16, 1, 4, 1), (8, 4, 8, 8), (16, 2, 1, 1)])
@pytest.mark.parametrize("mask", [dict(causal=True, key_begin=0, key_end=8), dict(causal=False, key_begin=2, key_end=5), dict(causal=True, key_begin=0, key_end=0),
                                  dict(causal=True, key_begin=1, key_end=7, window=3, query_offset=-1), dict(causal=False, key_begin=0, key_end=8, query_offset=4, window=5)])
def test_masks_keep_the_tokens_that_a_query_sees(tokens, heads, E, Ti, mask):
    P = params(10, 5, 2, 3)
    o = P.oracle
    desc = AttnDesc(tokens, heads, E, 1, Ti)
    for g in range(desc.groups()):
        key, i, _ = _key_of(desc, P.n, g)
        assert np.array_equal(o.score_keys(desc, g), key)
        at = i + mask.get("query_offset", 0)
        want = [mask["key_begin"] <= k < mask["key_end"] and (not mask["causal"] or k <= a) and (not mask.get("window") or a - k < mask["window"])
                for k, a in zip(key, at)]
        assert np.array_equal(o.mask_slots(desc, g, **mask), np.array(want, dtype=float))


def test_masked_and_subtracted_maps_decrypt_to_the_definition():
    P = params(10, 5, 2, 3)
    o, cl = P.oracle, Client(P, 60)
    desc = AttnDesc(8, 4, 2, 1, 2)
    g = inputs.rng(61, 0)
    a, b = g.uniform(-1, 1, (desc.groups(), P.n)), g.uniform(-1, 1, (desc.groups(), P.n))
    A, B = (np.stack([cl.encrypt_slots(z, SCALE, 4) for z in m]) for m in (a, b))
    w = np.array([0.8, -0.25, 0.0, 1.5])
    _, _, h = o.score_places(desc)
    D = o.attention_difference(desc, A, B, w)
    mask = dict(causal=True, key_begin=0, key_end=7)
    M = o.attention_mask(desc, A, **mask)
    for x in range(desc.groups()):
        assert np.abs(cl.decrypt_slots(D[x], SCALE) - (a[x] - w[h] * b[x])).max() < 2 * TOL
        assert np.abs(cl.decrypt_slots(M[x], SCALE) - a[x] * o.mask_slots(desc, x, **mask)).max() < TOL
