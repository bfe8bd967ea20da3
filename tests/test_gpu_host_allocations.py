"""Host allocations that fail inside the attention's and the positions' entry points end as a status, whichever of them it is; the next call works.

The calls run in a process of their own, whose `operator new` fails once, at a chosen call from the library."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include <dlfcn.h>
#include <stdlib.h>
#include <string.h>
#include <new>
static thread_local long left = -1;
static thread_local bool hit = false;
extern "C" void fail_at(long k) { left = k; hit = false; }
extern "C" int failed() { left = -1; return hit; }
static void *get(size_t n, void *from) {
    if (left >= 0) {
        Dl_info i;
        if (dladdr(from, &i) && i.dli_fname && strstr(i.dli_fname, "libckks_b200") && left-- == 0) { hit = true; throw std::bad_alloc(); }
    }
    void *p = malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void *operator new(size_t n) { return get(n, __builtin_return_address(0)); }
void *operator new[](size_t n) { return get(n, __builtin_return_address(0)); }
void operator delete(void *p) noexcept { free(p); }
void operator delete[](void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }
void operator delete[](void *p, size_t) noexcept { free(p); }
"""

CHILD = r"""
import ctypes as C
import sys
import numpy as np
import torch
from oracle.ckks_oracle import AttnDesc
from paper_2609_12378_b200 import binding
from tests.gpu_util import context, key_dev
from tests.harness import params
from tests.test_gpu_positions import EXP, RSQRT, _dev_cts, _dev_keys, _keys, _residues, _table

shim = C.CDLL(sys.argv[1])
shim.fail_at.argtypes = [C.c_long]
L = binding.load()
armed = {"name": None}
for name in binding.EXPORTS:
    def wrap(f, name):
        def call(*a):
            if armed["name"] != name:
                return f(*a)
            armed["name"] = None
            shim.fail_at(armed["k"])
            rc = f(*a)
            armed["hit"], armed["rc"] = bool(shim.failed()), rc
            return rc
        return call
    setattr(L, name, wrap(getattr(L, name), name))


def words(x):
    if isinstance(x, (list, tuple)):
        return [w for y in x for w in words(y)]
    return [x.data.cpu().numpy().tobytes()] if isinstance(x, binding.Ciphertext) else [repr(x)]


def every_allocation(name, call, failed=binding.ERR_CUDA):
    want, k = words(call()), 0
    while True:
        armed.update(name=name, k=k, hit=False, rc=None)
        try:
            got = call()
        except Exception:
            got = None
        if not armed["hit"]:
            assert got is not None and words(got) == want, name
            break
        assert armed["rc"] == failed, (name, k, armed["rc"])
        if k % 8 == 0:
            assert words(call()) == want, (name, k)
        k += 1
        assert k < 5000
    print(name, k, flush=True)
    assert k > 0, name


P, ctx = params(10, 13, 4, 4), context(10, 13, 4, 4)
o, level = P.oracle, 13
desc = AttnDesc(8, 2, 4, 2, 2)
shape = dict(tokens=8, heads=2, diag_block=4)
pshape = (16, 4, 8, 2)
rots = set()
for gb in (1, 2):
    rots |= set(ctx.attention_rotations(8, 2, 4, gb))
for kind in (0, 1, 2):
    rots |= set(ctx.attention_pack_rotations(kind, 2, *pshape))
a = (16, 2, 8)
rots |= set(ctx.rotary_rotations(*a, layout="interleaved"))
keys = _dev_keys(_keys(P, 5, sorted(rots)))
rlk = key_dev(_keys(P, 6, [0]).popitem()[1], 0)
q, k2, v = (_dev_cts(_residues(P, s, level, 2)) for s in (1, 2, 3))
S, T = _dev_cts(_residues(P, 4, level - 1, 2)), _dev_cts(_residues(P, 5, level - 1, 2))
w = torch.tensor([0.5, 0.25], dtype=torch.float64, device="cuda")
poly = (0.5, 1, EXP, [RSQRT], rlk, keys)
mask = dict(causal=True, key_end=7)
host_only = [("ckks_attention_rotations", lambda: ctx.attention_rotations(8, 2, 4, 2)),
             ("ckks_attention_pack_rotations", lambda: ctx.attention_pack_rotations(1, 2, *pshape))]
for name, call in host_only:
    every_allocation(name, call)
d, pd, sd = binding.CAttnDesc(8, 2, 4, 2, 2), binding.CAttnDesc(16, 4, 8, 1, 2), binding.Context._softmax_desc(0.5, 1, EXP, [RSQRT])
B = C.byref
for name, args in (("ckks_attention_scores_workspace_bytes", (B(d), level, 2)), ("ckks_attention_values_workspace_bytes", (B(d), level)),
                   ("ckks_softmax_rows_workspace_bytes", (B(d), B(sd), level)), ("ckks_attention_workspace_bytes", (B(d), B(sd), level, 2)),
                   ("ckks_attention_mask_workspace_bytes", (B(d), level)), ("ckks_attention_difference_workspace_bytes", (B(d), level)),
                   ("ckks_attention_masked_workspace_bytes", (B(d), B(sd), level, 2)), ("ckks_attention_differential_workspace_bytes", (B(d), B(sd), level, 2)),
                   ("ckks_attention_pack_workspace_bytes", (B(pd), 1, level, 2))):
    every_allocation(name, lambda: getattr(L, name)(ctx._h, *args), failed=0)
for gb in (1, 2):
    every_allocation("ckks_attention_scores", lambda: ctx.attention_scores(q, k2, rlk, keys, **shape, group_baby=gb))
every_allocation("ckks_softmax_rows", lambda: ctx.softmax_rows(S, *poly, **shape))
every_allocation("ckks_softmax_rows_masked", lambda: ctx.softmax_rows_masked(S, *poly, **shape, **mask))
every_allocation("ckks_attention_values", lambda: ctx.attention_values(S, v, rlk, keys, **shape))
every_allocation("ckks_attention", lambda: ctx.attention(q, k2, v, *poly, **shape))
every_allocation("ckks_attention_masked", lambda: ctx.attention_masked(q, k2, v, *poly, **shape, **mask))
every_allocation("ckks_attention_differential", lambda: ctx.attention_differential(q, k2, k2, q, v, w, *poly, **shape, masked=True, **mask))
every_allocation("ckks_attention_mask", lambda: ctx.attention_mask(S, **shape, **mask))
every_allocation("ckks_attention_difference", lambda: ctx.attention_difference(S, T, w, **shape))
shards = _dev_cts(_residues(P, 7, level, 8))
for kind in (0, 1, 2):
    every_allocation("ckks_attention_pack", lambda: ctx.attention_pack(kind, shards[:2] if kind == 2 else shards, 2, keys, *pshape))
_, _, cos, sin = _table(8, 16, 8)
every_allocation("ckks_rotary", lambda: ctx.rotary(q, [0, 8], cos, sin, keys, *a, layout="interleaved"))
pk = _dev_cts(_residues(P, 9, level - 1, 2))
fresh = lambda: [binding.Ciphertext(torch.empty_like(c.data), 0.0) for c in pk]  # noqa: E731
every_allocation("ckks_cache_append", lambda: ctx.cache_append(q, v, [1, 0], [(0, 8, 0), (1, 3, 8)], pk, pk, cos, sin, keys, *a, layout="interleaved",
                                                               out_k=fresh(), out_v=fresh()))
assert ctx.device_status() == binding.OK
print("done")
"""


def test_failed_allocations_end_as_a_status(tmp_path):
    (tmp_path / "shim.cpp").write_text(SHIM)
    shim = str(tmp_path / "shim.so")
    subprocess.run(["g++", "-O1", "-fPIC", "-shared", "-o", shim, str(tmp_path / "shim.cpp"), "-ldl"], check=True)
    env = dict(os.environ, LD_PRELOAD=shim, PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", CHILD, shim], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("done"), (r.returncode, r.stdout[-1500:], r.stderr[-3000:])
