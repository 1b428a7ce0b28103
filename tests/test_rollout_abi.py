"""The rollout entry points without a GPU: prototypes, refusals, the oracle's
own pins."""

import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle.kl import KIND_CE, KIND_FORWARD, kl_ref
from oracle.rollout import distill_ref, top_ref, verify_probs_ref
from paper_2606_12370_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "specverify_rollout.h")
FAKE = 0x10000  # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def prototypes():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return {m.group(1): [a.strip() for a in m.group(2).split(",")] for m in
            re.finditer(r"\b(?:spec_status|size_t)\s+(spec_\w+)\s*\(([^;]*?)\)\s*;", src, re.S)}


def test_exports_and_prototypes(lib):
    p = prototypes()
    assert set(p) == {"spec_top_logits", "spec_top_logits_workspace_size", "spec_distill_loss_fwd_bwd",
                      "spec_distill_workspace_size", "spec_verify_probs", "spec_verify_probs_workspace_size"}
    for name, args in p.items():
        assert len(getattr(lib, name).argtypes) == len(args), name
        for a, t in zip(args, getattr(lib, name).argtypes):
            want = ctypes.c_void_p if "*" in a else {"int64_t": ctypes.c_int64, "float": ctypes.c_float,
                                                     "size_t": ctypes.c_size_t}.get(a.split()[0], ctypes.c_int)
            assert t is want, (name, a)
    assert int(re.search(r"#define SPEC_MAX_LIST (\d+)", open(HEADER).read()).group(1)) == binding.SPEC_MAX_LIST


def test_workspace_sizes(lib):
    top, dis, pro = (lib.spec_top_logits_workspace_size, lib.spec_distill_workspace_size,
                     lib.spec_verify_probs_workspace_size)
    for bad in ((0, 1, 9, 4, 1), (1, 0, 9, 4, 1), (1, 1, 0, 4, 1), (1, 1, 9, 0, 1), (1, 1, 9, 257, 1), (1, 1, 9, 4, 2),
                (1, 1, (1 << 31) - 1, 4, 1), (1 << 24, 1, 9, 4, 1)):
        assert top(*bad) == 0 and dis(*bad) == 0, bad
    assert dis(1, 9, 9, 4, 1) == 0 and top(1, 9, 9, 4, 1) > 0
    for bad in ((0, 1, 9, 1), (1, -1, 9, 1), (1, 9, 9, 1), (1, 1, 0, 1), (1, 1, 9, 3), (1 << 24, 0, 9, 0)):
        assert pro(*bad) == 0, bad
    assert pro(1, 0, 1, 0) > 0
    for f, a in ((top, (4, 3, 151936, 64, 1)), (dis, (4096, 3, 151936, 64, 1)), (pro, (256, 3, 151936, 0))):
        assert f(*a) % 256 == 0 and f(*a) >= 256


TOP = dict(z=FAKE, sn=300, sk=100, dtype=1, N=4, K=3, V=100, M=8, temp=None, ts=1.0, ids=FAKE, val=FAKE, lz=None,
           ws=FAKE, wsb=1 << 30, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=5), 2), (dict(M=257), 2), (dict(M=0), 1), (dict(N=0), 1), (dict(K=0), 1), (dict(V=0), 1),
    (dict(N=1 << 24), 1), (dict(z=None), 1), (dict(ids=None), 1), (dict(val=None), 1), (dict(sn=-1), 1),
    (dict(sk=-1), 1), (dict(sn=1 << 62), 1), (dict(ts=0.0), 1), (dict(ts=float("nan")), 1),
    (dict(ts=float("inf")), 1), (dict(ws=None), 4), (dict(wsb=8), 4), (dict(ws=FAKE + 8), 1)])
def test_top_argument_errors(lib, kw, status):
    assert lib.spec_top_logits(*{**TOP, **kw}.values()) == status


DISTILL = dict(z=FAKE, sn=300, sk=100, dtype=1, N=4, K=3, V=100, ids=FAKE, val=FAKE, ln=24, lk=8, M=8, lz=None, on=3,
               ok=1, T=1.0, kind=0, scale=1.0, loss=FAKE, ps=None, grad=FAKE, gd=0, ws=FAKE, wsb=1 << 30, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), 2), (dict(K=9), 2), (dict(M=257), 2), (dict(gd=2), 2), (dict(dtype=0, gd=1), 2), (dict(N=0), 1),
    (dict(K=0), 1), (dict(V=-5), 1), (dict(M=0), 1), (dict(z=None), 1), (dict(ids=None), 1), (dict(val=None), 1),
    (dict(loss=None), 1), (dict(sn=-1), 1), (dict(lk=-1), 1), (dict(lz=FAKE, on=-1), 1), (dict(ln=1 << 61), 1),
    (dict(lz=FAKE, on=1 << 61), 1), (dict(T=0.0), 1), (dict(T=float("nan")), 1), (dict(kind=2), 1), (dict(kind=-1), 1),
    (dict(scale=float("inf")), 1), (dict(ws=None), 4), (dict(wsb=64), 4), (dict(ws=FAKE + 4), 1)])
def test_distill_argument_errors(lib, kw, status):
    assert lib.spec_distill_loss_fwd_bwd(*{**DISTILL, **kw}.values()) == status


PROBS = dict(p=FAKE, psb=400, psk=100, q=FAKE, qsb=300, qsk=100, dtype=0, B=4, K=3, V=100, ids=FAKE, ua=FAKE, us=FAKE,
             lens=None, acc=FAKE, em=FAKE, ov=None, ws=FAKE, wsb=1 << 30, stream=None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), 2), (dict(K=9), 2), (dict(K=-1), 1), (dict(B=0), 1), (dict(V=0), 1), (dict(p=None), 1),
    (dict(us=None), 1), (dict(ids=None), 1), (dict(ua=None), 1), (dict(acc=None), 1), (dict(em=None), 1),
    (dict(psk=-1), 1), (dict(qsb=-1), 1), (dict(psb=1 << 61), 1), (dict(qsk=1 << 61), 1), (dict(ws=None), 4),
    (dict(wsb=16), 4), (dict(ws=FAKE + 4), 1)])
def test_probs_argument_errors(lib, kw, status):
    assert lib.spec_verify_probs(*{**PROBS, **kw}.values()) == status


def test_binding_refusals():
    z = torch.zeros((2, 3, 10))
    with pytest.raises(ValueError, match="GPU"):
        binding.top_logits(z, 4)
    with pytest.raises(ValueError, match="GPU"):
        binding.distill_loss_fwd_bwd(z, torch.zeros((2, 3, 4), dtype=torch.int32), torch.zeros((2, 3, 4)))
    with pytest.raises(ValueError, match="GPU"):
        binding.verify_probs(z, None, torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, 2), torch.zeros(2))
    with pytest.raises(ValueError):
        binding.top_logits(torch.zeros((2, 10, 3)).transpose(1, 2), 4)
    with pytest.raises(ValueError):
        binding.top_logits(torch.zeros(10), 4)


CLIENT = r"""
#include <stdio.h>
#include "specverify_rollout.h"
int main(void) {
  printf("%d %d\n", SPEC_MAX_LIST, spec_version());
  printf("%zu\n", spec_verify_probs_workspace_size(256, 3, 151936, SPEC_F32));
  printf("%d\n", (int)spec_top_logits(NULL, 0, 0, SPEC_BF16, 1, 1, 8, 4, NULL, 1.0f, NULL, NULL, NULL, NULL, 0, NULL));
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_c99_client(lib, tmp_path):
    (tmp_path / "c.c").write_text(CLIENT)
    libdir = os.path.dirname(os.path.abspath(lib._name))
    r = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I" + os.path.join(ROOT, "include"),
                        str(tmp_path / "c.c"), "-o", str(tmp_path / "c"), "-L" + libdir, "-lspecverify",
                        "-Wl,-rpath," + libdir], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    out = subprocess.run([str(tmp_path / "c")], capture_output=True, text=True, timeout=120).stdout.split()
    assert out == ["256", str(lib.spec_version()), str(lib.spec_verify_probs_workspace_size(256, 3, 151936, 0)), "1"]


# ---- the oracle's pins ----------------------------------------------------------------

def test_oracle_top():
    z = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0], [-np.inf] * 5, [0.0, np.nan, 0, 0, 0]])
    r = top_ref(z, 4, 2.0)
    assert r["ids"].tolist() == [[1, 2, 4, 0], [-1] * 4, [-1] * 4]
    assert abs(r["logz"][0] - np.log(np.exp([0.5, 1.5, 1.5, 1.0]).sum())) < 1e-15
    assert r["logz"][1] == -np.inf and np.isnan(r["logz"][2])


@pytest.mark.parametrize("kind,code", [("forward", KIND_FORWARD), ("ce", KIND_CE)])
def test_oracle_distill_is_kl_for_whole_lists(kind, code):
    rng = np.random.default_rng(1)
    t, z = rng.standard_normal((2, 3, 2, 17)) * 2
    ids = np.broadcast_to(rng.permutation(17), (3, 2, 17))
    full = distill_ref(z, ids, np.take_along_axis(t, ids, -1), None, 0.7, kind, 1.3)
    ref = kl_ref(t, z, 0.7, code, 1.3)
    assert np.allclose(full["per_step"], ref["per_step"], rtol=1e-12)
    assert np.allclose(full["grad"], ref["grad"], rtol=1e-10, atol=1e-15)


@pytest.mark.parametrize("kind", ["forward", "ce"])
@pytest.mark.parametrize("tail", [True, False])
def test_oracle_distill_gradient(kind, tail):
    rng = np.random.default_rng(2)
    t, z = rng.standard_normal((2, 1, 2, 12))
    ids = np.argsort(-t, -1)[..., :5]
    val = np.take_along_axis(t, ids, -1)
    lz = np.log(np.exp(t / 0.5).sum(-1)) if tail else None
    g = distill_ref(z, ids, val, lz, 0.5, kind)["grad"]
    for n, k, v in np.ndindex(z.shape):
        a, b = z.copy(), z.copy()
        a[n, k, v] += 1e-6
        b[n, k, v] -= 1e-6
        d = (distill_ref(a, ids, val, lz, 0.5, kind)["loss"] - distill_ref(b, ids, val, lz, 0.5, kind)["loss"]) / 2e-6
        assert abs(d - g[n, k, v]) < 1e-8


def test_oracle_probs_frequencies():
    """The emitted token is distributed as p_n, whatever the draft."""
    rng = np.random.default_rng(3)
    V, R = 6, 40000
    p, q = rng.dirichlet(np.ones(V), size=2)
    ids = rng.choice(V, size=(R, 1), p=q)
    out = verify_probs_ref(np.broadcast_to(p, (R, 2, V)), np.broadcast_to(q, (R, 1, V)), ids, rng.random((R, 1)),
                           rng.random(R))
    f = np.bincount(out["emitted"][:, 0], minlength=V) / R
    assert np.all(np.abs(f - p) < 5 * np.sqrt(p / R))
    assert abs((out["accept_len"] == 1).mean() - np.minimum(p, q).sum()) < 0.02
    hot = verify_probs_ref(np.broadcast_to(p, (R, 2, V)), None, np.full((R, 1), 2), rng.random((R, 1)), rng.random(R))
    f = np.bincount(hot["emitted"][:, 0], minlength=V) / R
    assert np.all(np.abs(f - p) < 5 * np.sqrt(p / R))
