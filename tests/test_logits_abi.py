"""The calls on rows of logits refuse bad arguments before they touch the GPU (no kernel is launched in this file)."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1708_02983_amd", "libeasgd_hip.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libeasgd_hip.so not built (run __graft_entry__.build())")

EINVAL, EWORKSPACE, ERANGE = -1, -3, -4
FAKE = 0x10000        # never dereferenced: every call below must fail validation first, or has no rows


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


def test_declared_and_exported(hip):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "easgd.h")).read(), flags=re.S)
    for name in ("easgd_top_logits", "easgd_distill_loss", "easgd_distill_grad", "easgd_distill", "easgd_sample_tokens", "easgd_grad_distill"):
        assert re.search(rf"\b{name}\s*\(", text) and hasattr(hip.lib(), name) and callable(getattr(hip, name))
    assert re.search(r"EASGD_MAX_TOP\s+256\b", text) and hip.MAX_TOP == 256


class Call:
    """A call with good arguments, of which each test replaces some."""

    def __init__(self, lib, name):
        self.lib, self.name = lib, name
        rows = dict(logits=FAKE, dtype=0, rows=2, V=100, ld=100)
        teacher = dict(rows, indices=FAKE, values=FAKE, teacher_lse=None, k=5, labels=None, temperature=1.0, hard=0.0)
        scratch = dict(workspace=FAKE, workspace_bytes=1 << 40)
        self.args = {
            "easgd_top_logits": dict(rows, k=5, temperature=1.0, values=FAKE, indices=FAKE, lse=FAKE, **scratch),
            "easgd_distill_loss": dict(teacher, loss=FAKE, state=FAKE, **scratch),
            "easgd_distill_grad": dict(teacher, state=FAKE, dloss=FAKE, scale=1.0, dlogits=FAKE, dld=100),
            "easgd_distill": dict(teacher, scale=1.0, loss=FAKE, dlogits=FAKE, dld=100, **scratch),
            "easgd_sample_tokens": dict(rows, u=FAKE, temperature=FAKE, top_k=FAKE, top_p=FAKE, min_p=FAKE, tokens=FAKE, logprob=FAKE, **scratch),
        }[name]

    def __call__(self, **changes):
        assert set(changes) <= set(self.args)
        return getattr(self.lib, self.name)(*{**self.args, **changes}.values(), None)

    def has(self, *names):
        return all(n in self.args for n in names)


NAMES = ("easgd_top_logits", "easgd_distill_loss", "easgd_distill_grad", "easgd_distill", "easgd_sample_tokens")


@pytest.mark.parametrize("name", NAMES)
def test_refusals(hip, name):
    call = Call(hip.lib(), name)
    last = lambda: hip.lib().easgd_last_error().decode()
    bad = [dict(logits=None), dict(logits=FAKE + 2), dict(dtype=3), dict(dtype=-1), dict(V=0), dict(V=-5), dict(ld=99), dict(ld=0), dict(logits=FAKE + 1, dtype=1)]
    if call.has("k"):
        bad += [dict(k=0), dict(k=257), dict(k=-1)]
    if call.has("k", "temperature"):
        bad += [dict(temperature=t) for t in (0.0, -1.0, 1e-7, 1e7, float("inf"), float("nan"))]
    if call.has("hard"):
        bad += [dict(hard=h, labels=FAKE) for h in (-0.1, 1.1, float("nan"))] + [dict(hard=0.5, labels=None)]
        bad += [dict(indices=None), dict(values=None), dict(teacher_lse=FAKE + 2), dict(labels=FAKE + 1)]
    if call.has("scale"):
        bad += [dict(scale=float("inf")), dict(scale=float("nan")), dict(dlogits=None), dict(dld=99), dict(dlogits=FAKE + 2)]
    if name == "easgd_distill_grad":
        bad += [dict(state=None), dict(dloss=FAKE + 2)]
    for out in ("values", "indices", "loss", "u", "tokens"):
        if out in call.args:
            bad += [{out: None}]
    for other in ("values", "indices", "lse", "loss", "state", "u", "temperature", "top_k", "top_p", "min_p", "tokens", "logprob"):
        if isinstance(call.args.get(other), int):
            bad += [{other: FAKE + 2}]
    for changes in bad:
        assert call(**changes) == EINVAL, changes
        assert last().startswith(name + ":"), (changes, last())
    far = [dict(V=(1 << 20) + 1, ld=1 << 21), dict(rows=1 << 22), dict(ld=1 << 60)]
    if call.has("dld"):
        far += [dict(V=(1 << 20) + 1, ld=1 << 21, dld=1 << 21), dict(dld=1 << 60)]
    for changes in far:
        assert call(**changes) == ERANGE, changes
    # no rows: nothing to do, whatever the pointers are
    assert call(rows=0) == 0 and call(rows=0, logits=None) == 0
    assert call(rows=0, V=0) == EINVAL


@pytest.mark.parametrize("name", [n for n in NAMES if n != "easgd_distill_grad"])
def test_workspaces(hip, name):
    """Where a call asks for a workspace it has to be there, aligned and large enough; sizes are multiples of 256 bytes."""
    lib = hip.lib()
    call = Call(lib, name)
    asked = 0
    for rows, V in ((1, 10), (1, 1 << 20), (3, 50001), (16, 262144), (256, 131072), (4096, 131072), (100000, 5)):
        if name == "easgd_sample_tokens":
            need = lib.easgd_sample_tokens_workspace_bytes(rows, V)
        elif name == "easgd_top_logits":
            need = lib.easgd_top_logits_workspace_bytes(rows, V, 5)
        else:
            need = lib.easgd_distill_workspace_bytes(rows, V, 5)
        assert need % 256 == 0 and need <= 1 << 30
        if need:
            asked += 1
            wide = dict(dld=V) if call.has("dld") else {}
            for changes in (dict(workspace=None), dict(workspace=FAKE + 128), dict(workspace_bytes=need - 1)):
                assert call(rows=rows, V=V, ld=V, **wide, **changes) == EWORKSPACE, (rows, V, changes)
                assert name in lib.easgd_last_error().decode()


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu(hip):
    z = torch.randn(3, 10)
    idx, val = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)
    with pytest.raises(TypeError, match="logits must be a CUDA/HIP tensor"):
        hip.easgd_top_logits(z, 2)
    with pytest.raises(TypeError, match="logits must be a CUDA/HIP tensor"):
        hip.easgd_distill(z, idx, val)
    with pytest.raises(TypeError, match="logits must be a CUDA/HIP tensor"):
        hip.easgd_sample_tokens(z, torch.rand(3))


def test_the_network_call_refuses_too(hip):
    lib = hip.lib()
    dims = (ctypes.c_int * 2)(784, 10)
    good = dict(dims=dims, n_layers=1, W=FAKE, ld=7852, X=FAKE, indices=FAKE, values=FAKE, teacher_lse=None, k=3, labels=None, P=1, b=1,
                temperature=1.0, hard=0.0, G=FAKE, loss=None, workspace=FAKE, workspace_bytes=1 << 30)
    call = lambda **changes: lib.easgd_grad_distill(*{**good, **changes}.values(), None)
    for changes in (dict(W=None), dict(X=None), dict(G=None), dict(indices=None), dict(values=None), dict(k=0), dict(k=257), dict(temperature=0.0),
                    dict(hard=0.5), dict(hard=2.0, labels=FAKE), dict(n_layers=0), dict(P=0), dict(b=0), dict(ld=7000), dict(indices=FAKE + 2), dict(X=FAKE + 4),
                    dict(dims=(ctypes.c_int * 2)(784, 1025), ld=1 << 20)):
        assert call(**changes) == EINVAL, changes
        assert lib.easgd_last_error().decode().startswith("easgd_grad_distill:"), changes
    assert call(workspace=None) == EWORKSPACE and call(workspace_bytes=16) == EWORKSPACE
