"""The calls on given tokens, norms and AdamW rounds refuse bad arguments before they touch the GPU (no kernel is launched in this file)."""
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
NAN, INF = float("nan"), float("inf")
NAMES = ("easgd_score_tokens", "easgd_score_tokens_grad", "easgd_token_loss", "easgd_grad_norms", "adamw_round", "adamw_round_8bit", "easgd_grad_token_loss")


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


def test_declared_and_exported(hip):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "easgd.h")).read(), flags=re.S)
    for name in NAMES:
        assert re.search(rf"\b{name}\s*\(", text) and hasattr(hip.lib(), name)
    assert hip.version() >= 514 and hip.ADAMW_BLOCK == 256


class Call:
    """A call with good arguments, of which each test replaces some."""

    def __init__(self, lib, name):
        self.lib, self.name = lib, name
        rows = dict(logits=FAKE, dtype=0, rows=2, V=100, ld=100)
        scratch = dict(workspace=FAKE, workspace_bytes=1 << 40)
        replicas = dict(G=FAKE, dtype=0, Wc=FAKE, P=2, N=1000, ld=1000)
        rule = dict(ends=FAKE, rates=FAKE, decays=FAKE, tensors=3, clip=FAKE, eta=0.1, eta_at=None, rho=0.1, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01,
                    step=1, step_at=None)
        self.args = {
            "easgd_score_tokens": dict(rows, tokens=FAKE, temperature=1.0, logprob=FAKE, entropy=FAKE, rank=FAKE, k=5, top_logprob=FAKE, top_indices=FAKE,
                                       state=FAKE, **scratch),
            "easgd_score_tokens_grad": dict(rows, tokens=FAKE, temperature=1.0, state=FAKE, dlogprob=FAKE, dentropy=FAKE, scale=1.0, dlogits=FAKE << 8, dld=100),
            "easgd_token_loss": dict(rows, tokens=FAKE, weight=FAKE, bonus=0.1, temperature=1.0, scale=1.0, loss=FAKE, logprob=FAKE, entropy=FAKE,
                                     dlogits=FAKE << 8, dld=100, **scratch),
            "easgd_grad_norms": dict(G=FAKE, dtype=0, P=2, N=1000, ld=1000, max_norm=1.0, norm=FAKE, clip=FAKE, **scratch),
            "adamw_round": dict(W=FAKE, M=FAKE, S=FAKE, **replicas, **rule),
            "adamw_round_8bit": dict(W=FAKE, M=FAKE, S=FAKE, M_scale=FAKE, S_scale=FAKE, **replicas, **rule, seed=0),
        }[name]

    def __call__(self, **changes):
        assert set(changes) <= set(self.args), changes
        return getattr(self.lib, self.name)(*{**self.args, **changes}.values(), None)


def refused(hip, name, bad, code=EINVAL):
    call = Call(hip.lib(), name)
    for changes in bad:
        assert call(**changes) == code, changes
        assert hip.lib().easgd_last_error().decode().startswith(name + ":"), (changes, hip.lib().easgd_last_error())


ROWS = [dict(logits=None), dict(logits=FAKE + 2), dict(dtype=3), dict(dtype=-1), dict(V=0), dict(V=-5), dict(ld=99), dict(ld=0), dict(logits=FAKE + 1, dtype=1),
        *(dict(temperature=t) for t in (0.0, -1.0, 1e-7, 1e7, INF, NAN)), dict(tokens=FAKE + 2)]
FAR = [dict(V=(1 << 20) + 1, ld=1 << 21), dict(rows=1 << 22), dict(ld=1 << 60)]


def test_score(hip):
    name = "easgd_score_tokens"
    refused(hip, name, ROWS + [dict(k=-1), dict(k=257), dict(tokens=None), dict(tokens=None, rank=None), dict(tokens=None, logprob=None), dict(top_logprob=None),
                               dict(top_indices=None), dict(logprob=FAKE + 2), dict(entropy=FAKE + 1), dict(rank=FAKE + 2), dict(top_logprob=FAKE + 2),
                               dict(top_indices=FAKE + 1), dict(state=FAKE + 8),
                               dict(k=0, logprob=None, entropy=None, rank=None, state=None)])
    refused(hip, name, FAR, ERANGE)
    call = Call(hip.lib(), name)
    assert call(rows=0) == 0 and call(rows=0, logits=None, tokens=FAKE) == 0 and call(rows=0, V=0) == EINVAL


def test_score_grad(hip):
    name = "easgd_score_tokens_grad"
    refused(hip, name, ROWS + [dict(state=None), dict(state=FAKE + 8), dict(dlogits=None), dict(dlogprob=None, dentropy=None), dict(tokens=None), dict(dlogprob=FAKE + 2),
                               dict(dentropy=FAKE + 2), dict(scale=INF), dict(scale=NAN), dict(dld=99), dict(dlogits=(FAKE << 8) + 2), dict(dlogits=FAKE),
                               dict(dlogits=FAKE + 400)])
    refused(hip, name, FAR[:2] + [dict(ld=1 << 60, dld=1 << 60), dict(dld=1 << 60)], ERANGE)
    assert Call(hip.lib(), name)(rows=0) == 0


def test_token_loss(hip):
    name = "easgd_token_loss"
    refused(hip, name, ROWS + [dict(tokens=None), dict(weight=FAKE + 2), dict(bonus=INF), dict(bonus=NAN), dict(scale=INF), dict(loss=None), dict(loss=FAKE + 2),
                               dict(logprob=FAKE + 1), dict(entropy=FAKE + 2), dict(dlogits=None), dict(dld=99), dict(dlogits=(FAKE << 8) + 2), dict(dlogits=FAKE)])
    refused(hip, name, FAR[:2] + [dict(ld=1 << 60, dld=1 << 60), dict(dld=1 << 60)], ERANGE)
    assert Call(hip.lib(), name)(rows=0) == 0


def test_norms(hip):
    name = "easgd_grad_norms"
    refused(hip, name, [dict(G=None), dict(G=FAKE + 2), dict(G=FAKE + 1, dtype=2), dict(dtype=7), dict(P=0), dict(N=0), dict(ld=999), dict(max_norm=0.0), dict(max_norm=-1.0),
                        dict(max_norm=NAN), dict(norm=None), dict(norm=FAKE + 2), dict(clip=FAKE + 1)])
    refused(hip, name, [dict(N=(1 << 34) + 1, ld=1 << 35), dict(P=65536), dict(ld=1 << 60)], ERANGE)


@pytest.mark.parametrize("name", ["adamw_round", "adamw_round_8bit"])
def test_adamw(hip, name):
    bad = [dict(W=None), dict(M=None), dict(S=None), dict(G=None), dict(W=FAKE + 2), dict(G=FAKE + 2), dict(G=FAKE + 1, dtype=1), dict(dtype=3), dict(Wc=FAKE + 1),
           dict(P=0), dict(P=-1), dict(N=0), dict(ld=999), dict(tensors=-1), dict(ends=None), dict(rates=None), dict(decays=None), dict(ends=FAKE + 4), dict(rates=FAKE + 2),
           dict(decays=FAKE + 1), dict(clip=FAKE + 2), dict(eta_at=FAKE + 2), dict(step_at=FAKE + 4), dict(step=0), dict(step=-3), dict(Wc=None),
           *(dict(beta1=b) for b in (-0.1, 1.0, NAN)), *(dict(beta2=b) for b in (-0.1, 1.0, NAN)), *(dict(eps=e) for e in (0.0, -1e-8, 1e-31, 1e31, INF, NAN)),
           dict(eta=INF), dict(eta=NAN), dict(rho=NAN), dict(decay=INF)]
    if name == "adamw_round":
        bad += [dict(M=FAKE + 2), dict(S=FAKE + 2)]
    else:
        bad += [dict(M_scale=None), dict(S_scale=None), dict(M_scale=FAKE + 2), dict(S_scale=FAKE + 1)]
    refused(hip, name, bad)
    refused(hip, name, [dict(N=(1 << 34) + 1, ld=1 << 35), dict(P=65536), dict(ld=1 << 60)], ERANGE)


def test_workspaces(hip):
    lib, asked = hip.lib(), 0
    for rows, V in ((1, 10), (1, 1 << 20), (3, 50001), (16, 262144), (256, 131072), (4096, 131072), (100000, 5)):
        for k in (0, 5, 256):
            need = lib.easgd_score_tokens_workspace_bytes(rows, V, k)
            assert need % 256 == 0 and need <= 1 << 30
            if need:
                asked += 1
                for changes in (dict(workspace=None), dict(workspace=FAKE + 128), dict(workspace_bytes=need - 1)):
                    assert Call(lib, "easgd_score_tokens")(rows=rows, V=V, ld=V, k=k, **changes) == EWORKSPACE
        need = lib.easgd_token_loss_workspace_bytes(rows, V)
        assert need % 256 == 0
        if need:
            asked += 1
            assert Call(lib, "easgd_token_loss")(rows=rows, V=V, ld=V, dld=V, dlogits=1 << 50, workspace_bytes=need - 1) == EWORKSPACE
    for P, N in ((1, 1), (3, 1 << 20), (16, 1863690), (65535, 100)):
        need = lib.easgd_grad_norms_workspace_bytes(P, N)
        assert need % 256 == 0 and need <= 1 << 24
        if need:
            asked += 1
            assert Call(lib, "easgd_grad_norms")(P=P, N=N, ld=N, workspace_bytes=need - 1) == EWORKSPACE
    assert asked > 12
    assert lib.easgd_score_tokens_workspace_bytes(5, 100, 257) == 0 and lib.easgd_grad_norms_workspace_bytes(0, 5) == 0


def test_the_network_call(hip):
    lib = hip.lib()
    dims = (ctypes.c_int * 2)(784, 10)
    good = dict(dims=dims, n_layers=1, W=FAKE, ld=7852, X=FAKE, tokens=FAKE, weight=None, P=1, b=1, bonus=0.0, temperature=1.0, G=FAKE, loss=None, logprob=None,
                entropy=None, workspace=FAKE, workspace_bytes=1 << 30)
    call = lambda **changes: lib.easgd_grad_token_loss(*{**good, **changes}.values(), None)
    for changes in (dict(W=None), dict(X=None), dict(G=None), dict(tokens=None), dict(tokens=FAKE + 2), dict(weight=FAKE + 2), dict(bonus=NAN), dict(temperature=0.0),
                    dict(logprob=FAKE + 2), dict(entropy=FAKE + 1), dict(n_layers=0), dict(P=0), dict(b=0), dict(ld=7000), dict(X=FAKE + 4),
                    dict(dims=(ctypes.c_int * 2)(784, 1025), ld=1 << 20)):
        assert call(**changes) == EINVAL, changes
        assert lib.easgd_last_error().decode().startswith("easgd_grad_token_loss:"), changes
    assert call(workspace=None) == EWORKSPACE and call(workspace_bytes=16) == EWORKSPACE


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu(hip):
    z, t = torch.randn(3, 10), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: hip.easgd_score_tokens(z, t), lambda: hip.easgd_score_tokens_grad(z, t, z), lambda: hip.easgd_token_loss(z, t)):
        with pytest.raises(TypeError, match="logits must be a CUDA/HIP tensor"):
            call()
    with pytest.raises(TypeError, match="G must be a CUDA/HIP tensor"):
        hip.easgd_grad_norms(z)
    with pytest.raises(TypeError, match="W must be a CUDA/HIP tensor"):
        hip.adamw_round(z, z, z, z, 1, 0.1)
