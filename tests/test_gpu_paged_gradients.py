"""Tensors whose gradients or tangents would be lost are refused."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
DEV = "cuda"


def _coop():
    import paper_2311_00591_amd as coop
    return coop


def _announce(label):
    print(f"[gpu case] paged: {label}", flush=True)
    sys.stdout.flush()


def _calls():
    """(function, its floating-point tensors, the others), for an e4m3 pool."""
    coop = _coop()
    rnd = lambda *s: torch.randn(s, device=DEV, dtype=BF16)
    pool = dict(k_cache=rnd(4, 16, 2, 64).to(E4M3), v_cache=rnd(4, 16, 2, 64).to(E4M3),
                k_scale=torch.ones(2, device=DEV), v_scale=torch.ones(2, device=DEV))
    rows = dict(k=rnd(3, 2, 64), v=rnd(3, 2, 64))
    attend = dict(table=torch.arange(4, dtype=torch.int32, device=DEV).view(1, 4),
                  lengths=torch.tensor([40], device=DEV), token_offsets=torch.tensor([0, 3], device=DEV))
    return [(coop.cache_write, {**rows, **pool}, dict(slots=torch.arange(3, device=DEV))),
            (coop.tree_attention, {"q": rnd(3, 4, 64), **rows, **pool, "out": rnd(3, 4, 64)}, attend)]


@pytest.mark.parametrize("which", [0, 1])
def test_gradients_are_refused(which):
    _announce(f"gradients refused, {which}")
    call, tensors, rest = _calls()[which]
    call(**tensors, **rest)
    for name, t in tensors.items():
        needs = t.detach().requires_grad_()
        with pytest.raises(ValueError, match=f"{name} requires gradients"):
            call(**{**tensors, name: needs}, **rest)
        with torch.no_grad():
            call(**{**tensors, name: needs}, **rest)
        call(**{**tensors, name: needs.detach()}, **rest)
    torch.cuda.synchronize()


@pytest.mark.parametrize("which", [0, 1])
def test_tangents_are_refused(which):
    from torch.autograd import forward_ad
    _announce(f"tangents refused, {which}")
    call, tensors, rest = _calls()[which]
    with forward_ad.dual_level():
        call(**tensors, **rest)
        for name in ("k", "v"):
            dual = forward_ad.make_dual(tensors[name], torch.ones_like(tensors[name]))
            with pytest.raises(ValueError, match=f"{name} carries a tangent"):
                call(**{**tensors, name: dual}, **rest)
    call(**tensors, **rest)
    torch.cuda.synchronize()
