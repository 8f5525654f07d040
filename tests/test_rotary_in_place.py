"""What dropit_rotary refuses beside its types: places that belong to two values, gradients that would be lost.  Needs no GPU."""
import pytest
import torch

import paper_2202_13808_b200 as dropit
from paper_2202_13808_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def _call(q, k, device="cpu", **kw):
    length = q.shape[-3]
    return dropit.dropit_rotary(q, k, torch.zeros(length, 1, dtype=torch.int32, device=device), dropit.dropit_rotary_plan(q.shape[-1], (q.shape[-1],)), **kw)


def _buffer(*shape):
    return torch.zeros(*shape)


D = 16
SHARING = {
    "the same tensor": lambda b: (b.view(2, 8, 4, D), b.view(2, 8, 4, D)),
    "tokens": lambda b: (b.view(1, 16, 4, D)[:, :10], b.view(1, 16, 4, D)[:, 6:]),
    "one token": lambda b: (b.view(1, 16, 4, D)[:, :8], b.view(1, 16, 4, D)[:, 7:15]),
    "sequences": lambda b: (b.view(4, 4, 4, D)[:3], b.view(4, 4, 4, D)[1:]),
    "heads": lambda b: (b.view(2, 8, 4, D)[:, :, :3], b.view(2, 8, 4, D)[:, :, 2:]),
    "half a head": lambda b: (b.as_strided((2, 8, 2, D), (512, 64, 16, 1)), b.as_strided((2, 8, 2, D), (512, 64, 16, 1), 24)),
    "heads in front of the tokens": lambda b: (b.view(2, 4, 8, D)[:, :, :5].transpose(1, 2), b.view(2, 4, 8, D)[:, :, 3:].transpose(1, 2)),
    "a head and a token": lambda b: (b.view(1, 16, 4, D)[:, :15, 3:], b.as_strided((1, 15, 1, D), (1024, 64, 64, 1), 48 + 64)),
    "other strides": lambda b: (b.view(2, 8, 4, D), b.view(2, 4, 8, D).transpose(1, 2)),
}
APART = {
    "one projection": lambda b: (b.view(2, 4, 2, 4, D)[:, :, 0], b.view(2, 4, 2, 4, D)[:, :, 1]),
    "groups of heads": lambda b: (b.view(2, 8, 4, D)[:, :, :3], b.view(2, 8, 4, D)[:, :, 3:]),
    "heads by turns": lambda b: (b.view(2, 8, 4, D)[:, :, ::2], b.view(2, 8, 4, D)[:, :, 1::2]),
    "tokens by turns": lambda b: (b.view(2, 8, 4, D)[:, ::2], b.view(2, 8, 4, D)[:, 1::2]),
    "halves of a sequence": lambda b: (b.view(2, 8, 4, D)[:, :4], b.view(2, 8, 4, D)[:, 4:]),
    "sequences": lambda b: (b.view(4, 4, 4, D)[:2], b.view(4, 4, 4, D)[2:]),
    "heads in front of the tokens": lambda b: (b.view(2, 4, 8, D)[:, :3].transpose(1, 2), b.view(2, 4, 8, D)[:, 3:].transpose(1, 2)),
    "channels": lambda b: (b.view(2, 8, 2, 2 * D)[..., :D], b.view(2, 8, 2, 2 * D)[..., D:]),
    "one sequence": lambda b: (b.view(16, 4, D)[:, :1], b.view(16, 4, D)[:, 1:]),
    "memory of their own": lambda b: (b.view(2, 8, 4, D), torch.zeros_like(b).view(2, 8, 4, D)),
    "other strides, other places": lambda b: (b[:512].view(2, 4, 4, D), b[512:].view(2, 4, 4, D).transpose(1, 2)),
    "an empty one": lambda b: (b.view(2, 8, 4, D), b.view(2, 8, 4, D)[:, :, :0]),
}


@pytest.mark.parametrize("how", sorted(SHARING))
def test_queries_and_keys_that_share_values(how):
    for q, k in (SHARING[how](_buffer(1024)), SHARING[how](_buffer(1024))[::-1]):
        with pytest.raises(ValueError, match="share"):
            _call(q, k, in_place=True)


@pytest.mark.parametrize("how", sorted(APART))
def test_queries_and_keys_that_do_not(how):
    for q, k in (APART[how](_buffer(1024)), APART[how](_buffer(1024))[::-1]):
        with pytest.raises(ValueError, match="CUDA tensor"):       # every other check has passed
            _call(q, k, in_place=True)


def test_every_pair_of_views_against_the_places_they_name():
    """Strided views of one small buffer, drawn at random: refused if and only if they name a place twice (views of other strides that lie between one
    another may be refused although they do not)."""
    rng = torch.Generator().manual_seed(1)
    pick = lambda *c: c[int(torch.randint(len(c), (1,), generator=rng))]
    refused = taken = 0
    for _ in range(3000):
        b = _buffer(600)
        sizes = (pick(1, 2), pick(1, 2, 3), pick(1, 2, 3), 4)
        strides = (pick(0, 96, 128, 200), pick(4, 8, 16, 24, 48), pick(4, 6, 8, 12, 24), 1)
        same = pick(True, True, False)
        other = strides if same else (pick(96, 128, 200), pick(4, 8, 24, 48), pick(4, 8, 12), 1)
        q = b.as_strided(sizes, strides, pick(0, 4, 8, 10))
        k = b.as_strided((sizes[0], sizes[1], pick(1, 2), 4), other, pick(0, 4, 8, 12, 24, 96, 99, 300))
        at = torch.arange(600)
        places = [at.as_strided(t.shape, t.stride(), t.storage_offset()).flatten().tolist() for t in (q, k)]
        clash = any(len(set(p)) < len(p) for p in places) or bool(set(places[0]) & set(places[1]))
        with pytest.raises(ValueError) as e:
            _call(q, k, in_place=True)
        told = "CUDA tensor" not in str(e.value)
        assert told or not clash, (q.shape, q.stride(), q.storage_offset(), k.shape, k.stride(), k.storage_offset())
        refused, taken = refused + told, taken + (not told)
    assert refused > 300 and taken > 300


def test_a_view_that_meets_itself():
    for size, stride in (((1, 4, 2, D), (0, 8, 64, 1)), ((1, 4, 2, D), (0, 64, 8, 1)), ((2, 4, 2, D), (64, 64, 16, 1)), ((2, 4, 2, D), (0, 32, 16, 1))):
        with pytest.raises(ValueError, match="place"):
            _call(_buffer(1024).as_strided(size, stride), None, in_place=True)
        with pytest.raises(ValueError, match="place"):
            _call(_buffer(*size), _buffer(1024).as_strided(size, stride), in_place=True)


def test_gradients_that_would_be_lost():
    q, k, at = torch.zeros(1, 4, 2, D, requires_grad=True), torch.zeros(1, 4, 2, D), torch.zeros(4, 1)
    for a, b in ((q, k), (k, q), (q * 1, None)):
        with pytest.raises(RuntimeError, match="gradient"):
            _call(a, b, in_place=True)
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):
        _call(q, k, in_place=True)
    with pytest.raises(ValueError, match="CUDA tensor"):
        _call(q, k)
    # fp32 positions are values that a model could learn, but the rotation has no gradient for them
    rot, at = dropit.DropITRotary(D, (D,)), at.requires_grad_(True)
    for f in (lambda: rot(q, k, at), lambda: rot(k, None, at)):
        with pytest.raises(RuntimeError, match="positions"):
            f()
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):
        rot(q, k, at)


@pytest.mark.gpu
@pytest.mark.parametrize("how", sorted(APART))
def test_in_place_is_what_the_copy_is(cuda_device, how):
    b = torch.randn(1024, generator=torch.Generator(device=cuda_device).manual_seed(1), device=cuda_device)
    q, k = APART[how](b)
    at = torch.arange(q.shape[-3], device=cuda_device).unsqueeze(1)
    plan = dropit.dropit_rotary_plan(D, (D,))
    before = b.clone()
    want = dropit.dropit_rotary(q, k, at, plan)
    assert torch.equal(b, before)
    got = dropit.dropit_rotary(q, k, at, plan, in_place=True)
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and got[0].data_ptr() == q.data_ptr()
