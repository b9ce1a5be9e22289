"""What the bindings' objects point at stays theirs when they are copied, or their weights'
owners are given others."""
import copy
import ctypes
import gc
import pickle

import pytest

from paper_2504_03651_amd import echo, norm, rope


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r))])
def test_a_copied_rope_points_at_its_own_description(how):
    """The library is handed the address of a copy's own echo_rope_t, which is that of the
    original only where they share it."""
    import torch
    first = rope.Rope(96, 32, layout="interleaved", theta=500000.0, device="cpu")
    r = how(first)
    assert r.at == ctypes.addressof(r.c)
    want = bytes(first.c)
    del first
    gc.collect()
    assert ctypes.string_at(r.at, ctypes.sizeof(rope.CRope)) == want
    assert torch.equal(r.frequencies, rope.Rope(96, 32, theta=500000.0, device="cpu").frequencies)


def test_a_norms_pointers_are_not_copied_away_from_their_tensors():
    n = norm.Norm(64, pre="rms")
    for how in (copy.deepcopy, pickle.dumps):
        with pytest.raises(ValueError, match="pointers"):
            how(n)
    again = copy.copy(n)
    assert again.c is n.c and again.at == ctypes.addressof(n.c)


@pytest.mark.gpu
def test_weights_stay_those_that_a_norm_was_made_with():
    """A parameter that is given another tensor lets go of its memory; the norm does not."""
    import torch
    H = 4096
    w = torch.nn.Parameter(torch.full((H,), 2.0, device="cuda"))
    n = norm.Norm(H, pre="rms", pre_weight=w, pre_eps=0.0)
    x, y = torch.ones(3, H, device="cuda"), torch.empty(3, H, device="cuda")
    w.data = torch.full((H,), 5.0, device="cuda")
    other = [torch.full((H,), 7.0, device="cuda") for _ in range(64)]   # the memory, had it been let go
    norm.join(n, None, x, y=y)
    assert (y == 2).all() and len(other) == 64


def _ropes():
    import torch
    r = rope.Rope(64, device="cpu")
    f = r.frequencies
    for freq, what in [(f.float(), "dtype"), (f[:16].clone(), "shape"), (f[None], "shape"),
                       (torch.stack([f, f], 1)[:, 0], "not contiguous")]:
        r.frequencies = freq
        yield r, what


def test_rotate_refuses_frequencies_of_another_type_or_length():
    """They are read as R / 2 numbers of 64 bits."""
    import torch
    for r, what in _ropes():
        with pytest.raises(echo.EchoError, match="rope.frequencies.*" + what):
            rope.rotate(r, torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64))


@pytest.mark.gpu
def test_rotate_refuses_them_on_the_gpu():
    import torch
    for r, what in _ropes():
        r.frequencies = r.frequencies.cuda() if what != "not contiguous" else torch.ones(32, 2, dtype=torch.float64,
                                                                                         device="cuda")[:, 0]
        with pytest.raises(echo.EchoError, match="rope.frequencies.*" + what):
            rope.rotate(r, torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, 64, device="cuda"))
