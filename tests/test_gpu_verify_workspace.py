"""The verification's workspace holds what the call's own rows need: none of a
draft's predictions where there are none."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


@pytest.mark.parametrize("tau", [1.0, 0.0])
def test_without_a_draft(P, tau):
    import torch
    T, V = 12, 50000
    size = lambda rows: P.lib().puro_verify_drafts_workspace_size(3, T, rows, V)      # noqa: E731
    assert size(0) < size(T - 3)
    g = torch.Generator(device="cuda").manual_seed(1)
    z, u = torch.randn(T, V, generator=g, device="cuda"), torch.rand(T, generator=g, device="cuda")
    ids = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    off = torch.tensor([0, 4, 8, T], dtype=torch.int32, device="cuda")
    room = torch.full((size(0) + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    got = P.verify_drafts(z, None, ids, off, u, u[:3].contiguous(), temperature=tau, ws=room[:size(0)])
    want = P.verify_drafts(z, None, ids, off, u, u[:3].contiguous(), temperature=tau)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (room[size(0):] == 0x5A).all().item()
    # a draft of fewer rows than the target's takes as much as those need
    zq = torch.randn(T - 3, V, generator=g, device="cuda")
    room = torch.full((size(T - 3) + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    got = P.verify_drafts(z, zq, ids, off, u, u[:3].contiguous(), temperature=tau, ws=room[:size(T - 3)])
    want = P.verify_drafts(z, zq, ids, off, u, u[:3].contiguous(), temperature=tau)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (room[size(T - 3):] == 0x5A).all().item()
