"""The workspace of gla_norm_bwd: partial sums for dweight and dbias, no more than the call writes, and none where they are not wanted."""
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla


def test_sizes():
    # two fp32 sums for each weight from 4096 waves at most, of which those of a work-group make one where it stays with a head
    for B, H, T, D in ((1, 1 << 17, 1, 32), (2, 1 << 17, 3, 8192), (1, 70000, 5, 64), (1, 40000, 1, 128)):
        assert gla.gla_norm_bwd_workspace_bytes(B, H, T, D) <= 2 * 4 * H * D + 255
    for D in (16, 64, 100, 128, 384, 1152, 2048, 4096, 8192):
        for B, H, T in ((1, 1, 100000), (2, 16, 4096), (3, 7, 50), (64, 1, 1)):
            n = gla.gla_norm_bwd_workspace_bytes(B, H, T, D)
            assert 2 * 4 * H * D <= n <= 2 * 4 * D * max(H * B * T, 256) + 255


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B,H,T,D", [(1, 3, 700, 20), (2, 16, 300, 64), (1, 5, 2000, 72), (1, 1, 3000, 160), (1, 2, 500, 1152), (1, 1, 90, 2048), (1, 1, 90, 8192),
                                     (1, 3000, 2, 32)])
def test_what_a_call_writes(B, H, T, D, layout):
    """What lies behind the workspace is left alone; without weights so is the workspace, and the other gradients are the same."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gen = torch.Generator(device="cuda:0").manual_seed(D)
    lead = (B, H, T) if layout == 0 else (B, T, H)
    x, do, r = (torch.randn(*lead, D, generator=gen, device="cuda:0").to(torch.bfloat16) for _ in range(3))
    n = gla.gla_norm_bwd_workspace_bytes(B, H, T, D)
    room = torch.full((n + 4096,), 99, dtype=torch.uint8, device="cuda:0")
    first = gla.gla_norm_bwd(x, do, r_pre=r, layout=layout, want_d_weight=True, workspace=room[:n])
    own = gla.gla_norm_bwd(x, do, r_pre=r, layout=layout, want_d_weight=True)
    torch.cuda.synchronize()
    assert bool((room[n:] == 99).all()) and not bool((room[:n] == 99).all())
    assert all(torch.equal(a, b) for a, b in zip(first, own))
    room.fill_(99)
    second = gla.gla_norm_bwd(x, do, r_pre=r, layout=layout, want_d_weight=False, workspace=room[:n])
    torch.cuda.synchronize()
    assert bool((room == 99).all()) and second[2:] == (None, None)
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
