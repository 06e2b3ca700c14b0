"""The gradients of norm and rotation write their workspace and the gains' gradients
and nothing beside them: called with exactly the bytes they ask for, between guards."""
import pytest
import torch

import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu

EPS = 1e-6


# grid, heads q / kv, D: few groups of tokens (workgroups along the heads), and more than 1,024
@pytest.mark.parametrize("grid,hq,hkv,D", [((1, 1, 3), 10, 2, 128), ((4, 9, 5), 12, 6, 64), ((12, 40, 40), 2, 1, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_workspace_and_gains_are_kept_to(grid, hq, hkv, D, dtype):
    p = vsa2.make_problem(1, hq, hkv, D, *grid, 4, 4, 4, 1, 1, 1,
                          vsa2.VSA2_BF16 if dtype == torch.bfloat16 else vsa2.VSA2_F32)
    t, h, w = (-(-m // 4) * 4 for m in grid)
    n, L = grid[0] * grid[1] * grid[2], t * h * w
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1, n, hq + 2 * hkv, D, generator=g, device="cuda").to(dtype)
    q, k, _ = (y.transpose(1, 2) for y in x.split([hq, hkv, hkv], 2))
    dy = [torch.randn(1, m, L, D, generator=g, device="cuda").to(dtype) for m in (hq, hkv, hkv)]
    gains = [1 + 0.1 * torch.randn(D, generator=g, device="cuda") for _ in range(2)]
    want = vsa2.qk_norm_rope_bwd(p, *dy, q=q, k=k, q_gain=gains[0], k_gain=gains[1], eps=EPS)

    st, need = vsa2.vsa2_qk_norm_rope_workspace(p)
    assert st == 0 and need > 0
    ws = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")      # NaN wherever it is read unwritten
    dgain = torch.full((2, D + 512), 7.0, device="cuda")
    dx = torch.empty_like(x)

    def rows(t):
        return vsa2.vsa2_rows(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))

    out = [y.transpose(1, 2) for y in dx.split([hq, hkv, hkv], 2)]
    at = [row[256:256 + D] for row in dgain]
    st = vsa2.vsa2_qk_norm_rope_bwd(p, None, EPS, rows(q), gains[0].data_ptr(), dy[0].data_ptr(), rows(out[0]),
                                    at[0].data_ptr(), rows(k), gains[1].data_ptr(), dy[1].data_ptr(), rows(out[1]),
                                    at[1].data_ptr(), dy[2].data_ptr(), rows(out[2]), ws.data_ptr() + 256, need,
                                    torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    for a, b in zip((*out, *at), want):
        assert torch.equal(a, b)
    assert (ws[:256] == 0xff).all() and (ws[256 + need:] == 0xff).all()
    assert (dgain[:, :256] == 7).all() and (dgain[:, 256 + D:] == 7).all()
