"""linattn_rotary on more tokens than one dimension of a launch holds."""
import numpy as np
import pytest

from oracle import decay_oracle as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode,n", [("f32", (1 << 27) + 9), ("bf16", (1 << 24) + 9)])
@pytest.mark.parametrize("kind,dims", [("adjacent", (128,)), ("halves", (44, 42, 42))])
def test_more_workgroups_than_a_grid_s_first_dimension(mode, n, kind, dims):
    """In place, 64 GiB in fp32: the rows at both ends and where the launch goes on in another dimension."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    d, dt = 128, torch.float32 if mode == "f32" else torch.bfloat16
    if torch.cuda.mem_get_info()[0] < n * d * (4 if mode == "f32" else 2) + (4 << 30):
        pytest.skip("needs the memory for its tensor")
    q = torch.zeros((1, 1, n, d), dtype=dt, device="cuda")
    marks = [0, 1, (1 << 23) - 1, 1 << 23, (1 << 24) - 1, 1 << 24, n - 2, n - 1] + ([(1 << 26) + 3, (1 << 27) - 1, 1 << 27] if mode == "f32" else [])
    at = torch.tensor(marks, device="cuda")
    q[0, 0, at] = 1.0
    grid = None if len(dims) == 1 else (1, 30, 52)
    got, _ = G.rotary(q, dims=dims, grid=grid, pairs=kind, q_out=q)
    assert got is q
    pos = np.array(marks)[:, None] if grid is None else np.stack((np.array(marks) // 1560, np.array(marks) // 52 % 30, np.array(marks) % 52), 1)
    want, err = O.rotary(np.ones((len(marks), d)), pos, dims, kind, 10000.0, False)
    u = 2.0 ** -24 if mode == "f32" else 2.0 ** -8
    assert (np.abs(G.to_host_f64(q[0, 0, at]) - want) <= err + u * np.abs(want)).all()
    q[0, 0, at] = 0.0
    assert not any(part.any() for part in q[0, 0].split(1 << 24))
    del q, got
    torch.cuda.empty_cache()
