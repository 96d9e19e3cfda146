"""README's step of questions over a DevicePool, from the fork to the release in one graph: the eager step's bits."""

import os
import re

import pytest
import torch

from test_gpu_pages import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def test_the_step_is_captured_as_the_readme_says(ap):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        block, = [x for x in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "DevicePool" in x]
    at, end = block.index("pool.fork"), block.index("pool.check")
    before, step, after = block[:at], block[at:end], block[end:]
    torch.manual_seed(4)
    n, n_q = 333, 18
    k, v = (torch.randn(28, n, 4, 128, device="cuda").bfloat16() for _ in range(2))
    new = torch.randn(28, n_q, 36, 128, device="cuda").bfloat16()

    def inputs():
        q_rot, out = (torch.full((n_q, 28, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return dict(ap=ap, torch=torch, k=k, v=v, n=n, n_q=n_q, q_rot=q_rot, out=out, video=i32([0]), video_rows=i32([n]),
                    parents=i32([0, 0, 0]), questions=i32([1, 2, 3]), new_rows=i32([5, 1, 12]), bounds=i32([0, 3]),
                    nothing=i32([0, 0, 0]), rotary=ap.Rotary(128), positions=i32([n + i for i in range(n_q)]),
                    project=lambda layer: (new[layer][:, :28], new[layer][:, 28:32], new[layer][:, 32:]))

    captured = inputs()
    exec(before, captured)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        exec(step, captured)
    for counts in ([5, 1, 12], [3, 9, 2], [1, 0, 1]):
        eager = inputs()
        eager["new_rows"].copy_(i32(counts))
        exec(before + step + after, eager)
        captured["new_rows"].copy_(i32(counts))
        captured["out"].fill_(7.0)
        graph.replay()
        exec(after, captured)                                              # raises if a call could not be carried out
        assert ap.apack_device_error(captured["ws"]) == 0
        assert torch.equal(captured["out"], eager["out"])
        assert (captured["out"][sum(counts):] == 7).all() and not (captured["out"][:sum(counts)] == 7).all()
        assert captured["pool"].lengths[:5].tolist() == [n, 0, 0, 0, 0]
        assert int(captured["pool"].tables.free_count) == 4096 - -(-n // 16)
