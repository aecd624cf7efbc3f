"""Tensors of one call on several devices are refused before anything of theirs is read (no GPU: tensors without memory)."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode


@pytest.fixture(scope="module")
def spf():
    from paper_2603_02631_b200.build import build_library
    build_library()
    import paper_2603_02631_b200 as mod
    return mod


L, HQ, HKV, D, M, N, BLOCK = 2, 4, 2, 64, 8, 300, 128
WHERE = ("q", "k_pools", "k_scales", "block_table", "importance", "lse")


def _prompt(spf, at):
    """A prompt's tensors on cuda:0, those that `at` names elsewhere ("k_pools" and "k_scales": the last layer's)."""
    def new(name, shape, dtype, layer=None):
        device = at.get(name, "cuda:0") if layer in (None, L - 1) else at.get("q", "cuda:0")
        return torch.empty(shape, dtype=dtype, device=device)

    return spf.PagedFp8PromptBuffers(
        new("q", (L, HQ, M, D), torch.bfloat16), [new("k_pools", (4, HKV, BLOCK, D), torch.uint8, l) for l in range(L)],
        [new("k_scales", (4, HKV, BLOCK // 64), torch.float32, l) for l in range(L)], new("block_table", (3,), torch.int32), N,
        new("importance", (N,), torch.float32), new("lse", (L, HQ, M), torch.float32))


@pytest.mark.parametrize("name", WHERE)
def test_score_paged_fp8_wants_a_prompt_on_one_device(spf, name):
    with FakeTensorMode(), pytest.raises(ValueError, match="another device"):
        spf.spf_score_paged_fp8_workspace_bytes([_prompt(spf, {name: "cuda:1"})])


def test_score_paged_fp8_wants_all_prompts_on_one_device(spf):
    elsewhere = {name: "cuda:1" for name in WHERE}
    for prompts in ([{"q": "cuda:1"}], [elsewhere, {}]):
        with FakeTensorMode(), pytest.raises(ValueError, match="another device"):
            spf.spf_score_paged_fp8_workspace_bytes([_prompt(spf, at) for at in prompts])


@pytest.mark.parametrize("name", ["workspace", "dev_status"])
def test_score_paged_fp8_wants_workspace_and_status_there_too(spf, name):
    with FakeTensorMode():
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:1" if name == "workspace" else "cuda:0")
        status = torch.empty(1, dtype=torch.int32, device="cuda:1" if name == "dev_status" else "cuda:0")
        with pytest.raises(ValueError, match="another device"):
            spf.spf_score_paged_fp8([_prompt(spf, {})], ws, dev_status=status)


def test_score_paged_fp8_wants_a_contiguous_workspace(spf):
    with FakeTensorMode(), pytest.raises(TypeError, match="contiguous"):
        spf.spf_score_paged_fp8([_prompt(spf, {})], torch.empty((64, 2048), dtype=torch.uint8, device="cuda:0")[:, :1024])
