"""Caches and queries with a size of zero are refused as all else is, with the extension module and without it."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [None, False])
@pytest.mark.parametrize("P,H,page,D,B,Hq,Sq", [(4, 0, 16, 64, 1, 4, 1), (4, 2, 16, 0, 1, 4, 1), (0, 2, 16, 64, 1, 4, 1), (4, 2, 0, 64, 1, 4, 1), (4, 2, 16, 64, 0, 4, 1),
                                               (4, 2, 16, 64, 1, 0, 1), (4, 2, 16, 64, 1, 4, 0)])
def test_sizes_of_zero(native, P, H, page, D, B, Hq, Sq, monkeypatch):
    import torch
    from paper_2604_18616_amd import binding
    monkeypatch.setattr(binding, "_native", native)
    cache = binding.kv_fp8_cache(P, H, page, D)
    bf16 = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    table, n = torch.zeros((B, 2), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    calls = [lambda: binding.attn_kv_fp8(bf16(B, Hq, Sq, D), cache, table, n)]
    if Hq and Sq:
        calls += [lambda: binding.kv_fp8_write(cache, bf16(B, H, Sq, D), bf16(B, H, Sq, D), table, n), lambda: binding.kv_fp8_read(cache, table, n, 4)]
    for call in calls:
        with pytest.raises((ValueError, binding.AttnError)):
            call()
    torch.cuda.synchronize()
