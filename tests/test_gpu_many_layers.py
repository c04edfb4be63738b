"""Read-back of more layers than a launch's grid has room for."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("flags", [0, 8, 16])
def test_all_layers_at_once(flags):
    import torch
    from paper_2502_11517_b200 import binding, build
    build()
    layers, m = 65535 + 3, 3
    pool = binding.Pool(layers, 1, 1, 64, 1, 1, 1, 4, flags=flags)
    pool.request_begin()
    # whole numbers of up to 7, a 7 in every group of 32 (whose scale in 4 bits is then 1): every kind of pool holds them as they are
    k = ((torch.arange(layers, device="cuda")[:, None, None, None] + torch.arange(m, device="cuda")[None, :, None, None]) % 7 + 1).float()
    k = k.expand(layers, m, 1, 64).to(torch.bfloat16).contiguous()
    k[..., ::32] = 7
    v = (-k).contiguous()
    pool.kv_append_run(0, 0, m, k, v)
    got_k, got_v = pool.kv_read_layers(0, 0, 0, m)
    assert torch.equal(got_k, k) and torch.equal(got_v, v)
    got_k, got_v = pool.kv_read_layers(0, 0, 1, m - 1, layer_begin=1)
    assert torch.equal(got_k, k[1:, 1:]) and torch.equal(got_v, v[1:, 1:])
    assert pool.status() == 0
    pool.close()
