"""The binding's descriptors of paged tensors: what a kernel would misread is refused when the descriptor is made, a descriptor of another
device when a serving call is given it.  No GPU: the device is the last thing that is looked at."""
import types

import pytest
import torch

from paper_2609_04774_b200 import binding

BF, U8, F32 = torch.bfloat16, torch.uint8, torch.float32


def pages(n=6, page=16, heads=2, dim=128, dtype=BF):
    return torch.zeros(n, page, heads, dim, dtype=dtype)


def refused(word, make, *args):
    with pytest.raises(binding.CpArgumentError) as e:
        make(*args)
    assert e.value.code == binding.CP_ERR_INVALID_ARG and word in str(e.value), str(e.value)


def test_bf16_caches():
    k = pages()
    refused("CUDA device", binding.make_cache, k, pages())                     # all but the device is in order
    refused("torch.bfloat16", binding.make_cache, pages(dtype=U8), pages(dtype=U8))
    refused("torch.bfloat16", binding.make_cache, pages(dtype=torch.float16), pages(dtype=torch.float16))
    refused("agree", binding.make_cache, k, pages(n=5))
    refused("agree", binding.make_cache, k, pages(dtype=U8))
    refused("agree", binding.make_cache, k, pages(page=32)[:, ::2])
    refused("unit stride", binding.make_cache, k.transpose(2, 3), k.transpose(2, 3))
    refused("unit stride", binding.make_cache, k[0], k[0])
    refused("unit stride", binding.make_cache_fp8, k[0].to(U8), k[0].to(U8), torch.ones(2), torch.ones(2))


def test_e4m3_caches():
    k, s = pages(dtype=U8), torch.ones(2)
    refused("CUDA device", binding.make_cache_fp8, k, pages(dtype=U8), s, s)
    refused("CUDA device", binding.make_cache_fp8, k.view(torch.float8_e4m3fn), k.view(torch.float8_e4m3fn), s, s)
    refused("torch.uint8", binding.make_cache_fp8, pages(), pages(), s, s)
    refused("torch.uint8", binding.make_cache_fp8, k.view(torch.float8_e5m2), k.view(torch.float8_e5m2), s, s)
    refused("agree", binding.make_cache_fp8, k, pages(n=5, dtype=U8), s, s)
    refused("k_scale", binding.make_cache_fp8, k, k, s.double(), s)
    refused("v_scale", binding.make_cache_fp8, k, k, s, s.to(BF))
    refused("v_scale", binding.make_cache_fp8, k, k, s, torch.ones(3))
    refused("k_scale", binding.make_cache_fp8, k, k, torch.ones(1).expand(2), s)


def test_page_pools():
    k = torch.zeros(3, 6, 16, 2, 128, dtype=BF)
    refused("CUDA device", binding.make_page_pool, k, k)
    refused("CUDA device", binding.make_page_pool, k.view(U8)[..., :128], k.view(U8)[..., :128])
    refused("layers", binding.make_page_pool, k, k[:2])
    refused("layers", binding.make_page_pool, [], [])
    refused("agree", binding.make_page_pool, k, [pages(), pages(), pages(n=7)])
    refused("torch.bfloat16", binding.make_page_pool, k.float(), k.float())


def test_descriptors_of_another_device():
    on = [types.SimpleNamespace(device=i) for i in (0, 1)]
    for kind in (binding.cp_kv_cache, binding.cp_kv_cache_fp8, binding.cp_page_pool):
        d = kind()
        assert binding._described(on[1], d, kind)                              # made by hand: nothing is known of its tensors
        d.device = 0
        assert binding._described(on[0], d, kind)
        refused("cuda:0", binding._described, on[1], d, kind)
    refused("takes a cp_kv_cache", binding._described, on[0], binding.cp_kv_cache_fp8(), binding.cp_kv_cache)
