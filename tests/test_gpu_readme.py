"""README's example run as it stands there, over two layers: the stored rows are those of the dense path, the samples' attention
is that of the prompt's kept rows and their own."""
import pytest
import torch

from paper_2601_07667_b200 import binding
from paper_2601_07667_b200 import inputs as I

from asl_check import make_path, to_dev
from pages_check import ints
from readme_check import example

pytestmark = pytest.mark.gpu


def test_the_example_of_the_paged_cache():
    wl = I.workload("C3", n_q_heads=32, n_kv_heads=8, seqlens=(900,), budgets=(200,), layers=2)
    L, n = 2, 5
    path, dense = make_path(wl), make_path(wl)
    x = [I.layer_inputs(wl, layer, seed=layer) for layer in range(L)]
    q_obs, k, v = ([to_dev(x[layer][name]) for layer in range(L)] for name in ("q_obs", "k", "v"))
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)        # noqa: E731
    k_new, v_new, q = rand(L, n, 8, 128), rand(L, n, 8, 128), rand(L, n, 32, 128)
    given = dict(binding=binding, L=L, path=path, q_obs=q_obs, k=k, v=v, k_new=k_new, v_new=v_new, q=q, n_tokens=n,
                 budget=ints([200] + [-1] * 63), prompt_slots=ints([0]), parent=ints([-1] + [0] * n + [-1] * (63 - n)),
                 slots=ints(range(1, n + 1)), cu_q=ints(range(n + 1)), want=ints([-1] + [201] * n + [-1] * (63 - n)), to=ints([-1] * 64))
    exec(example(), given)
    cache = given["cache"]
    cache.check()
    table = cache.table.cpu()
    for layer in range(L):
        dense.run_layer(q_obs[layer], k[layer], v[layer], layer)
        dense.join()
        rows = [pool[layer, table[0, :4].long().cuda()].transpose(0, 1).reshape(8, 256, 128)[:, :200] for pool in (cache.k, cache.v)]
        for got, ref in zip(rows, (dense.k_out, dense.v_out)):
            assert torch.equal(got.view(torch.int16), ref.view(torch.int16))
        for i in range(n):
            kk = torch.cat([rows[0].transpose(0, 1), k_new[layer, i:i + 1]]).double().repeat_interleave(4, dim=1)
            vv = torch.cat([rows[1].transpose(0, 1), v_new[layer, i:i + 1]]).double().repeat_interleave(4, dim=1)
            w = torch.softmax(torch.einsum("hd,nhd->hn", q[layer, i].double(), kk) / 128 ** 0.5, dim=1)
            ref, scale = torch.einsum("hn,nhd->hd", w, vv), torch.einsum("hn,nhd->hd", w, vv.abs())
            # a logit is a sum of 128 products in fp32, each step half of 2^-23; weights and the result are rounded to bf16 (2^-8 each),
            # sums run in fp32 over 201 keys, 2^x is good to 2^-22
            x_off = torch.einsum("hd,nhd->hn", q[layer, i].double().abs(), kk.abs()).amax(1, keepdim=True) / 128 ** 0.5 * 130 * 2.0 ** -24
            tol = 2.0 ** -8 * ref.abs() + scale * (2.0 ** -8 + 2 * x_off + 201 * 2.0 ** -24 + 2.0 ** -20) * 1.01
            assert ((given["outs"][layer][i].double() - ref).abs() <= tol).all()
    path.close(), dense.close()
