"""The small language model: bounds of its default type (fp32), rows that belong to no sequence, repeatable gradients."""
import math

import pytest
import torch

from test_gpu_diff_lm import DEV, reference

pytestmark = pytest.mark.gpu


def poison():
    """NaN in the memory that the next small tensors get."""
    kept = [torch.full((n,), math.nan, device=DEV) for n in (1 << 10, 1 << 13, 1 << 15, 1 << 17) for _ in range(40)]
    torch.cuda.synchronize()
    del kept


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_no_sequence(dtype):
    """Rows that no sequence has: their logits are finite, and the gradients are those without them."""
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    tokens, positions, starts, _ = copying_batch(5, 20, 50, seed=1)
    n, extra = tokens.numel(), 37
    gen = torch.Generator(device=DEV).manual_seed(2)
    dz = torch.randn(n, 50, generator=gen, device=DEV).bfloat16().float()
    runs = []
    for more in (0, extra):
        lm = DiffLM(50, layers=2, heads=4, kv_heads=2, head_dim=32, seed=3, dtype=dtype)
        t = torch.cat([tokens, torch.zeros(more, dtype=tokens.dtype, device=DEV)])
        p = torch.cat([positions, torch.zeros(1, more, dtype=torch.int32, device=DEV)], 1)
        poison()
        z = lm.forward(t, p, starts, 40)
        assert torch.isfinite(z).all()
        poison()
        lm.backward(torch.cat([dz, torch.zeros(more, 50, device=DEV)]))
        runs.append((z[:n].double(), {k: g.double() for k, g in lm.g.items()}))
    # the same sums over other tiles: fp32 products, whose results are rounded to bf16 in the bf16 model
    tol = 1e-5 if dtype is torch.float32 else 2e-2
    (z0, g0), (z1, g1) = runs
    assert (z0 - z1).norm() <= tol * z0.norm()
    for k in g0:
        assert (g0[k] - g1[k]).norm() <= tol * g0[k].norm(), k


def test_gradients_repeat():
    """The same batch, the same bits, with few words under many rows."""
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    lm = DiffLM(7, layers=1, heads=4, kv_heads=2, head_dim=32, seed=3)
    tokens, positions, starts, _ = copying_batch(300, 20, 7, seed=1)
    first = None
    for _ in range(8):
        z = lm.forward(tokens, positions, starts, 40)
        lm.backward(torch.cos(z))
        got = {k: g.clone() for k, g in lm.g.items()}
        first = first or got
        for k, g in got.items():
            assert torch.equal(g, first[k]), k


def test_decoder_fills_its_room():
    """As many tokens as there is room for and no more; a sequence that begins anew goes on beside the others."""
    from paper_2010_02838_amd.diff_lm import DiffLM
    lm = DiffLM(20, layers=1, heads=2, kv_heads=1, head_dim=16, seed=2)
    words = torch.randint(0, 20, (2, 6), generator=torch.Generator().manual_seed(1)).to(DEV)
    decoder = lm.decoder(2, 6)
    first = [decoder.step(words[:, t]) for t in range(6)]
    for _ in range(2):
        with pytest.raises(ValueError):
            decoder.step(words[:, 0])
    decoder.lens.zero_()
    for t in range(6):
        assert torch.equal(decoder.step(words[:, t]), first[t])
    with pytest.raises(ValueError):
        decoder.step(words[:, 0])


def test_width_that_the_heads_do_not_have():
    """A residual stream narrower than all heads together: gradients as those of the square model (1e-4), and a decoder of its size."""
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    lm = DiffLM(30, layers=2, heads=16, kv_heads=4, head_dim=64, lambda_init=0.5, seed=3, width=96)
    for i in range(2):
        lm.w["lam%d" % i].copy_(torch.linspace(-0.3, 0.9, 16))
    tokens, positions, starts, _ = copying_batch(3, 12, 30, seed=1)
    z = lm.forward(tokens, positions, starts, 24)
    dz = torch.randn(z.shape, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    lm.backward(dz)
    want, grads = reference(lm, tokens, starts, positions, dz)
    assert (z.double().cpu() - want).norm() <= 1e-4 * want.norm()
    for n, g in grads.items():
        assert (lm.g[n].double().cpu() - g).norm() <= 1e-4 * g.norm(), n
    decoder, first = lm.decoder(1, 24), tokens[:int(starts[1])]
    for t, word in enumerate(first):
        got = decoder.step(word[None])[0]
        assert (got - z[t]).norm() <= 1e-4 * z[t].norm(), t


@pytest.mark.parametrize("kv_heads", [1, 4])
def test_gradients_of_an_fp32_network(kv_heads):
    """The default model is fp32 throughout.  A gradient passes some thirty sums of up to 256 terms, each rounded to a few times 2^-24 of its terms; the
    difference of the two maps at a lambda near one and the sums of either sign cost one to two digits of that: 1e-4."""
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    lm = DiffLM(50, layers=2, heads=4, kv_heads=kv_heads, head_dim=32, lambda_init=0.5, seed=3)
    for i in range(2):
        lm.w["lam%d" % i].copy_(torch.tensor([0.3, -0.2, 0.0, 0.9]))
    tokens, positions, starts, _ = copying_batch(5, 20, 50, seed=1)
    z = lm.forward(tokens, positions, starts, 40)
    dz = torch.randn(z.shape, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    lm.backward(dz)
    want, grads = reference(lm, tokens, starts, positions, dz)
    assert (z.double().cpu() - want).norm() <= 1e-4 * want.norm()
    for n, g in grads.items():
        assert (lm.g[n].double().cpu() - g).norm() <= 1e-4 * g.norm(), n


def test_lambdas_gradient_of_a_bf16_network(monkeypatch):
    """lambda's gradient is a sum of products of either sign, dO (P_2 v) of all rows and channels, which cancels; some six bf16 roundings in front of each of them,
    1.7e-3 as a 2-norm, are 4e-3 of the root of the products' squares, five times that where a row's channels share one (2e-2)."""
    from paper_2010_02838_amd import binding as B
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    lm = DiffLM(50, layers=1, heads=4, kv_heads=2, head_dim=64, lambda_init=0.2, seed=5, dtype=torch.bfloat16)
    tokens, positions, starts, _ = copying_batch(4, 30, 50, seed=2)
    z = lm.forward(tokens, positions, starts, 60)
    dz = torch.randn(z.shape, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16().float()
    call, products = B.codistill_diff_attention_backward, []

    def keep(desc, q, k, v, lam, out, o_second, lse, dout, *rest):
        products.append(o_second.double() * dout.double())
        call(desc, q, k, v, lam, out, o_second, lse, dout, *rest)

    monkeypatch.setattr(B, "codistill_diff_attention_backward", keep)
    lm.backward(dz)
    _, grads = reference(lm, tokens, starts, positions, dz)
    size = products[0].square().sum((0, 2)).sqrt().cpu()
    assert (lm.g["lam0"].double().cpu() - grads["lam0"]).norm() <= 2e-2 * size.norm()


def test_decoding_in_fp32():
    """Token by token against the cache and in one pass: the same fp32 products in other orders, rounded to a few times 2^-24 some thirty times: 1e-4."""
    from paper_2010_02838_amd.diff_lm import DiffLM
    lm = DiffLM(50, layers=2, heads=4, kv_heads=2, head_dim=32, seed=4)
    gen = torch.Generator(device=DEV).manual_seed(5)
    T = 140
    words = torch.randint(0, 50, (3, T), generator=gen, device=DEV)
    starts = torch.arange(4, dtype=torch.int32, device=DEV) * T
    positions = torch.arange(T, dtype=torch.int32, device=DEV).repeat(3)[None]
    z = lm.forward(words.flatten(), positions, starts, T).view(3, T, -1)
    dec = lm.decoder(3, T)
    for t in range(T):
        got = dec.step(words[:, t])
        assert (got - z[:, t]).norm() <= 1e-4 * z[:, t].norm(), t
