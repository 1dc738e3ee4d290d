"""The word model in each type: a step's gradients against torch's own derivative in 64 bits."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.mark.parametrize("dtype", list(U))
def test_gradients_of_a_large_batch(dtype):
    """Gradients of the mean over 65,536 tokens, each some 1e-7 and smaller before they are summed.

    Twelve values on the way are rounded to the type (the input, five parameters,
    three results, G, dh, da and db), each within u of itself; a parameter's
    gradient is a sum over tokens, off by the root of the sum of their squares
    at best and by 12 u of the whole at worst where all errors agree; the layer
    norm and the activations multiply an error of theirs by 2 at most.  In
    single precision the sums count for more: 3 (65,536 + 8) u at worst.
    """
    from paper_2007_08725_amd.word_model import WordModel
    K, V, rows = 32, 6000, 65536
    gen = torch.Generator().manual_seed(3)
    theta = (torch.rand(rows, K, generator=gen) ** 4).cuda()
    words = torch.randint(0, V, (rows,), generator=gen, dtype=torch.int32).cuda()
    model = WordModel(K, V, 32, dtype=dtype)
    p = {n: t.double().requires_grad_() for n, t in model.params.items()}
    model.step(theta, words)
    got = {n: m[0] / 0.1 for n, m in model._moments.items()}  # the first step's average is a tenth of the gradient
    grads = {n: torch.zeros_like(t) for n, t in p.items()}
    for part in range(0, rows, 8192):
        t, w = theta[part:part + 8192].double(), words[part:part + 8192].long()
        x = torch.nn.functional.layer_norm(t, (K,), p["norm_weight"], p["norm_bias"], 1e-5)
        a = x @ p["w_gate"].t()
        z = (a * torch.sigmoid(a) * (x @ p["w_value"].t())) @ p["weight"].t() + p["bias"]
        loss = (torch.logsumexp(z, 1) - z.gather(1, w[:, None])[:, 0]).sum() / rows
        for n, d in zip(p, torch.autograd.grad(loss, list(p.values()))):
            grads[n] += d
    room = 24 * U[dtype] if dtype != torch.float32 else 3 * (rows + 8) * U[dtype]
    for n, want in grads.items():
        assert float((got[n].double() - want).norm()) <= room * float(want.norm()), n
