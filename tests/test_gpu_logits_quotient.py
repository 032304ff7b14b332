"""The repetition penalty's quotient alone: x / repetition rounded once, so err <= 2^-24 |x / repetition|, half a unit in the
last place of a normal result, or half the smallest subnormal, 2^-150, below."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["prompt", "history"])
@pytest.mark.parametrize("rows,vocab", [(6, 4099), (40, 128256), (100, 128256)])
def test_the_quotient_is_rounded_once(dtype, where, rows, vocab):
    from paper_2502_02534_amd import binding as B
    g = torch.Generator().manual_seed(rows)
    x = (4 * torch.randn((rows, vocab), generator=g)).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    rep = 0.5 + 1.5 * torch.rand(rows, generator=g)
    rep[:6] = torch.tensor([1.3, 3.0, 2.0 ** 127, 2.9e38, 2.0 ** -130, 1.0])  # reciprocals that are subnormal or past the range
    kw = {}
    if where == "prompt":
        kw["prompt_bits"] = torch.full((rows, -(-vocab // 32)), -1, dtype=torch.int32, device=DEV)
        seen = torch.ones(vocab, dtype=torch.bool)
    else:
        tokens = torch.randperm(vocab, generator=g)[:1500].to(torch.int32)
        kw["tokens"] = tokens.expand(rows, -1).contiguous().to(DEV)
        kw["token_lens"] = torch.full((rows,), 1500, dtype=torch.int32, device=DEV)
        seen = torch.zeros(vocab, dtype=torch.bool)
        seen[tokens.long()] = True
    x_dev, rep_dev, out = x.to(DEV), rep.to(DEV), torch.empty((rows, vocab), device=DEV)
    print(f"quotient {dtype} {where} {rows} x {vocab}", flush=True)
    B.penalize_logits(x_dev, B.SPD_F32 if dtype == "f32" else B.SPD_BF16, rows, vocab, vocab,
                      B.make_penalties(repetition=rep_dev, **kw), out, vocab)
    torch.cuda.synchronize()
    x, rho = x.double(), rep.double()[:, None]
    want = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
    big = want.abs() > torch.finfo(torch.float32).max
    got = out.cpu().double()
    assert torch.equal(got[big], torch.sign(want[big]) * float("inf"))
    assert bool(((got - want).abs()[~big] <= (2.0 ** -24 * want.abs()[~big]).clamp(min=2.0 ** -150)).all())
