"""GPU tests of the operators around the tied weight at the ends of their arguments' ranges, against the 64-bit
definitions (oracle/tied_oracle.py)."""
import numpy as np
import pytest
import torch

import paper_1905_04035_b200 as dst
from oracle import tied_oracle as o

pytestmark = pytest.mark.gpu
U = 2.0 ** -24                                              # half a step of fp32, relative
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw_tokens(x, u, **settings):
    """(tokens, prob) of dst_sample with one value of each setting for all rows."""
    rows = x.shape[0]
    full = lambda v, d=torch.float32: torch.full((rows,), v, dtype=d, device="cuda")  # noqa: E731
    args = {name: full(v, torch.int32 if name == "top_k" else torch.float32) for name, v in settings.items() if v is not None}
    tokens, prob = full(-7, torch.int64), full(-7.0)
    dst.dst_sample(x, u if torch.is_tensor(u) else full(u), tokens, prob=prob, **args)
    return tokens.cpu().numpy(), prob.cpu().numpy()


# (rows, vocab): a row in one CTA as a list or not, a row over two, four and eight CTAs, more rows than CTAs at once
@pytest.mark.parametrize("rows,vocab", [(3, 700), (2, 2000), (40, 4100), (20, 9000), (1, 33708), (400, 3000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top_k,top_p", [(None, None), (40, None), (None, 0.9), (40, 0.9)])
def test_temperatures_not_above_zero_take_the_largest_logit_whatever_the_filters(rows, vocab, dtype, top_k, top_p):
    x = (torch.randn(rows, vocab, generator=torch.Generator().manual_seed(vocab)) * 3).to(TYPES[dtype])
    want = x.float().numpy().argmax(-1)                                          # the first of equal ones
    x = x.cuda()
    for t in (-1.0, -0.5, -1e-30, -1e30, float("-inf"), -0.0, 0.0, float("nan")):
        for min_p in (None, 1e-30, 0.1, 1.0, 2.0):
            tokens, prob = draw_tokens(x, 0.75, temperature=t, top_k=top_k, top_p=top_p, min_p=min_p)
            assert np.array_equal(tokens, want) and (prob == 1).all(), (t, min_p)


@pytest.mark.parametrize("n,d", [(1, 8), (37, 64), (300, 512), (5, 61), (70, 1021)])
@pytest.mark.parametrize("wt,ot,it", [("f32", "f32", torch.int64), ("bf16", "bf16", torch.int32), ("f32", "bf16", torch.int32), ("bf16", "f32", torch.int64)])
@pytest.mark.parametrize("positions,p", [(0, 0.0), (3, 0.25)])
def test_a_lookup_in_an_empty_table_gives_zeros_and_counts_every_index(n, d, wt, ot, it, positions, p):
    weight = torch.empty(0, d, dtype=TYPES[wt], device="cuda")
    assert weight.data_ptr() == 0                                                # there is nothing to read
    idx = torch.arange(n, device="cuda").sub_(n // 2).to(it)
    position = torch.ones(positions, d, device="cuda") if positions else None
    out = torch.full((n, d), float("nan"), dtype=TYPES[ot], device="cuda")
    result = torch.full((3,), 7, dtype=torch.int64, device="cuda")
    dst.dst_embed(idx, weight, out, scale=3.0, position=position, p=p, seed=5, result=result)
    assert (out == 0).all() and result.tolist() == [4, n, 0]


def check_draws(X, x, u, temperature, **settings):
    """Tokens and probs of every row against the definition; rows where a decision hangs on the exponential's last bits
    (nearer than 2^-18 of the sums) may differ, and are counted."""
    rows = x.shape[0]
    tokens, prob = draw_tokens(x, torch.tensor(u, dtype=torch.float32, device="cuda"), temperature=temperature, **settings)
    unsure = 0
    for r in range(rows):
        token, p, margin = o.sample(X[r], float(np.float32(u[r])), float(np.float32(1.0 if temperature is None else temperature)), settings.get("top_k") or 0,
                                    float(np.float32(settings.get("top_p") or 1.0)), float(np.float32(settings.get("min_p") or 0.0)))
        if margin < 2.0 ** -18 and token != tokens[r]:
            unsure += 1
            continue
        assert token == tokens[r] and abs(p - prob[r]) <= 2.0 ** -18, (r, token, tokens[r], p, prob[r], settings)
    assert unsure <= 1 + rows // 50


# rows of 1025 to 2048 entries, and many rows of any length, are one CTA's
@pytest.mark.parametrize("rows,vocab", [(1, 2000), (5, 1100), (1, 4099), (80, 33708)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("most,rest", [(1e-40, 1e-42), (1e-37, 0.0), (1e-40, 0.0), (0.0, -1e-38), (3e-36, 0.0)])
def test_top_k_of_logits_whose_differences_are_next_to_nothing(rows, vocab, dtype, most, rest):
    x = torch.full((rows, vocab), rest).to(TYPES[dtype])
    x[:, 7] = most
    x[:, 900] = (most + rest) / 2
    X = x.float().numpy()
    u = np.random.default_rng(vocab).integers(0, 1 << 24, rows) / 2.0 ** 24
    for k in (2, 40, 200):
        check_draws(X, x.cuda(), u, None, top_k=k)
        check_draws(X, x.cuda(), u, None, top_k=k, top_p=0.5, min_p=0.5)


@pytest.mark.parametrize("rows,vocab", [(3, 3000), (100, 1500), (2, 33708)])
@pytest.mark.parametrize("temperature", [2e-37, 1e-38, 4e-39])
@pytest.mark.parametrize("settings", [dict(top_p=0.5), dict(top_p=0.95), dict(top_k=1200), dict(top_k=1200, top_p=0.8, min_p=0.01), dict(min_p=0.05)])
def test_temperatures_whose_steps_are_next_to_nothing(rows, vocab, temperature, settings):
    """Logits as close together as the temperature is small, so that their weights are ordinary ones."""
    g = np.random.default_rng(vocab)
    X = (-np.abs(g.standard_normal((rows, vocab))) * 4 * temperature).astype(np.float32)
    assert len(np.unique(X)) > 1000
    check_draws(X, torch.from_numpy(X).cuda(), g.integers(0, 1 << 24, rows) / 2.0 ** 24, temperature, **settings)


def test_a_single_column_has_no_order_of_its_own():
    """[n, 1] tensors whose rows are one element apart, whatever stride their single column reports."""
    n = 300
    x = torch.randn(1, n, device="cuda").t()
    assert x.stride() == (1, n)
    out = torch.empty(1, n, device="cuda").t()
    dst.dst_dropout(x, out, 0.0, 1, scale=2.0)
    assert torch.equal(out, x * 2)
    q = dst.Fp8Matrix(n, 1)
    dst.dst_quantize_fp8(x, q)
    assert (q.dequantize() - x).abs().max() <= x.abs().max() / 16
    idx = torch.arange(n - 1, -1, -1, device="cuda")
    dst.dst_embed(idx, x, out)
    assert torch.equal(out, x.flip(0))
    tokens = torch.full((n,), -7, device="cuda")
    dst.dst_sample(x, torch.full((n,), 0.5, device="cuda"), tokens)
    assert (tokens == 0).all()


# M, N, K whose tiles fill the GPU, so that the inner dimension is summed in one part: the tile of two CTAs, and the side of at
# most 16, 32, 64 and 128 rows as a or as b
@pytest.mark.parametrize("M,N,K", [(4736, 1024, 16384), (5, 19000, 16384), (30, 19000, 9000), (19000, 60, 9000), (19000, 100, 9000)])
def test_an_fp32_result_does_not_pay_for_an_early_block_that_outweighs_the_rest(M, N, K):
    """Every element is one product B in the first block, nothing up to column 768, and 2^-6 B spread over what follows.

    The first six blocks sum to B exactly.  Stretches of six blocks after them may lose 2u of their own sum for every one of
    their 768 additions (additions in tensor memory truncate, at worst), and joining a stretch rounds to nearest, u of the sum:
        768 2u R + stretches u (B + R)             R the sum of the rest
    that is 35 u B for K = 9000 and 45 u B for 16384.  Summed on in tensor memory, every 32 elements after the first block are
    truncated at B itself, which is off by 285 and 1065 u B."""
    g = torch.Generator(device="cuda").manual_seed(K)

    def matrix(rows, small):
        x = torch.rand(rows, K, device="cuda", generator=g).to(torch.bfloat16).add_(1).mul_(small)
        x[:, 0], x[:, 1:768] = 448, 0
        m = dst.Fp8Matrix(rows, K)
        dst.dst_quantize_fp8(x, m)
        return m

    a, b = matrix(M, 0.09 * 15616 / (K - 768)), matrix(N, 1.0)
    out = torch.full((M, N), float("nan"), device="cuda")
    dst.dst_matmul_fp8(a, b, out, torch.empty(max(dst.dst_matmul_fp8_workspace_bytes(M, N, K), 256), dtype=torch.uint8, device="cuda"))
    rows, cols = torch.arange(0, M, max(1, M // 40), device="cuda"), torch.arange(0, N, max(1, N // 40), device="cuda")
    A, B = a.dequantize()[rows].double(), b.dequantize()[cols].double()
    first, rest = A[:, :1] @ B[:, :1].T, A[:, 768:] @ B[:, 768:].T
    stretches = -(-(K - 768) // 768)
    bound = 768 * 2 * U * rest + stretches * U * (first + rest)
    error = (out[rows][:, cols].double() - (first + rest)).abs()
    assert (error <= bound).all(), (float((error / (U * first)).max()), float((bound / (U * first)).max()))


def test_weights_next_to_a_power_of_two():
    """Rows [0, z] with z around every -k ln 2, where the weight is next to 2^(31 - k): the second entry is never lost.  Its
    weight is at least 2^11, and a uniform number of 1 - 2^-24 takes the last 2^-24 of the sum, 2^8 at most."""
    z = np.concatenate([np.float32(-k * np.log(2)) + np.arange(-300, 301, dtype=np.float32) * np.spacing(np.float32(k * np.log(2))) for k in range(1, 20)]).astype(np.float32)
    x = torch.from_numpy(np.stack([np.zeros_like(z), z], -1)).cuda()
    tokens, prob = draw_tokens(x, 1 - 2.0 ** -24)
    e = np.exp(z.astype(np.float64))
    assert (tokens == 1).all() and np.abs(prob / (e / (1 + e)) - 1).max() <= 2.0 ** -11
