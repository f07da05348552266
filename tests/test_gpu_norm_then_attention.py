"""The norm and rotation in front of the package's attentions, as a transformer block runs them."""
import pytest
import torch

from tests import cache_reference as ref
from tests.test_gpu_cache import ints, rotation, sb  # noqa: F401  (sb: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [0, 1], ids=["heads first", "tokens first"])
@pytest.mark.parametrize("B, N, H, d, block", [(2, 517, 3, 128, 128), (1, 1000, 2, 64, 64)])
def test_norm_then_attention(sb, B, N, H, d, block, layout):  # noqa: F811
    """q and k of a fused projection are normed and rotated into the layout that the dense and the routed attention read, and, for the same
    sequence, over a cache: each against softmax attention in 64 bits over what it was given."""
    g = torch.Generator().manual_seed(N)
    fused = torch.randn(B, N, 3 * H, d, generator=g).bfloat16()
    weight = 1 + 0.1 * torch.randn(d, generator=g)
    cos, sin = rotation(N, d)
    x = fused.cuda()
    shape = (B, H, N, d) if layout == sb.SOL_LAYOUT_BHND else (B, N, H, d)
    tokens_first = lambda t: t if layout == sb.SOL_LAYOUT_BNHD else t.transpose(1, 2)  # noqa: E731
    q, k, v, out = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    tokens_first(v).copy_(x[:, :, 2 * H:])
    # (the projection's views as inputs: the strides of inputs and outputs need not be alike)
    ins = [t if layout == sb.SOL_LAYOUT_BNHD else t.transpose(1, 2) for t in (x[:, :, :H], x[:, :, H:2 * H])]
    sb.sol_attn_qk_norm_rope(*ins, q, k, cos.cuda(), sin.cuda(), q_weight=weight.cuda(), k_weight=weight.cuda(), interleaved=True, layout=layout)
    at = torch.arange(N, dtype=torch.int32).expand(B, N)
    for t, i in ((q, 0), (k, H)):
        want, tol = ref.norm_rope(fused[:, :, i:i + H], weight, cos, sin, at, 1e-6, True)
        assert ((tokens_first(t).cpu().double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all()
    qd, kd, vd = (tokens_first(t).cpu().double().transpose(1, 2) for t in (q, k, v))
    softmax = lambda a, b, c: torch.softmax(a @ b.transpose(-1, -2) * d ** -0.5, -1) @ c  # noqa: E731
    want = softmax(qd, kd, vd)
    ws = sb.make_workspace(B, H, N, d, block, block)
    # dense, then routed with a threshold below every score, which selects all; both keep weights in bf16 (2^-8 of |v|, beside out's rounding)
    for mode in (sb.SOL_MODE_DENSE, sb.SOL_MODE_SOL):
        out.fill_(9)
        sb.sol_attn_forward_ex(q, k, v, out, ws, block, block, threshold=-1e6, mode=mode, layout=layout)
        got = tokens_first(out).cpu().double().transpose(1, 2)
        assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -8 * softmax(qd, kd, vd.abs()) + 1e-5).all(), mode
    # over the 4-bit cache: the first sequence's keys and values as the cache holds them
    cache, slots = sb.make_cache(-(-N // 64), 64, H, d), torch.arange(N, dtype=torch.int32, device="cuda")
    rows = [tokens_first(t)[0].contiguous() for t in (q, k, v)]
    sb.sol_attn_cache_append(rows[1], rows[2], slots, cache)
    held, cached = [torch.empty_like(rows[1]) for _ in range(2)], torch.empty_like(rows[0])
    sb.sol_attn_cache_read(cache, slots, *held)
    sb.sol_attn_cache_attention(rows[0], ints([0, N]), ints([N]), ints([list(range(cache.pages))]), cache, cached, N,
                                sb.make_cache_workspace(N, H, H, d), causal=False)
    kc, vc = (t.cpu().double().transpose(0, 1) for t in held)
    want = softmax(qd[0], kc, vc)
    assert ((cached.cpu().double().transpose(0, 1) - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * softmax(qd[0], kc, vc.abs()) + 1e-5).all()
