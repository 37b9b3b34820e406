"""The weight that a prompt's queries give each key, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from helpers import nan_bytes, to64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


@pytest.fixture(scope="module")
def gen():
    from paper_2410_17980_amd import inputs
    return inputs


def activations(gen, B, H, Hkv, Tq, T, d, seed, kind="mixed"):
    q, _, _ = gen.gaussian(B, H, Tq, d, seed=seed, dtype="f32")
    _, k, _ = gen.gaussian(B, Hkv, T, d, seed=seed + 1, dtype="f32")
    far = (6.0 * d ** 0.5) ** 0.5
    for h in range(Hkv):
        if kind == "sharp":
            k[:, h] *= 40.0
        elif kind == "far" or (kind == "mixed" and h % 3 == 2):
            k[:, h, :, d - 1] = -far
            q[:, h * (H // Hkv):(h + 1) * (H // Hkv), :, d - 1] = far
        elif h % 3 == 1:
            k[:, h] *= 3.0
    return q.to(torch.bfloat16), k.to(torch.bfloat16)


def check(sb, oracle, q, k, T=None, lens=None, qlens=None, cap=None):
    """A weight's relative error is rel = (T + 64) 2^-23 + 8 dz (T factors 1 + e, dz: d products and sums in fp32), and a key's sum adds
    the errors of Tq G weights that are at most what the queries have to give: one each.  The sums themselves: fp32, at most
    Tq G roundings of a number no larger than the result."""
    B, H, Tq, d = q.shape
    Hkv, n = k.shape[1], k.shape[2]
    cap = cap or n
    bound = n if T is None else T
    kd = torch.full((B, Hkv, cap, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    kd[:, :, :n] = k.cuda()
    qd = q.cuda()
    at = [min(max(x, 0), bound) for x in lens] if lens is not None else [bound] * B
    nq = [min(max(x, 0), Tq) for x in qlens] if qlens is not None else [Tq] * B
    for b in range(B):                                   # padding is anything at all
        kd[b, :, at[b]:] = float("nan")
        qd[b, :, nq[b]:] = float("nan")
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    was = torch.rand(B, Hkv, cap, generator=torch.Generator().manual_seed(3)).cuda()
    out = torch.full_like(was, -7.0)
    ws = nan_bytes(sb.sb_attn_key_weight_workspace_bytes(B, H, Hkv, Tq, bound, d))
    got = sb.sb_attn_key_weight(qd, kd, T=bound, lens=ints(lens), qlens=ints(qlens), score=was, score_out=out, workspace=ws)
    torch.cuda.synchronize()
    assert got is out
    G, worst = H // Hkv, 0.0
    for b in range(B):
        one = lambda x, m: to64(x)[b:b + 1, :, :m]
        want = oracle.key_weight(one(q, nq[b]), one(k, at[b]))[0]
        dz = d * U * float((one(q, nq[b]).__abs__().max(initial=0.0)) * np.abs(one(k, at[b])).sum(-1).max(initial=0.0)) / np.sqrt(d) / 4
        rel = (at[b] + 64) * 2 * U + 8 * dz
        for g in range(Hkv):
            s = to64(out)[b, g]
            ref = want[g] + to64(was)[b, g, :at[b]]
            err = np.abs(s[:at[b]] - ref)
            tol = rel * (1.0 + want[g]) + (nq[b] * G + 2) * U * ref
            worst = max(worst, float((err / tol).max(initial=0.0)))
            assert (err <= tol).all(), (b, g, float((err - tol).max()))
            assert (s[at[b]:] == -7.0).all()
    again = was.clone()
    assert sb.sb_attn_key_weight(qd, kd, T=bound, lens=ints(lens), qlens=ints(qlens), score=again) is again
    fresh = sb.sb_attn_key_weight(qd, kd, T=bound, lens=ints(lens), qlens=ints(qlens))
    for b in range(B):
        assert torch.equal(again[b, :, :at[b]], out[b, :, :at[b]]) and torch.equal(again[b, :, at[b]:], was[b, :, at[b]:])
        assert torch.allclose(fresh[b, :, :at[b]] + was[b, :, :at[b]], out[b, :, :at[b]], rtol=1e-6, atol=1e-6)
    print(f"{worst:.3f} of the bound")


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 3, 31, 32, 33, 64, 65, 127, 128, 129, 200, 333])
def test_prompts(sb, oracle, gen, T, d):
    check(sb, oracle, *activations(gen, 2, 3, 3, T, T, d, seed=T + d))


@pytest.mark.parametrize("Tq,T", [(1, 1), (1, 2), (1, 700), (5, 700), (32, 700), (33, 700), (64, 129), (100, 101), (40, 2500)])
@pytest.mark.parametrize("d", [64, 128])
def test_windows(sb, oracle, gen, Tq, T, d):
    check(sb, oracle, *activations(gen, 2, 6, 3, Tq, T, d, seed=Tq + T))


@pytest.mark.parametrize("H,Hkv", [(2, 1), (3, 1), (12, 4), (5, 1), (8, 1), (20, 2)])
def test_grouped_heads(sb, oracle, gen, H, Hkv):
    check(sb, oracle, *activations(gen, 1, H, Hkv, 150, 150, 64, seed=H))


@pytest.mark.parametrize("B,H,Hkv,T,d", [(22, 12, 4, 261, 64), (27, 12, 12, 150, 32), (16, 64, 8, 70, 32), (9, 56, 7, 130, 128), (5, 90, 45, 200, 64)])
def test_grids_of_many_units(sb, oracle, gen, B, H, Hkv, T, d):
    """Four units a workgroup, more workgroups than the chip holds, kv heads that do and do not divide the chip: every head is there once."""
    check(sb, oracle, *activations(gen, B, H, Hkv, T, T, d, seed=B))


@pytest.mark.parametrize("kind", ["far", "sharp", "near"])
@pytest.mark.parametrize("d", [32, 128])
def test_kinds_of_heads(sb, oracle, gen, kind, d):
    check(sb, oracle, *activations(gen, 1, 3, 3, 500, 500, d, seed=5, kind=kind))


@pytest.mark.parametrize("d", [32, 64, 128])
def test_padded_batches(sb, oracle, gen, d):
    lens = [0, 1, 2, 33, 150, 260, 300, 999, -4]
    q, k = activations(gen, len(lens), 2, 2, 300, 300, d, seed=d)
    check(sb, oracle, q, k, lens=lens, qlens=lens)
    # windows of different lengths, one longer than its entry
    check(sb, oracle, q[:, :, :70].contiguous(), k, lens=[0, 1, 2, 33, 150, 260, 300, 80, 70], qlens=[0, 0, 1, 33, 70, 7, 64, 70, 70])
    check(sb, oracle, q[:, :, :70].contiguous(), k, lens=[300] * 9, cap=310)


def test_bound_below_the_capacity(sb, oracle, gen):
    q, k = activations(gen, 2, 4, 2, 50, 400, 64, seed=4)
    check(sb, oracle, q, k[:, :, :200].contiguous(), cap=1111)
    check(sb, oracle, q, k, T=123, cap=401)


def test_sums_to_what_the_forward_takes(sb, gen):
    """All keys' weights are what the forward takes off the stick: sum over keys = sum over queries of 1 - exp(m)."""
    q, k = (t.cuda() for t in activations(gen, 2, 6, 3, 1500, 1500, 128, seed=6))
    s = sb.sb_attn_key_weight(q, k)
    _, m = sb.sb_attn_fwd_gqa(q, k, k)
    taken = (1.0 - torch.exp(m.double())).view(2, 3, -1).sum(-1)
    assert torch.allclose(s.double().sum(-1), taken, rtol=1e-4)


def test_one_token_is_what_decode_gives(sb, gen):
    """One query whose own key is the last row: the weights that decode on the rows before it gives (4-bit rows, so that both read the same)."""
    q, k = (t.cuda() for t in activations(gen, 2, 6, 3, 1, 2500, 64, seed=7))
    cache = [torch.zeros(2, 3, 2528, w, dtype=torch.uint8, device="cuda") for w in (32, 2, 32, 2)]
    sb.sb_attn_kv4_store(k, k, *cache)
    k4, _ = sb.sb_attn_kv4_load(*cache, 2500)
    _, a = sb.sb_attn_decode_kv4(q[:, :, 0].contiguous(), *cache, T=2499, score_out=torch.zeros(2, 3, 2528, device="cuda"))
    b = sb.sb_attn_key_weight(q, k4)
    assert torch.allclose(a[:, :, :2499], b[:, :, :2499], rtol=1e-3, atol=1e-6) and (b[:, :, 2499] == 0).all()


def test_nan_in_a_key(sb, gen):
    q, k = (t.cuda() for t in activations(gen, 1, 2, 2, 200, 200, 64, seed=8, kind="far"))
    s = sb.sb_attn_key_weight(q, k)
    kx = k.clone()
    kx[0, 1, 100, 3] = float("nan")
    sx = sb.sb_attn_key_weight(q, kx)
    assert torch.equal(s[0, 0], sx[0, 0]) and sx[0, 1, 100].isnan()
    assert torch.isfinite(sx[0, 1, 101:]).all()          # keys nearer than it


def test_captured(sb, gen):
    q, k = (t.cuda() for t in activations(gen, 3, 4, 2, 130, 900, 64, seed=9))
    lens = torch.tensor([900, 130, 500], dtype=torch.int32, device="cuda")
    out = torch.zeros(3, 2, 900, device="cuda")
    ws = nan_bytes(sb.sb_attn_key_weight_workspace_bytes(3, 4, 2, 130, 900, 64))
    step = lambda: sb.sb_attn_key_weight(q, k, lens=lens, score_out=out, workspace=ws)
    want = []
    lengths = ([900, 130, 500], [140, 200, 900], [0, 1, 131])
    for x in lengths:
        lens.copy_(torch.tensor(x, dtype=torch.int32))
        out.fill_(-1.0)
        step()
        want.append(out.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(2):
        for x, w in zip(lengths, want):
            lens.copy_(torch.tensor(x, dtype=torch.int32))
            out.fill_(-1.0)
            ws.random_(0, 255)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)


def test_refusals(sb):
    q = torch.zeros(2, 4, 8, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    s = torch.zeros(2, 2, 16, device="cuda")
    for call, why in ((lambda: sb.sb_attn_key_weight(q.float(), k), "must be torch.bfloat16"), (lambda: sb.sb_attn_key_weight(q, k[:1]), "has shape"),
                      (lambda: sb.sb_attn_key_weight(q, k, T=7), "bad shape"), (lambda: sb.sb_attn_key_weight(q, k, T=17), "bad shape"),
                      (lambda: sb.sb_attn_key_weight(q[:, :3].contiguous(), k), "bad shape"), (lambda: sb.sb_attn_key_weight(q, k, score=s[:, :, :8]), "contiguous"),
                      (lambda: sb.sb_attn_key_weight(q, k, score=s.double()), "must be torch.float32"), (lambda: sb.sb_attn_key_weight(q, k.cpu()), "must live on the GPU"),
                      (lambda: sb.sb_attn_key_weight(q, k, qlens=torch.zeros(3, dtype=torch.int32, device="cuda")), "has shape"),
                      (lambda: sb.sb_attn_key_weight(q, k, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")), "workspace")):
        with pytest.raises(sb.SbAttnError, match=why):
            call()
