"""One layer of forked rollouts as a program runs it: norm, projections, rotary append
into the caches, attention over the shared prefix, projection, gated residual and norm,
for a step of several tokens and one of single tokens, against the same layer in 64 bits.

Every stage rounds its output to bf16 (2^-8 relative, about 2^-9.8 in the mean square),
as the projections and the attention's weights do. Six such roundings of independent
sign in a row stay below 6 x 2^-8 relative in the 2-norm; h divides by the deviation of
the stream, whose rounding enters at the same size.
"""

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def rel(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("heads, kv_heads, interleaved", [(4, 4, True), (4, 2, False)])
def test_layer_of_forked_rollouts(heads, kv_heads, interleaved):
    d, prefix, capacity = 64, 333, 40
    hidden, kv = heads * d, kv_heads * d
    g = torch.Generator().manual_seed(heads * 10 + kv_heads)
    r = lambda *s: torch.randn(*s, generator=g)
    w_in = (r(hidden + 2 * kv, hidden) / hidden ** 0.5).to(BF16)
    w_out = (r(hidden, hidden) / hidden ** 0.5).to(BF16)
    weight, gate = 1 + 0.1 * r(hidden), r(1, hidden)
    scale, shift = 0.2 * r(1, hidden), 0.2 * r(1, hidden)
    freqs, amplitude = ispa.rotary_frequencies(d // 2, device="cpu")
    prefix_k, prefix_v = r(prefix, kv).to(BF16), r(prefix, kv).to(BF16)
    gpu = lambda t: t.to(DEV)
    caches = [torch.zeros(3, capacity, kv, dtype=BF16, device=DEV) for _ in range(2)]
    own = [[torch.zeros(0, kv, dtype=torch.float64)] * 3 for _ in range(2)]
    lens = torch.zeros(3, dtype=torch.int32, device=DEV)

    for counts in ([5, 0, 9], [1, 1, 1], [1, 3, 0]):
        rows = sum(counts)
        starts = [0]
        for m in counts:
            starts.append(starts[-1] + m)
        x = r(rows, hidden)
        # the layer
        start = torch.tensor(starts, dtype=torch.int32, device=DEV)
        _, h = ispa.norm_residual(gpu(x), norm="layer", scale=gpu(scale), shift=gpu(shift))
        qkv = ispa.project(h, gpu(w_in), out_dtype=BF16)
        slots, positions, after = ispa.slot_map(start, lens, capacity, rows, first_position=prefix)
        before = lens.tolist()
        q = ispa.rotary_append(qkv[:, :hidden], qkv[:, hidden:hidden + kv], qkv[:, hidden + kv:], positions, slots,
                               gpu(freqs), heads, *caches, n_kv_heads=kv_heads, interleaved=interleaved,
                               amplitude=amplitude)
        lens = after
        a, _ = ispa.attn_shared(q, gpu(prefix_k), gpu(prefix_v), *caches, start, lens, heads, n_kv_heads=kv_heads)
        y = ispa.project(a, gpu(w_out), out_dtype=BF16)
        x_out, h_out = ispa.norm_residual(gpu(x), y, norm="rms", weight=gpu(weight), gate=gpu(gate))
        torch.cuda.synchronize()
        # the same in 64 bits
        X = x.double()
        H = (X - X.mean(1, keepdim=True)) / (X.var(1, unbiased=False, keepdim=True) + 1e-6).sqrt()
        H = H * (1 + scale.double()) + shift.double()
        QKV = H @ w_in.double().t()
        at = torch.tensor([prefix + before[b] + i for b, m in enumerate(counts) for i in range(m)]).double()
        angle = (at[:, None] * freqs)[:, None]

        def turn(t):
            t = t.view(rows, -1, d)
            i, k = (slice(0, d, 2), slice(1, d, 2)) if interleaved else (slice(0, d // 2), slice(d // 2, d))
            out = torch.empty_like(t)
            out[..., i] = t[..., i] * angle.cos() - t[..., k] * angle.sin()
            out[..., k] = t[..., i] * angle.sin() + t[..., k] * angle.cos()
            return out.flatten(1)

        Q, K, V = turn(QKV[:, :hidden]), turn(QKV[:, hidden:hidden + kv]), QKV[:, hidden + kv:]
        A = torch.zeros(rows, hidden, dtype=torch.float64)
        for b, m in enumerate(counts):
            s = slice(starts[b], starts[b + 1])
            own[0][b], own[1][b] = torch.cat((own[0][b], K[s])), torch.cat((own[1][b], V[s]))
            keys, values = torch.cat((prefix_k.double(), own[0][b])), torch.cat((prefix_v.double(), own[1][b]))
            for n in range(heads):
                c = n // (heads // kv_heads) * d
                w = torch.softmax(Q[s, n * d:(n + 1) * d] @ keys[:, c:c + d].t() / d ** 0.5, 1)
                A[s, n * d:(n + 1) * d] = w @ values[:, c:c + d]
        Xo = X + gate.double() * (A @ w_out.double().t())
        Ho = Xo / (Xo.pow(2).mean(1, keepdim=True) + 1e-6).sqrt() * weight.double()
        assert lens.tolist() == [len(k) for k in own[0]]
        bound = 6 * 2.0 ** -8
        assert rel(a, A) <= bound and rel(x_out, Xo) <= bound and rel(h_out, Ho) <= bound
        for b, n in enumerate(lens.tolist()):
            assert rel(caches[0][b, :n], own[0][b]) <= bound if n else True
            assert not caches[0][b, n:].any() and not caches[1][b, n:].any()
