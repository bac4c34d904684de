"""The training step's operators together, as a program uses them (MI355X):
lookup -> the ranks' embedding gradients -> encode -> rank sum -> gradient norm
-> clipped AdamW step -> lookup, over several steps, beside a second matrix
whose gradient goes through the geometry-aware branch and is decoded.

Each call is checked against the oracle on the call's own inputs, so a wrong
order on the stream or a stale buffer shows.  Scales are per rank and 128
columns; the encode's codes equal the oracle's bit for bit, the rank mean too.
"""

import numpy as np
import pytest
import torch

from oracle import codec, train
from synth import factor_inputs, gradient_set

pytestmark = pytest.mark.gpu

gift = pytest.importorskip("paper_2607_07494_amd.gift")
DEV = "cuda"
F = np.float32
N, T, V, d = 3, 300, 500, 256          # ranks, tokens a rank, vocabulary, width
M2, R = 320, 16                        # the second matrix [M2, d], rank of its transform
LR, MAX_NORM, SCALE = 1e-2, 1e-2, 16.0


def bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


@pytest.mark.parametrize("moments", ["f32", "e4m3"])
def test_steps_of_a_small_model(moments):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    stream = torch.cuda.Stream()
    ctx = gift.Context(stream=stream.cuda_stream)
    gen = torch.Generator().manual_seed(1)
    table, w2 = (torch.randn(s, generator=gen).mul_(0.02).to(DEV) for s in ((V, d), (M2, d)))
    copies = [table.bfloat16(), w2.bfloat16()]
    rows = torch.empty((N, T, d), dtype=torch.bfloat16, device=DEV)
    grads = torch.empty((N, V, d), device=DEV)
    codes, scales = torch.empty((N, V, d), dtype=torch.uint8, device=DEV), torch.empty((N, 1, 2), device=DEV)
    g2 = torch.from_numpy(gradient_set(3, 4, N, M2, d)).to(DEV)
    codes2, scales2 = torch.empty((N, M2, d), dtype=torch.uint8, device=DEV), torch.empty((N, 1, 2), device=DEV)
    mean, mean2, out2 = (torch.empty(s, device=DEV) for s in ((V, d), (M2, d), (M2, d)))
    norm = torch.empty(2, device=DEV)
    factor = gift.Factor(ctx, M2, d, R, gift.SIDE_INPUT, seed=5)
    factor.update(acts=torch.from_numpy(factor_inputs(6, 1024, d)[0]).to(DEV), iters=4)
    opt = gift.AdamW(ctx, [table, w2], weight_decay=[0.0, 0.1], moments=moments, seed=9, copies=copies)
    torch.cuda.synchronize()
    U, cf, ci, s2 = (x.cpu().numpy().astype(np.float64) for x in factor.export(gift.SIDE_INPUT))
    torch.cuda.synchronize()
    fA = codec.Factor(U, cf, ci, float(s2[0]))
    old_copy = copies[0].float().cpu().numpy()
    for step in range(1, 4):
        tokens = torch.randint(-3, V, (N, T), generator=gen)
        dout = (torch.randn((N, T, d), generator=gen) * 1e-3).bfloat16()
        tok_g, dout_g = tokens.to(DEV), dout.to(DEV)
        before = [table.cpu().numpy(), w2.cpu().numpy()]
        state = {k: v.cpu().numpy().copy() for k, v in opt.state.items()}
        torch.cuda.synchronize()
        # one pass of the program, nothing waits in between
        gift.embedding(ctx, copies[0], tok_g, rows, scale=SCALE)
        gift.embedding_grad(ctx, tok_g, dout_g, grads, scale=SCALE)
        gift.encode(ctx, None, grads, codes, scales, 0, 128)
        gift.reduce_local(ctx, codes, scales, mean, 0, 128)
        gift.encode(ctx, factor, g2, codes2, scales2, 0, 128)
        gift.reduce_local(ctx, codes2, scales2, mean2, 0, 128)
        gift.decode(ctx, factor, mean2, out2)
        gift.grad_norm(ctx, [mean, out2], norm, max_norm=MAX_NORM)
        opt.step([mean, out2], lr=LR, grad_scale=norm[1:])
        torch.cuda.synchronize()
        # the lookup read the copy of the step before
        want = train.lookup(old_copy, tokens.numpy(), SCALE)
        np.testing.assert_array_equal(bits(rows), train.to_bf16(want))
        # embedding gradient: at most 64 + L / 8 + 4 roundings of 2^-24 of the magnitudes' sum, L <= T
        g = train.lookup_grad(tokens.numpy(), dout.float().numpy(), V, SCALE)
        size = train.lookup_grad(tokens.numpy(), dout.float().abs().numpy(), V, SCALE)
        assert np.all(np.abs(grads.cpu().numpy() - g) <= (64 + T / 8 + 4) * 2.0 ** -24 * size)
        ref_codes, ref_scales = codec.quantize_transformed(grads.cpu().numpy(), 0, 128)
        np.testing.assert_array_equal(codes.cpu().numpy(), ref_codes)
        np.testing.assert_array_equal(scales.cpu().numpy(), ref_scales)
        np.testing.assert_array_equal(mean.cpu().numpy(), codec.reduce_local(ref_codes, ref_scales, 0, 128))
        want2 = codec.round_trip(g2.cpu().numpy(), fA, None, 0, 128)
        assert np.linalg.norm(out2.cpu().numpy() - want2) <= 2e-3 * np.linalg.norm(want2)
        # norm, clip, step
        averaged = [mean.cpu().numpy(), out2.cpu().numpy()]
        n, coef = train.grad_norm(averaged, MAX_NORM)
        got_n, got_c = norm.cpu().numpy()
        assert abs(got_n - n) <= 2.0 ** -23 * n and abs(got_c - coef) <= 2.0 ** -23 * coef and coef < 1
        for k, (p, gr, at, decay) in enumerate(zip((table, w2), averaged, opt.starts, (0.0, 0.1))):
            flat, count = gr.ravel(), gr.size
            if moments == "f32":
                old = [state[x][at:at + count] for x in "mv"]
            else:
                old = [train.decode_moment(state[x][at:at + count], state[x + "_scales"][at // 256:at // 256 + -(-count // 256)])
                       for x in "mv"]
            m, v = train.adamw_moments(*old, flat, 0.9, 0.95, got_c)
            got = p.cpu().numpy()
            if moments == "f32":
                want_p = train.adamw_param(before[k].ravel(), m, v, LR, 0.9, 0.95, 1e-8, decay, step)
                np.testing.assert_array_equal(got.ravel(), want_p)
                np.testing.assert_array_equal(opt.state["m"][at:at + count].cpu().numpy(), m)
            else:
                r = train.random_numbers(count, k, step, 9)
                for x, values, keep in (("m", m, False), ("v", v, True)):
                    c, s = train.stochastic_codes(values, r, keep)
                    np.testing.assert_array_equal(opt.state[x][at:at + count].cpu().numpy(), c)
                    np.testing.assert_array_equal(opt.state[x + "_scales"][at // 256:at // 256 + s.size].cpu().numpy(), s)
                # (the step's own float32 bound is pinned where it is tested alone: here 2^-18 of an update of at most
                # 10 lr, the first steps' |m| / sqrt(v) after bias correction being below 10)
                want_p, _, _ = train.adamw_formula(before[k].ravel(), *old, flat, LR, 0.9, 0.95, 1e-8, decay, step, float(got_c))
                assert np.all(np.abs(got.ravel() - want_p) <= 2.0 ** -22 * np.abs(want_p) + 2.0 ** -18 * 10 * LR)
            np.testing.assert_array_equal(bits(copies[k]), train.to_bf16(got).reshape(got.shape))
        old_copy = copies[0].float().cpu().numpy()
    factor.close()
    ctx.close()
