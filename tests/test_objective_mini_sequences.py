"""Host side of the LM head's other objectives: mini-sequences that are made of a call's M.  No kernel is launched here."""
import os

import pytest

import paper_2407_15892_amd as mst


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(mst.binding.LIB_PATH):
        from paper_2407_15892_amd.build import build
        build()


# few logits a row and many rows of a long hidden size: by the logits alone one mini-sequence would do, whose rows x d are 2^30 or more
LONG = [(131072, 8192, 512, 2), (131072, 8192, 512, 128), (262144, 4096, 256, 256), (131073, 8192, 512, 2), (1 << 20, 1024, 8, 2), (1 << 18, 65536, 8, 300)]


@pytest.mark.parametrize("S,d,V,M", LONG)
@pytest.mark.parametrize("K", [0, 8])
def test_a_mini_sequence_stays_within_the_limits_of_its_offsets(S, d, V, M, K):
    plain = mst.mst_workspace_bytes(S, d, V, M)                        # the caller's M is a valid one
    fwd, bwd, saved = mst.mst_objective_bytes(S, d, V, M, K)
    rows = -(-S // M)
    assert rows * d < 1 << 30 and bwd >= plain[1]
    most = ((1 << 30) - 1) // d                                        # rows of the longest mini-sequence there may be
    assert bwd == 4 * V * -(-S // -(-S // most))


@pytest.mark.parametrize("S,d,V,M", [(131072, 8192, 512, 1), (1 << 18, 65536, 8, 10)])
def test_a_call_that_leaves_no_valid_mini_sequence_is_refused(S, d, V, M):
    for call in (lambda: mst.mst_workspace_bytes(S, d, V, M), lambda: mst.mst_objective_bytes(S, d, V, M)):
        with pytest.raises(mst.MstError) as e:
            call()
        assert e.value.status == -2


@pytest.mark.parametrize("d", [0, -8])
def test_no_hidden_size_is_refused(d):
    with pytest.raises(mst.MstError) as e:
        mst.mst_objective_bytes(64, d, 100, 1)
    assert e.value.status == -2


@pytest.mark.gpu
@pytest.mark.parametrize("K", [0, 8])
def test_rows_of_two_long_mini_sequences(K):
    """Outputs and gradients are those of calls of half of the rows each."""
    import torch
    S, d, V = 131072, 8192, 512
    g = torch.Generator(device="cuda").manual_seed(11)
    H = torch.empty((S, d), dtype=torch.bfloat16, device="cuda")
    for r in range(0, S, 16384):
        H[r:r + 16384] = torch.randn((16384, d), generator=g, device="cuda")
    W = (torch.randn((V, d), generator=g, device="cuda") * 2 / d ** 0.5).bfloat16()
    labels = torch.randint(0, V, (S,), generator=g, device="cuda", dtype=torch.int32)
    labels[::7] = -100
    index = torch.randint(-1, V, (S, K), generator=g, device="cuda", dtype=torch.int32)
    logits, teacher_lse = torch.randn((S, K), generator=g, device="cuda"), torch.full((S,), 6.0, device="cuda")

    def call(rows, M):
        n = rows.stop - rows.start
        f, b, sv = mst.mst_objective_bytes(n, d, V, M, K)
        ws, saved = (torch.empty(x, dtype=torch.uint8, device="cuda") for x in (max(f, b), sv))
        loss, nll, other = torch.empty(1, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        dH, dW = torch.empty((n, d), dtype=torch.bfloat16, device="cuda"), torch.empty((V, d), device="cuda")
        if K:
            mst.mst_lmhead_distill_fwd(H[rows], W, index[rows], logits[rows], M, ws, loss, saved=saved, teacher_lse=teacher_lse[rows],
                                       labels=labels[rows], label_coef=0.5, divisor=S, nll=nll, kd=other)
            mst.mst_lmhead_distill_bwd(H[rows], W, K, M, 1.0, saved, ws, dH, dW)
        else:
            mst.mst_lmhead_wce_fwd(H[rows], W, labels[rows], -100, M, ws, loss, saved=saved, divisor=S, nll=nll, lse=other)
            mst.mst_lmhead_wce_bwd(H[rows], W, M, 1.0, saved, ws, dH, dW)
        return loss.double().item(), nll, other, dH, dW

    whole = call(slice(0, S), 2)
    parts = [call(slice(a, a + S // 2), 1) for a in (0, S // 2)]
    assert abs(whole[0] - sum(p[0] for p in parts)) <= 8 * 2.0 ** -24 * sum(p[0] for p in parts)
    assert torch.equal(whole[1], torch.cat([p[1] for p in parts])) and torch.equal(whole[2], torch.cat([p[2] for p in parts]))
    for a, part in zip((0, S // 2), parts):
        for r in range(0, S // 2, 16384):
            dH, ref = whole[3][a + r:a + r + 16384].double(), part[3][r:r + 16384].double()
            # the same logits' gradient, another split of the contraction and a bf16 rounding each: two half steps and little more
            assert ((dH - ref).abs() <= 2 * 2.0 ** -8 * ref.abs() + 2.0 ** -12 * ref.abs().amax(1, keepdim=True)).all()
    # dW: the same terms in other float32 sums, chains of at most 4096 additions of 32 products each.  Every one rounds a partial sum, none of
    # which is much larger than the row's largest entry, by half a step at most; independent of each other 4 sqrt(4096) half steps, on both sides
    dW = sum(p[4].double() for p in parts)
    assert ((whole[4].double() - dW).abs() <= 2 * 4 * 64 * 2.0 ** -24 * dW.abs().amax(1, keepdim=True)).all()
