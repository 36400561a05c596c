"""The LM head's other objectives on the GPU under bounds without room for cancellation: labels, weights, caps and a second exponential
beside each other on every tile of the forward, teachers stored in bfloat16, and the weights' gradient from parts of the rows in large tiles."""
from functools import partial

import pytest

import paper_2407_15892_amd as mst
from tests import test_gpu_objective_edges as edges
from tests.objective_gpu_harness import Problem, Run
from tests.objective_tight_bounds import check

pytestmark = pytest.mark.gpu

SIZES = [(20, 64, 300), (130, 72, 9000), (200, 72, 12800), (400, 72, 12800), (1500, 64, 12800)]      # tiles of 64 x 32, of 256 x 32, 64, 128 and 256


def run_and_check(p):
    r = Run(p)
    r.forward()
    r.backward()
    print(check(p, r.outputs(), p.oracle()))
    return r


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("o", [
    dict(K=40, tail=True),
    dict(K=40, tail=True, label_coef=0.5, temperature=2.0, weights=True),
    dict(K=64, tail=True, label_coef=0.3, teacher_coef=0.7, temperature=4.0, softcap=30.0),
    dict(K=70, label_coef=0.5, temperature=0.5, weights=True, softcap=8.0),
    dict(K=5, tail=True, label_coef=0.25, temperature=3.0, softcap=50.0, weights=True, divisor=12345),
    dict(weights=True, z_coef=1e-3, softcap=30.0),
    dict(z_coef=1e-2, divisor=77),
], ids=str)
def test_outputs_gradients_and_the_loss_of_their_sum(S, d, V, o):
    run_and_check(Problem(S, d, V, **o))


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("K", [1, 20, 64, 100, 256])
@pytest.mark.parametrize("tail", [False, True])
def test_teachers_in_bfloat16(S, d, V, K, tail):
    p = Problem(S, d, V, K=K, tail=tail, label_coef=0.5, temperature=2.0, weights=True, teacher="bf16")
    run_and_check(p)


EDGES = {name: getattr(edges, name) for name in (
    "test_an_index_that_comes_twice_counts_once", "test_what_is_not_asked_for_may_hold_anything", "test_labels_that_only_count", "test_all_entries_in_one_tile",
    "test_teacher_that_gives_more_than_1", "test_rows_of_weight_zero", "test_ignore_index_that_is_an_entry_of_the_vocabulary",
    "test_values_that_are_not_finite_stay_in_their_rows", "test_calls_repeat_bit_by_bit_and_share_nothing", "test_a_captured_step_follows_its_inputs")}
EDGES.update({"test_logits_of_minus_infinity-%s" % t: partial(edges.test_logits_of_minus_infinity, tail=t) for t in (False, True)})
EDGES.update({"test_indices_out_of_range-%s" % b: partial(edges.test_indices_out_of_range, bad=b) for b in ("label", "entry", "far entry")})
EDGES.update({"test_masks_of_the_lowest_value_and_shares_that_are_next_to_nothing-%s-%s" % (t, T):
              partial(edges.test_masks_of_the_lowest_value_and_shares_that_are_next_to_nothing, tail=t, temperature=T)
              for t in (False, True) for T in (0.02, 1.0)})


@pytest.mark.parametrize("S,d,V,rows", [(130, 72, 9000, 32), (200, 72, 12800, 64), (400, 72, 12800, 128)])
@pytest.mark.parametrize("name", EDGES)
def test_edges_on_the_tiles_in_between(name, S, d, V, rows):
    """More tiles of 32 x 256 than half of the compute units, and not yet one of 256 x 256 for each."""
    assert mst.mst_forward_tile_rows(S, d, V, 1) == rows and -(-S // 32) * -(-V // 256) > 128
    EDGES[name](S=S, d=d, V=V)


@pytest.mark.parametrize("S,d,V", [(12289, 264, 1153), (13001, 280, 1473), (16384, 512, 1000)])
@pytest.mark.parametrize("o", [dict(K=7, tail=True, label_coef=0.5, temperature=2.0, weights=True), dict(softcap=4.0, z_coef=1e-3, weights=True)],
                         ids=["distill", "wce"])
def test_weights_gradient_from_parts_of_the_rows_in_large_tiles(S, d, V, o):
    """16 to 22 parts in tiles of 256 x 256, the last one short; vocabulary and hidden size on a tile's edge or not.  Launches that are counted
    under dH's reduce: the sum of dW's parts, for distillation the entries; dH itself is in one part."""
    p = Problem(S, d, V, **o)
    r = Run(p)
    r.forward()
    mst.mst_profile_enable(1)
    try:
        r.backward()
        r.torch.cuda.synchronize()
        counts = {k: v[2] for k, v in mst.mst_profile_collect().items()}
    finally:
        mst.mst_profile_enable(0)
    assert counts["bwd_gemm_dw"] == 1 and counts["bwd_dh_reduce"] == (2 if p.K else 1), counts
    first = r.dW.clone()
    r.backward(M=S // 300)
    assert r.torch.equal(first, r.dW)
    print(check(p, r.outputs(), p.oracle()))
