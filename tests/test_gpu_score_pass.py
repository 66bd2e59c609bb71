"""Engine.score_pass of passes that failed, and of tokens that are no 32-bit numbers."""
import numpy as np
import pytest

from s2d2_inputs import generate_prompts, generate_weights, get_config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["t_bf16_128", "t_f32"])
def test_scores_of_a_verifier_pass_that_timed_out_are_refused(name):
    from paper_2603_25702_b200 import Engine, S2D2Error
    wl = get_config(name)
    eng = Engine(wl.model, block_size=wl.block_size, max_batch=wl.batch, max_seq_len=256, kv_page_tokens=wl.kv_page_tokens, seed=1)
    eng.load_weights(generate_weights(wl.model, seed=0))
    ids = eng.prefill(generate_prompts(wl))

    def code(fn, *a):
        with pytest.raises(S2D2Error) as e:
            fn(*a)
        return e.value.code

    st = eng.draft_block(ids)
    n = sum(s.n_masked for s in st)
    assert code(eng.score_pass, 1, 1) == -4                          # no verifier pass yet
    eng.verify_block(ids, [1] * len(ids))
    draft = eng.score_pass(0, n, None, 5)
    eng.score_pass(1, 1)
    eng.debug_set_status(10)                                         # as a verifier pass leaves it that gave up on a wait
    assert code(eng.score_pass, 1, 1) == -5
    assert code(eng.score_pass, 1, 1) == -5                          # still
    again = eng.score_pass(0, n, None, 5)                            # the draft pass was checked when it returned
    assert all(np.array_equal(draft[k], again[k]) for k in draft)
    assert code(eng.accept_and_commit, ids, [1] * len(ids)) == -5    # not taken away from the step
    assert code(eng.score_pass, 1, 1) == -4                          # reported: those logits stay invalid
    again = eng.score_pass(0, n, None, 5)
    assert all(np.array_equal(draft[k], again[k]) for k in draft)
    eng.accept_and_commit(ids, [1] * len(ids))
    st = eng.draft_block(ids)
    n = sum(s.n_masked for s in st)
    eng.verify_block(ids, [1] * len(ids))
    for which in (0, 1):                                             # passes that succeed are scored again
        x = eng.debug_copy_logits(which, n).astype(np.float64)
        m = x.max(axis=1, keepdims=True)
        lse = (m + np.log(np.exp(x - m).sum(axis=1, keepdims=True)))[:, 0]
        # 32-bit sums of at most 4096 terms, tests of the scores themselves bound them closer
        assert np.abs(eng.score_pass(which, x.shape[0])["lse"] - lse).max() <= 4096 * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse).max()
    eng.accept_and_commit(ids, [1] * len(ids))
    # a draft pass that times out is reported by draft_block, and has no scores
    eng.debug_set_status(10)
    assert code(eng.draft_block, ids) == -5
    assert code(eng.score_pass, 0, 1) == -4
    st = eng.draft_block(ids)
    n = sum(s.n_masked for s in st)
    got = eng.score_pass(0, n, np.full(n, 2 ** 32 + 1))
    assert np.isfinite(got["lse"]).all() and np.isnan(got["logprob"]).all() and (got["rank"] == -1).all()
    eng.close()
