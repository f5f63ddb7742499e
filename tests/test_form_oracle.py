"""The numpy oracle of students with a form of attention against the C oracle of the plain ones."""
import numpy as np

from oracle import sp_form_oracle
from oracle.sp_oracle import OracleConfig
from paper_2408_12526_amd import sp, synth


def test_plain_form_is_the_plain_forward(oracle64):
    s = synth.StudentShape(K=2, layers=2, hidden=128, heads=2, ffn=256, vocab=50, max_pos=40, classes=3)
    rng = np.random.default_rng(0)
    blob = synth.make_weights(rng, s, std=0.05, ln_random=True, qk_std=0.2)
    lengths = np.array([7, 1, 40], np.int32)
    ids, cu = synth.make_ids(rng, int(lengths.sum()), s.vocab), sp.sp_pack(lengths)
    cfg = OracleConfig(s.K, s.layers, s.hidden, s.heads, s.ffn, s.vocab, s.max_pos, s.classes, s.ln_eps)
    want = oracle64.forward(cfg, blob, ids, cu, 2)
    got = sp_form_oracle.forward([synth.student_views(blob, s, m) for m in range(2)], s.heads, s.layers, s.ln_eps, ids, cu, 2)
    assert np.abs(got - want).max() < 1e-10
    far = sp_form_oracle.forward([synth.student_views(blob, s, m) for m in range(2)], s.heads, s.layers, s.ln_eps, ids, cu, 2, window=(2, 2))
    assert np.abs(far - want).max() > 1e-4
