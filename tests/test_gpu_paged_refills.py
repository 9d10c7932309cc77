"""Paged steps whose refills bring more rows than a pass carries: each request against a standalone oracle run, teacher-forced, as in the tests of paged steps."""
import numpy as np
import pytest

import dmtd_inputs as di
import paper_2510_11958_amd as pkg
from oracle import dmtd_oracle as O
from parity_util import engine_config, norm_err, oracle_config
from test_gpu_paged_steps import SHAPES, TOL

pytestmark = pytest.mark.gpu


class Requests:
    def __init__(self, name, lengths, page, n_late, literal):
        """lengths: tokens that each request has room for."""
        self.sh, self.n_late, self.page = SHAPES[name], n_late, page
        blob = di.make_weight_blob(self.sh, seed=5, gain_sigma=0.2)
        self.room = max(lengths)
        self.eng = pkg.Engine(engine_config(self.sh, self.room, len(lengths), full_pos_add_embed=literal), blob)
        ocfg = oracle_config(self.sh, full_pos_add_embed=literal)
        w = O.unpack_weights(blob, ocfg, np.float64)
        self.orcs = [O.DmtdOracle(ocfg, w, self.room + 1) for _ in lengths]
        self.text = [di.make_prompts(self.sh.vocab, 1, n, seed=50 + i)[0] for i, n in enumerate(lengths)]
        self.at, self.worst = [0] * len(lengths), 0.0
        self.eng.paged_begin(page)

    def step(self, work, full):
        """work: (slot, new tokens); full: of all of them, or the slots of which.  A first step is a prompt's."""
        fulls = [bool(full) if isinstance(full, bool) else s in full for s, _ in work]
        toks = [self.text[s][self.at[s]:self.at[s] + n] for s, n in work]
        self.eng.paged_step([s for s, _ in work], toks, [int(f) for f in fulls], self.n_late)
        z = self.eng.logits()
        for j, (s, n) in enumerate(work):
            o = self.orcs[s]
            if self.at[s] == 0:
                o.prefill(toks[j], self.n_late)
            else:
                for i, t in enumerate(toks[j]):          # tau 1: a full step; a cycle without end: a late-only one
                    o.decode_cycle(1 if fulls[j] else 1 << 20, self.n_late, max_new=1, forced=[int(t)])
                    assert not fulls[j] or n == 1
            self.at[s] += n
            self.worst = max(self.worst, norm_err(z[j], o.last_logits.astype(np.float64)))
            state = self.eng.paged_state(s)
            assert (state["n_tok"], state["n_front"]) == (o.n_tok, o.n_front)
        assert state["free_pages"] == len(self.at) * self.room // self.page - sum(-(-n // self.page) for n in self.at)
        assert self.worst < TOL[self.sh.dtype], self.worst


@pytest.mark.parametrize("page, literal, n_late", [(16, False, 2), (32, True, 1), (256, False, 1)])
def test_refills_of_several_passes(page, literal, n_late):
    """An fp32 model's pass carries 128 rows: refills of 192 (two parts) beside 62 (with the second part), then of 300 (three parts) between others that fit, and one of 128."""
    r = Requests("fp32", [512, 512, 512], page, n_late, literal)
    r.step([(0, 20), (1, 7), (2, 50)], True)
    r.step([(0, 101), (2, 3)], False)
    r.step([(0, 90), (1, 30)], False)
    r.step([(1, 31)], False)
    r.step([(1, 1), (0, 1), (2, 1)], True)          # 62, 192, 4
    r.step([(2, 1), (0, 1)], True)
    for n in (128, 128, 43):
        r.step([(1, n)], False)
    r.step([(0, 100)], False)
    r.step([(2, 127)], False)
    r.step([(0, 1), (1, 1)], True)                  # 101, 300; slot 2's wait
    r.step([(2, 1)], True)                          # 128
    r.step([(0, 1), (1, 1), (2, 1)], False)
    r.step([(0, 1), (1, 1), (2, 1)], True)


def test_a_refill_of_several_requests():
    """A bf16 model's pass carries 2048 rows: six refills of 441, four in one pass and two in the next."""
    r = Requests("bf16_hd64", [512] * 6, 64, 1, False)
    r.step([(s, 10 + s) for s in range(6)], True)
    r.step([(s, 440) for s in (3, 0, 5)], False)
    r.step([(s, 440) for s in (1, 2, 4)], False)
    r.step([(s, 1) for s in (5, 4, 3, 2, 1, 0)], True)
    r.step([(s, 1) for s in range(6)], False)
    r.step([(s, 1) for s in (0, 3)], True)


@pytest.mark.parametrize("literal", [False, True])
def test_a_refill_of_one_long_request(literal):
    """Of 2101 rows, in parts of 2048 and 53, the second of which takes another request's."""
    r = Requests("bf16", [2300, 2300], 16, 2, literal)
    r.step([(1, 5), (0, 9)], True)
    r.step([(0, 2000)], False)
    r.step([(0, 100), (1, 3)], False)
    r.step([(0, 1), (1, 1)], True)
    r.step([(0, 1), (1, 1)], False)
    r.step([(1, 1), (0, 1)], True)


@pytest.mark.parametrize("literal", [False, True])
@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_refills_beside_late_only_rows(name, literal):
    """Late-only rows of some requests, in front of, between and behind those whose refills take several passes; n_late = all layers: none take any."""
    room, most = (400, 100) if name == "fp32" else (700, 600)          # a pass: 128 rows, 2048
    for n_late in (2, SHAPES[name].n_layers):
        r = Requests(name, [room] * 6, 16, n_late, literal)
        r.step([(s, 5 + s) for s in range(6)], True)
        for s in range(6):
            r.step([(s, most)], False)
        if name == "fp32":
            r.step([(1, 90)], False)
        r.step([(0, 2), (1, 1), (2, 3), (3, 1), (4, 1), (5, 4)], {1, 3, 4})
        r.step([(5, 1), (4, 1), (2, 1), (0, 1)], {5, 0, 2})
        r.step([(s, 1) for s in range(6)], False)
        r.step([(s, 1) for s in range(6)], True)
