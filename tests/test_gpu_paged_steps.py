"""Paged steps of a context: requests that come and go, each compared with a standalone oracle run of its own (rows of different requests do not mix), teacher-forced, every
step's logits and every token where the oracle's margin allows."""
import ctypes as C

import numpy as np
import pytest

import dmtd_inputs as di
import paper_2510_11958_amd as pkg
from oracle import dmtd_oracle as O
from parity_util import MARGIN, engine_config, norm_err, oracle_config, top2_margin

TOL = {"fp32": 1e-4, "bf16": 2e-2}      # of the other parity tests: the same kernels but for the attention, whose sums are as exact

SHAPES = {
    "fp32": di.ModelShape(4, 128, 4, 2, 64, 192, 130, dtype="fp32"),
    "bf16": di.ModelShape(4, 256, 8, 2, 128, 512, 1000, dtype="bf16"),
    "bf16_hd64": di.ModelShape(3, 256, 4, 2, 64, 512, 700, dtype="bf16"),
}


class Server:
    """The engine, and per slot an oracle, the request's whole token string, its cycle length and how far it is."""

    def __init__(self, name, slots, max_seq_len, page, n_late, literal=False, seed=5):
        self.sh, self.n_late, self.literal, self.max_seq_len = SHAPES[name], n_late, literal, max_seq_len
        blob = di.make_weight_blob(self.sh, seed=seed, gain_sigma=0.2)
        self.eng = pkg.Engine(engine_config(self.sh, max_seq_len, slots, full_pos_add_embed=literal), blob)
        self.ocfg = oracle_config(self.sh, full_pos_add_embed=literal)
        self.w = O.unpack_weights(blob, self.ocfg, np.float64)
        self.eng.paged_begin(page)
        self.req, self.worst, self.checked = {}, 0.0, 0

    def arrive(self, slot, prompt_len, tau, total, seed):
        text = di.make_prompts(self.sh.vocab, 1, total, seed=seed)[0]
        self.req[slot] = dict(text=text, prompt=prompt_len, tau=tau, at=0, phase=0, orc=O.DmtdOracle(self.ocfg, self.w, self.max_seq_len + 1))

    def leave(self, slot):
        self.eng.paged_release(slot)
        del self.req[slot]

    def step(self, work):
        """work: (slot, tokens to bring; for a request past its prompt 1).  Compares the logits of every request whose last token is one the oracle answers."""
        slots, toks, full = [], [], []
        for slot, count in work:
            r = self.req[slot]
            slots.append(slot)
            toks.append(r["text"][r["at"]:r["at"] + count])
            if r["at"] < r["prompt"]:
                assert r["at"] + count <= r["prompt"]
                full.append(1)
            else:
                full.append(1 if r["phase"] >= r["tau"] else 0)
                r["phase"] = 1 if full[-1] else r["phase"] + 1
        out = self.eng.paged_step(slots, toks, full, self.n_late)
        z = self.eng.logits()
        assert z.shape == (len(slots), self.sh.vocab)
        for j, (slot, count) in enumerate(work):
            r = self.req[slot]
            in_prompt = r["at"] < r["prompt"]
            r["at"] += count
            assert int(out[j]) == int(np.argmax(z[j]))
            if in_prompt:
                if r["at"] < r["prompt"]:
                    continue
                r["orc"].prefill(r["text"][:r["prompt"]], self.n_late)
                r["phase"] = 1
            else:
                r["orc"].decode_cycle(r["tau"], self.n_late, max_new=1, forced=[int(r["text"][r["at"] - 1])])
            ref = r["orc"].last_logits.astype(np.float64)
            self.worst = max(self.worst, norm_err(z[j], ref))
            if top2_margin(ref) > MARGIN:
                assert int(out[j]) == int(np.argmax(ref)), (slot, r["at"])
                self.checked += 1
            s = self.eng.paged_state(slot)
            assert (s["n_tok"], s["n_front"]) == (r["orc"].n_tok, r["orc"].n_front)

    def done(self):
        assert self.worst < TOL[self.sh.dtype], self.worst


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("page, literal, n_late", [(16, False, 2), (32, True, 1), (256, False, 1)])
def test_requests_come_and_go(name, page, literal, n_late):
    s = Server(name, 5, 300, page, n_late, literal)
    s.arrive(3, 20, 3, 120, 11)
    s.step([(3, 20)])
    for _ in range(4):
        s.step([(3, 1)])
    s.arrive(0, 70, 1, 200, 12)                          # a long prompt in chunks beside the first request's tokens
    s.arrive(4, 1, 2, 60, 13)                            # a prompt of one token
    s.step([(0, 33), (3, 1), (4, 1)])
    s.step([(4, 1), (0, 36)])
    s.step([(3, 1), (0, 1), (4, 1)])
    for _ in range(5):
        s.step([(4, 1), (3, 1), (0, 1)])
    s.leave(3)
    s.arrive(3, 130, 4, 250, 14)                         # its slot again
    s.arrive(1, 17, 5, 80, 15)
    s.step([(1, 17), (3, 100), (0, 1), (4, 1)])          # (an fp32 model's pass carries 128 rows)
    s.step([(3, 30), (4, 1)])
    for _ in range(11):
        s.step([(0, 1), (1, 1), (3, 1), (4, 1)])
    s.leave(0)
    s.step([(3, 1)])
    s.step([(1, 1), (3, 1)])
    s.done()
    assert s.checked > 20


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_all_layers_late(name):
    """n_late = all layers: nothing passes the front layers; the literal reading adds the embedding once more at full positions."""
    for literal in (False, True):
        s = Server(name, 2, 100, 16, SHAPES[name].n_layers, literal)
        s.arrive(0, 30, 2, 60, 21)
        s.arrive(1, 5, 3, 60, 22)
        s.step([(1, 5), (0, 30)])
        for _ in range(6):
            s.step([(0, 1), (1, 1)])
        s.done()


@pytest.mark.gpu
def test_many_rows():
    """A step of more than 192 rows: the wide projections' layout of rows."""
    s = Server("bf16", 3, 600, 64, 2)
    s.arrive(0, 500, 2, 520, 31)
    s.arrive(1, 210, 3, 300, 32)
    s.arrive(2, 9, 1, 60, 33)
    s.step([(2, 9)])
    s.step([(0, 400), (1, 210), (2, 1)])
    s.step([(0, 100), (1, 1), (2, 1)])
    for _ in range(4):
        s.step([(0, 1), (1, 1), (2, 1)])
    s.done()


@pytest.mark.gpu
def test_many_requests():
    """More requests than the tiled projections' rows: single tokens, and the head, in the wide layout of rows; the slots named out of order."""
    n = 200
    s = Server("bf16", n, 32, 16, 2)
    for slot in range(n):
        s.arrive(slot, 1 + slot % 3, 1 + slot % 4, 12, 100 + slot)
    order = np.random.RandomState(3).permutation(n).tolist()
    s.step([(slot, s.req[slot]["prompt"]) for slot in order])
    for _ in range(3):
        s.step([(slot, 1) for slot in order])
    s.step([(slot, 1) for slot in order if slot % 50 != 7])          # 196 of them
    for slot in order[:9]:
        s.leave(slot)
    s.step([(slot, 1) for slot in order[9:]])                        # 191
    s.done()


@pytest.mark.gpu
def test_pool_and_slots_run_out():
    s = Server("fp32", 3, 64, 16, 2)                    # 12 pages
    eng = s.eng
    assert eng.paged_state(0) == {"n_tok": 0, "n_front": 0, "free_pages": 12}
    s.arrive(0, 60, 2, 64, 41)
    s.arrive(1, 60, 2, 64, 42)
    s.arrive(2, 33, 2, 64, 43)
    s.step([(0, 60)])
    s.step([(1, 60)])
    s.step([(2, 33)])
    assert eng.paged_state(2)["free_pages"] == 1

    def refused(code, slots, toks, full, n_late=2):
        before = [eng.paged_state(i) for i in range(3)]
        with pytest.raises(pkg.DmtdError) as e:
            eng.paged_step(slots, toks, full, n_late)
        assert e.value.code == code
        assert [eng.paged_state(i) for i in range(3)] == before

    refused(pkg.DMTD_ECAPACITY, [0], [[1] * 5], [1])                  # max_seq_len
    refused(pkg.DMTD_EINVAL, [0, 0], [[1], [1]], [1, 1])
    refused(pkg.DMTD_EINVAL, [3], [[1]], [1])
    refused(pkg.DMTD_EINVAL, [0], [[130]], [1])
    refused(pkg.DMTD_EINVAL, [0, 1], [[1], []], [1, 1])
    refused(pkg.DMTD_EINVAL, [0], [[1]], [1], n_late=5)
    s.step([(0, 1)])                                                  # a late-only step
    refused(pkg.DMTD_ESTATE, [0], [[1]], [1], n_late=1)               # a token awaits its refill
    s.step([(0, 1), (1, 1), (2, 1)])
    s.leave(1)
    assert eng.paged_state(0)["free_pages"] == 5
    s.arrive(1, 64, 2, 64, 44)
    s.step([(1, 64)])
    for _ in range(2):
        s.step([(0, 1), (2, 1)])
    s.done()
    with pytest.raises(pkg.DmtdError):
        eng.paged_release(3)
    for call in (lambda: eng.prefill(np.ones((1, 4))), lambda: eng.masked_forward(np.ones((1, 4)), np.ones(4), 2), lambda: eng.read_kv(0, 0, 4),
                 lambda: eng.set_n_early(1), lambda: eng.decode(2, 2, 1), lambda: eng.paged_begin(16)):
        with pytest.raises(pkg.DmtdError) as e:
            call()
        assert e.value.code == pkg.DMTD_ESTATE
    eng.set_sampling(1.0, 5, 1)
    refused(pkg.DMTD_ESTATE, [0], [[1]], [1])
    eng.set_sampling(0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_reset_gives_the_context_back(name):
    """Prefill and decoding behind paged steps and a reset are those of a fresh context, bit for bit; and paged steps can follow again."""
    sh = SHAPES[name]
    blob = di.make_weight_blob(sh, seed=7)
    prompt = di.make_prompts(sh.vocab, 2, 40, seed=8)

    def run(eng):
        first = eng.prefill(prompt)
        z0 = eng.logits()
        out = eng.decode(3, 2, 7)
        return first, z0, out, eng.logits()

    fresh = run(pkg.Engine(engine_config(sh, 128, 2), blob))
    eng = pkg.Engine(engine_config(sh, 128, 2), blob)
    for _ in range(2):
        eng.paged_begin(32)
        with pytest.raises(pkg.DmtdError):
            eng.logits()
        eng.paged_step([1, 0], [prompt[0][:30], prompt[1][:9]], [1, 1], 2)
        eng.paged_step([0], [[3]], [0], 2)
        assert eng.logits().shape == (1, sh.vocab)
        eng.reset()
        for a, b in zip(fresh, run(eng)):
            assert np.array_equal(a, b)
        eng.reset()


def test_paged_begin_refuses_without_a_gpu():
    cfg = pkg.ModelConfig(4, 64, 4, 2, 64, 96, 50, dtype="fp32", max_seq_len=64, dry_run=True)
    lib, cc = pkg.load_library(), cfg.to_c()
    assert lib.dmtd_paged_step_bytes(C.byref(cc), 16) > 0
    for page in (0, 8, 24, 512, -16):
        assert lib.dmtd_paged_step_bytes(C.byref(cc), page) == 0
    assert lib.dmtd_paged_step_bytes(C.byref(pkg.ModelConfig(**{**cfg.__dict__, "head_dim": 48}).to_c()), 16) == 0
    assert lib.dmtd_paged_step_bytes(C.byref(cc), 128) == 0            # 64 positions hold no page of 128
    eng = pkg.Engine(cfg)
    for call, code in ((lambda: eng.paged_begin(16), pkg.DMTD_ESTATE), (lambda: eng.paged_begin(8), pkg.DMTD_EINVAL),
                       (lambda: eng.paged_step([0], [[1]], [1], 2), pkg.DMTD_ESTATE), (lambda: eng.paged_release(0), pkg.DMTD_ESTATE), (lambda: eng.paged_state(0), pkg.DMTD_EINVAL)):
        with pytest.raises(pkg.DmtdError) as e:
            call()
        assert e.value.code == code
    assert lib.dmtd_paged_begin(None, 16, None, 0) == pkg.DMTD_EINVAL
    assert lib.dmtd_paged_step(None, 1, None, None, None, None, 1, None) == pkg.DMTD_EINVAL
    assert lib.dmtd_paged_release(None, 0) == pkg.DMTD_EINVAL
