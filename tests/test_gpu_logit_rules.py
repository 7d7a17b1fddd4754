"""Penalties, biases, masks and temperature on logits, with their log-sums and best tokens, against the oracle in 64 bits."""
from dataclasses import dataclass, replace

import numpy as np
import pytest
import torch

from oracle import draft_oracle as oracle
from paper_2510_11062_amd import api
from tests.rollout_case import DTYPES, U16, U32, assert_within, host64, i32, rounded, to_dev

TOKEN_RANGE, SEQLENS, RULE = 4, 8, 512


@dataclass
class Rows:
    """A batch on the host: None where there is no such rule."""
    logits: np.ndarray
    dtype: torch.dtype
    new: np.ndarray = None              # rows of each sequence; None: one
    tokens: list = None                 # a list for each sequence
    size: tuple = ()
    prompt: list = None                 # a list for each group
    drafted: np.ndarray = None
    parent: np.ndarray = None
    repetition: np.ndarray = None
    presence: np.ndarray = None
    frequency: np.ndarray = None
    temperature: np.ndarray = None
    bias: list = None                   # [(token, value), ..] for each sequence
    allowed: np.ndarray = None          # [masks, V]
    mask_row: np.ndarray = None

    @property
    def n_seq(self):
        return len(self.logits) if self.new is None else len(self.new)

    def start(self):
        return np.arange(self.n_seq + 1) if self.new is None else np.concatenate([[0], np.cumsum(self.new)]).astype(int)

    def ways(self):
        start = self.start()
        return [w for s in range(self.n_seq) for w in oracle.paths(self.parent[start[s]:start[s + 1]])[0]]

    def device(self, dev, spare=3, **over):
        """A LogitRules; lists stand in rows that are longer than they are, with tokens behind their ends that nobody counts."""
        f32 = lambda a: None if a is None else to_dev(a, torch.float32, dev)

        def lists(rows):
            m = np.zeros((len(rows), max([len(r) for r in rows] + [0]) + spare), np.int64)
            for r, row in zip(m, rows):
                r[:len(row)] = row
            return i32(m, dev), i32([len(r) for r in rows], dev)

        t = dict(cu_q=None if self.new is None else i32(self.start(), dev))
        if self.tokens is not None:
            t["tokens"], t["length"] = lists(self.tokens)
        if self.prompt is not None:
            t["prompt"], t["prompt_len"] = lists(self.prompt)
            t["group_seq"] = i32(np.concatenate([[0], np.cumsum(self.size)]), dev)
        if self.parent is not None:
            t["drafted"] = i32(self.drafted, dev)
            t["ancestors"] = torch.from_numpy(oracle.as_bits([sum(1 << i for i in w) for w in self.ways()])).to(dev)
        for name in ("repetition", "presence", "frequency", "temperature"):
            t[name] = f32(getattr(self, name))
        if self.bias is not None:
            flat = [e for row in self.bias for e in row]
            t["bias_cu"] = i32(np.concatenate([[0], np.cumsum([len(r) for r in self.bias])]), dev)
            t["bias_token"], t["bias"] = i32([e[0] for e in flat], dev), to_dev(np.array([e[1] for e in flat], dtype=np.float64), torch.float32, dev)
        if self.allowed is not None:
            m, V = self.allowed.shape
            bits = np.zeros((m, -(-V // 32) * 32), np.uint8)
            bits[:, :V] = self.allowed
            bits[:, V:] = 1      # behind the last token: nobody looks
            t["allowed"] = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).to(dev)
            t["mask_row"] = i32(self.mask_row, dev)
        t.update(over)
        return api.LogitRules(**t)

    def want(self):
        """The oracle's rows."""
        V = self.logits.shape[1]
        group = np.searchsorted(np.cumsum(self.size), np.arange(self.n_seq), side="right") if self.prompt is not None else None
        penalties = any(getattr(self, x) is not None for x in ("repetition", "presence", "frequency"))
        of = lambda name, s, other: other if getattr(self, name) is None else float(np.float32(getattr(self, name)[s]))
        start, ways = self.start(), self.ways() if self.parent is not None else None
        rows = []
        for s in range(self.n_seq):
            for t in range(start[s], start[s + 1]):
                prompt = self.prompt[group[s]] if group is not None and group[s] < len(self.prompt) else []
                behind = list(self.tokens[s]) if self.tokens is not None else []
                if ways is not None:
                    behind += [self.drafted[start[s] + i] for i in ways[t]]
                if not penalties:
                    prompt, behind = [], []
                inside = lambda x: [v for v in x if 0 <= v < V]
                bias = {v: float(np.float32(b)) for v, b in self.bias[s] if 0 <= v < V} if self.bias is not None else {}
                allowed = self.allowed[self.mask_row[t]] if self.allowed is not None and self.mask_row[t] >= 0 else None
                with np.errstate(invalid="ignore"):
                    rows.append(oracle.sampling_row(self.logits[t], inside(prompt), inside(behind), of("repetition", s, 1.0), of("presence", s, 0.0),
                                                    of("frequency", s, 0.0), of("temperature", s, 1.0), bias, allowed))
        return rows


def compare(o, want, out_dtype=None, what=""):
    """Every rounding on the way to out is one of 2^-24 of what is rounded (`size` adds those up; the temperature takes two), and out's own.
    lse: a shift of the exponents is one of lse.  The scale of the exponents is off by 3 roundings, the difference in them by one, of at most
    the largest |out|; a lane adds 32 terms, lanes and wavefronts 8 times, workgroups V / 8192 times, each of these one rounding of
    the sum, and so do exponential and logarithm (one unit, two roundings each).  best: within the error of the largest."""
    for t, (out, lse, best, size) in enumerate(want):
        real = np.isfinite(out)
        bound = 1.01 * U32 * size + 1e-37
        if "out" in o and o["out"] is not None:
            got = host64(o["out"][t])
            assert np.array_equal(np.isnan(got), np.isnan(out)) and np.array_equal(np.isinf(got), np.isinf(out)), f"{what} row {t}"
            inf = np.isinf(out)
            assert np.array_equal(got[inf], out[inf]), f"{what} row {t}"
            own = bound[real] + (U16 * (np.abs(out[real]) + bound[real]) if o["out"].dtype == torch.bfloat16 else 0)
            assert_within(got[real], out[real], own, f"{what} row {t}")
        if o.get("lse") is not None:
            got = float(o["lse"][t])
            if not np.isfinite(lse):
                assert got == lse or (np.isnan(got) and np.isnan(lse)), f"{what} row {t}: {got} for {lse}"
            else:
                most = np.abs(out[real]).max()
                assert abs(got - lse) <= bound[real].max() + U32 * (8 * most + 50 + len(out) / 8192 + 8 * abs(lse)), f"{what} row {t}: {got} for {lse}"
        if o.get("best") is not None:
            got = int(o["best"][t])
            if best < 0:
                assert got == -1, f"{what} row {t}"
            else:
                near = 2 * bound[best] if np.isfinite(out[best]) else 0
                assert got == best or (got >= 0 and out[got] >= out[best] - near - 2 * bound[got] and out[got] != out[best]), f"{what} row {t}: {got} for {best}"


def apply(r, dev, **kw):
    rules = r.device(dev)
    return api.at_grpo_logit_rules(rules, to_dev(r.logits, r.dtype, dev), **kw)


def draw(rs, dtype, V, n_seq, new=None, size=(), own=40, prompt=60, biases=5, masks=3, penalties=True, temperature=True):
    dtype = DTYPES[dtype]
    n = n_seq if new is None else int(sum(new))
    r = Rows(rounded(rs.normal(size=(n, V)) * 3, dtype), dtype, None if new is None else np.array(new))
    r.tokens = [rs.integers(0, V, rs.integers(0, own + 1)) for _ in range(n_seq)]
    if len(size):
        r.size, r.prompt = size, [rs.integers(0, V, rs.integers(0, prompt + 1)) for _ in size]
    if new is not None:
        r.drafted = rs.integers(0, V, n)
        r.parent = np.concatenate([[j - rs.integers(1, j + 1) if j else -1 for j in range(m)] for m in new]).astype(int)
    if penalties:
        r.repetition, r.presence, r.frequency = rs.uniform(0.8, 1.6, n_seq), rs.uniform(-0.3, 1, n_seq), rs.uniform(-0.2, 0.7, n_seq)
    if temperature:
        r.temperature = rs.uniform(0.3, 2, n_seq)
    if biases:
        r.bias = [[(int(rs.integers(0, V)), float(rs.normal() * 3)) for _ in range(rs.integers(0, biases + 1))] for _ in range(n_seq)]
    if masks:
        r.allowed = rs.random((masks, V)) < rs.choice([0.01, 0.5, 0.97], (masks, 1))
        r.mask_row = rs.integers(-1, masks, n)
    return r


SIZES = [1, 7, 8, 31, 33, 100, 2047, 2048, 2049, 8191, 8192, 8193, 20001]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", SIZES)
def test_against_the_oracle(gpu_device, dtype, V):
    rs = np.random.default_rng(V)
    for new, size in ((None, (2, 0, 3)), ([3, 1, 0, 8, 2], (1, 3)), ([64, 70], ()), ([1], (1,))):
        n_seq = 5 if new is None else len(new)
        if new == [64, 70]:      # only the first 64 of a sequence's tokens have bits
            r = draw(rs, dtype, V, n_seq, [64, 60], size)
        else:
            r = draw(rs, dtype, V, n_seq, new, size)
        word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
        want = r.want()
        compare(apply(r, gpu_device, data_error=word), want, what=f"{new}")
        compare(apply(r, gpu_device, out_dtype=torch.float32), want, what=f"{new} to float32")
        assert int(word) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_large_vocabulary(gpu_device, dtype):
    r = draw(np.random.default_rng(1), dtype, 151936, 4, [2, 1, 1, 3], (1, 3), own=3000, prompt=9000, biases=300)
    compare(apply(r, gpu_device), r.want())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rule", ["repetition", "presence", "frequency", "temperature", "bias", "allowed", "none", "tokens", "prompt", "parent"])
def test_one_rule_alone(gpu_device, dtype, rule):
    rs = np.random.default_rng(len(rule))
    r = draw(rs, dtype, 300, 6, [2, 1, 4, 1, 1, 3], (2, 4), own=400, prompt=500)
    if rule in ("tokens", "prompt", "parent"):      # of the lists, with all penalties
        r = replace(r, bias=None, allowed=None, temperature=None, **{x: None for x in ("tokens", "prompt", "parent") if x != rule})
    else:
        r = replace(r, **{x: None for x in ("repetition", "presence", "frequency", "temperature", "bias", "allowed") if x != rule})
    compare(apply(r, gpu_device), r.want())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_wanted(gpu_device, dtype):
    r = draw(np.random.default_rng(8), dtype, 8200, 5, None, (5,))
    want, full = r.want(), apply(r, gpu_device)
    for out in (False, True):
        for lse in (False, True):
            for best in (False, True):
                if not (out or lse or best):
                    continue
                o = apply(r, gpu_device, want_out=out, want_lse=lse, want_best=best)
                for name, on in (("out", out), ("lse", lse), ("best", best)):
                    assert (o[name] is not None) == on and (not on or torch.equal(o[name], full[name])), (name, out, lse, best)
    compare(full, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 8195])
def test_strides_places_and_the_logits_themselves(gpu_device, dtype, V):
    r = draw(np.random.default_rng(9), dtype, V, 4, None, (4,))
    want = apply(r, gpu_device)
    rules, rows = r.device(gpu_device), to_dev(r.logits, r.dtype, gpu_device)
    for off_in, off_out, wide in ((0, 0, 8), (1, 0, 5), (0, 3, 7), (5, 2, 1), (3, 3, 11)):
        store = torch.full((4, V + wide + 8), float("nan"), dtype=r.dtype, device=gpu_device)
        view = store[:, off_in:off_in + V]
        view.copy_(rows)
        to = torch.full((4, V + wide + 9), -5.0, dtype=r.dtype, device=gpu_device)
        out = to[:, off_out:off_out + V]
        o = api.at_grpo_logit_rules(rules, view, out=out)
        assert o["out"].data_ptr() == out.data_ptr() and torch.equal(o["out"], want["out"]) and torch.equal(o["lse"], want["lse"]) and torch.equal(o["best"], want["best"])
        assert (to[:, :off_out] == -5).all() and (to[:, off_out + V:] == -5).all()
        before = store.clone()
        api.at_grpo_logit_rules(rules, view, out=view)
        assert torch.equal(view, want["out"])
        before[:, off_in:off_in + V] = want["out"]
        assert torch.equal(store.nan_to_num(7), before.nan_to_num(7))
    both = torch.full((4, 2 * V + 3), -5.0, dtype=r.dtype, device=gpu_device)      # beside each other in rows of one buffer
    for a, b in ((0, V + 3), (V + 1, 0)):
        both[:, a:a + V] = rows
        assert torch.equal(api.at_grpo_logit_rules(rules, both[:, a:a + V], out=both[:, b:b + V])["out"], want["out"])
        assert torch.equal(both[:, a:a + V], rows) and torch.equal(both[:, b:b + V], want["out"])
    with pytest.raises(api.AtGrpoError):
        api.at_grpo_logit_rules(rules, both[:, :V], out=both[:, V - 1:2 * V - 1])
    with pytest.raises(api.AtGrpoError):
        flat = torch.zeros(8 * V, dtype=r.dtype, device=gpu_device)
        api.at_grpo_logit_rules(rules, flat[:4 * V].view(4, V), out=flat[1:4 * V + 1].view(4, V))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 9000])
def test_the_lowest_of_equal_tokens(gpu_device, dtype, V):
    rs = np.random.default_rng(2)
    r = Rows(rounded(rs.normal(size=(12, V)), DTYPES[dtype]), DTYPES[dtype])
    at = [sorted(rs.choice(V, 3, replace=False)) for _ in range(12)]
    for t in range(12):
        r.logits[t, at[t]] = 9.0
    r.temperature = rs.uniform(0.2, 3, 12)
    assert apply(r, gpu_device)["best"].tolist() == [a[0] for a in at]
    r.logits[:] = 0
    r.logits[:, 0] = -0.0
    assert apply(r, gpu_device)["best"].tolist() == [0] * 12
    r.allowed, r.mask_row = np.zeros((2, V), bool), np.arange(12) % 2
    r.allowed[0, V - 1] = r.allowed[1, 5:9] = True
    o = apply(r, gpu_device)
    assert o["best"].tolist() == [V - 1, 5] * 6
    assert o["lse"].tolist()[0] == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 8300])
def test_nothing_left_and_numbers_at_the_ends_of_the_range(gpu_device, dtype, V):
    rs = np.random.default_rng(3)
    t = DTYPES[dtype]
    low, high = float(torch.finfo(t).min), float(torch.finfo(t).max)
    r = Rows(rounded(rs.normal(size=(12, V)), t), t)
    r.allowed = np.ones((3, V), bool)
    r.allowed[0] = False                                   # nothing
    r.allowed[1, [4, V - 2]] = False
    r.mask_row = np.array([0, 1, 1, 1, -1, -1, -1, -1, -1, -1, 2, -1])
    r.logits[1, [4, V - 2]] = np.nan                       # masked
    r.logits[2, [4, V - 2]] = np.inf, high
    r.logits[3, 7] = np.nan                                # not masked
    r.logits[4, 7] = np.inf
    r.logits[5] = -np.inf                                  # nothing, without a mask
    r.logits[6, 1:] = -np.inf
    r.logits[7] = low
    r.logits[8] = high
    r.logits[9] = np.nan
    r.logits[10, :3] = low
    r.logits[11, [3, 9]] = np.inf, np.nan
    want = r.want()
    with np.errstate(all="ignore"):
        o = apply(r, gpu_device)
    compare(o, [w for w in want])
    assert o["best"].tolist()[0] == -1 and o["best"].tolist()[5] == -1 and o["best"].tolist()[9] == -1 and int(o["best"][4]) == 7
    assert np.isneginf(host64(o["lse"])[[0, 5]]).all() and np.isnan(host64(o["lse"])[[3, 9, 11]]).all() and float(o["lse"][4]) == np.inf
    r.mask_row[:] = 0      # every row: also where what is masked is infinite or NaN
    o = apply(r, gpu_device)
    assert np.isneginf(host64(o["out"])).all() and o["best"].tolist() == [-1] * 12 and np.isneginf(host64(o["lse"])).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_biases(gpu_device, dtype):
    """Bans, the same token twice (the last counts), tokens outside the vocabulary, lists of none and of many."""
    rs = np.random.default_rng(4)
    for V in (64, 9000):
        r = Rows(rounded(rs.normal(size=(5, V)), DTYPES[dtype]), DTYPES[dtype])
        r.bias = [[(3, -np.inf), (7, 2.0), (3, 1.5)], [(V - 1, -np.inf), (0, np.inf)], [], [(v, float(v % 7)) for v in rs.integers(0, V, 5000)], [(-1, 5.0), (V, 6.0), (2 ** 31 - 1, 3.0), (9, 1.0)]]
        word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
        o = apply(r, gpu_device, data_error=word)
        compare(o, r.want())
        assert int(word) == TOKEN_RANGE and int(o["best"][1]) == 0 and bool(torch.isneginf(o["out"][1, V - 1]))


@pytest.mark.gpu
def test_counts_of_long_lists(gpu_device):
    """A token that occurs 70000 times, and lists longer than any workgroup's share."""
    rs = np.random.default_rng(6)
    r = Rows(rounded(rs.normal(size=(2, 9000)) * 4, torch.float32), torch.float32)
    r.tokens = [np.concatenate([np.full(70000, 8999), rs.integers(0, 9000, 30000)]), np.arange(9000)]
    r.frequency = np.array([0.001, 0.5])
    compare(apply(r, gpu_device), r.want())
    # with biases, whose numbers and the counts then have a word each: lists of any length, and of the most that share one
    r.bias = [[(8999, 1.0), (5, 2.0), (8999, -4.0)], [(v, float(v % 5)) for v in range(0, 9000, 7)]]
    compare(apply(r, gpu_device), r.want())
    for n in (65535, 65536):
        r.tokens = [np.full(n, 8999), np.arange(100)]
        compare(api.at_grpo_logit_rules(r.device(gpu_device, spare=0), to_dev(r.logits, r.dtype, gpu_device)), r.want(), what=f"{n}")
    r.tokens = [np.arange(50), np.arange(100)]
    for n in (32766, 32767, 32768):
        r.bias = [[(v, float(v % 5)) for v in rs.integers(0, 9000, n - 1)], [(3, 2.0)]]
        compare(apply(r, gpu_device), r.want(), what=f"{n} biases")


@pytest.mark.gpu
@pytest.mark.parametrize("what,bit", [("tokens", TOKEN_RANGE), ("prompt", TOKEN_RANGE), ("drafted", TOKEN_RANGE), ("length", SEQLENS), ("prompt_len", SEQLENS),
                                      ("group_seq", SEQLENS), ("cu_q", SEQLENS), ("bias_cu", SEQLENS), ("mask_row", RULE), ("repetition", RULE), ("presence", RULE),
                                      ("frequency", RULE), ("temperature", RULE)])
def test_data_that_is_none(gpu_device, what, bit):
    """Passed over, with its bit, and the other rows are as they are."""
    dev = gpu_device
    for wrong in (-1, -2 ** 31, 2 ** 31 - 1, 10 ** 6):
        r = draw(np.random.default_rng(7), "f32", 500, 4, [2, 3, 1, 2], (1, 3), biases=6)
        r.tokens, r.prompt, r.bias = [np.append(x, 3) for x in r.tokens], [np.append(x, 4) for x in r.prompt], [x + [(2, 1.0)] for x in r.bias]
        rules, word = r.device(dev), torch.zeros(1, dtype=torch.int32, device=dev)
        logits = to_dev(r.logits, r.dtype, dev)
        field = getattr(rules, what)
        changed, affected = r, {}
        if what in ("tokens", "prompt"):
            field[1, 0] = wrong
            rows = list(getattr(r, what))
            rows[1] = np.append(rows[1][1:], wrong)
            changed = replace(r, **{what: rows})
        elif what == "drafted":
            field[2] = wrong
            d = r.drafted.copy()
            d[2] = wrong
            changed = replace(r, drafted=d)
        elif what in ("length", "prompt_len"):
            field[1] = wrong
            name = dict(length="tokens", prompt_len="prompt")[what]
            rows = list(getattr(r, name))
            rows[1] = rows[1][:0]
            changed = replace(r, **{name: rows})
        elif what == "group_seq":
            field[2] = wrong if wrong > 0 else 5
            changed = replace(r, prompt=[r.prompt[0], r.prompt[1][:0]])
        elif what == "bias_cu":
            field[4] = wrong
            changed = replace(r, bias=r.bias[:3] + [[]])
        elif what == "mask_row":
            if wrong == -1:
                continue
            field[4] = wrong
            m = r.mask_row.copy()
            m[4] = -1
            changed = replace(r, mask_row=m)
        elif what == "cu_q":
            field[4] = wrong if wrong > 0 else 9      # the last sequence's rows are nobody's
            one = lambda a, x: np.append(a[:3], x)
            changed = replace(r, repetition=one(r.repetition, 1), presence=one(r.presence, 0), frequency=one(r.frequency, 0), temperature=one(r.temperature, 1),
                              bias=r.bias[:3] + [[]])
        else:
            field[1] = {-1: float("nan"), -2 ** 31: float("inf"), 2 ** 31 - 1: -float("inf"), 10 ** 6: float("nan")}[wrong]
            a = getattr(r, what).copy()
            a[1] = 1 if what in ("repetition", "temperature") else 0
            changed = replace(r, **{what: a})
        compare(api.at_grpo_logit_rules(rules, logits, data_error=word), changed.want(), what=f"{what} {wrong}")
        assert int(word) == bit, (what, wrong)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [0.0, -1.0, 1e-40])
def test_settings_that_are_not_positive(gpu_device, value):
    r = draw(np.random.default_rng(11), "f32", 500, 3)
    for name in ("repetition", "temperature"):
        a = getattr(r, name).copy()
        a[2] = value
        word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
        o = apply(replace(r, **{name: a}), gpu_device, data_error=word)
        a = a.copy()
        a[2] = 1
        compare(o, replace(r, **{name: a}).want())
        assert int(word) == RULE


@pytest.mark.gpu
@pytest.mark.parametrize("V", [500, 9000])
def test_a_temperature_at_the_end_of_the_range(gpu_device, V):
    """Its reciprocal is finite, and times log2 e it is not.  out: the reciprocal's rounding and the product's, neither of which is of small
    numbers; lse: ln of a count (two roundings and the exponential's unit), or the largest itself."""
    logits = torch.full((2, V), -1.0)
    logits[0, 3::7], logits[1], logits[1, V - 2] = 0.0, 0.0, 1.0
    temperature, word = torch.full((2,), 3.5e-39), torch.zeros(1, dtype=torch.int32, device=gpu_device)
    rules = api.LogitRules(temperature=temperature.to(gpu_device))
    o = api.at_grpo_logit_rules(rules, logits.to(gpu_device), data_error=word)
    want = logits.double() / temperature.double()[:, None]
    assert int(word) == 0 and o["best"].tolist() == [3, V - 2]
    assert ((o["out"].cpu().double() - want).abs() <= 2.01 * U32 * want.abs()).all()
    n = np.log(len(range(3, V, 7)))
    assert abs(float(o["lse"][0]) - n) <= 8 * U32 * n and abs(float(o["lse"][1]) - float(want[1].max())) <= 3.01 * U32 * float(want[1].max())


@pytest.mark.gpu
@pytest.mark.parametrize("biases", [False, True])
def test_quotients_past_the_range(gpu_device, biases):
    """A repetition so small that what occurs in front is multiplied out of the range: infinite, no NaN."""
    V, r = 700, np.float32(1e-38)
    logits = torch.zeros(2, V)
    logits[:, 5], logits[0, 9], logits[1, 9] = 2.0, 10.0, -10.0
    dev, i32 = gpu_device, lambda x: torch.tensor(x, dtype=torch.int32, device=gpu_device)
    more = dict(bias_cu=i32([0, 1, 1]), bias_token=i32([600]), bias=torch.zeros(1, device=dev)) if biases else {}
    rules = api.LogitRules(tokens=i32([[5, 9], [5, 9]]), length=i32([2, 2]), repetition=torch.full((2,), float(r)).to(dev), **more)
    word = torch.zeros(1, dtype=torch.int32, device=dev)
    o = api.at_grpo_logit_rules(rules, logits.to(dev), data_error=word)
    out, two = o["out"].cpu(), 2 / float(r)
    assert int(word) == 0 and o["best"].tolist() == [9, 5] and float(out[0, 9]) == float("inf") == float(o["lse"][0])
    assert all(abs(float(out[t, 5]) - two) <= 1.01 * U32 * two for t in (0, 1)) and abs(float(o["lse"][1]) - two) <= 3.01 * U32 * two
    assert abs(float(out[1, 9]) + 10 * float(r)) <= 1.01 * U32 * 10 * float(r)
    rest = [v for v in range(V) if v not in (5, 9)]
    assert (out[:, rest] == 0).all()


@pytest.mark.gpu
def test_rows_of_no_sequence(gpu_device):
    """In front of the first and behind the last: their masks and nothing else."""
    r = draw(np.random.default_rng(12), "f32", 700, 3, [2, 1, 2], (3,))
    want = r.want()
    more = rounded(np.random.default_rng(13).normal(size=(4, 700)), torch.float32)
    rules = r.device(gpu_device)
    rules.cu_q += 1
    pad = lambda t, x: torch.cat((torch.full((1,), x, dtype=t.dtype, device=t.device), t, torch.full((3,), x, dtype=t.dtype, device=t.device)))
    rules.drafted, rules.ancestors, rules.mask_row = pad(rules.drafted, 0), pad(rules.ancestors, -1), pad(rules.mask_row, 1)
    logits = to_dev(np.concatenate([more[:1], r.logits, more[1:]]), torch.float32, gpu_device)
    word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    o = api.at_grpo_logit_rules(rules, logits, data_error=word)
    alone = [oracle.sampling_row(x, [], [], 1, 0, 0, 1, {}, r.allowed[1]) for x in more]
    compare(o, alone[:1] + want + alone[1:])
    assert int(word) == 0


@pytest.mark.gpu
def test_no_rows_and_one(gpu_device):
    o = api.at_grpo_logit_rules(api.LogitRules(), torch.zeros(0, 50, device=gpu_device))
    assert o["out"].shape == (0, 50) and o["lse"].shape == (0,) and o["best"].shape == (0,)
    r = draw(np.random.default_rng(14), "bf16", 1, 1)
    compare(apply(r, gpu_device), r.want())


@pytest.mark.gpu
def test_many_rows(gpu_device):
    """More workgroups than 16 bits count."""
    rs = np.random.default_rng(15)
    n = 70001
    logits = torch.randn(n, 33, device=gpu_device, generator=torch.Generator(device=gpu_device).manual_seed(0))
    temperature = torch.from_numpy(rs.uniform(0.5, 2, n)).float().to(gpu_device)
    o = api.at_grpo_logit_rules(api.LogitRules(temperature=temperature), logits)
    x = logits.double() / temperature.double()[:, None]
    assert torch.equal(o["best"].long(), logits.argmax(1))
    assert float((o["out"].double() - x).abs().max()) <= 4 * U32 * float(x.abs().max())
    assert float((o["lse"].double() - torch.logsumexp(x, 1)).abs().max()) <= U32 * (8 * float(x.abs().max()) + 60)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("biases", [0, 20])
def test_several_chunks_a_workgroup(gpu_device, dtype, biases):
    """Rows enough that a workgroup has more than one chunk of them: some of them against the oracle, all against the same rows few at a time."""
    rs = np.random.default_rng(18)
    V, new = 50003, [1 + i % 3 for i in range(1000)]
    r = draw(rs, dtype, 300, 1000, new, (400, 600), biases=biases)      # lists of the first 300 tokens ..
    n = sum(new)
    spread = lambda v: int(v) * 165 % V                                 # .. spread over all
    r.tokens, r.prompt = [[spread(v) for v in x] for x in r.tokens], [[spread(v) for v in x] for x in r.prompt]
    r.drafted = np.array([spread(v) for v in r.drafted])
    r.bias = None if r.bias is None else [[(spread(v), b) for v, b in x] for x in r.bias]
    r.allowed = rs.random((3, V)) < 0.7
    logits = torch.randn(n, V, generator=torch.Generator().manual_seed(3)).to(r.dtype)
    r.logits = np.zeros((n, 1))
    rules, dev_logits = r.device(gpu_device), logits.to(gpu_device)
    o = api.at_grpo_logit_rules(rules, dev_logits)
    start = r.start()
    for s in (0, 1, 2, 399, 400, 998, 999):
        rows = slice(start[s], start[s + 1])
        part = Rows(logits[rows].double().numpy(), r.dtype, np.array(new[s:s + 1]), r.tokens[s:s + 1], (1,), r.prompt[:1] if s < 400 else r.prompt[1:], r.drafted[rows],
                    r.parent[rows], r.repetition[s:s + 1], r.presence[s:s + 1], r.frequency[s:s + 1], r.temperature[s:s + 1],
                    None if r.bias is None else r.bias[s:s + 1], r.allowed, r.mask_row[rows])
        few = apply(part, gpu_device)
        compare({k: o[k][rows] for k in ("out", "lse", "best")}, part.want(), what=f"sequence {s}")
        assert torch.equal(few["out"], o["out"][rows]) and torch.equal(few["best"], o["best"][rows]), s
        assert float((few["lse"] - o["lse"][rows]).abs().max()) <= 40 * U32 * float(few["lse"].abs().max().clamp(min=1))      # sums in another order


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_streams_and_graphs(gpu_device, dtype):
    r = draw(np.random.default_rng(16), dtype, 8300, 4, [2, 1, 4, 1], (1, 3))
    rules, logits = r.device(gpu_device), to_dev(r.logits, r.dtype, gpu_device)
    fn = lambda: api.at_grpo_logit_rules(rules, logits)
    names = ("out", "lse", "best")
    side, g = torch.cuda.Stream(device=gpu_device), torch.cuda.CUDAGraph()
    want = fn()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = fn()
    side.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in names)
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            out = fn()
    for step in range(3):
        logits.mul_(-1.25)
        rules.length.sub_(1).clamp_(min=0)
        rules.temperature.mul_(1.1)
        want = fn()
        for n in names:
            out[n].fill_(3)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in names), step


REFUSALS = {
    "logits on the host": lambda r, x: (r, x.cpu()),
    "whole numbers": lambda r, x: (r, x.int()),
    "three dimensions": lambda r, x: (r, x[None]),
    "columns apart": lambda r, x: (r, x.repeat(1, 2)[:, ::2]),
    "rows that overlap": lambda r, x: (r, x[:1].expand(4, -1)),
    "lengths of another number": lambda r, x: (replace(r, length=r.length[:3]), x),
    "lengths in 64 bits": lambda r, x: (replace(r, length=r.length.long()), x),
    "tokens without lengths": lambda r, x: (replace(r, length=None), x),
    "tokens of fewer sequences": lambda r, x: (replace(r, tokens=r.tokens[:3]), x),
    "prompts without groups": lambda r, x: (replace(r, group_seq=None), x),
    "prompts of more groups": lambda r, x: (replace(r, prompt=r.prompt.repeat(2, 1)), x),
    "settings in 64 bits": lambda r, x: (replace(r, temperature=r.temperature.double()), x),
    "a mask of too few columns": lambda r, x: (replace(r, allowed=r.allowed[:, :-1].contiguous()), x),
    "masks without rows": lambda r, x: (replace(r, mask_row=None), x),
    "biases without tokens": lambda r, x: (replace(r, bias_token=None), x),
    "fewer values than tokens": lambda r, x: (replace(r, bias=r.bias[:-1]), x),
    "paths without tokens": lambda r, x: (replace(r, ancestors=torch.zeros(4, dtype=torch.int64, device=x.device)), x),
    "settings on the host": lambda r, x: (replace(r, presence=r.presence.cpu()), x),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", REFUSALS)
def test_refusals(gpu_device, name):
    r = draw(np.random.default_rng(17), "f32", 100, 4, None, (4,))
    r.bias[0] = [(1, 1.0), (2, 2.0)]
    rules, logits = REFUSALS[name](r.device(gpu_device), to_dev(r.logits, r.dtype, gpu_device))
    with pytest.raises(api.AtGrpoError):
        api.at_grpo_logit_rules(rules, logits)


@pytest.mark.gpu
def test_refused_outputs(gpu_device):
    x = torch.zeros(4, 100, device=gpu_device)
    for kw in (dict(out=x[:3].clone()), dict(out=x.bfloat16()), dict(out_dtype=torch.bfloat16), dict(out_dtype=torch.float16), dict(out=x.cpu()),
               dict(want_out=False, want_lse=False, want_best=False), dict(data_error=torch.zeros(2, dtype=torch.int32, device=gpu_device))):
        with pytest.raises(api.AtGrpoError):
            api.at_grpo_logit_rules(api.LogitRules(), x, **kw)
