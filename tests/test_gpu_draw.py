"""Draws from given numbers on the GPU against the oracle: tokens bit for bit, log-probabilities to
float32 rounding (half a step, 2^-24, of the value; the logarithm itself is taken in 64 bits on both sides, whose
differences of a unit can move a value across a midpoint: one step, 2^-23)."""
import numpy as np
import pytest
import torch

import synth
from oracle import draw as D

pytestmark = pytest.mark.gpu

tadm = pytest.importorskip("paper_2609_37924_amd")

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

F = np.float32
INF, NAN = np.inf, np.nan
_models = {}


def model(V):
    if V not in _models:
        _models[V] = tadm.tadm_model_create(tadm.make_config(synth.get_config("tiny", vocab=V), max_batch=1, max_seq=64))
        tadm.tadm_set_stream(_models[V], torch.cuda.current_stream().cuda_stream)
    return _models[V]


@pytest.fixture(scope="module", autouse=True)
def _close():
    yield
    for m in _models.values():
        tadm.tadm_model_destroy(m)
    _models.clear()


def scratch(m, R):
    size = tadm.tadm_sample_rows_work(m, R)
    return torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda")  # nothing relies on what it holds


def check(rows, u, settings, ld=None, shift=0):
    """rows [R, V]; settings: name -> array [R].  ld: floats between rows, shift: floats before the first."""
    R, V = rows.shape
    ld = ld or V
    m = model(V)
    flat = torch.full((shift + R * ld + 8,), NAN, device="cuda")
    logits = flat[shift:shift + R * ld].view(R, ld)[:, :V]
    logits.copy_(torch.from_numpy(np.ascontiguousarray(rows)))
    dev = {k: torch.from_numpy(np.asarray(v, dtype=np.int32 if k == "top_k" else F)).cuda() for k, v in settings.items()}
    ud = torch.from_numpy(np.asarray(u, dtype=F)).cuda()
    token = torch.full((R + 1,), 77, dtype=torch.int32, device="cuda")
    logp = torch.full((R + 1,), 77.0, device="cuda")
    work = scratch(m, R)
    tadm.tadm_sample_rows(m, logits, tadm.row_settings(**dev), ud, token[:R], logp[:R], work)
    torch.cuda.synchronize()
    assert token[R] == 77 and logp[R] == 77.0
    got, lp = token[:R].cpu().numpy(), logp[:R].cpu().numpy().astype(np.float64)
    for r in range(R):
        ref, ref_lp = D.draw(rows[r], F(u[r]), **{k: np.asarray(v)[r] for k, v in settings.items()})
        assert got[r] == ref, (r, got[r], ref, {k: np.asarray(v)[r] for k, v in settings.items()})
        assert lp[r] == ref_lp or abs(lp[r] - ref_lp) <= 2.0 ** -23 * abs(ref_lp) + 1e-300, (r, lp[r], ref_lp)
    # the tokens alone
    again = torch.full((R,), 55, dtype=torch.int32, device="cuda")
    tadm.tadm_sample_rows(m, logits, tadm.row_settings(**dev), ud, again, None, work)
    assert torch.equal(again, token[:R])


def mixed(rng, R):
    return dict(temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 2.5], size=R), top_k=rng.choice([0, 0, 1, 2, 20, 500, 10 ** 6, -4], size=R),
                top_p=rng.choice([1.0, 0.999, 0.9, 0.5, 1e-9], size=R), min_p=rng.choice([0.0, 0.0, 0.01, 0.3], size=R))


@pytest.mark.parametrize("V", [1000, 32768])
@pytest.mark.parametrize("R", [3, 600])
def test_temperatures_at_the_ends_of_float32(V, R):
    """l' = l (1 / t) in float32: +-inf where that overflows, and -1 for a row of which nothing finite is left."""
    rng = np.random.default_rng(V + R)
    rows = rng.normal(size=(R, V)).astype(F)
    rows[::3] = -5 - np.abs(rows[::3])  # none but -inf at 1e-38
    rows[1::3, ::7] += 9  # several +inf at 1e-38
    tiny = np.where(np.arange(R) % 3 < 2, 1e-38, 1e-30)
    assert D.draw(rows[0], F(0.5), temperature=tiny[0])[0] == -1 and D.draw(rows[1], F(0.5), temperature=tiny[1])[0] >= 0
    check(rows, rng.random(R), dict(temperature=tiny))
    check(rows, rng.random(R), dict(temperature=tiny, top_k=[5] * R, top_p=[0.7] * R))
    check(rows, rng.random(R), dict(temperature=np.where(tiny < 1e-35, 3e38, np.inf)))


@pytest.mark.parametrize("V", [1, 2, 3, 5, 63, 64, 257, 1000, 4097, 16384, 16385, 32768, 32771, 50304, 128256, 262143, 262144])
def test_rows_with_settings_of_their_own(V):
    rng = np.random.default_rng(V)
    R = 24 if V < 20000 else 12
    rows = (rng.normal(size=(R, V)) * rng.uniform(0.02, 4.0, size=(R, 1))).astype(F)
    if V > 10:
        rows[rng.random(rows.shape) < 0.2] = -INF
        rows[::3, V // 3] = NAN
        rows[:, V // 2] = 1.0
    check(rows, rng.random(R), mixed(rng, R))


@pytest.mark.parametrize("name", ["temperature", "top_k", "top_p", "min_p", None])
@pytest.mark.parametrize("V", [300, 40000])
def test_one_setting_alone(name, V):
    rng = np.random.default_rng(V + len(name or ""))
    rows = (rng.normal(size=(16, V)) * 2).astype(F)
    s = mixed(rng, 16)
    check(rows, rng.random(16), {name: s[name]} if name else {})


@pytest.mark.parametrize("ld, shift", [(1000, 0), (1003, 0), (1003, 1), (2048, 3), (1001, 2)])
def test_rows_at_any_float(ld, shift):
    rng = np.random.default_rng(ld + shift)
    check((rng.normal(size=(9, 1000)) * 3).astype(F), rng.random(9), mixed(rng, 9), ld, shift)


FLAT = {
    "equal": lambda rng, V: np.zeros(V),
    "two values": lambda rng, V: rng.choice([0.0, -0.25], size=V),
    "signed zeros": lambda rng, V: rng.choice([0.0, -0.0, -1.0], size=V),
    "one bin": lambda rng, V: rng.uniform(3.0, 3.0 + 2.0 ** -8, size=V),
    "one digit": lambda rng, V: 100.0 + rng.uniform(0, 2.0 ** -17, size=V),
    "neighbours": lambda rng, V: np.nextafter(F(2), F(3)) + rng.choice([0.0, 2.0 ** -22], size=V),
    "tiny differences": lambda rng, V: rng.choice([0.0, 1e-9, 2e-9, 1e-38], size=V),
}


@pytest.mark.parametrize("V", [3000, 33000, 262144])
@pytest.mark.parametrize("kind", list(FLAT))
def test_rows_whose_entries_hardly_differ(kind, V):
    """More entries in a bin, in its digits, and with the same value, than a list holds."""
    rng = np.random.default_rng(V + len(kind))
    R = 8
    rows = np.stack([FLAT[kind](rng, V) for _ in range(R)]).astype(F)
    s = dict(temperature=np.ones(R), top_k=[0, 1500, V // 2, 0, V - 1, 2, 1025, 0],
             top_p=[0.5, 1.0, 0.5, 0.999, 0.9, 1.0, 0.7, 1.0], min_p=np.zeros(R))
    check(rows, rng.random(R), s)


def test_ends_of_the_settings():
    rng = np.random.default_rng(8)
    s = []
    for t in (0.0, -1.0, NAN, 1e-30, 1e30, 1.0):
        for k in (0, -2 ** 31, 2 ** 31 - 1, 3):
            for p in (-1.0, 0.0, NAN, INF, 1e-45, 1.0 - 2.0 ** -24):
                for q in (NAN, -1.0, 1e-45, 1.0, INF):
                    s.append((t, k, p, q))
    t, k, p, q = (np.array(x) for x in zip(*s))
    rows = (rng.normal(size=(len(s), 130)) * 3).astype(F)
    check(rows, rng.random(len(s)), dict(temperature=t, top_k=k, top_p=p, min_p=q))


@pytest.mark.parametrize("V", [130, 40000])
def test_ends_of_the_numbers(V):
    rng = np.random.default_rng(9)
    u = np.array([0.0, -0.0, -1.0, NAN, 1.0, 2.0, INF, 1.0 - 2.0 ** -24, 2.0 ** -24, 2.0 ** -25, 2.0 ** -149, 0.5], dtype=F)
    rows = (rng.normal(size=(len(u), V)) * 3).astype(F)
    rows[5, 0] = rows[4, V - 1] = 9.0
    check(rows, u, dict(top_p=np.where(np.arange(len(u)) % 2, 1.0, 0.9)))


@pytest.mark.parametrize("V", [130, 40000])
def test_rows_of_infinities(V):
    rows = np.zeros((9, V), dtype=F)
    rows[0] = -INF
    rows[1] = NAN
    rows[2, ::2], rows[2, 1::2] = NAN, -INF
    rows[3] = -INF
    rows[3, V - 1] = -3e38
    rows[4, [5, 99]] = INF
    rows[5] = INF
    rows[6, 7], rows[6, 8], rows[6, 9] = 3e38, -3e38, NAN
    rows[7] = -3e38
    rows[8, 3:] = -INF
    n = len(rows)
    for s in (dict(), dict(top_k=[2] * n), dict(top_p=[0.6] * n), dict(temperature=[0.01] * n, top_p=[0.6] * n), dict(temperature=[0.0] * n)):
        check(rows, np.linspace(0.05, 0.95, n), s)


def test_captured_draws_read_their_settings_at_each_replay():
    rng = np.random.default_rng(10)
    R, V = 6, 50304
    m = model(V)
    logits, u = torch.zeros(R, V, device="cuda"), torch.zeros(R, device="cuda")
    dev = {k: torch.from_numpy(v.astype(np.int32 if k == "top_k" else F)).cuda() for k, v in mixed(rng, R).items()}
    token, logp, work = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda"), scratch(m, R)
    settings = tadm.row_settings(**dev)
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    side.wait_stream(main)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        tadm.tadm_set_stream(m, side.cuda_stream)
        try:
            with torch.cuda.graph(graph, stream=side):
                tadm.tadm_sample_rows(m, logits, settings, u, token, logp, work)
        finally:
            tadm.tadm_set_stream(m, main.cuda_stream)
    main.wait_stream(side)
    for seed in range(4):
        rng = np.random.default_rng(seed)
        s = mixed(rng, R)
        rows, x = (rng.normal(size=(R, V)) * 2).astype(F), rng.random(R).astype(F)
        logits.copy_(torch.from_numpy(rows))
        u.copy_(torch.from_numpy(x))
        for k, v in s.items():
            dev[k].copy_(torch.from_numpy(v.astype(np.int32 if k == "top_k" else F)))
        graph.replay()
        torch.cuda.synchronize()
        ref = [D.draw(rows[r], x[r], **{k: v[r] for k, v in s.items()}) for r in range(R)]
        assert token.tolist() == [t for t, _ in ref]
        eager = torch.zeros_like(token)
        tadm.tadm_sample_rows(m, logits, settings, u, eager, None, work)
        assert torch.equal(eager, token)


@pytest.mark.parametrize("V", [700, 5000, 9001])
def test_more_rows_than_split(V):
    """A block a row: ordinary rows and rows whose entries hardly differ, which overflow the list."""
    rng = np.random.default_rng(V)
    R = 530
    rows = (rng.normal(size=(R, V)) * rng.uniform(0.02, 4.0, size=(R, 1))).astype(F)
    for i, kind in enumerate(FLAT):
        rows[i::40] = FLAT[kind](rng, V)
    rows[11::40] = -INF
    check(rows, rng.random(R), mixed(rng, R), V + 2)


def test_scratch_is_asked_for():
    m = model(50304)
    logits, u, token = torch.zeros(4, 50304, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    size = tadm.tadm_sample_rows_work(m, 4)
    assert size > 0 and tadm.tadm_sample_rows_work(m, 0) == 0
    for work in (None, torch.zeros(size - 16, dtype=torch.uint8, device="cuda"), torch.zeros(size + 16, dtype=torch.uint8, device="cuda")[8:]):
        with pytest.raises(tadm.TadmError, match="scratch"):
            tadm.tadm_sample_rows(m, logits, None, u, token, None, work)
    with pytest.raises(tadm.TadmError, match="apart"):
        tadm.tadm_sample_rows(m, logits[:, :100].contiguous(), None, u, token, None, torch.zeros(size, dtype=torch.uint8, device="cuda"))
    assert tadm.tadm_sample_rows_work(m, 5000) == 0  # a block a row needs none
